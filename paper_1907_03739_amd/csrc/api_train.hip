// C ABI of the operators in pvconv_train.h: argument validation on the host,
// then launches on the caller's stream. Nothing is enqueued when validation
// fails.
#include <math.h>

#include "pv_args.h"
#include "pv_train.h"

namespace {

inline bool misaligned(const void* p, size_t to) { return ((uintptr_t)p & (to - 1)) != 0; }

// The byte range of rows of channels.
inline size_t row_bytes(long long rows, int c, int ld, pvconv_dtype dt) {
    return rows > 0 ? ((size_t)(rows - 1) * (size_t)ld + (size_t)c) * esize(dt) : 0;
}

inline pvconv_status check_ws(const void* ws, size_t bytes, size_t need) {
    return need && (!ws || misaligned(ws, 256) || bytes < need) ? PVCONV_EWORKSPACE : PVCONV_OK;
}

inline bool norm_sizes_ok(int B, int N, int C, int groups) {
    return B >= 0 && N >= 0 && C >= 1 && C <= PVCONV_MAX_NORM_CHANNELS && groups >= 1 &&
           C % groups == 0 && sizes_fit(B, N);
}
inline bool norm_act_ok(pvconv_act a) { return act_ok(a) || a == PVCONV_ACT_SILU; }

inline bool fp8_sizes_ok(int M, int K, int N) {
    return M >= 0 && M <= (1 << 30) && K >= 1 && N >= 1 && K <= PVCONV_FP8_MAX_CHANNELS &&
           N <= PVCONV_FP8_MAX_CHANNELS &&
           (long long)pv_fp8_blocks(M) * pv_fp8_blocks(K > N ? K : N) <= (1LL << 26);
}
inline size_t fp8_bytes(int rows, int cols) {
    return (size_t)rows * pv_fp8_blocks(cols) * PVCONV_FP8_BLOCK;
}

inline bool int8_sizes_ok(int M, int K, int N) {
    const auto blocks = [](int n) { return ((long long)n + PVCONV_INT8_BLOCK - 1) / PVCONV_INT8_BLOCK; };
    return M >= 0 && M <= (1 << 30) && K >= 1 && N >= 1 && K <= PVCONV_INT8_MAX_CHANNELS &&
           N <= PVCONV_INT8_MAX_CHANNELS && blocks(M) * blocks(K > N ? K : N) <= (1LL << 26);
}
inline size_t int8_bytes(int rows, int cols) {
    return (size_t)rows * (((size_t)cols + PVCONV_INT8_BLOCK - 1) / PVCONV_INT8_BLOCK) *
           PVCONV_INT8_BLOCK;
}

// Byte ranges of which none may overlap an output.
struct Ranges {
    const void* p[16];
    size_t bytes[16];
    int n = 0;
    void add(const void* q, size_t b) {
        if (q && b) {
            p[n] = q;
            bytes[n++] = b;
        }
    }
    // adds an output; false where it overlaps what is there
    bool output(const void* q, size_t b) {
        if (!q || !b) return true;
        for (int i = 0; i < n; i++)
            if (bytes_overlap(q, b, p[i], bytes[i])) return false;
        add(q, b);
        return true;
    }
};

inline bool ce_sizes_ok(int M, int K, int V) {
    return M >= 0 && M <= (1 << 24) && K >= 1 && K <= PVCONV_CE_MAX_CHANNELS && V >= 1 &&
           V <= PVCONV_MAX_CLASSES;
}
// The arguments that a forward and a backward share; `r` gets the inputs' ranges.
pvconv_status check_ce(PvLinearCe& a, pvconv_dtype x_dt, pvconv_dtype w_dt, pvconv_dtype dx_dt,
                       pvconv_dtype dw_dt, Ranges& r) {
    if (!ce_sizes_ok(a.M, a.K, a.V) || !dtype_ok(x_dt) || !dtype_ok(w_dt) || !dtype_ok(dx_dt) ||
        !dtype_ok(dw_dt))
        return PVCONV_EINVAL;
    if (a.x.ld == 0) a.x.ld = a.K;
    if (a.w.ld == 0) a.w.ld = a.K;
    if (a.dx.ld == 0) a.dx.ld = a.K;
    if (a.x.ld < a.K || a.w.ld < a.K || a.dx.ld < a.K) return PVCONV_EINVAL;
    a.dw.ld = a.K;
    a.x.bf16 = x_dt == PVCONV_BF16;
    a.w.bf16 = w_dt == PVCONV_BF16;
    a.dx.bf16 = dx_dt == PVCONV_BF16;
    a.dw.bf16 = dw_dt == PVCONV_BF16;
    if (a.M > 0 && (!a.x.p || !a.w.p || !a.labels)) return PVCONV_EINVAL;
    if (misaligned(a.x.p, esize(x_dt)) || misaligned(a.w.p, esize(w_dt)) ||
        misaligned(a.bias, 4) || misaligned(a.labels, 4) || misaligned(a.weight, 4) ||
        misaligned(a.loss, 4) || misaligned(a.lse, 4) || misaligned(a.dx.p, esize(dx_dt)) ||
        misaligned(a.dw.p, esize(dw_dt)) || misaligned(a.dbias, 4))
        return PVCONV_EINVAL;
    const size_t mb = (size_t)a.M * 4, vb = (size_t)a.V * 4;
    r.add(a.w.p, row_bytes(a.V, a.K, a.w.ld, w_dt));
    r.add(a.bias, vb);
    r.add(a.labels, mb);
    r.add(a.weight, mb);
    if (a.dx.p && (overlap(a.x.p, a.M, a.K, a.x.ld, x_dt, a.dx.p, a.K, a.dx.ld, dx_dt) ||
                   !r.output(a.dx.p, row_bytes(a.M, a.K, a.dx.ld, dx_dt))))
        return PVCONV_EINVAL;
    r.add(a.x.p, row_bytes(a.M, a.K, a.x.ld, x_dt));
    if (!r.output(a.dw.p, row_bytes(a.V, a.K, a.K, dw_dt)) || !r.output(a.dbias, vb))
        return PVCONV_EINVAL;
    return PVCONV_OK;
}

pvconv_status check_distill(const void* z, pvconv_dtype z_dt, int& z_ld, int M, int V,
                            const float* t_val, const int32_t* t_class, int top,
                            const int32_t* labels, float temperature, float alpha) {
    if (M < 0 || M > (1 << 30) || V < 1 || V > PVCONV_MAX_CLASSES || top < 1 ||
        top > PVCONV_MAX_TOP || !dtype_ok(z_dt))
        return PVCONV_EINVAL;
    if (!(temperature > 0.f) || isinf(temperature) || isinf(1.f / temperature) ||
        !(alpha >= 0.f && alpha <= 1.f))
        return PVCONV_EINVAL;
    if (z_ld == 0) z_ld = V;
    if (z_ld < V) return PVCONV_EINVAL;
    if (M == 0) return PVCONV_OK;
    if (!z || !t_val || !t_class) return PVCONV_EINVAL;
    if (misaligned(z, esize(z_dt)) || misaligned(t_val, 4) || misaligned(t_class, 4) ||
        misaligned(labels, 4))
        return PVCONV_EINVAL;
    return PVCONV_OK;
}

pvconv_status check_dz(const void* z, pvconv_dtype z_dt, int z_ld, const void* dz,
                       pvconv_dtype dz_dt, int& dz_ld, int M, int V, const float* t_val,
                       const int32_t* t_class, int top) {
    if (!dtype_ok(dz_dt)) return PVCONV_EINVAL;
    if (dz_ld == 0) dz_ld = V;
    if (dz_ld < V) return PVCONV_EINVAL;
    if (M == 0) return PVCONV_OK;
    const size_t tb = (size_t)M * top * 4, db = row_bytes(M, V, dz_ld, dz_dt);
    if (!dz || misaligned(dz, esize(dz_dt))) return PVCONV_EINVAL;
    if (overlap(z, M, V, z_ld, z_dt, dz, V, dz_ld, dz_dt) || bytes_overlap(dz, db, t_val, tb) ||
        bytes_overlap(dz, db, t_class, tb))
        return PVCONV_EINVAL;
    return PVCONV_OK;
}

}  // namespace

extern "C" {

size_t pvconv_group_norm_act_workspace_size(int B, int N, int C, int groups) {
    return norm_sizes_ok(B, N, C, groups) ? pv_group_norm_ws_bytes(B, N, C, groups) : 0;
}

pvconv_status pvconv_group_norm_act(const void* x, pvconv_dtype x_dt, int x_ld, int B, int N,
                                    int C, int groups, const int32_t* lengths,
                                    const float* gamma, const float* beta, float eps,
                                    pvconv_act act, float slope, void* y, pvconv_dtype y_dt,
                                    int y_ld, float* stats, void* workspace,
                                    size_t workspace_bytes, void* stream) {
    if (!norm_sizes_ok(B, N, C, groups) || !dtype_ok(x_dt) || !dtype_ok(y_dt) ||
        !norm_act_ok(act) || !(eps >= 0.f))
        return PVCONV_EINVAL;
    if (x_ld == 0) x_ld = C;
    if (y_ld == 0) y_ld = C;
    if (x_ld < C || y_ld < C) return PVCONV_EINVAL;
    if (B == 0) return PVCONV_OK;
    if (N == 0 && !stats) return PVCONV_OK;
    if ((N > 0 && (!x || !y)) || !gamma || !beta) return PVCONV_EINVAL;
    if (misaligned(x, esize(x_dt)) || misaligned(y, esize(y_dt)) || misaligned(gamma, 4) ||
        misaligned(beta, 4) || misaligned(stats, 4) || misaligned(lengths, 4))
        return PVCONV_EINVAL;
    const long long M = (long long)B * N;
    const size_t yb = row_bytes(M, C, y_ld, y_dt), sb = stats ? (size_t)B * groups * 8 : 0;
    if (overlap(x, M, C, x_ld, x_dt, y, C, y_ld, y_dt) ||
        bytes_overlap(y, yb, gamma, (size_t)C * 4) || bytes_overlap(y, yb, beta, (size_t)C * 4) ||
        bytes_overlap(y, yb, stats, sb) ||
        bytes_overlap(x, row_bytes(M, C, x_ld, x_dt), stats, sb))
        return PVCONV_EINVAL;
    const pvconv_status st =
        check_ws(workspace, workspace_bytes, pv_group_norm_ws_bytes(B, N, C, groups));
    if (st != PVCONV_OK) return st;
    return pv_launch_group_norm(
        PvNorm{B, N, C, groups, lengths, gamma, beta, eps, act, slope},
        PvRows{(void*)x, x_dt == PVCONV_BF16, x_ld}, PvRows{y, y_dt == PVCONV_BF16, y_ld}, stats,
        workspace, as_stream(stream));
}

size_t pvconv_group_norm_act_backward_workspace_size(int B, int N, int C, int groups) {
    return norm_sizes_ok(B, N, C, groups) ? pv_group_norm_bwd_ws_bytes(B, N, C, groups) : 0;
}

pvconv_status pvconv_group_norm_act_backward(
    const void* dy, pvconv_dtype dy_dt, int dy_ld, const void* x, pvconv_dtype x_dt, int x_ld,
    int B, int N, int C, int groups, const int32_t* lengths, const float* stats,
    const float* gamma, const float* beta, pvconv_act act, float slope, void* dx,
    pvconv_dtype dx_dt, int dx_ld, float* dgamma, float* dbeta, void* workspace,
    size_t workspace_bytes, void* stream) {
    if (!norm_sizes_ok(B, N, C, groups) || !dtype_ok(x_dt) || !dtype_ok(dy_dt) ||
        !dtype_ok(dx_dt) || !norm_act_ok(act))
        return PVCONV_EINVAL;
    if (x_ld == 0) x_ld = C;
    if (dy_ld == 0) dy_ld = C;
    if (dx_ld == 0) dx_ld = C;
    if (x_ld < C || dy_ld < C || dx_ld < C) return PVCONV_EINVAL;
    const long long M = (long long)B * N;
    if (M > 0 && (!dy || !x || !stats || !dx || !gamma || !beta)) return PVCONV_EINVAL;
    if (misaligned(x, esize(x_dt)) || misaligned(dy, esize(dy_dt)) ||
        misaligned(dx, esize(dx_dt)) || misaligned(gamma, 4) || misaligned(beta, 4) ||
        misaligned(stats, 4) || misaligned(lengths, 4) || misaligned(dgamma, 4) ||
        misaligned(dbeta, 4))
        return PVCONV_EINVAL;
    const size_t cb = (size_t)C * 4, db = row_bytes(M, C, dx_ld, dx_dt);
    if (overlap(x, M, C, x_ld, x_dt, dx, C, dx_ld, dx_dt) ||
        overlap(dy, M, C, dy_ld, dy_dt, dx, C, dx_ld, dx_dt) ||
        bytes_overlap(dx, db, gamma, cb) || bytes_overlap(dx, db, beta, cb) ||
        bytes_overlap(dx, db, stats, (size_t)B * groups * 8) ||
        bytes_overlap(dx, db, dgamma, dgamma ? cb : 0) ||
        bytes_overlap(dx, db, dbeta, dbeta ? cb : 0) ||
        bytes_overlap(dgamma, dgamma ? cb : 0, dbeta, dbeta ? cb : 0) ||
        bytes_overlap(gamma, cb, dgamma, dgamma ? cb : 0) ||
        bytes_overlap(gamma, cb, dbeta, dbeta ? cb : 0) ||
        bytes_overlap(beta, cb, dgamma, dgamma ? cb : 0) ||
        bytes_overlap(beta, cb, dbeta, dbeta ? cb : 0))
        return PVCONV_EINVAL;
    const pvconv_status st =
        check_ws(workspace, workspace_bytes, pv_group_norm_bwd_ws_bytes(B, N, C, groups));
    if (st != PVCONV_OK) return st;
    return pv_launch_group_norm_bwd(
        PvNorm{B, N, C, groups, lengths, gamma, beta, 0.f, act, slope},
        PvRows{(void*)dy, dy_dt == PVCONV_BF16, dy_ld},
        PvRows{(void*)x, x_dt == PVCONV_BF16, x_ld}, PvRows{dx, dx_dt == PVCONV_BF16, dx_ld},
        stats, dgamma, dbeta, workspace, as_stream(stream));
}

pvconv_status pvconv_fp8_quantize_weight(const void* w, pvconv_dtype w_dt, int w_ld, int N,
                                         int K, uint8_t* weight, uint8_t* scale,
                                         uint8_t* weight_t, uint8_t* scale_t, void* stream) {
    if (!fp8_sizes_ok(0, K, N) || !dtype_ok(w_dt)) return PVCONV_EINVAL;
    if (w_ld == 0) w_ld = K;
    if (w_ld < K || !w || !weight || !scale || (!weight_t) != (!scale_t)) return PVCONV_EINVAL;
    if (misaligned(w, esize(w_dt)) || misaligned(weight, 16) || misaligned(weight_t, 16))
        return PVCONV_EINVAL;
    const size_t wb = row_bytes(N, K, w_ld, w_dt), qb = fp8_bytes(N, K),
                 sb = (size_t)pv_fp8_blocks(N) * pv_fp8_blocks(K),
                 tb = weight_t ? fp8_bytes(K, N) : 0, ub = weight_t ? sb : 0;
    if (bytes_overlap(w, wb, weight, qb) || bytes_overlap(w, wb, scale, sb) ||
        bytes_overlap(w, wb, weight_t, tb) || bytes_overlap(w, wb, scale_t, ub) ||
        bytes_overlap(weight, qb, scale, sb) || bytes_overlap(weight, qb, weight_t, tb) ||
        bytes_overlap(weight, qb, scale_t, ub) || bytes_overlap(scale, sb, weight_t, tb) ||
        bytes_overlap(scale, sb, scale_t, ub) || bytes_overlap(weight_t, tb, scale_t, ub))
        return PVCONV_EINVAL;
    return pv_launch_fp8_quantize_weight(PvRows{(void*)w, w_dt == PVCONV_BF16, w_ld}, N, K,
                                         weight, scale, weight_t, scale_t, as_stream(stream));
}

size_t pvconv_fp8_linear_workspace_size(int M, int K, int N) {
    return fp8_sizes_ok(M, K, N) ? pv_fp8_linear_ws_bytes(M, K, N) : 0;
}

pvconv_status pvconv_fp8_linear(const void* x, pvconv_dtype x_dt, int x_ld, int M, int K, int N,
                                const uint8_t* weight, const uint8_t* scale, const float* bias,
                                pvconv_act act, float slope, void* y, pvconv_dtype y_dt,
                                int y_ld, void* workspace, size_t workspace_bytes,
                                void* stream) {
    if (!fp8_sizes_ok(M, K, N) || !dtype_ok(x_dt) || !dtype_ok(y_dt) || !act_ok(act))
        return PVCONV_EINVAL;
    if (x_ld == 0) x_ld = K;
    if (y_ld == 0) y_ld = N;
    if (x_ld < K || y_ld < N) return PVCONV_EINVAL;
    if (M == 0) return PVCONV_OK;
    if (!x || !weight || !scale || !y) return PVCONV_EINVAL;
    if (misaligned(x, esize(x_dt)) || misaligned(weight, 16) || misaligned(bias, 4) ||
        misaligned(y, esize(y_dt)))
        return PVCONV_EINVAL;
    const size_t yb = row_bytes(M, N, y_ld, y_dt);
    if (overlap(x, M, K, x_ld, x_dt, y, N, y_ld, y_dt) ||
        bytes_overlap(y, yb, weight, fp8_bytes(N, K)) ||
        bytes_overlap(y, yb, scale, (size_t)pv_fp8_blocks(N) * pv_fp8_blocks(K)) ||
        bytes_overlap(y, yb, bias, bias ? (size_t)N * 4 : 0))
        return PVCONV_EINVAL;
    const pvconv_status st = check_ws(workspace, workspace_bytes, pv_fp8_linear_ws_bytes(M, K, N));
    if (st != PVCONV_OK) return st;
    return pv_launch_fp8_linear(PvRows{(void*)x, x_dt == PVCONV_BF16, x_ld}, M, K, N, weight,
                                scale, bias, act, slope, PvRows{y, y_dt == PVCONV_BF16, y_ld},
                                workspace, as_stream(stream));
}

size_t pvconv_fp8_linear_backward_workspace_size(int M, int K, int N) {
    return fp8_sizes_ok(M, K, N) ? pv_fp8_linear_bwd_ws_bytes(M, K, N) : 0;
}

pvconv_status pvconv_fp8_linear_backward(const void* dy, pvconv_dtype dy_dt, int dy_ld,
                                         const void* x, pvconv_dtype x_dt, int x_ld, int M,
                                         int K, int N, const uint8_t* weight_t,
                                         const uint8_t* scale_t, void* dx, pvconv_dtype dx_dt,
                                         int dx_ld, float* dw, float* dbias, void* workspace,
                                         size_t workspace_bytes, void* stream) {
    if (!fp8_sizes_ok(M, K, N) || !dtype_ok(dy_dt) || !dtype_ok(x_dt) || !dtype_ok(dx_dt))
        return PVCONV_EINVAL;
    if (dy_ld == 0) dy_ld = N;
    if (x_ld == 0) x_ld = K;
    if (dx_ld == 0) dx_ld = K;
    if (dy_ld < N || x_ld < K || dx_ld < K) return PVCONV_EINVAL;
    if (!dx && !dw && !dbias) return PVCONV_EINVAL;
    if (M == 0 && !dw && !dbias) return PVCONV_OK;
    if (M > 0 && (!dy || (dw && !x) || (dx && (!weight_t || !scale_t)))) return PVCONV_EINVAL;
    if (misaligned(dy, esize(dy_dt)) || misaligned(x, esize(x_dt)) ||
        misaligned(dx, esize(dx_dt)) || misaligned(weight_t, 16) || misaligned(dw, 4) ||
        misaligned(dbias, 4))
        return PVCONV_EINVAL;
    const size_t yb = row_bytes(M, N, dy_ld, dy_dt), xb = dw ? row_bytes(M, K, x_ld, x_dt) : 0,
                 wb = dw ? (size_t)N * K * 4 : 0, bb = dbias ? (size_t)N * 4 : 0,
                 qb = dx ? fp8_bytes(K, N) : 0,
                 sb = dx ? (size_t)pv_fp8_blocks(N) * pv_fp8_blocks(K) : 0,
                 db = dx ? row_bytes(M, K, dx_ld, dx_dt) : 0;
    if ((dx && (overlap(dy, M, N, dy_ld, dy_dt, dx, K, dx_ld, dx_dt) ||
                (dw && overlap(x, M, K, x_ld, x_dt, dx, K, dx_ld, dx_dt)))) ||
        bytes_overlap(dx, db, weight_t, qb) || bytes_overlap(dx, db, scale_t, sb) ||
        bytes_overlap(dx, db, dw, wb) || bytes_overlap(dx, db, dbias, bb) ||
        bytes_overlap(dw, wb, dy, yb) || bytes_overlap(dw, wb, x, xb) ||
        bytes_overlap(dw, wb, weight_t, qb) || bytes_overlap(dw, wb, scale_t, sb) ||
        bytes_overlap(dw, wb, dbias, bb) || bytes_overlap(dbias, bb, dy, yb) ||
        bytes_overlap(dbias, bb, x, xb) || bytes_overlap(dbias, bb, weight_t, qb) ||
        bytes_overlap(dbias, bb, scale_t, sb))
        return PVCONV_EINVAL;
    const pvconv_status st =
        check_ws(workspace, workspace_bytes, pv_fp8_linear_bwd_ws_bytes(M, K, N));
    if (st != PVCONV_OK) return st;
    return pv_launch_fp8_linear_bwd(
        PvRows{(void*)dy, dy_dt == PVCONV_BF16, dy_ld},
        PvRows{(void*)x, x_dt == PVCONV_BF16, x_ld}, M, K, N, weight_t, scale_t,
        PvRows{dx, dx_dt == PVCONV_BF16, dx_ld}, dw, dbias, workspace, as_stream(stream));
}

pvconv_status pvconv_int8_quantize(const void* x, pvconv_dtype x_dt, int x_ld, int R, int K,
                                   int8_t* q, float* scale, void* stream) {
    if (!int8_sizes_ok(0, K, 1) || R < 0 || R > (1 << 30) || !dtype_ok(x_dt)) return PVCONV_EINVAL;
    if (x_ld == 0) x_ld = K;
    if (x_ld < K) return PVCONV_EINVAL;
    if (R == 0) return PVCONV_OK;
    if (!x || !q || !scale || misaligned(x, esize(x_dt)) || misaligned(q, 16) ||
        misaligned(scale, 4))
        return PVCONV_EINVAL;
    Ranges r;
    r.add(x, row_bytes(R, K, x_ld, x_dt));
    if (!r.output(q, int8_bytes(R, K)) || !r.output(scale, (size_t)R * 4)) return PVCONV_EINVAL;
    return pv_launch_int8_quantize(PvRows{(void*)x, x_dt == PVCONV_BF16, x_ld}, R, K, q, scale,
                                   as_stream(stream));
}

size_t pvconv_int8_linear_workspace_size(int M, int K, int N) {
    return int8_sizes_ok(M, K, N) ? pv_int8_linear_ws_bytes(M, K, N, false) : 0;
}
size_t pvconv_int8_linear_rows_workspace_size(int M, int K, int N) {
    return int8_sizes_ok(M, K, N) ? pv_int8_linear_ws_bytes(M, K, N, true) : 0;
}

pvconv_status pvconv_int8_linear(const void* x, pvconv_dtype x_dt, int x_ld, int M, int K, int N,
                                 const int8_t* weight, const float* scale, const float* bias,
                                 pvconv_act act, float slope, void* y, pvconv_dtype y_dt,
                                 int y_ld, int8_t* rows, float* row_scale, void* workspace,
                                 size_t workspace_bytes, void* stream) {
    if (!int8_sizes_ok(M, K, N) || !dtype_ok(x_dt) || !dtype_ok(y_dt) || !act_ok(act))
        return PVCONV_EINVAL;
    if (x_ld == 0) x_ld = K;
    if (y_ld == 0) y_ld = N;
    if (x_ld < K || y_ld < N || (!rows) != (!row_scale)) return PVCONV_EINVAL;
    if (M == 0) return PVCONV_OK;
    if (!x || !weight || !scale || !y) return PVCONV_EINVAL;
    if (misaligned(x, esize(x_dt)) || misaligned(weight, 16) || misaligned(scale, 4) ||
        misaligned(bias, 4) || misaligned(y, esize(y_dt)) || misaligned(rows, 16) ||
        misaligned(row_scale, 4))
        return PVCONV_EINVAL;
    Ranges r;
    r.add(weight, int8_bytes(N, K));
    r.add(scale, (size_t)N * 4);
    r.add(bias, (size_t)N * 4);
    if (overlap(x, M, K, x_ld, x_dt, y, N, y_ld, y_dt) ||
        !r.output(y, row_bytes(M, N, y_ld, y_dt)))
        return PVCONV_EINVAL;
    r.add(x, row_bytes(M, K, x_ld, x_dt));
    if (!r.output(rows, int8_bytes(M, K)) || !r.output(row_scale, (size_t)M * 4))
        return PVCONV_EINVAL;
    const pvconv_status st = check_ws(workspace, workspace_bytes,
                                      pv_int8_linear_ws_bytes(M, K, N, rows != nullptr));
    if (st != PVCONV_OK) return st;
    return pv_launch_int8_linear(PvRows{(void*)x, x_dt == PVCONV_BF16, x_ld}, M, K, N, weight,
                                 scale, bias, act, slope, PvRows{y, y_dt == PVCONV_BF16, y_ld},
                                 rows, row_scale, workspace, as_stream(stream));
}

pvconv_status pvconv_int8_linear_rows(const int8_t* rows, const float* row_scale, int M, int K,
                                      int N, const int8_t* weight, const float* scale,
                                      const float* bias, pvconv_act act, float slope, void* y,
                                      pvconv_dtype y_dt, int y_ld, void* workspace,
                                      size_t workspace_bytes, void* stream) {
    if (!int8_sizes_ok(M, K, N) || !dtype_ok(y_dt) || !act_ok(act)) return PVCONV_EINVAL;
    if (y_ld == 0) y_ld = N;
    if (y_ld < N) return PVCONV_EINVAL;
    if (M == 0) return PVCONV_OK;
    if (!rows || !row_scale || !weight || !scale || !y) return PVCONV_EINVAL;
    if (misaligned(rows, 16) || misaligned(row_scale, 4) || misaligned(weight, 16) ||
        misaligned(scale, 4) || misaligned(bias, 4) || misaligned(y, esize(y_dt)))
        return PVCONV_EINVAL;
    Ranges r;
    r.add(rows, int8_bytes(M, K));
    r.add(row_scale, (size_t)M * 4);
    r.add(weight, int8_bytes(N, K));
    r.add(scale, (size_t)N * 4);
    r.add(bias, (size_t)N * 4);
    if (!r.output(y, row_bytes(M, N, y_ld, y_dt))) return PVCONV_EINVAL;
    const pvconv_status st =
        check_ws(workspace, workspace_bytes, pv_int8_linear_ws_bytes(M, K, N, true));
    if (st != PVCONV_OK) return st;
    return pv_launch_int8_linear_rows(rows, row_scale, M, K, N, weight, scale, bias, act, slope,
                                      PvRows{y, y_dt == PVCONV_BF16, y_ld}, workspace,
                                      as_stream(stream));
}

size_t pvconv_int8_linear_backward_workspace_size(int M, int K, int N) {
    return int8_sizes_ok(M, K, N) ? pv_int8_linear_bwd_ws_bytes(M, K, N) : 0;
}

pvconv_status pvconv_int8_linear_backward(const void* dy, pvconv_dtype dy_dt, int dy_ld,
                                          const int8_t* rows, const float* row_scale, int M,
                                          int K, int N, const int8_t* weight,
                                          const float* scale, void* dx, pvconv_dtype dx_dt,
                                          int dx_ld, float* dw, float* dbias, void* workspace,
                                          size_t workspace_bytes, void* stream) {
    if (!int8_sizes_ok(M, K, N) || !dtype_ok(dy_dt) || !dtype_ok(dx_dt)) return PVCONV_EINVAL;
    if (dy_ld == 0) dy_ld = N;
    if (dx_ld == 0) dx_ld = K;
    if (dy_ld < N || dx_ld < K || (!dx && !dw && !dbias)) return PVCONV_EINVAL;
    if (M == 0 && !dw && !dbias) return PVCONV_OK;
    if (M > 0 && (!dy || (dw && (!rows || !row_scale)) || (dx && (!weight || !scale))))
        return PVCONV_EINVAL;
    if (misaligned(dy, esize(dy_dt)) || misaligned(rows, 16) || misaligned(row_scale, 4) ||
        misaligned(weight, 16) || misaligned(scale, 4) || misaligned(dx, esize(dx_dt)) ||
        misaligned(dw, 4) || misaligned(dbias, 4))
        return PVCONV_EINVAL;
    Ranges r;
    if (dw) {
        r.add(rows, int8_bytes(M, K));
        r.add(row_scale, (size_t)M * 4);
    }
    if (dx) {
        r.add(weight, int8_bytes(N, K));
        r.add(scale, (size_t)N * 4);
    }
    if ((dx && overlap(dy, M, N, dy_ld, dy_dt, dx, K, dx_ld, dx_dt)) ||
        !r.output(dx, row_bytes(M, K, dx_ld, dx_dt)))
        return PVCONV_EINVAL;
    r.add(dy, row_bytes(M, N, dy_ld, dy_dt));
    if (!r.output(dw, (size_t)N * K * 4) || !r.output(dbias, (size_t)N * 4)) return PVCONV_EINVAL;
    const pvconv_status st =
        check_ws(workspace, workspace_bytes, pv_int8_linear_bwd_ws_bytes(M, K, N));
    if (st != PVCONV_OK) return st;
    return pv_launch_int8_linear_bwd(PvRows{(void*)dy, dy_dt == PVCONV_BF16, dy_ld}, rows,
                                     row_scale, M, K, N, weight, scale,
                                     PvRows{dx, dx_dt == PVCONV_BF16, dx_ld}, dw, dbias,
                                     workspace, as_stream(stream));
}

size_t pvconv_distill_topk_workspace_size(int, int) { return 0; }

pvconv_status pvconv_distill_topk(const void* z, pvconv_dtype z_dt, int z_ld, int M, int V,
                                  const float* t_val, const int32_t* t_class, int top,
                                  const int32_t* labels, float temperature, float alpha,
                                  const float* row_weight, float* loss, float* lse, void* dz,
                                  pvconv_dtype dz_dt, int dz_ld, void*, size_t, void* stream) {
    pvconv_status st =
        check_distill(z, z_dt, z_ld, M, V, t_val, t_class, top, labels, temperature, alpha);
    if (st != PVCONV_OK) return st;
    if (dz) {
        st = check_dz(z, z_dt, z_ld, dz, dz_dt, dz_ld, M, V, t_val, t_class, top);
        if (st != PVCONV_OK) return st;
    }
    if (M == 0) return PVCONV_OK;
    if (!loss || misaligned(loss, 4) || misaligned(lse, 4) || misaligned(row_weight, 4))
        return PVCONV_EINVAL;
    const size_t zb = row_bytes(M, V, z_ld, z_dt), db = dz ? row_bytes(M, V, dz_ld, dz_dt) : 0,
                 lb = (size_t)M * 4, eb = lse ? (size_t)M * 8 : 0, tb = (size_t)M * top * 4;
    if (bytes_overlap(loss, lb, z, zb) || bytes_overlap(lse, eb, z, zb) ||
        bytes_overlap(loss, lb, lse, eb) || bytes_overlap(loss, lb, dz, db) ||
        bytes_overlap(lse, eb, dz, db) || bytes_overlap(loss, lb, t_val, tb) ||
        bytes_overlap(loss, lb, t_class, tb) || bytes_overlap(lse, eb, t_val, tb) ||
        bytes_overlap(lse, eb, t_class, tb) || bytes_overlap(loss, lb, labels, labels ? lb : 0) ||
        bytes_overlap(lse, eb, labels, labels ? lb : 0) ||
        bytes_overlap(dz, db, labels, labels ? lb : 0) ||
        bytes_overlap(loss, lb, row_weight, row_weight ? lb : 0) ||
        bytes_overlap(lse, eb, row_weight, row_weight ? lb : 0) ||
        bytes_overlap(dz, db, row_weight, row_weight ? lb : 0))
        return PVCONV_EINVAL;
    return pv_launch_distill(PvDistill{PvRows{(void*)z, z_dt == PVCONV_BF16, z_ld}, M, V, t_val,
                                       t_class, top, labels, temperature, alpha},
                             row_weight, loss, lse, PvRows{dz, dz_dt == PVCONV_BF16, dz_ld},
                             as_stream(stream));
}

pvconv_status pvconv_distill_topk_backward(const void* z, pvconv_dtype z_dt, int z_ld, int M,
                                           int V, const float* t_val, const int32_t* t_class,
                                           int top, const int32_t* labels, float temperature,
                                           float alpha, const float* lse, const float* dloss,
                                           void* dz, pvconv_dtype dz_dt, int dz_ld,
                                           void* stream) {
    pvconv_status st =
        check_distill(z, z_dt, z_ld, M, V, t_val, t_class, top, labels, temperature, alpha);
    if (st != PVCONV_OK) return st;
    st = check_dz(z, z_dt, z_ld, dz, dz_dt, dz_ld, M, V, t_val, t_class, top);
    if (st != PVCONV_OK) return st;
    if (M == 0) return PVCONV_OK;
    if (!lse || misaligned(lse, 4) || misaligned(dloss, 4)) return PVCONV_EINVAL;
    const size_t db = row_bytes(M, V, dz_ld, dz_dt), lb = (size_t)M * 4;
    if (bytes_overlap(dz, db, lse, 2 * lb) || bytes_overlap(dz, db, dloss, dloss ? lb : 0) ||
        bytes_overlap(dz, db, labels, labels ? lb : 0))
        return PVCONV_EINVAL;
    return pv_launch_distill_bwd(PvDistill{PvRows{(void*)z, z_dt == PVCONV_BF16, z_ld}, M, V,
                                           t_val, t_class, top, labels, temperature, alpha},
                                 lse, dloss, PvRows{dz, dz_dt == PVCONV_BF16, dz_ld},
                                 as_stream(stream));
}

size_t pvconv_linear_cross_entropy_workspace_size(int M, int K, int V, pvconv_dtype x_dt,
                                                  pvconv_dtype w_dt, pvconv_dtype dx_dt,
                                                  pvconv_dtype dw_dt, int want_grad) {
    if (!ce_sizes_ok(M, K, V) || !dtype_ok(x_dt) || !dtype_ok(w_dt) || !dtype_ok(dx_dt) ||
        !dtype_ok(dw_dt))
        return 0;
    PvLinearCe a{};
    float some;  // a gradient that is wanted: any address
    a.M = M;
    a.K = K;
    a.V = V;
    a.x.bf16 = x_dt == PVCONV_BF16;
    a.w.bf16 = w_dt == PVCONV_BF16;
    a.dx = PvRows{want_grad ? &some : nullptr, dx_dt == PVCONV_BF16, K};
    a.dw = PvRows{want_grad ? &some : nullptr, dw_dt == PVCONV_BF16, K};
    a.dbias = want_grad ? &some : nullptr;
    return pv_linear_ce_ws_bytes(a, true, want_grad != 0);
}

pvconv_status pvconv_linear_cross_entropy(
    const void* x, pvconv_dtype x_dt, int x_ld, const void* w, pvconv_dtype w_dt, int w_ld, int M,
    int K, int V, const float* bias, const int32_t* labels, const float* row_weight, float* loss,
    float* lse, void* dx, pvconv_dtype dx_dt, int dx_ld, void* dw, pvconv_dtype dw_dt,
    float* dbias, void* workspace, size_t workspace_bytes, void* stream) {
    PvLinearCe a{PvRows{(void*)x, false, x_ld}, PvRows{(void*)w, false, w_ld}, M, K, V, bias,
                 labels, row_weight, loss, lse, PvRows{dx, false, dx_ld}, PvRows{dw, false, 0},
                 dbias};
    Ranges r;
    pvconv_status st = check_ce(a, x_dt, w_dt, dx_dt, dw_dt, r);
    if (st != PVCONV_OK) return st;
    if (M == 0 && !dw && !dbias) return PVCONV_OK;
    if (M > 0 && !loss) return PVCONV_EINVAL;
    if (!r.output(loss, (size_t)M * 4) || !r.output(lse, (size_t)M * 4)) return PVCONV_EINVAL;
    st = check_ws(workspace, workspace_bytes,
                  pv_linear_ce_ws_bytes(a, true, dx || dw || dbias));
    if (st != PVCONV_OK) return st;
    return pv_launch_linear_ce(a, true, workspace, as_stream(stream));
}

pvconv_status pvconv_linear_cross_entropy_backward(
    const void* x, pvconv_dtype x_dt, int x_ld, const void* w, pvconv_dtype w_dt, int w_ld, int M,
    int K, int V, const float* bias, const int32_t* labels, const float* lse, const float* dloss,
    void* dx, pvconv_dtype dx_dt, int dx_ld, void* dw, pvconv_dtype dw_dt, float* dbias,
    void* workspace, size_t workspace_bytes, void* stream) {
    PvLinearCe a{PvRows{(void*)x, false, x_ld}, PvRows{(void*)w, false, w_ld}, M, K, V, bias,
                 labels, dloss, nullptr, (float*)lse, PvRows{dx, false, dx_ld},
                 PvRows{dw, false, 0}, dbias};
    Ranges r;
    if (M > 0 && lse) r.add(lse, (size_t)M * 4);
    pvconv_status st = check_ce(a, x_dt, w_dt, dx_dt, dw_dt, r);
    if (st != PVCONV_OK) return st;
    if (!dx && !dw && !dbias) return PVCONV_EINVAL;
    if (M == 0 && !dw && !dbias) return PVCONV_OK;
    if (M > 0 && !lse) return PVCONV_EINVAL;
    st = check_ws(workspace, workspace_bytes, pv_linear_ce_ws_bytes(a, false, true));
    if (st != PVCONV_OK) return st;
    return pv_launch_linear_ce(a, false, workspace, as_stream(stream));
}

}  // extern "C"
