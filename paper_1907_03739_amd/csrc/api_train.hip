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

}  // extern "C"
