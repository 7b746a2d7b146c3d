// Distillation loss against a teacher's top logits, and its gradient
// (pvconv_train.h).
//
// A team of threads owns a row: it takes the row's maximum and its sums of
// exponentials at temperatures 1 and T in one pass, the teacher's term over the
// stored entries, and writes the gradient in a second pass. Bound by HBM: z
// read (twice where a gradient is written), dz written.
#include "pv_train.h"

namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ bool bad_class(int c, int V) { return (unsigned)c >= (unsigned)V; }

// Reductions over a team: TEAM consecutive threads, a power of two up to a
// wave, or the whole workgroup (through LDS, in wave order).
template <int TEAM, typename Op>
__device__ __forceinline__ float team_reduce(float v, Op op, float* lds) {
#pragma unroll
    for (int m = 1; m < (TEAM < 64 ? TEAM : 64); m <<= 1) v = op(v, __shfl_xor(v, m));
    if constexpr (TEAM > 64) {
        __syncthreads();
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
        __syncthreads();
        v = lds[0];
#pragma unroll
        for (int w = 1; w < TEAM / 64; w++) v = op(v, lds[w]);
    }
    return v;
}
struct Max {
    __device__ float operator()(float a, float b) const { return fmaxf(a, b); }
};
struct Add {
    __device__ float operator()(float a, float b) const { return a + b; }
};

// The teacher's side of a row: maximum and sum of its present entries at
// temperature T (has: some entry has weight).
struct Teacher {
    float max, inv;
    bool has;
};
template <int TEAM>
__device__ __forceinline__ Teacher teacher_of(const PvDistill& d, size_t row, int lane, float tau,
                                              float* lds) {
    float m = -INFINITY, s = 0.f;
    for (int j = lane; j < d.top; j += TEAM)
        if (!bad_class(d.t_class[row * d.top + j], d.V))
            m = fmaxf(m, d.t_val[row * d.top + j] * tau);
    m = team_reduce<TEAM>(m, Max(), lds);
    const float base = m == -INFINITY ? 0.f : m;
    for (int j = lane; j < d.top; j += TEAM)
        if (!bad_class(d.t_class[row * d.top + j], d.V))
            s += __expf(d.t_val[row * d.top + j] * tau - base);
    s = team_reduce<TEAM>(s, Add(), lds);
    // s is 0 only where every present value is -inf; a NaN keeps its row NaN
    return Teacher{base, s == 0.f ? 0.f : 1.f / s, !(s == 0.f)};
}

struct Weights {  // of the two terms for a row
    float kl, ce;
    int label;
};

// The gradient of one logit before the entries of its class: w_kl T q + w_ce q1.
__device__ __forceinline__ float soft_grad(float z, float tau, const Weights& w, float lse1,
                                           float lset) {
    float g = 0.f;
    if (w.kl != 0.f) g = w.kl * __expf(fmaf(z, tau, -lset));
    if (w.ce != 0.f) g = fmaf(w.ce, __expf(z - lse1), g);
    return g;
}

// dz of a row from its statistics. The entries' and the label's classes get
// their whole value from the thread that owns the entry, after the others.
template <int TEAM>
__device__ __forceinline__ void row_gradient(const PvDistill& d, size_t row, int lane, float tau,
                                             const Teacher& t, const Weights& w, float lse1,
                                             float lset, float scale, bool empty,
                                             const PvRows& dz) {
    const size_t in = row * d.z.ld, out = row * dz.ld;
    const bool zero = scale == 0.f || empty;
    for (int c = lane; c < d.V; c += TEAM)
        pv_store_one(dz.p, dz.bf16, out + c,
                     zero ? 0.f
                          : scale * soft_grad(pv_load_one(d.z.p, d.z.bf16, in + c), tau, w, lse1,
                                              lset));
    if (zero) return;
    if constexpr (TEAM > 64) __syncthreads();
    const int entries = w.kl != 0.f ? d.top : 0;
    for (int j = lane; j <= entries; j += TEAM) {
        const int c = j < entries ? d.t_class[row * d.top + j] : (w.ce != 0.f ? w.label : -1);
        if (bad_class(c, d.V)) continue;
        float p = 0.f;
        for (int i = 0; i < entries; i++)
            if (d.t_class[row * d.top + i] == c)
                p += __expf(d.t_val[row * d.top + i] * tau - t.max);
        float g = soft_grad(pv_load_one(d.z.p, d.z.bf16, in + c), tau, w, lse1, lset) -
                  w.kl * p * t.inv;
        if (w.ce != 0.f && c == w.label) g -= w.ce;
        pv_store_one(dz.p, dz.bf16, out + c, scale * g);
    }
}

__device__ __forceinline__ Weights weights_of(const PvDistill& d, size_t row, bool has) {
    Weights w;
    w.label = d.labels ? d.labels[row] : -1;
    w.kl = has ? d.alpha * d.temperature : 0.f;
    w.ce = bad_class(w.label, d.V) ? 0.f : 1.f - d.alpha;
    return w;
}

template <int TEAM>
__global__ __launch_bounds__(kThreads) void pv_distill_kernel(PvDistill d, const float* weight,
                                                              float* loss, float* lse,
                                                              PvRows dz) {
    __shared__ float lds[kThreads / 64];
    const int lane = threadIdx.x % TEAM;
    const float tau = 1.f / d.temperature;
    const bool soft = d.alpha > 0.f, hard = d.labels && d.alpha < 1.f;
    for (size_t row = (size_t)blockIdx.x * (kThreads / TEAM) + threadIdx.x / TEAM; row < (size_t)d.M;
         row += (size_t)gridDim.x * (kThreads / TEAM)) {
        const size_t in = row * d.z.ld;
        float m = -INFINITY, s1 = 0.f, st = 0.f;
        for (int c = lane; c < d.V; c += TEAM) {
            const float z = pv_load_one(d.z.p, d.z.bf16, in + c);
            if (z > m) {
                const float e = m - z;
                s1 *= __expf(e);
                st *= __expf(e * tau);
                m = z;
            }
            const float e = z == -INFINITY ? -INFINITY : z - m;
            s1 += __expf(e);
            st += __expf(e * tau);
        }
        const float top = team_reduce<TEAM>(m, Max(), lds);
        const float e = m == -INFINITY ? -INFINITY : m - top;
        // a NaN in s1, st survives the rescaling
        s1 = team_reduce<TEAM>(s1 * __expf(e), Add(), lds);
        st = team_reduce<TEAM>(st * __expf(e * tau), Add(), lds);
        const bool empty = s1 == 0.f;
        const float lse1 = top + __logf(s1), lset = top * tau + __logf(st);
        const Teacher t = soft ? teacher_of<TEAM>(d, row, lane, tau, lds) : Teacher{0.f, 0.f, false};
        const Weights w = weights_of(d, row, t.has);
        float kl = 0.f;
        if (w.kl != 0.f && !empty)
            for (int j = lane; j < d.top; j += TEAM) {
                const int c = d.t_class[row * d.top + j];
                if (bad_class(c, d.V)) continue;
                const float u = d.t_val[row * d.top + j] * tau - t.max;
                const float p = __expf(u) * t.inv;
                const float z = pv_load_one(d.z.p, d.z.bf16, in + c);
                if (!(p == 0.f)) kl += p * (u + __logf(t.inv) - (z * tau - lset));
            }
        kl = team_reduce<TEAM>(kl, Add(), lds);
        if (lane == 0) {
            float l = 0.f;
            if (!empty) {
                l = w.kl * d.temperature * kl;
                if (w.ce != 0.f) l += w.ce * (lse1 - pv_load_one(d.z.p, d.z.bf16, in + w.label));
            }
            loss[row] = l;
            if (lse) {
                lse[2 * row] = hard ? lse1 : 0.f;
                lse[2 * row + 1] = soft ? lset : 0.f;
            }
        }
        if (dz.p)
            row_gradient<TEAM>(d, row, lane, tau, t, w, lse1, lset, weight ? weight[row] : 1.f,
                               empty, dz);
    }
}

template <int TEAM>
__global__ __launch_bounds__(kThreads) void pv_distill_bwd_kernel(PvDistill d, const float* lse,
                                                                  const float* dloss, PvRows dz) {
    __shared__ float lds[kThreads / 64];
    const int lane = threadIdx.x % TEAM;
    const float tau = 1.f / d.temperature;
    const bool soft = d.alpha > 0.f;
    for (size_t row = (size_t)blockIdx.x * (kThreads / TEAM) + threadIdx.x / TEAM; row < (size_t)d.M;
         row += (size_t)gridDim.x * (kThreads / TEAM)) {
        const float lse1 = lse[2 * row], lset = lse[2 * row + 1];
        const Teacher t = soft ? teacher_of<TEAM>(d, row, lane, tau, lds) : Teacher{0.f, 0.f, false};
        const Weights w = weights_of(d, row, t.has);
        // the statistics of a row of -inf are -inf
        const bool empty = lse1 == -INFINITY || lset == -INFINITY;
        row_gradient<TEAM>(d, row, lane, tau, t, w, lse1, lset, dloss ? dloss[row] : 1.f, empty,
                           dz);
    }
}

constexpr int kTeamV = 1024;  // classes from which a workgroup owns a row

unsigned grid_of(size_t blocks) { return (unsigned)(blocks < 65536 ? blocks : 65536); }

}  // namespace

size_t pv_distill_ws_bytes(int M, int V) {
    (void)M;
    (void)V;
    return 0;
}

pvconv_status pv_launch_distill(const PvDistill& d, const float* row_weight, float* loss,
                                float* lse, const PvRows& dz, void* ws, hipStream_t s) {
    (void)ws;
    if (d.V >= kTeamV)
        pv_distill_kernel<kThreads><<<grid_of(d.M), kThreads, 0, s>>>(d, row_weight, loss, lse, dz);
    else
        pv_distill_kernel<16><<<grid_of((d.M + 15) / 16), kThreads, 0, s>>>(d, row_weight, loss,
                                                                            lse, dz);
    return pv_launch_status();
}

pvconv_status pv_launch_distill_bwd(const PvDistill& d, const float* lse, const float* dloss,
                                    const PvRows& dz, hipStream_t s) {
    if (d.V >= kTeamV)
        pv_distill_bwd_kernel<kThreads><<<grid_of(d.M), kThreads, 0, s>>>(d, lse, dloss, dz);
    else
        pv_distill_bwd_kernel<16><<<grid_of((d.M + 15) / 16), kThreads, 0, s>>>(d, lse, dloss, dz);
    return pv_launch_status();
}
