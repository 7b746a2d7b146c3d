// Group normalisation with an activation, channels last, and its gradients
// (pvconv_train.h).
//
// A group of a cloud that fits the registers of a workgroup is read once, by one
// launch a direction (pv_gn_held_*: up to 8192 vectors), where hold_of finds that
// faster. The others take two launches: the first sums a share ("chunk") of a
// cloud's rows over a slab of whole groups; the second adds the chunks' sums of its
// groups in a fixed order and applies them to a chunk of rows. Bound by HBM: there
// x (and dy) are read twice, y (dx) is written once. 16 x 32768 x 128, 8 groups,
// bf16: sums 27 us (4.9 TB/s) and apply 47 (5.7), backward 58 (4.6) and 72 (5.6).
#include <type_traits>

#include "pv_train.h"

namespace {

constexpr int kThreads = 256;
constexpr int kRowsAhead = 4;  // rows a thread loads before it uses the first

// How the work is dealt: items (cloud, slab of channels, chunk of rows).
struct Deal {
    int CG;      // channels a group
    int slab;    // channels a slab: whole groups
    int slabs;
    int chunk;   // rows a chunk
    int chunks;
    size_t items;
};

// A slab is at most about 128 channels (or one group): 256 bytes of a bf16 row; of
// groups that are no whole vectors, as many as make whole ones, up to kMixedSlab.
// Chunks are for about kItems items, of kMinElements at least: an item adds the
// sums of its cloud's chunks (kSums pairs at most, 128 KB from the L2), which has
// to stay short beside its own rows.
constexpr int kSlab = 128, kMixedSlab = 256, kItems = 1024, kSums = 8192, kMinElements = 8192;

Deal deal(int B, int N, int C, int groups) {
    Deal d;
    d.CG = C / groups;
    int k = kSlab / d.CG;
    k = k < 1 ? 1 : (k > groups ? groups : k);
    const int odd = d.CG % 8 == 0 ? 1 : (d.CG % 4 == 0 ? 2 : (d.CG % 2 == 0 ? 4 : 8));
    if (odd > 1 && (size_t)odd * d.CG <= kMixedSlab) {
        k = k < odd ? odd : k / odd * odd;
        k = k > groups ? groups : k;
    }
    d.slab = k * d.CG;
    d.slabs = (groups + k - 1) / k;
    const size_t per = (size_t)(B > 0 ? B : 1) * d.slabs;
    size_t chunks = (kItems + per - 1) / per;
    if (chunks > (size_t)kSums / k) chunks = kSums / k < 1 ? 1 : kSums / k;
    const int rows = (kMinElements + d.slab - 1) / d.slab;
    const size_t most = ((size_t)N + rows - 1) / rows;
    if (chunks > most) chunks = most;
    if (chunks < 1) chunks = 1;
    d.chunk = (int)(((size_t)N + chunks - 1) / chunks);
    if (d.chunk < 1) d.chunk = 1;
    d.chunks = (int)(((size_t)N + d.chunk - 1) / d.chunk);
    if (d.chunks < 1) d.chunks = 1;
    d.items = (size_t)B * d.slabs * d.chunks;
    return d;
}

// One item and this thread's place in it: `cols` threads along the slab's
// vectors, `par` rows in parallel.
template <int VEC>
struct Place {
    int b, s, chunk, rows0, rows1, c0, width, cols, par, col, row, n;
    // (arrays that fit the card have fewer than 2^32 items: 32-bit divisions)
    __device__ Place(size_t item, const Deal& d, int N, int C, const int32_t* lengths) {
        const uint32_t r = (uint32_t)item / (uint32_t)d.chunks;
        chunk = (int)((uint32_t)item - r * (uint32_t)d.chunks);
        b = (int)(r / (uint32_t)d.slabs);
        s = (int)(r - (uint32_t)b * (uint32_t)d.slabs);
        n = lengths ? min(max(lengths[b], 0), N) : N;
        c0 = s * d.slab;
        width = min(d.slab, C - c0);
        const int vecs = width / VEC;
        cols = min(vecs, kThreads);
        par = kThreads / cols;
        row = threadIdx.x / cols;
        col = threadIdx.x - row * cols;
        if (row >= par) row = 1 << 30;  // beyond every row
        rows0 = chunk * d.chunk;
        rows1 = min(rows0 + d.chunk, N);
    }
};

// The types of the arrays of a call: all bf16, all fp32, or looked up per load.
enum Types { kBf16, kF32, kMixed };
// A vector of a row as it lies in memory, so that several can be in flight
// before the first is turned into floats.
template <int TYPES, int VEC>
struct Raw {
    static constexpr int kWords = TYPES == kBf16 ? (VEC + 1) / 2 : VEC;
    static constexpr bool kStreams = TYPES != kMixed && kWords == 4;
    uint32_t w[kWords];
    // ONCE: past the caches' normal order (streams() has the rule)
    template <bool ONCE = false>
    __device__ __forceinline__ void load(const PvRows& x, size_t row, int c) {
        const size_t at = row * x.ld + c;
        if constexpr (ONCE && kStreams) {
            typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
            const u32x4 v = __builtin_nontemporal_load(
                (const u32x4*)((const char*)x.p + at * (TYPES == kBf16 ? 2 : 4)));
#pragma unroll
            for (int i = 0; i < 4; i++) w[i] = v[i];
        } else if constexpr (TYPES == kBf16) {
            const uint16_t* p = (const uint16_t*)x.p + at;
            if constexpr (VEC == 1)
                w[0] = *p;
            else
                __builtin_memcpy(w, __builtin_assume_aligned(p, VEC * 2), VEC * 2);
        } else {
            float v[VEC];
            if (TYPES == kMixed && x.bf16)
                pv_load_vec<true, VEC>(x.p, at, v);
            else
                pv_load_vec<false, VEC>(x.p, at, v);
            __builtin_memcpy(w, v, VEC * 4);
        }
    }
    __device__ __forceinline__ float get(int i) const {
        if constexpr (TYPES == kBf16)
            return __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
        else
            return __uint_as_float(w[i]);
    }
};
template <int TYPES, int VEC>
__device__ __forceinline__ void store_row(const PvRows& x, size_t row, int c,
                                          const float (&v)[VEC]) {
    const size_t at = row * x.ld + c;
    if (TYPES == kBf16 || (TYPES == kMixed && x.bf16))
        pv_store_vec<true, VEC>(x.p, at, v);
    else
        pv_store_vec<false, VEC>(x.p, at, v);
}

// The activation and its derivative: SiLU, or a slope for v < 0 (1: none).
template <bool SILU>
__device__ __forceinline__ float act_of(float v, float neg) {
    if (SILU) return v * __builtin_amdgcn_rcpf(1.f + __expf(-v));
    return v >= 0.f ? v : v * neg;
}
template <bool SILU>
__device__ __forceinline__ float dact_of(float v, float neg) {
    if (SILU) {
        const float s = __builtin_amdgcn_rcpf(1.f + __expf(-v));
        return s * fmaf(v, 1.f - s, 1.f);
    }
    return v > 0.f ? 1.f : neg;
}

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) v += __shfl_xor(v, m);
    return v;
}

template <int VEC>
__device__ __forceinline__ void load_params(const PvNorm& n, int c, float (&ga)[VEC],
                                            float (&be)[VEC]) {
#pragma unroll
    for (int i = 0; i < VEC; i++) {
        ga[i] = n.gamma[c + i];
        be[i] = n.beta[c + i];
    }
}

// The value that a group's sums are about: its first channel of the cloud's first
// row. Without it, E[x^2] - mean^2 would lose the square of mean / spread, which
// leaves no digit of the variance where a mean is 2^26 spreads away; about an element
// of the group both terms are of the spread's size (unless that element lies as far
// from the others). The difference of two 32-bit values keeps 53 bits.
template <int TYPES>
__device__ __forceinline__ double pivot_of(const PvRows& x, int b, const PvNorm& n, int c) {
    Raw<TYPES, 1> f;
    f.load(x, (size_t)b * n.N, c);
    return (double)f.get(0);
}

// part[item of (b, slab, chunk)][group in slab] = sums of x - pivot and of its
// square, in 64 bits.
template <int TYPES, int VEC, bool ONCE>
__global__ __launch_bounds__(kThreads) void pv_gn_sums_kernel(PvNorm n, Deal d, PvRows x,
                                                              double2* part, int per) {
    __shared__ double2 red[kThreads];
    for (size_t item = blockIdx.x; item < d.items; item += gridDim.x) {
        const Place<VEC> p(item, d, n.N, n.C, n.lengths);
        const int rows1 = min(p.rows1, p.n);
        const int vecs = p.width / VEC, gv = d.CG / VEC, ng = p.width / d.CG;
        for (int v0 = 0; v0 < vecs; v0 += p.cols) {
            double s = 0., ss = 0.;
            const int c = p.c0 + (v0 + p.col) * VEC;
            if (v0 + p.col < vecs && p.rows0 < rows1) {
                const double pivot = pivot_of<TYPES>(x, p.b, n, c / d.CG * d.CG);
                for (int k = p.rows0 + p.row; k < rows1; k += p.par * kRowsAhead) {
                    Raw<TYPES, VEC> f[kRowsAhead];
#pragma unroll
                    for (int u = 0; u < kRowsAhead; u++)
                        f[u].template load<ONCE>(
                            x, (size_t)p.b * n.N + min(k + u * p.par, rows1 - 1), c);
#pragma unroll
                    for (int u = 0; u < kRowsAhead; u++)
                        if (k + u * p.par < rows1)
#pragma unroll
                            for (int i = 0; i < VEC; i++) {
                                const double v = (double)f[u].get(i) - pivot;
                                s += v;
                                ss = fma(v, v, ss);
                            }
                }
            }
            __syncthreads();
            red[threadIdx.x] = make_double2(s, ss);
            __syncthreads();
            // the groups that this run of columns touches
            const int g0 = v0 / gv, g1 = min((v0 + p.cols + gv - 1) / gv, ng);
            for (int g = g0 + (threadIdx.x >> 6); g < g1; g += kThreads / 64) {
                const int a = max(g * gv - v0, 0),
                          z = min((g + 1) * gv - v0, min(p.cols, vecs - v0));
                double t = 0., tt = 0.;
                const int w = z - a, m = w * p.par;
                for (int i = threadIdx.x & 63; i < m; i += 64) {
                    const double2 e = red[(i / w) * p.cols + a + i % w];
                    t += e.x;
                    tt += e.y;
                }
                t = wave_sum(t);
                tt = wave_sum(tt);
                if ((threadIdx.x & 63) == 0) {
                    double2* o = part + item * per + g;
                    // a group wider than the workgroup comes in several runs
                    if (g * gv < v0) {
                        t += o->x;
                        tt += o->y;
                    }
                    *o = make_double2(t, tt);
                }
            }
        }
    }
}

// The same where groups are no whole vectors (MIX in the kernels below): sums a
// channel, then a group. The slab is one run of vectors.
template <int TYPES, int VEC, bool ONCE>
__global__ __launch_bounds__(kThreads) void pv_gn_mixed_sums_kernel(PvNorm n, Deal d, PvRows x,
                                                                    double2* part, int per) {
    __shared__ double2 red[kThreads * VEC];
    __shared__ double2 chan[kMixedSlab];
    for (size_t item = blockIdx.x; item < d.items; item += gridDim.x) {
        const Place<VEC> p(item, d, n.N, n.C, n.lengths);
        const int rows1 = min(p.rows1, p.n), c = p.c0 + p.col * VEC;
        double s[VEC], ss[VEC], pivot[VEC];
#pragma unroll
        for (int i = 0; i < VEC; i++) {
            s[i] = ss[i] = 0.;
            pivot[i] = n.N > 0 ? pivot_of<TYPES>(x, p.b, n, (c + i) / d.CG * d.CG) : 0.;
        }
        for (int k = p.rows0 + p.row; k < rows1; k += p.par * kRowsAhead) {
            Raw<TYPES, VEC> f[kRowsAhead];
#pragma unroll
            for (int u = 0; u < kRowsAhead; u++)
                f[u].template load<ONCE>(
                    x, (size_t)p.b * n.N + min(k + u * p.par, rows1 - 1), c);
#pragma unroll
            for (int u = 0; u < kRowsAhead; u++)
                if (k + u * p.par < rows1)
#pragma unroll
                    for (int i = 0; i < VEC; i++) {
                        const double v = (double)f[u].get(i) - pivot[i];
                        s[i] += v;
                        ss[i] = fma(v, v, ss[i]);
                    }
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < VEC; i++) red[threadIdx.x * VEC + i] = make_double2(s[i], ss[i]);
        __syncthreads();
        for (int i = threadIdx.x; i < p.width; i += kThreads) {
            double t = 0., tt = 0.;
            for (int r = 0; r < p.par; r++) {
                t += red[r * p.width + i].x;
                tt += red[r * p.width + i].y;
            }
            chan[i] = make_double2(t, tt);
        }
        __syncthreads();
        for (int g = threadIdx.x >> 6; g < p.width / d.CG; g += kThreads / 64) {
            double t = 0., tt = 0.;
            for (int i = threadIdx.x & 63; i < d.CG; i += 64) {
                t += chan[g * d.CG + i].x;
                tt += chan[g * d.CG + i].y;
            }
            t = wave_sum(t);
            tt = wave_sum(tt);
            if ((threadIdx.x & 63) == 0) part[item * per + g] = make_double2(t, tt);
        }
    }
}

// The pairs of the groups that channels c .. lie in.
template <bool MIX, int VEC>
__device__ __forceinline__ void of_groups(const float2* v, int c, int CG, float (&a)[VEC],
                                          float (&b)[VEC]) {
    const float2 first = v[c / CG];
#pragma unroll
    for (int i = 0; i < VEC; i++) {
        const float2 e = MIX ? v[(c + i) / CG] : first;
        a[i] = e.x;
        b[i] = e.y;
    }
}

// A group's two sums over its cloud's chunks, by a wave, in a fixed order.
__device__ __forceinline__ double2 add_chunks(const double2* part, int per, int chunks,
                                              size_t first, int g) {
    double t = 0., tt = 0.;
    for (int i = threadIdx.x & 63; i < chunks; i += 64) {
        const double2 e = part[(first + i) * per + g];
        t += e.x;
        tt += e.y;
    }
    return make_double2(wave_sum(t), wave_sum(tt));
}

__device__ __forceinline__ float2 stats_of(double sum, double squares, double pivot, double count,
                                           float eps) {
    const double off = sum / count, var = squares / count - off * off;
    return make_float2((float)(pivot + off),
                       (float)(1. / sqrt((var < 0. ? 0. : var) + (double)eps)));
}

template <int TYPES, bool SILU, int VEC, bool MIX, bool ONCE>
__global__ __launch_bounds__(kThreads) void pv_gn_apply_kernel(PvNorm n, Deal d, PvRows x,
                                                               PvRows y, float neg,
                                                               const double2* part, int per,
                                                               float2* stats) {
    extern __shared__ float2 st[];
    for (size_t item = blockIdx.x; item < d.items; item += gridDim.x) {
        const Place<VEC> p(item, d, n.N, n.C, n.lengths);
        const int ng = p.width / d.CG, vecs = p.width / VEC;
        const int last = min(p.rows1, p.n) - 1;  // the last row that is read
        __syncthreads();
        for (int g = threadIdx.x >> 6; g < ng; g += kThreads / 64) {
            const double2 t = add_chunks(part, per, d.chunks, item - p.chunk, g);
            if ((threadIdx.x & 63) == 0) {
                st[g] = make_float2(0.f, 0.f);
                if (p.n > 0)
                    st[g] = stats_of(t.x, t.y, pivot_of<TYPES>(x, p.b, n, p.c0 + g * d.CG),
                                     (double)p.n * d.CG, n.eps);
                if (stats && p.chunk == 0) stats[(size_t)p.b * n.groups + p.c0 / d.CG + g] = st[g];
            }
        }
        __syncthreads();
        for (int v = p.col; v < vecs; v += p.cols) {
            const int c = p.c0 + v * VEC;
            float mean[VEC], rstd[VEC], ga[VEC], be[VEC];
            of_groups<MIX, VEC>(st, v * VEC, d.CG, mean, rstd);
            load_params<VEC>(n, c, ga, be);
            for (int k = p.rows0 + p.row; k < p.rows1; k += p.par * kRowsAhead) {
                Raw<TYPES, VEC> f[kRowsAhead];
#pragma unroll
                for (int u = 0; u < kRowsAhead; u++)
                    f[u].template load<ONCE>(
                        x, (size_t)p.b * n.N + max(min(k + u * p.par, last), 0), c);
#pragma unroll
                for (int u = 0; u < kRowsAhead; u++) {
                    const int ku = k + u * p.par;
                    if (ku >= p.rows1) break;
                    float r[VEC];
#pragma unroll
                    for (int j = 0; j < VEC; j++)
                        r[j] = act_of<SILU>(
                            fmaf(ga[j], (f[u].get(j) - mean[j]) * rstd[j], be[j]), neg);
                    if (ku > last)
#pragma unroll
                        for (int j = 0; j < VEC; j++) r[j] = 0.f;
                    store_row<TYPES, VEC>(y, (size_t)p.b * n.N + ku, c, r);
                }
            }
        }
    }
}

// chan[b * chunks + chunk][c] = (sum dv xh, sum dv) over the chunk's rows, and
// part[item][group in slab] = their sums over the group's channels, times
// gamma: (sum gamma dv, sum gamma dv xh).
template <int TYPES, bool SILU, int VEC, bool MIX, bool ONCE>
__global__ __launch_bounds__(kThreads) void pv_gn_bwd_sums_kernel(PvNorm n, Deal d, PvRows dy,
                                                                  PvRows x, float neg,
                                                                  const float2* stats,
                                                                  float2* chan, double2* part,
                                                                  int per) {
    __shared__ float2 red[kThreads * VEC];
    for (size_t item = blockIdx.x; item < d.items; item += gridDim.x) {
        const Place<VEC> p(item, d, n.N, n.C, n.lengths);
        const int rows1 = min(p.rows1, p.n), vecs = p.width / VEC;
        float2* out = chan + ((size_t)p.b * d.chunks + p.chunk) * n.C + p.c0;
        for (int v0 = 0; v0 < vecs; v0 += p.cols) {
            const int c = p.c0 + (v0 + p.col) * VEC;
            float s[VEC], h[VEC];
#pragma unroll
            for (int i = 0; i < VEC; i++) s[i] = h[i] = 0.f;
            if (v0 + p.col < vecs) {
                float mean[VEC], rstd[VEC], ga[VEC], be[VEC];
                of_groups<MIX, VEC>(stats + (size_t)p.b * n.groups, c, d.CG, mean, rstd);
                load_params<VEC>(n, c, ga, be);
                for (int k = p.rows0 + p.row; k < rows1; k += p.par * kRowsAhead) {
                    Raw<TYPES, VEC> f[kRowsAhead], g[kRowsAhead];
#pragma unroll
                    for (int u = 0; u < kRowsAhead; u++) {
                        const size_t row = (size_t)p.b * n.N + min(k + u * p.par, rows1 - 1);
                        f[u].template load<ONCE>(x, row, c);
                        g[u].template load<ONCE>(dy, row, c);
                    }
#pragma unroll
                    for (int u = 0; u < kRowsAhead; u++) {
                        if (k + u * p.par >= rows1) break;
#pragma unroll
                        for (int i = 0; i < VEC; i++) {
                            const float xh = (f[u].get(i) - mean[i]) * rstd[i];
                            const float dv =
                                g[u].get(i) * dact_of<SILU>(fmaf(ga[i], xh, be[i]), neg);
                            s[i] += dv;
                            h[i] = fmaf(dv, xh, h[i]);
                        }
                    }
                }
            }
            __syncthreads();
#pragma unroll
            for (int i = 0; i < VEC; i++) red[threadIdx.x * VEC + i] = make_float2(h[i], s[i]);
            __syncthreads();
            const int run = min(p.cols, vecs - v0) * VEC;
            for (int i = threadIdx.x; i < run; i += kThreads) {
                float2 t = make_float2(0.f, 0.f);
                for (int r = 0; r < p.par; r++) {
                    const float2 e = red[r * p.cols * VEC + i];
                    t.x += e.x;
                    t.y += e.y;
                }
                out[v0 * VEC + i] = t;
            }
        }
        __syncthreads();
        for (int g = threadIdx.x >> 6; g < p.width / d.CG; g += kThreads / 64) {
            double t = 0., u = 0.;
            for (int i = threadIdx.x & 63; i < d.CG; i += 64) {
                const float2 e = out[g * d.CG + i];
                const double ga = (double)n.gamma[p.c0 + g * d.CG + i];
                t = fma(ga, (double)e.y, t);
                u = fma(ga, (double)e.x, u);
            }
            t = wave_sum(t);
            u = wave_sum(u);
            if ((threadIdx.x & 63) == 0) part[item * per + g] = make_double2(t, u);
        }
    }
}

// The first `params` workgroups add the chunks' sums of 16 channels into dgamma and
// dbeta, 16 threads a channel, each a share of the chunks (first, since each has a
// long way: behind the others they ran 18 us on at 16 x 32768 x 128).
constexpr int kParamChannels = 16;
__device__ __forceinline__ void add_params(size_t rows, int C, const float2* chan, float* dgamma,
                                           float* dbeta, double2* red) {
    constexpr int kShares = kThreads / kParamChannels;
    const int ch = threadIdx.x % kParamChannels, share = threadIdx.x / kParamChannels;
    const int c = (int)blockIdx.x * kParamChannels + ch;
    double t = 0., u = 0.;
    if (c < C)
        for (size_t r = share; r < rows; r += 4 * kShares) {
            float2 e[4];
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const size_t at = r + i * kShares;
                e[i] = chan[(at < rows ? at : r) * C + c];
            }
#pragma unroll
            for (int i = 0; i < 4; i++)
                if (r + i * kShares < rows) {
                    t += (double)e[i].x;
                    u += (double)e[i].y;
                }
        }
    red[threadIdx.x] = make_double2(t, u);
    __syncthreads();
    if (share == 0 && c < C) {
        for (int w = 1; w < kShares; w++) {
            t += red[ch + kParamChannels * w].x;
            u += red[ch + kParamChannels * w].y;
        }
        if (dgamma) dgamma[c] = (float)t;
        if (dbeta) dbeta[c] = (float)u;
    }
}

template <int TYPES, bool SILU, int VEC, bool MIX, bool ONCE>
__global__ __launch_bounds__(kThreads) void pv_gn_bwd_apply_kernel(
    PvNorm n, Deal d, PvRows dy, PvRows x, PvRows dx, float neg, const float2* stats,
    const float2* chan, const double2* part, int per, float* dgamma, float* dbeta, unsigned params) {
    extern __shared__ float2 gs[];  // per group: mean(gamma dv), mean(gamma dv xh)
    __shared__ double2 red[kThreads];
    if (blockIdx.x < params) {
        add_params((size_t)n.B * d.chunks, n.C, chan, dgamma, dbeta, red);
        return;
    }
    for (size_t item = blockIdx.x - params; item < d.items; item += gridDim.x - params) {
        const Place<VEC> p(item, d, n.N, n.C, n.lengths);
        const int ng = p.width / d.CG, vecs = p.width / VEC;
        const int last = min(p.rows1, p.n) - 1;  // the last row that is read
        __syncthreads();
        for (int g = threadIdx.x >> 6; g < ng; g += kThreads / 64) {
            const double2 t = add_chunks(part, per, d.chunks, item - p.chunk, g);
            const double cnt = p.n > 0 ? (double)p.n * d.CG : 1.;
            if ((threadIdx.x & 63) == 0)
                gs[g] = make_float2((float)(t.x / cnt), (float)(t.y / cnt));
        }
        __syncthreads();
        for (int v = p.col; v < vecs; v += p.cols) {
            const int c = p.c0 + v * VEC;
            float m1[VEC], m2[VEC], mean[VEC], rstd[VEC], ga[VEC], be[VEC];
            of_groups<MIX, VEC>(gs, v * VEC, d.CG, m1, m2);
            of_groups<MIX, VEC>(stats + (size_t)p.b * n.groups, c, d.CG, mean, rstd);
            load_params<VEC>(n, c, ga, be);
            for (int k = p.rows0 + p.row; k < p.rows1; k += p.par * kRowsAhead) {
                Raw<TYPES, VEC> f[kRowsAhead], g[kRowsAhead];
#pragma unroll
                for (int u = 0; u < kRowsAhead; u++) {
                    const size_t row = (size_t)p.b * n.N + max(min(k + u * p.par, last), 0);
                    f[u].template load<ONCE>(x, row, c);
                    g[u].template load<ONCE>(dy, row, c);
                }
#pragma unroll
                for (int u = 0; u < kRowsAhead; u++) {
                    const int ku = k + u * p.par;
                    if (ku >= p.rows1) break;
                    float r[VEC];
#pragma unroll
                    for (int j = 0; j < VEC; j++) {
                        const float xh = (f[u].get(j) - mean[j]) * rstd[j];
                        const float dv = g[u].get(j) * dact_of<SILU>(fmaf(ga[j], xh, be[j]), neg);
                        r[j] = rstd[j] * (fmaf(ga[j], dv, -m1[j]) - xh * m2[j]);
                    }
                    if (ku > last)
#pragma unroll
                        for (int j = 0; j < VEC; j++) r[j] = 0.f;
                    store_row<TYPES, VEC>(dx, (size_t)p.b * n.N + ku, c, r);
                }
            }
        }
    }
}

// ---------------------------------------------------------------------------
// Groups held in registers: a workgroup of T threads a (cloud, group), U vectors
// a thread, rows in parallel over the threads. The mean is summed first, the
// squares about it then, both from the registers.
// 16 x 2048 x 128, 8 groups, bf16: 12.5 us, of which 3 would move the bytes; 32 clouds
// of them: 14.6, backward 21: bound by a workgroup's chain of load, two sums and
// store, one a CU.
// ---------------------------------------------------------------------------
template <int T>
__device__ __forceinline__ double group_sum(double a, double* lds) {
    a = wave_sum(a);
    if constexpr (T > 64) {
        __syncthreads();
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = a;
        __syncthreads();
        a = 0.;
#pragma unroll
        for (int w = 0; w < T / 64; w++) a += lds[w];
    }
    return a;
}
template <int T>
__device__ __forceinline__ double2 group_sum(double a, double b, double2* lds) {
    a = wave_sum(a);
    b = wave_sum(b);
    if constexpr (T > 64) {
        __syncthreads();
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = make_double2(a, b);
        __syncthreads();
        a = b = 0.;
#pragma unroll
        for (int w = 0; w < T / 64; w++) {
            a += lds[w].x;
            b += lds[w].y;
        }
    }
    return make_double2(a, b);
}

template <int T, int VEC>
struct Held {
    int b, g, c, n, par, row;  // cloud, group, first channel, valid rows; this thread's place
    bool active;
    __device__ Held(const PvNorm& p, size_t item) {
        g = (int)((uint32_t)item % (uint32_t)p.groups);
        b = (int)((uint32_t)item / (uint32_t)p.groups);
        n = p.lengths ? min(max(p.lengths[b], 0), p.N) : p.N;
        const int CG = p.C / p.groups, cols = CG / VEC;
        par = T / cols;
        row = threadIdx.x / cols;
        active = row < par;
        c = g * CG + (threadIdx.x - row * cols) * VEC;
    }
};

// Workgroups go round the XCDs: each XCD takes a run of (cloud, group), so that
// the groups of a cloud, whose rows share cache lines, share an L2.
__device__ __forceinline__ size_t run_of_xcd(size_t items) {
    const size_t run = (items + 7) / 8;
    const size_t i = (size_t)(blockIdx.x & 7) * run + (blockIdx.x >> 3);
    return (blockIdx.x >> 3) < run && i < items ? i : items;
}

template <int T, int U, int TYPES, bool SILU, int VEC>
__global__ __launch_bounds__(T) void pv_gn_held_kernel(PvNorm n, PvRows x, PvRows y, float neg,
                                                       float2* stats) {
    __shared__ double lds[T / 64];
    const size_t item = run_of_xcd((size_t)n.B * n.groups);
    if (item >= (size_t)n.B * n.groups) return;
    const Held<T, VEC> p(n, item);
    Raw<TYPES, VEC> f[U];
    float ga[VEC], be[VEC];
    if (p.active) {
        load_params<VEC>(n, p.c, ga, be);
#pragma unroll
        for (int u = 0; u < U; u++)
            f[u].load(x, (size_t)p.b * n.N + max(min(p.row + u * p.par, p.n - 1), 0), p.c);
    }
    double s = 0.;
    if (p.active)
#pragma unroll
        for (int u = 0; u < U; u++)
            if (p.row + u * p.par < p.n)
#pragma unroll
                for (int i = 0; i < VEC; i++) s += (double)f[u].get(i);
    const double cnt = (double)p.n * (n.C / n.groups);
    const double mean = cnt > 0. ? group_sum<T>(s, lds) / cnt : 0.;
    double q = 0.;
    if (p.active)
#pragma unroll
        for (int u = 0; u < U; u++)
            if (p.row + u * p.par < p.n)
#pragma unroll
                for (int i = 0; i < VEC; i++) {
                    const double d = (double)f[u].get(i) - mean;
                    q = fma(d, d, q);
                }
    float2 st = make_float2(0.f, 0.f);
    if (cnt > 0.)
        st = make_float2((float)mean,
                         (float)(1. / sqrt(group_sum<T>(q, lds) / cnt + (double)n.eps)));
    if (stats && threadIdx.x == 0) stats[item] = st;
    if (!p.active) return;
#pragma unroll
    for (int u = 0; u < U; u++) {
        const int k = p.row + u * p.par;
        if (k >= n.N) continue;
        float r[VEC];
#pragma unroll
        for (int i = 0; i < VEC; i++)
            r[i] = act_of<SILU>(fmaf(ga[i], (f[u].get(i) - st.x) * st.y, be[i]), neg);
        if (k >= p.n)
#pragma unroll
            for (int i = 0; i < VEC; i++) r[i] = 0.f;
        store_row<TYPES, VEC>(y, (size_t)p.b * n.N + k, p.c, r);
    }
}

// chan[b][c] = (sum dv xh, sum dv), or dgamma and dbeta themselves of one cloud.
template <int T, int U, int TYPES, bool SILU, int VEC>
__global__ __launch_bounds__(T) void pv_gn_held_bwd_kernel(PvNorm n, PvRows dy, PvRows x, PvRows dx,
                                                           float neg, const float2* stats,
                                                           float2* chan, float* dgamma,
                                                           float* dbeta) {
    __shared__ double2 lds[T / 64];
    extern __shared__ float2 red[];  // [T * VEC]
    const size_t item = run_of_xcd((size_t)n.B * n.groups);
    if (item >= (size_t)n.B * n.groups) return;
    const Held<T, VEC> p(n, item);
    const int CG = n.C / n.groups;
    const float2 st = stats[item];
    // dy times the activation's derivative: held from the sums on, of four vectors of 8
    // of two (more would spill)
    constexpr int kKept = U * VEC > 24 ? U / 2 : U;
    Raw<TYPES, VEC> f[U], g[U];
    float kept[kKept][VEC];
    float ga[VEC], be[VEC], h[VEC], s[VEC];
#pragma unroll
    for (int i = 0; i < VEC; i++) h[i] = s[i] = 0.f;
    double t = 0., tt = 0.;
    if (p.active) {
        load_params<VEC>(n, p.c, ga, be);
#pragma unroll
        for (int u = 0; u < U; u++) {
            const size_t row = (size_t)p.b * n.N + max(min(p.row + u * p.par, p.n - 1), 0);
            f[u].load(x, row, p.c);
            g[u].load(dy, row, p.c);
        }
#pragma unroll
        for (int u = 0; u < U; u++)
            if (p.row + u * p.par < p.n)
#pragma unroll
                for (int i = 0; i < VEC; i++) {
                    const float xh = (f[u].get(i) - st.x) * st.y;
                    const float dv = g[u].get(i) * dact_of<SILU>(fmaf(ga[i], xh, be[i]), neg);
                    s[i] += dv;
                    h[i] = fmaf(dv, xh, h[i]);
                    if (u < kKept) kept[u][i] = dv;
                }
#pragma unroll
        for (int i = 0; i < VEC; i++) {
            t = fma((double)ga[i], (double)s[i], t);
            tt = fma((double)ga[i], (double)h[i], tt);
            red[threadIdx.x * VEC + i] = make_float2(h[i], s[i]);
        }
    }
    const double2 sum = group_sum<T>(t, tt, lds);  // (also the barrier after red)
    // the channels' sums over the rows in parallel: shares of them a thread each,
    // then a wave a channel over the shares
    const int parts = min(min(T / CG, 64), p.par);
    auto keep = [&](int i, double a, double b) {
        const int c = p.g * CG + i;
        if (chan) {
            chan[(size_t)p.b * n.C + c] = make_float2((float)a, (float)b);
        } else {
            if (dgamma) dgamma[c] = (float)a;
            if (dbeta) dbeta[c] = (float)b;
        }
    };
    if (parts > 1) {
        const int i = threadIdx.x % CG, part = threadIdx.x / CG;
        float2 e = make_float2(0.f, 0.f);
        if (part < parts)
            for (int r = part; r < p.par; r += parts) {
                e.x += red[r * CG + i].x;
                e.y += red[r * CG + i].y;
            }
        __syncthreads();
        if (part < parts) red[part * CG + i] = e;
        __syncthreads();
        const int lane = threadIdx.x & 63;
        for (int c = threadIdx.x >> 6; c < CG; c += T / 64) {
            const float2 v = lane < parts ? red[lane * CG + c] : make_float2(0.f, 0.f);
            const double a = wave_sum((double)v.x), b = wave_sum((double)v.y);
            if (lane == 0) keep(c, a, b);
        }
    } else {
        for (int i = threadIdx.x; i < CG; i += T) {
            double a = 0., b = 0.;
            for (int r = 0; r < p.par; r++) {
                a += (double)red[r * CG + i].x;
                b += (double)red[r * CG + i].y;
            }
            keep(i, a, b);
        }
    }
    if (!p.active) return;
    const double cnt = p.n > 0 ? (double)p.n * CG : 1.;
    const float m1 = (float)(sum.x / cnt), m2 = (float)(sum.y / cnt);
    load_params<VEC>(n, p.c, ga, be);  // (again: not held over the sums)
#pragma unroll
    for (int u = 0; u < U; u++) {
        const int k = p.row + u * p.par;
        if (k >= n.N) continue;
        float r[VEC];
#pragma unroll
        for (int i = 0; i < VEC; i++) {
            const float xh = (f[u].get(i) - st.x) * st.y;
            const float dv =
                u < kKept ? kept[u < kKept ? u : 0][i]
                          : g[u].get(i) * dact_of<SILU>(fmaf(ga[i], xh, be[i]), neg);
            r[i] = st.y * (fmaf(ga[i], dv, -m1) - xh * m2);
        }
        if (k >= p.n)
#pragma unroll
            for (int i = 0; i < VEC; i++) r[i] = 0.f;
        store_row<TYPES, VEC>(dx, (size_t)p.b * n.N + k, p.c, r);
    }
}

// dgamma, dbeta from the clouds' sums, 16 channels a workgroup, in cloud order
__global__ __launch_bounds__(kThreads) void pv_gn_params_kernel(int B, int C, const float2* chan,
                                                                float* dgamma, float* dbeta) {
    __shared__ double2 red[kThreads];
    add_params((size_t)B, C, chan, dgamma, dbeta, red);
}

unsigned grid_of(size_t items) { return (unsigned)(items < (1u << 20) ? items : 1u << 20); }

int types_of(const PvRows* r, int count) {
    int bf16 = 0;
    for (int i = 0; i < count; i++) bf16 += r[i].bf16 ? 1 : 0;
    return bf16 == count ? kBf16 : (bf16 == 0 ? kF32 : kMixed);
}
// Vector width: whole vectors in a group and a row, aligned rows, 16 bytes at
// most of the widest type.
int width_for(int CG, const PvRows* r, int count) {
    const int most = types_of(r, count) == kBf16 ? 8 : 4;
    int v = most;
    for (int i = 0; i < count; i++) {
        const int w = pv_vec_width(most, r[i].bf16 ? 2 : 4, r[i].p, CG, r[i].ld);
        v = w < v ? w : v;
    }
    return v;
}
// The vector width of the two launches: vectors across groups (MIX) where those of
// a group are narrower and a slab is whole vectors.
struct Width {
    int vec;
    bool mix;
};
Width width_of_rows(const Deal& d, int C, const PvRows* r, int count) {
    const int own = width_for(d.CG, r, count), rows = width_for(C, r, count);
    if (rows > own && d.slab <= kMixedSlab && d.slab % rows == 0) return {rows, true};
    return {own, false};
}

// f with the call's types, activation and vector width as constants
template <typename F>
void with_kind(int types, bool silu, int vec, F f) {
    auto vecs = [&](auto T, auto S) {
        switch (vec) {
            case 8:
                if constexpr (decltype(T)::value == kBf16) f(T, S, std::integral_constant<int, 8>());
                break;
            case 4: f(T, S, std::integral_constant<int, 4>()); break;
            case 2: f(T, S, std::integral_constant<int, 2>()); break;
            default: f(T, S, std::integral_constant<int, 1>()); break;
        }
    };
    auto acts = [&](auto T) {
        if (silu)
            vecs(T, std::true_type());
        else
            vecs(T, std::false_type());
    };
    switch (types) {
        case kBf16: acts(std::integral_constant<int, kBf16>()); break;
        case kF32: acts(std::integral_constant<int, kF32>()); break;
        default: acts(std::integral_constant<int, kMixed>()); break;
    }
}

// Whether the two launches, whose reads of a line lie far apart, read past the
// caches' normal order: where x and what is streamed beside it (y, or a gradient's dy)
// come near what the Infinity Cache holds (256 MiB). us, streaming / not, of an input
// that was just written and of one that comes from memory:
//   forward     8 x 32768 x 128 bf16 (x 64 MB) 37.4 / 36.7, 42.6 / 42.2; 12 of them
//               55 / 54, 63 / 68; 16: 65 / 70, 74 / 89; 32: 129 / 142, 133 / 168
//   gradient    6: 55.4 / 54.8, 55.5 / 58.0; 12: 104 / 104, 105 / 119; 16: 122 / 125,
//               127 / 144; 32: 240 / 281, 241 / 279; 12 x 24000 x 96 fp32: 126 / 124,
//               130 / 139 (and 130 / 119 where both lie in the cache)
constexpr size_t kStreamBytes = (size_t)224 << 20;
bool streams(const PvNorm& n, const PvRows& a, const PvRows& b) {
    return (size_t)n.B * n.N * n.C * ((a.bf16 ? 2 : 4) + (b.bf16 ? 2 : 4)) >= kStreamBytes;
}
// f with whether to stream as a constant, for vectors that can
template <int TYPES, int VEC, typename F>
void with_stream(bool once, F f) {
    if constexpr (Raw<TYPES, VEC>::kStreams) {
        if (once) {
            f(std::true_type());
            return;
        }
    }
    f(std::false_type());
}

// Whether a group is held in the registers of a workgroup, and of which: vectors a
// thread of 256 (kSmallU) or of 1024 (kLargeU, kLargeBwdU: a gradient holds x and
// dy), one (cloud, group) a workgroup. Where it fits, it is held unless the two
// launches are faster (us, held / two launches, bf16 but where noted):
// - Forward, 256 threads: workgroups for more than one round of the chip that are
//   less than half full, several to an item of the two launches (16384 x 1 x 128, 8
//   groups: 237 / 87; 4096 x 16 x 128, 8 groups: 64 / 34; but 256 x 64 x 128, 8
//   groups: 7.9 / 9.4, and 65536 x 3 x 64 in one group, fp32: 117 / 210).
// - Forward, 1024 threads: more than two workgroups a CU (256 x 512 x 128, 8
//   groups: 49 / 28; where both go by single elements more than four, 31 x 1000 x
//   96 of wider rows, 32 groups: 19 / 29), or few of them with much to read each
//   (1 x 8192 x 64, 8 groups: 17.0 / 9.6; but 1 x 4096 x 128, 32 groups: 10.5 / 16.9).
// - Gradient: where a workgroup adds its channels' sums a wave a channel, groups of
//   more than 32 channels (64 x 3 x 512, 8 groups, fp32: 15 / 8; but 1 x 1 x 1088 in 8
//   groups, whose threads add a channel each: 4.1 / 7.8, 512 x 20 x 640 in 4 groups:
//   19 / 25); many workgroups
//   (16384 x 1 x 128, 8 groups: 1020 / 176; of 1024 threads, 256 x 512 x 128, 8
//   groups: 68 / 41) unless they are full (64 x 256 x 256, 32 groups, fp32: 19 / 28);
//   and few with much to read each (4 x 2048 x 128, 8 groups: 15.6 / 12.2; 32 clouds:
//   21 / 27).
constexpr int kSmallT = 256, kSmallU = 2, kLargeT = 1024, kLargeU = 8, kLargeBwdU = 4;
constexpr int kHeldChannels = 32;
enum Hold { kNot, kSmall, kLarge };
Hold hold_of(const PvNorm& n, const Deal& d, int vec, bool gradient) {
    if (n.N < 1) return kNot;
    const size_t groups = (size_t)n.B * n.groups;  // workgroups
    const int cols = d.CG / vec;
    // a thread adds a channel's sums of a gradient (else a wave does)
    auto by_threads = [&](int threads) { return d.CG > threads / 2 || cols > threads / 2; };
    if (cols <= kSmallT && n.N <= kSmallT / cols * kSmallU) {
        const int vectors = n.N * cols;
        const bool held =
            gradient ? by_threads(kSmallT) ||
                           (d.CG <= kHeldChannels && groups <= 2048 && groups * d.CG <= 8192) ||
                           (d.CG <= 8 && vec >= 4 && vectors >= kSmallT * 3 / 2)
                     : groups <= 4096 || vectors >= kSmallT || groups <= 3 * d.items;
        // HIP takes fewer than 2^32 threads a launch
        return held && (groups + 7) / 8 * 8 * kSmallT <= 0xffffffffu ? kSmall : kNot;
    }
    if (cols <= kLargeT && n.N <= kLargeT / cols * (gradient ? kLargeBwdU : kLargeU)) {
        const int values = n.N * d.CG;
        const size_t most = vec > 1 ? 512 : gradient ? 768 : 1024;
        const bool held = groups <= most &&
                          (gradient ? (d.CG <= kHeldChannels || by_threads(kLargeT)) &&
                                          (values <= 16384 || groups >= 192)
                                    : values <= 32768 || groups >= 96);
        return held ? kLarge : kNot;
    }
    return kNot;
}

float negative_slope(const PvNorm& n) {
    return n.act == PVCONV_ACT_LEAKY ? n.slope : (n.act == PVCONV_ACT_RELU ? 0.f : 1.f);
}

}  // namespace

size_t pv_group_norm_ws_bytes(int B, int N, int C, int groups) {
    const Deal d = deal(B, N, C, groups);
    return pv_align256(d.items * (d.slab / d.CG) * sizeof(double2));
}

size_t pv_group_norm_bwd_ws_bytes(int B, int N, int C, int groups) {
    const Deal d = deal(B, N, C, groups);
    return pv_group_norm_ws_bytes(B, N, C, groups) +
           pv_align256((size_t)B * d.chunks * C * sizeof(float2));
}

pvconv_status pv_launch_group_norm(const PvNorm& n, const PvRows& x, const PvRows& y,
                                   float* stats, void* ws, hipStream_t s) {
    const Deal d = deal(n.B, n.N, n.C, n.groups);
    const PvRows all[2] = {x, y};
    const int per = d.slab / d.CG;
    const float neg = negative_slope(n);
    const int types = types_of(all, 2), own = width_for(d.CG, all, 2);
    const bool silu = n.act == PVCONV_ACT_SILU;
    const Hold hold = hold_of(n, d, own, false);
    if (hold != kNot) {
        with_kind(types, silu, own, [&](auto T, auto S, auto V) {
            constexpr int TYPES = decltype(T)::value, VEC = decltype(V)::value;
            constexpr bool SILU = decltype(S)::value;
            const unsigned held = (unsigned)(((size_t)n.B * n.groups + 7) / 8 * 8);
            if (hold == kSmall)
                pv_gn_held_kernel<kSmallT, kSmallU, TYPES, SILU, VEC>
                    <<<held, kSmallT, 0, s>>>(n, x, y, neg, (float2*)stats);
            else
                pv_gn_held_kernel<kLargeT, kLargeU, TYPES, SILU, VEC>
                    <<<held, kLargeT, 0, s>>>(n, x, y, neg, (float2*)stats);
        });
        return pv_launch_status();
    }
    const Width w = width_of_rows(d, n.C, all, 2);
    const bool once = streams(n, x, y);
    with_kind(types, silu, w.vec, [&](auto T, auto S, auto V) {
        constexpr int TYPES = decltype(T)::value, VEC = decltype(V)::value;
        constexpr bool SILU = decltype(S)::value;
        const unsigned grid = grid_of(d.items);
        const size_t lds = per * sizeof(float2);
        double2* part = (double2*)ws;
        with_stream<TYPES, VEC>(once, [&](auto O) {
            constexpr bool ONCE = decltype(O)::value;
            if (w.mix) {
                pv_gn_mixed_sums_kernel<TYPES, VEC, ONCE>
                    <<<grid, kThreads, 0, s>>>(n, d, x, part, per);
                pv_gn_apply_kernel<TYPES, SILU, VEC, true, ONCE>
                    <<<grid, kThreads, lds, s>>>(n, d, x, y, neg, part, per, (float2*)stats);
            } else {
                pv_gn_sums_kernel<TYPES, VEC, ONCE><<<grid, kThreads, 0, s>>>(n, d, x, part, per);
                pv_gn_apply_kernel<TYPES, SILU, VEC, false, ONCE>
                    <<<grid, kThreads, lds, s>>>(n, d, x, y, neg, part, per, (float2*)stats);
            }
        });
    });
    return pv_launch_status();
}

pvconv_status pv_launch_group_norm_bwd(const PvNorm& norm, const PvRows& dy, const PvRows& x,
                                       const PvRows& dx, const float* stats, float* dgamma,
                                       float* dbeta, void* ws, hipStream_t s) {
    PvNorm n = norm;
    if (n.N == 0) n.B = 0;  // nothing to read: dgamma and dbeta are 0
    const Deal d = deal(n.B, n.N, n.C, n.groups);
    const PvRows all[3] = {dy, x, dx};
    const int per = d.slab / d.CG;
    const unsigned params =
        dgamma || dbeta ? (unsigned)((n.C + kParamChannels - 1) / kParamChannels) : 0;
    if (d.items == 0 && params == 0) return PVCONV_OK;
    double2* part = (double2*)ws;
    float2* chan = (float2*)((char*)ws + pv_group_norm_ws_bytes(n.B, n.N, n.C, n.groups));
    const float neg = negative_slope(n);
    const int types = types_of(all, 3), own = width_for(d.CG, all, 3);
    const bool silu = n.act == PVCONV_ACT_SILU;
    const Hold hold = n.B ? hold_of(n, d, own, true) : kNot;
    const float2* st = (const float2*)stats;
    if (hold != kNot) {
        float2* sums = n.B > 1 ? (float2*)ws : nullptr;
        with_kind(types, silu, own, [&](auto T, auto S, auto V) {
            constexpr int TYPES = decltype(T)::value, VEC = decltype(V)::value;
            constexpr bool SILU = decltype(S)::value;
            const unsigned held = (unsigned)(((size_t)n.B * n.groups + 7) / 8 * 8);
            if (hold == kSmall)
                pv_gn_held_bwd_kernel<kSmallT, kSmallU, TYPES, SILU, VEC>
                    <<<held, kSmallT, kSmallT * VEC * sizeof(float2), s>>>(
                        n, dy, x, dx, neg, st, sums, dgamma, dbeta);
            else
                pv_gn_held_bwd_kernel<kLargeT, kLargeBwdU, TYPES, SILU, VEC>
                    <<<held, kLargeT, kLargeT * VEC * sizeof(float2), s>>>(
                        n, dy, x, dx, neg, st, sums, dgamma, dbeta);
        });
        if (sums && params)
            pv_gn_params_kernel<<<params, kThreads, 0, s>>>(n.B, n.C, sums, dgamma, dbeta);
        return pv_launch_status();
    }
    const Width w = width_of_rows(d, n.C, all, 3);
    const bool once = streams(n, dy, x);
    with_kind(types, silu, w.vec, [&](auto T, auto S, auto V) {
        constexpr int TYPES = decltype(T)::value, VEC = decltype(V)::value;
        constexpr bool SILU = decltype(S)::value;
        auto go = [&](auto M, auto O) {
            constexpr bool MIX = decltype(M)::value, ONCE = decltype(O)::value;
            if (d.items)
                pv_gn_bwd_sums_kernel<TYPES, SILU, VEC, MIX, ONCE>
                    <<<grid_of(d.items), kThreads, 0, s>>>(n, d, dy, x, neg, st, chan, part, per);
            pv_gn_bwd_apply_kernel<TYPES, SILU, VEC, MIX, ONCE>
                <<<grid_of(d.items) + params, kThreads, per * sizeof(float2), s>>>(
                    n, d, dy, x, dx, neg, st, chan, part, per, dgamma, dbeta, params);
        };
        with_stream<TYPES, VEC>(once, [&](auto O) {
            if (w.mix)
                go(std::true_type(), O);
            else
                go(std::false_type(), O);
        });
    });
    return pv_launch_status();
}
