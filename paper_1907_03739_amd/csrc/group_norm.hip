// Group normalisation with an activation, channels last, and its gradients
// (pvconv_train.h).
//
// Two launches a direction. The first sums a share ("chunk") of a cloud's rows
// over a slab of whole groups; the second adds the chunks' sums of its groups
// in a fixed order and applies them to a chunk of rows. Bound by HBM: x (and
// dy) read twice, y (dx) written once.
#include <type_traits>

#include "pv_train.h"

namespace {

constexpr int kThreads = 256;

// How the work is dealt: items (cloud, slab of channels, chunk of rows).
struct Deal {
    int CG;      // channels a group
    int slab;    // channels a slab: whole groups
    int slabs;
    int chunk;   // rows a chunk
    int chunks;
    size_t items;
};

// A slab is at most about 128 channels (or one group), so that the sums that
// an item of the second launch adds stay few; chunks are small enough for
// about kItems items and not smaller than kMinRows rows.
constexpr int kSlab = 128, kItems = 2048, kMinRows = 16;

Deal deal(int B, int N, int C, int groups) {
    Deal d;
    d.CG = C / groups;
    int k = kSlab / d.CG;
    k = k < 1 ? 1 : (k > groups ? groups : k);
    d.slab = k * d.CG;
    d.slabs = (groups + k - 1) / k;
    const size_t per = (size_t)(B > 0 ? B : 1) * d.slabs;
    size_t chunks = (kItems + per - 1) / per;
    const size_t most = (size_t)(N + kMinRows - 1) / kMinRows;
    if (chunks > most) chunks = most;
    if (chunks < 1) chunks = 1;
    d.chunk = (int)(((size_t)N + chunks - 1) / chunks);
    if (d.chunk < 1) d.chunk = 1;
    d.chunks = (N + d.chunk - 1) / d.chunk;
    if (d.chunks < 1) d.chunks = 1;
    d.items = (size_t)B * d.slabs * d.chunks;
    return d;
}

// One item and this thread's place in it: `cols` threads along the slab's
// vectors, `par` rows in parallel.
template <int VEC>
struct Place {
    int b, s, chunk, rows0, rows1, c0, width, cols, par, col, row, n;
    __device__ Place(size_t item, const Deal& d, int N, int C, const int32_t* lengths) {
        chunk = (int)(item % d.chunks);
        const size_t r = item / d.chunks;
        s = (int)(r % d.slabs);
        b = (int)(r / d.slabs);
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

__device__ __forceinline__ float act_of(float v, int act, float slope) {
    if (act == PVCONV_ACT_SILU) return v * __builtin_amdgcn_rcpf(1.f + __expf(-v));
    return pv_activate(v, act, slope);
}
__device__ __forceinline__ float dact_of(float v, int act, float slope) {
    if (act == PVCONV_ACT_SILU) {
        const float s = __builtin_amdgcn_rcpf(1.f + __expf(-v));
        return s * fmaf(v, 1.f - s, 1.f);
    }
    if (act == PVCONV_ACT_NONE) return 1.f;
    return v > 0.f ? 1.f : (act == PVCONV_ACT_LEAKY ? slope : 0.f);
}

// Sum over the workgroup's threads that hold `group`'s share, in a fixed
// order: the wave that owns the group adds the entries lane-wise, then across.
__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) v += __shfl_xor(v, m);
    return v;
}

// part[item of (b, slab, chunk)][group in slab] = (sum, sum of squares), in 64
// bits: the subtraction that makes the variance of them loses nothing that 32
// bits could hold.
template <bool XB, int VEC>
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
            if (v0 + p.col < vecs)
                for (int k = p.rows0 + p.row; k < rows1; k += p.par) {
                    float f[VEC];
                    pv_load_vec<XB, VEC>(x.p, ((size_t)p.b * n.N + k) * x.ld + c, f);
#pragma unroll
                    for (int i = 0; i < VEC; i++) {
                        s += (double)f[i];
                        ss = fma((double)f[i], (double)f[i], ss);
                    }
                }
            __syncthreads();
            red[threadIdx.x] = make_double2(s, ss);
            __syncthreads();
            // the groups that this run of columns touches
            const int g0 = v0 / gv, g1 = min((v0 + p.cols + gv - 1) / gv, ng);
            for (int g = g0 + (threadIdx.x >> 6); g < g1; g += kThreads / 64) {
                const int a = max(g * gv - v0, 0), z = min((g + 1) * gv - v0, min(p.cols, vecs - v0));
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

// The statistics of the item's groups into st (mean, rstd), and out to `stats`
// by the items of chunk 0.
__device__ __forceinline__ void group_stats(const double2* part, int per, const Deal& d,
                                            size_t item, int chunk, int ng, int n, float eps,
                                            float2* st, float2* out) {
    const double2* p = part + (item - chunk) * per;
    for (int g = threadIdx.x >> 6; g < ng; g += kThreads / 64) {
        double t = 0., tt = 0.;
        for (int i = threadIdx.x & 63; i < d.chunks; i += 64) {
            const double2 e = p[(size_t)i * per + g];
            t += e.x;
            tt += e.y;
        }
        t = wave_sum(t);
        tt = wave_sum(tt);
        if ((threadIdx.x & 63) == 0) {
            const double cnt = (double)n * d.CG;
            float2 r = make_float2(0.f, 0.f);
            if (n > 0) {
                const double mean = t / cnt, var = tt / cnt - mean * mean;
                r.x = (float)mean;
                r.y = (float)(1. / sqrt((var < 0. ? 0. : var) + (double)eps));
            }
            st[g] = r;
            if (out && chunk == 0) out[g] = r;
        }
    }
}

template <bool XB, bool YB, int VEC>
__global__ __launch_bounds__(kThreads) void pv_gn_apply_kernel(PvNorm n, Deal d, PvRows x,
                                                               PvRows y, const double2* part,
                                                               int per, float2* stats) {
    extern __shared__ float2 st[];
    for (size_t item = blockIdx.x; item < d.items; item += gridDim.x) {
        const Place<VEC> p(item, d, n.N, n.C, n.lengths);
        const int ng = p.width / d.CG, vecs = p.width / VEC;
        __syncthreads();
        group_stats(part, per, d, item, p.chunk, ng, p.n, n.eps, st,
                    stats ? stats + (size_t)p.b * n.groups + p.c0 / d.CG : nullptr);
        __syncthreads();
        for (int v = p.col; v < vecs; v += p.cols) {
            const int c = p.c0 + v * VEC;
            const float2 m = st[v * VEC / d.CG];
            float a[VEC], be[VEC];
#pragma unroll
            for (int i = 0; i < VEC; i++) {
                a[i] = n.gamma[c + i];
                be[i] = n.beta[c + i];
            }
            for (int k = p.rows0 + p.row; k < p.rows1; k += p.par) {
                const size_t at = (size_t)p.b * n.N + k;
                float f[VEC];
                if (k < p.n) {
                    pv_load_vec<XB, VEC>(x.p, at * x.ld + c, f);
#pragma unroll
                    for (int i = 0; i < VEC; i++)
                        f[i] = act_of(fmaf(a[i], (f[i] - m.x) * m.y, be[i]), n.act, n.slope);
                } else {
#pragma unroll
                    for (int i = 0; i < VEC; i++) f[i] = 0.f;
                }
                pv_store_vec<YB, VEC>(y.p, at * y.ld + c, f);
            }
        }
    }
}

// part[b * chunks + chunk][c] = (sum dv xh, sum dv) over the chunk's rows.
template <bool DB, bool XB, int VEC>
__global__ __launch_bounds__(kThreads) void pv_gn_bwd_sums_kernel(PvNorm n, Deal d, PvRows dy,
                                                                  PvRows x, const float2* stats,
                                                                  float2* part) {
    __shared__ float2 red[kThreads * VEC];
    for (size_t item = blockIdx.x; item < d.items; item += gridDim.x) {
        const Place<VEC> p(item, d, n.N, n.C, n.lengths);
        const int rows1 = min(p.rows1, p.n), vecs = p.width / VEC;
        for (int v0 = 0; v0 < vecs; v0 += p.cols) {
            const int c = p.c0 + (v0 + p.col) * VEC;
            float s[VEC], h[VEC];
#pragma unroll
            for (int i = 0; i < VEC; i++) s[i] = h[i] = 0.f;
            if (v0 + p.col < vecs) {
                const float2 m = stats[(size_t)p.b * n.groups + c / d.CG];
                float ga[VEC], be[VEC];
#pragma unroll
                for (int i = 0; i < VEC; i++) {
                    ga[i] = n.gamma[c + i];
                    be[i] = n.beta[c + i];
                }
                for (int k = p.rows0 + p.row; k < rows1; k += p.par) {
                    const size_t at = (size_t)p.b * n.N + k;
                    float f[VEC], g[VEC];
                    pv_load_vec<XB, VEC>(x.p, at * x.ld + c, f);
                    pv_load_vec<DB, VEC>(dy.p, at * dy.ld + c, g);
#pragma unroll
                    for (int i = 0; i < VEC; i++) {
                        const float xh = (f[i] - m.x) * m.y;
                        const float dv = g[i] * dact_of(fmaf(ga[i], xh, be[i]), n.act, n.slope);
                        s[i] += dv;
                        h[i] = fmaf(dv, xh, h[i]);
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
                part[((size_t)p.b * d.chunks + p.chunk) * n.C + p.c0 + v0 * VEC + i] = t;
            }
        }
    }
}

// Items beyond d.items add the chunks' sums of 64 channels into dgamma, dbeta.
template <bool DB, bool XB, bool OB, int VEC>
__global__ __launch_bounds__(kThreads) void pv_gn_bwd_apply_kernel(
    PvNorm n, Deal d, PvRows dy, PvRows x, PvRows dx, const float2* stats, const float2* part,
    float* dgamma, float* dbeta, size_t items) {
    extern __shared__ float2 gs[];  // per group of the slab: mean(gamma dv), mean(gamma dv xh)
    __shared__ double2 red[kThreads];
    for (size_t item = blockIdx.x; item < items; item += gridDim.x) {
        if (item >= d.items) {
            const int c = (int)(item - d.items) * 64 + (threadIdx.x & 63);
            double t = 0., u = 0.;
            const size_t rows = (size_t)n.B * d.chunks;
            if (c < n.C)
                for (size_t r = threadIdx.x >> 6; r < rows; r += kThreads / 64) {
                    const float2 e = part[r * n.C + c];
                    t += (double)e.x;
                    u += (double)e.y;
                }
            __syncthreads();
            red[threadIdx.x] = make_double2(t, u);
            __syncthreads();
            if (threadIdx.x < 64 && c < n.C) {
                for (int w = 1; w < kThreads / 64; w++) {
                    t += red[threadIdx.x + 64 * w].x;
                    u += red[threadIdx.x + 64 * w].y;
                }
                if (dgamma) dgamma[c] = (float)t;
                if (dbeta) dbeta[c] = (float)u;
            }
            continue;
        }
        const Place<VEC> p(item, d, n.N, n.C, n.lengths);
        const int ng = p.width / d.CG, vecs = p.width / VEC;
        __syncthreads();
        for (int g = threadIdx.x >> 6; g < ng; g += kThreads / 64) {
            double t = 0., u = 0.;
            const int m = d.CG * d.chunks;
            for (int i = threadIdx.x & 63; i < m; i += 64) {
                const int c = p.c0 + g * d.CG + i % d.CG;
                const float2 e = part[((size_t)p.b * d.chunks + i / d.CG) * n.C + c];
                const double ga = (double)n.gamma[c];
                t = fma(ga, (double)e.y, t);
                u = fma(ga, (double)e.x, u);
            }
            t = wave_sum(t);
            u = wave_sum(u);
            const double cnt = p.n > 0 ? (double)p.n * d.CG : 1.;
            if ((threadIdx.x & 63) == 0) gs[g] = make_float2((float)(t / cnt), (float)(u / cnt));
        }
        __syncthreads();
        for (int v = p.col; v < vecs; v += p.cols) {
            const int c = p.c0 + v * VEC;
            const float2 q = gs[v * VEC / d.CG];
            const float2 m = stats[(size_t)p.b * n.groups + c / d.CG];
            float ga[VEC], be[VEC];
#pragma unroll
            for (int i = 0; i < VEC; i++) {
                ga[i] = n.gamma[c + i];
                be[i] = n.beta[c + i];
            }
            for (int k = p.rows0 + p.row; k < p.rows1; k += p.par) {
                const size_t at = (size_t)p.b * n.N + k;
                float f[VEC], g[VEC];
                if (k < p.n) {
                    pv_load_vec<XB, VEC>(x.p, at * x.ld + c, f);
                    pv_load_vec<DB, VEC>(dy.p, at * dy.ld + c, g);
#pragma unroll
                    for (int i = 0; i < VEC; i++) {
                        const float xh = (f[i] - m.x) * m.y;
                        const float dv = g[i] * dact_of(fmaf(ga[i], xh, be[i]), n.act, n.slope);
                        f[i] = m.y * (fmaf(ga[i], dv, -q.x) - xh * q.y);
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < VEC; i++) f[i] = 0.f;
                }
                pv_store_vec<OB, VEC>(dx.p, at * dx.ld + c, f);
            }
        }
    }
}

unsigned grid_of(size_t items) { return (unsigned)(items < (1u << 20) ? items : 1u << 20); }

// Vector width: whole vectors in a group, a row and a slab, and aligned rows.
int width_for(int CG, const PvRows* r, int count) {
    int v = 8;
    for (int i = 0; i < count; i++) {
        const int w = pv_vec_width(8, r[i].bf16 ? 2 : 4, r[i].p, CG, r[i].ld);
        v = w < v ? w : v;
    }
    return v;
}

template <typename F>
void with_vec(int v, F f) {
    switch (v) {
        case 8: f(std::integral_constant<int, 8>()); break;
        case 4: f(std::integral_constant<int, 4>()); break;
        case 2: f(std::integral_constant<int, 2>()); break;
        default: f(std::integral_constant<int, 1>()); break;
    }
}
template <typename F>
void with_bool(bool b, F f) {
    if (b)
        f(std::true_type());
    else
        f(std::false_type());
}

}  // namespace

size_t pv_group_norm_ws_bytes(int B, int N, int C, int groups) {
    const Deal d = deal(B, N, C, groups);
    return pv_align256(d.items * (d.slab / d.CG) * sizeof(double2));
}

size_t pv_group_norm_bwd_ws_bytes(int B, int N, int C, int groups) {
    const Deal d = deal(B, N, C, groups);
    return pv_align256((size_t)B * d.chunks * C * sizeof(float2));
}

pvconv_status pv_launch_group_norm(const PvNorm& n, const PvRows& x, const PvRows& y,
                                   float* stats, void* ws, hipStream_t s) {
    const Deal d = deal(n.B, n.N, n.C, n.groups);
    const PvRows all[2] = {x, y};
    const int per = d.slab / d.CG;
    const unsigned grid = grid_of(d.items);
    with_vec(width_for(d.CG, all, 2), [&](auto V) {
        with_bool(x.bf16, [&](auto XB) {
            constexpr int VEC = decltype(V)::value;
            pv_gn_sums_kernel<decltype(XB)::value, VEC>
                <<<grid, kThreads, 0, s>>>(n, d, x, (double2*)ws, per);
            with_bool(y.bf16, [&](auto YB) {
                pv_gn_apply_kernel<decltype(XB)::value, decltype(YB)::value, VEC>
                    <<<grid, kThreads, per * sizeof(float2), s>>>(n, d, x, y, (const double2*)ws,
                                                                  per, (float2*)stats);
            });
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
    const size_t items = d.items + (dgamma || dbeta ? (size_t)(n.C + 63) / 64 : 0);
    if (items == 0) return PVCONV_OK;
    with_vec(width_for(d.CG, all, 3), [&](auto V) {
        constexpr int VEC = decltype(V)::value;
        with_bool(dy.bf16, [&](auto DB) {
            with_bool(x.bf16, [&](auto XB) {
                if (d.items)
                    pv_gn_bwd_sums_kernel<decltype(DB)::value, decltype(XB)::value, VEC>
                        <<<grid_of(d.items), kThreads, 0, s>>>(n, d, dy, x, (const float2*)stats,
                                                               (float2*)ws);
                with_bool(dx.bf16, [&](auto OB) {
                    pv_gn_bwd_apply_kernel<decltype(DB)::value, decltype(XB)::value,
                                           decltype(OB)::value, VEC>
                        <<<grid_of(items), kThreads, per * sizeof(float2), s>>>(
                            n, d, dy, x, dx, (const float2*)stats, (const float2*)ws, dgamma,
                            dbeta, items);
                });
            });
        });
    });
    return pv_launch_status();
}
