// Operands of the products in pv_product.h, plain products and column sums.
#include "pv_product.h"

namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ float load_kind(const void* src, PvKind kind, size_t at) {
    if (kind == kPvF32) return ((const float*)src)[at];
    if (kind == kPvBf16) return pv_bf16_to_f32(((const uint16_t*)src)[at]);
    return (float)((const int8_t*)src)[at];
}

// Eight consecutive columns of a row from c0 on, zeros from C on.
template <PvKind KIND>
__device__ __forceinline__ void load8(const PvPack& k, size_t row, int c0, float (&v)[8]) {
    const size_t from = row * k.ld + c0;
    if (c0 + 8 > k.C) {
#pragma unroll
        for (int i = 0; i < 8; i++)  // (no branches, which would wait for one after another)
            v[i] = load_kind(k.src, KIND, row * k.ld + min(c0 + i, k.C - 1));
#pragma unroll
        for (int i = 0; i < 8; i++) v[i] = c0 + i < k.C ? v[i] : 0.f;
    } else if constexpr (KIND == kPvBf16) {
        const pv_u32x4 w = *(const pv_u32x4_any*)((const uint16_t*)k.src + from);
#pragma unroll
        for (int i = 0; i < 8; i++)
            v[i] = __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
    } else if constexpr (KIND == kPvF32) {
        const pv_u32x4 w = *(const pv_u32x4_any*)((const float*)k.src + from);
        const pv_u32x4 y = *(const pv_u32x4_any*)((const float*)k.src + from + 4);
#pragma unroll
        for (int i = 0; i < 8; i++) v[i] = __uint_as_float(i < 4 ? w[i] : y[i - 4]);
    } else {  // quantised rows begin on 128 bytes
        const uint2 w = *(const uint2*)((const int8_t*)k.src + from);
#pragma unroll
        for (int i = 0; i < 8; i++)
            v[i] = (float)(int8_t)((i < 4 ? w.x : w.y) >> (8 * (i & 3)));
    }
}

// The next bf16 part of v, which leaves v - part. The largest finite values would
// round to infinity: they are cut off instead.
__device__ __forceinline__ uint32_t next_part(float& v) {
    uint32_t h = pv_f32_to_bf16(v);
    const uint32_t u = __float_as_uint(v);
    const bool finite = (u & 0x7fffffffu) < 0x7f800000u;
    if (finite && (h & 0x7fffu) == 0x7f80u) h = u >> 16;
    v = finite ? v - pv_bf16_to_f32((uint16_t)h) : 0.f;
    return h;
}

// log2 of the threads of a row of `per` pieces: as many as leave an eighth of them idle at
// most, of few rows a third.
__host__ __device__ inline int pack_shift(int per, int rows) {
    const int idle = rows <= 4096 ? per / 3 : per / 8;
    int shift = 8;
    while (shift > 3 && ((per + (1 << shift) - 1) >> shift << shift) > per + idle) shift--;
    return shift;
}

// Rows of parts: eight consecutive columns a thread, both ends of the traffic in 16-byte
// pieces, a power of two of threads a row. Bound by memory.
template <PvKind KIND>
__device__ __forceinline__ void pack_rows(const PvPack& k, size_t block, size_t blocks) {
    const int per = (int)(k.pitch / 16);
    const int shift = pack_shift(per, k.rows);
    const int lead = threadIdx.x >> shift, first = threadIdx.x & ((1 << shift) - 1);
    const size_t rows = (size_t)kThreads >> shift;
    for (size_t row = block * rows + lead; row < (size_t)k.rows; row += blocks * rows) {
        const float rs = k.row_scale && row < (size_t)k.R ? k.row_scale[row] : 1.f;
        for (int piece = first; piece < per; piece += 1 << shift) {
            const int c0 = piece * 8;
            float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            if (row < (size_t)k.R) {
                load8<KIND>(k, row, c0, v);
                if (k.row_scale) {  // (NaN for a row that was not finite)
#pragma unroll
                    for (int i = 0; i < 8; i++) v[i] = c0 + i < k.C ? v[i] * rs : 0.f;
                }
                if (k.col_scale) {
#pragma unroll
                    for (int i = 0; i < 8; i++)
                        v[i] = c0 + i < k.C ? v[i] * k.col_scale[c0 + i] : 0.f;
                }
            }
            uint8_t* to = k.dst + row * k.pitch + (size_t)c0 * 2;
            if (KIND != kPvF32 && k.parts == 1 && !k.row_scale && !k.col_scale) {
                *(pv_u32x4*)to = pv_u32x4{pv_pack_bf16x2(v[0], v[1]), pv_pack_bf16x2(v[2], v[3]),
                                          pv_pack_bf16x2(v[4], v[5]), pv_pack_bf16x2(v[6], v[7])};
                continue;
            }
            for (int part = 0; part < k.parts; part++) {
                uint32_t q[8];
#pragma unroll
                for (int i = 0; i < 8; i++) q[i] = next_part(v[i]);
                *(pv_u32x4*)(to + part * k.part_bytes) =
                    pv_u32x4{q[0] | (q[1] << 16), q[2] | (q[3] << 16), q[4] | (q[5] << 16),
                             q[6] | (q[7] << 16)};
            }
        }
    }
}

// Sums of columns over runs of rows, in 64 bits: eight columns a thread, 64 a workgroup,
// whose 32 threads take every 32nd row of a column, four of them under way; of a single run,
// which would leave most CUs idle, eight columns and 256 threads.
__host__ __device__ inline int sum_groups(int R) { return pv_sum_runs(R) == 1 ? 1 : 8; }
template <PvKind KIND>
__device__ __forceinline__ void sum_columns(const PvPack& k, size_t block, size_t blocks,
                                            double (*part)[72]) {
    const int groups = sum_groups(k.R), leads = kThreads / groups;
    const size_t nb = (k.C + 8 * groups - 1) / (8 * groups),
                 total = nb * ((k.R + k.rows - 1) / k.rows);
    const int group = threadIdx.x & (groups - 1), lead = threadIdx.x / groups;
    constexpr int kAhead = 4;
    for (size_t t = block; t < total; t += blocks) {
        const int c0 = ((int)(t % nb) * groups + group) * 8;
        const size_t r0 = t / nb * k.rows;
        const int rows = (int)min((size_t)k.rows, (size_t)k.R - r0);
        double s[8] = {0., 0., 0., 0., 0., 0., 0., 0.};
        if (c0 < k.C)
            for (int i = lead; i < rows; i += leads * kAhead) {
                float v[kAhead][8];
#pragma unroll
                for (int u = 0; u < kAhead; u++)
                    load8<KIND>(k, r0 + min(i + leads * u, rows - 1), c0, v[u]);
#pragma unroll
                for (int u = 0; u < kAhead; u++)
                    if (i + leads * u < rows)
#pragma unroll
                        for (int q = 0; q < 8; q++) s[q] += (double)v[u][q];
            }
        // the threads of a wave that have the same columns, then the four waves
        for (int w = groups; w < 64; w <<= 1)
#pragma unroll
            for (int q = 0; q < 8; q++) s[q] += __shfl_xor(s[q], w);
        if ((int)(threadIdx.x & 63) < groups)
#pragma unroll
            for (int q = 0; q < 8; q++) part[threadIdx.x >> 6][group * 8 + q] = s[q];
        __syncthreads();
        const int c = (int)(t % nb) * groups * 8 + (int)threadIdx.x;
        if ((int)threadIdx.x < groups * 8 && c < k.C)
            k.sums[t / nb * k.C + c] = (float)(((part[0][threadIdx.x] + part[1][threadIdx.x]) +
                                                part[2][threadIdx.x]) + part[3][threadIdx.x]);
        __syncthreads();
    }
}

__global__ __launch_bounds__(kThreads) void pv_packs_kernel(PvPacks k) {
    __shared__ double part[4][72];
    int j = 0;
    while (j + 1 < k.n && blockIdx.x >= k.begin[j + 1]) j++;
    const size_t block = blockIdx.x - k.begin[j], blocks = k.begin[j + 1] - k.begin[j];
    const PvPack& job = k.job[j];
    if (job.sums) {
        if (job.kind == kPvBf16)
            sum_columns<kPvBf16>(job, block, blocks, part);
        else
            sum_columns<kPvF32>(job, block, blocks, part);
    } else if (job.kind == kPvBf16) {
        pack_rows<kPvBf16>(job, block, blocks);
    } else if (job.kind == kPvF32) {
        pack_rows<kPvF32>(job, block, blocks);
    } else {
        pack_rows<kPvInt8>(job, block, blocks);
    }
}

struct PlainEpi {
    PvPlain e;
    int N;
    template <int MI>
    __device__ __forceinline__ void tile(const PvProduct& p, int mw, int nw, int lane,
                                         const pv_f32x4 (&acc)[4][MI]) const {
        const int r = lane & 15, nb = nw + 8 * (lane >> 4);
#pragma unroll
        for (int i = 0; i < MI; i++) {
            const int m = mw + 16 * i + r;
            if (m >= p.M) continue;
            float v[16];
#pragma unroll
            for (int q = 0; q < 16; q++) v[q] = acc[q >> 2][i][q & 3];
            if (e.add) {
#pragma unroll
                for (int q = 0; q < 16; q += 4) {
                    const int n = pv_col(nb, q);
                    const float* from = e.add + (size_t)m * p.N + n;
                    if (n + 4 <= p.N) {
                        const pv_u32x4 w = *(const pv_u32x4_any*)from;
#pragma unroll
                        for (int u = 0; u < 4; u++) v[q + u] += __uint_as_float(w[u]);
                    } else {
#pragma unroll
                        for (int u = 0; u < 4; u++)
                            if (n + u < p.N) v[q + u] += from[u];
                    }
                }
            }
            pv_store_runs(e.out, m, nb, p.N, v);
        }
    }
    __device__ __forceinline__ void one(int m, int n, float v) const {
        if (e.add) v += e.add[(size_t)m * N + n];
        pv_store_one(e.out.p, e.out.bf16, (size_t)m * e.out.ld + n, v);
    }
};

// A wave a column: 64 runs at a time in 64 bits, in a fixed order, eight loads in flight.
__device__ __forceinline__ void sum_run(const PvSums& k, int c) {
    const int lane = threadIdx.x & 63;
    double s = 0.;
    for (int i0 = 0; i0 < k.n; i0 += 512) {
        float v[8];
#pragma unroll
        for (int u = 0; u < 8; u++)
            v[u] = k.runs[(size_t)min(i0 + 64 * u + lane, k.n - 1) * k.N + c];
#pragma unroll
        for (int u = 0; u < 8; u++)
            if (i0 + 64 * u + lane < k.n) s += (double)v[u];
    }
#pragma unroll
    for (int w = 1; w < 64; w <<= 1) s += __shfl_xor(s, w);
    if (lane == 0) k.out[c] = (float)s;
}
__device__ __forceinline__ void sum_runs(const PvSums& k, unsigned block) {
    const int c = (int)block * 4 + (threadIdx.x >> 6);
    if (c < k.N) sum_run(k, c);
}
__global__ __launch_bounds__(kThreads) void pv_sum_runs_kernel(PvSums k) {
    sum_runs(k, blockIdx.x);
}
// a product's splits and column sums
__global__ __launch_bounds__(kThreads) void pv_finish_kernel(PvProduct p, PlainEpi epi, PvSums k,
                                                             unsigned sums) {
    if (blockIdx.x < sums)
        sum_runs(k, blockIdx.x);
    else
        pv_join<false>(p, epi, blockIdx.x - sums, gridDim.x - sums);
}

// The same, a thread a column: many columns, whose neighbours lie side by side.
__global__ __launch_bounds__(kThreads) void pv_sum_runs_wide_kernel(PvSums k) {
    const int c = (int)blockIdx.x * kThreads + threadIdx.x;
    if (c >= k.N) return;
    double s = 0.;
    for (int i0 = 0; i0 < k.n; i0 += 8) {
        float v[8];
#pragma unroll
        for (int u = 0; u < 8; u++) v[u] = k.runs[(size_t)min(i0 + u, k.n - 1) * k.N + c];
#pragma unroll
        for (int u = 0; u < 8; u++)
            if (i0 + u < k.n) s += (double)v[u];
    }
    k.out[c] = (float)s;
}
constexpr int kWideSums = 4096;  // columns

// Two products, the first's a along k, the second's across it, a workgroup a tile, and
// column sums, in one launch. Products of few tiles leave CUs idle, and a launch costs as
// much as one of them. (us, two products, what joins their splits, sums / in one: 999 x 323,
// 1003 classes, fp32: 14 + 4 + 16 + 4 + 3 / 26; 777 x 203 -> 99, fp32: 4.5 + 5.2 + 2.9 /
// 13, two launches fewer; since with three stages of parts 21 and 11.)
struct Pair {
    PvProduct x, y;
    PlainEpi ex, ey;
    uint32_t x_blocks, y_blocks;
    PvSums sums;
};
__device__ __forceinline__ bool pair_sums(const Pair& k, int waves) {
    const uint32_t products = k.x_blocks + k.y_blocks;
    if (blockIdx.x < products) return false;
    for (int c = (int)(blockIdx.x - products) * waves + (int)(threadIdx.x >> 6); c < k.sums.N;
         c += (int)(gridDim.x - products) * waves)
        sum_run(k.sums, c);
    return true;
}
__global__ __launch_bounds__(PvTileS::kThreads, 1) void pv_pair_kernel(Pair k) {
    typedef PvTileS T;
    constexpr int SA = T::TM * kSlice, SB = T::TN * kSlice;
    __shared__ __align__(16) uint8_t la0[SA], la1[SA], la2[SA], la3[SA];
    __shared__ __align__(16) uint8_t lb0[SB], lb1[SB], lb2[SB], lb3[SB];
    const PvStages lds{la0, la1, la2, la3, lb0, lb1, lb2, lb3};
    if (pair_sums(k, T::kThreads / 64)) return;
    if (blockIdx.x < k.x_blocks)
        pv_product_tiles<false, false, true, T>(k.x, k.ex, blockIdx.x, k.x_blocks, lds);
    else
        pv_product_tiles<false, true, true, T>(k.y, k.ey, blockIdx.x - k.x_blocks, k.y_blocks, lds);
}
template <int PB>
__global__ __launch_bounds__(PvTileP::kThreads, 1) void pv_pair_parts_kernel(Pair k) {
    constexpr int SA = 3 * PvTileP::TM * kSlice, SB = PB * PvTileP::TN * kSlice;
    __shared__ __align__(16) uint8_t la0[SA], la1[SA], la2[SA], lb0[SB], lb1[SB], lb2[SB];
    const PvStages lds{la0, la1, la2, nullptr, lb0, lb1, lb2, nullptr};
    if (pair_sums(k, PvTileP::kThreads / 64)) return;
    if (blockIdx.x < k.x_blocks)
        pv_parts_tiles<false, true, 3, PB>(k.x, k.ex, blockIdx.x, k.x_blocks, lds);
    else
        pv_parts_tiles<true, true, 3, PB>(k.y, k.ey, blockIdx.x - k.x_blocks, k.y_blocks, lds);
}

}  // namespace

constexpr size_t kOneStep = 2048;  // workgroups: all of them at once
void pv_launch_packs(PvPacks& k, hipStream_t s) {
    k.begin[0] = 0;
    for (int j = 0; j < k.n; j++) {
        const PvPack& p = k.job[j];
        const int columns = 8 * sum_groups(p.R);
        size_t blocks = (size_t)pv_sum_runs(p.R) * ((p.C + columns - 1) / columns);
        if (!p.sums) {  // a step each, of many rows two
            const int rows = kThreads >> pack_shift((int)(p.pitch / 16), p.rows);
            blocks = ((size_t)p.rows + rows - 1) / rows;
            if (blocks > kOneStep) blocks = blocks < 2 * kOneStep ? kOneStep : blocks / 2;
        }
        k.begin[j + 1] = k.begin[j] + (unsigned)(blocks < (1u << 16) ? blocks : 1u << 16);
    }
    if (k.n && k.begin[k.n])
        hipLaunchKernelGGL(pv_packs_kernel, dim3(k.begin[k.n]), dim3(kThreads), 0, s, k);
}

void pv_launch_sum_runs(const PvSums& k, hipStream_t s) {
    if (!k.out) return;
    if (k.N >= kWideSums)
        hipLaunchKernelGGL(pv_sum_runs_wide_kernel, dim3((k.N + kThreads - 1) / kThreads),
                           dim3(kThreads), 0, s, k);
    else
        hipLaunchKernelGGL(pv_sum_runs_kernel, dim3((k.N + 3) / 4), dim3(kThreads), 0, s, k);
}

void pv_launch_plain(const PvProduct& p, bool a_across, const PvPlain& e, const PvSums& sums,
                     hipStream_t s) {
    const PlainEpi epi{e, p.N};
    if (a_across)
        pv_run_product<false, true, true>(p, epi, s);
    else
        pv_run_product<false, false, true>(p, epi, s);
    if (sums.out && sums.N < kWideSums && p.splits > 1 && pv_join_narrow(p)) {
        const unsigned blocks = (unsigned)(sums.N + 3) / 4;
        hipLaunchKernelGGL(pv_finish_kernel, dim3(blocks + pv_blocks((size_t)p.M * p.N, 64)),
                           dim3(kThreads), 0, s, p, epi, sums, blocks);
        return;
    }
    pv_run_join<false>(p, epi, s);
    pv_launch_sum_runs(sums, s);
}

// Unsplit, one round of workgroups (some of them for column sums), and expected to take no
// longer than one after the other.
constexpr float kLaunch = 3.f;  // us
constexpr size_t kSumBlocks = 8;
int pv_pair_size(const PvProduct& x, const PvProduct& y) {
    float best = x.us + y.us + kLaunch;
    int size = -1;
    auto choose = [&](const PvSizeCost& c) {
        const size_t blocks = pv_up(pv_tiles_of(x.M, x.N, c.tm, c.tn), 8) +
                              pv_up(pv_tiles_of(y.M, y.N, c.tm, c.tn), 8) + kSumBlocks;
        const int xs = x.slices * x.pairs, ys = y.slices * y.pairs;
        const float us = (float)(xs > ys ? xs : ys) * c.slice + c.rest;
        if (blocks > (size_t)c.slots || us > best) return;
        best = us;
        size = c.size;
    };
    for (const PvSizeCost& c : kPvCosts)
        if (c.size == kPvS) choose(c);
    if (x.a.parts == 3 && y.a.parts == 3 && x.b.parts == y.b.parts &&
        pv_all_parts(x.a.parts, x.b.parts))
        choose(pv_parts_cost(x.pairs));
    return size;
}
void pv_take_pair(PvProduct& p, int size) {
    p.size = size;
    p.per = p.slices * p.pairs;
    p.splits = 1;
}
void pv_launch_pair(const PvProduct& x, const PvPlain& ex, const PvProduct& y, const PvPlain& ey,
                    const PvSums& sums, hipStream_t s) {
    Pair k{x, y, PlainEpi{ex, x.N}, PlainEpi{ey, y.N}, 0, 0, sums};
    auto run = [&](auto kernel, auto tile) {
        typedef decltype(tile) T;
        auto tiles = [](PvProduct& p) {
            p.first = 0;
            p.count = (uint32_t)pv_tiles_of(p.M, p.N, T::TM, T::TN);
            return (uint32_t)pv_up(p.count, 8);
        };
        k.x_blocks = tiles(k.x);
        k.y_blocks = tiles(k.y);
        const unsigned products = k.x_blocks + k.y_blocks, waves = T::kThreads / 64,
                       most = T::kWorkgroups - products;
        unsigned more = sums.out ? ((unsigned)sums.N + waves - 1) / waves : 0;
        if (more > most) more = most;
        hipLaunchKernelGGL(kernel, dim3(products + more), dim3(T::kThreads), 0, s, k);
    };
    if (x.size == kPvS)
        run(pv_pair_kernel, PvTileS());
    else if (x.b.parts == 3)
        run(pv_pair_parts_kernel<3>, PvTileP());
    else
        run(pv_pair_parts_kernel<1>, PvTileP());
}
