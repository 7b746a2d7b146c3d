// Products a b^T of two row-major operands on the matrix cores, whose rows are
// whole slices of 128 bytes: 64 bf16 values (fp32 sums) or 128 8-bit integers
// (32-bit integer sums). The 8-bit integer layer and the linear cross entropy
// give it their epilogues.
//
// A 32-bit value can be an operand in up to three bf16 parts, h = bf16(v), m =
// bf16(v - h), l = bf16(v - h - m): 24 bits in all. The product of such operands
// is a sum of products of parts (a pair of parts is a run of slices like any
// other); hh + hm + mh + mm + hl + lh leaves out terms below 2^-26 of a product.
#pragma once

#include "pv_train.h"

typedef int pv_i32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t pv_u32x4 __attribute__((ext_vector_type(4)));
typedef pv_u32x4 pv_u32x4_any __attribute__((aligned(2)));
typedef __bf16 pv_b16x8 __attribute__((ext_vector_type(8)));

constexpr int kSlice = 128;  // bytes

__host__ __device__ static inline int pv_slices(int n, int per) { return (n + per - 1) / per; }
static inline size_t pv_up(size_t n, size_t to) { return (n + to - 1) / to * to; }

struct PvPanel {  // rows at p + part * part_bytes + row * pitch
    const uint8_t* p;
    size_t pitch, part_bytes;
    int parts;
};
struct PvProduct {
    PvPanel a, b;
    int M, N, slices;
    int pairs;
    uint32_t pa, pb;     // pair t multiplies part (pa >> 4t) & 15 of a by that of b
    int splits, per;     // slices (of all pairs) a split; partial sums where splits > 1
    uint32_t* partial;   // [splits][M][N], 32-bit words
    uint32_t first, count;  // the tiles of this launch (pv_run_tiles)
};

// The pairs of parts of two operands that a product needs: to 24 bits, or to 16 where
// neither has three parts.
static inline void pv_pairs(PvProduct& p, int parts_a, int parts_b) {
    p.pairs = 0;
    p.pa = p.pb = 0;
    const int orders = parts_a < 3 && parts_b < 3 ? 2 : 3;
    for (int order = 0; order < orders; order++)
        for (int i = 0; i <= order; i++) {
            const int j = order - i;
            if (i >= parts_a || j >= parts_b) continue;
            p.pa |= (uint32_t)i << (4 * p.pairs);
            p.pb |= (uint32_t)j << (4 * p.pairs);
            p.pairs++;
        }
}

// Tiles: WM x WN waves of 16 MI rows by 64 columns each.
template <int WM_, int WN_, int MI_>
struct PvTile {
    static constexpr int WM = WM_, WN = WN_, MI = MI_;
    static constexpr int TM = WM * MI * 16, TN = WN * 64, kThreads = 64 * WM * WN;
};
typedef PvTile<2, 2, 4> PvTileM;  // 128 x 128, two workgroups a CU
typedef PvTile<4, 1, 2> PvTileN;  // 128 x 64: few columns
typedef PvTile<2, 4, 8> PvTileL;  // 256 x 256

// Workgroups go round the XCDs; each XCD takes a run of tiles, eight tiles of rows
// by the columns in turn, so that its L2 serves both operands.
template <class T>
__device__ __forceinline__ bool pv_tile_of(const PvProduct& p, int& split, int& m0, int& n0) {
    const uint32_t mt = (uint32_t)(p.M + T::TM - 1) / T::TM, nt = (uint32_t)(p.N + T::TN - 1) / T::TN;
    const uint32_t run = (p.count + 7) / 8;
    uint32_t idx = (blockIdx.x & 7) * run + (blockIdx.x >> 3);
    if ((blockIdx.x >> 3) >= run || idx >= p.count) return false;
    idx += p.first;
    split = (int)(idx / (mt * nt));
    const uint32_t t = idx % (mt * nt), g = t / (8 * nt), r = t - g * 8 * nt;
    const uint32_t gm = min(8u, mt - g * 8);
    m0 = (int)((g * 8 + r % gm) * T::TM);
    n0 = (int)(r / gm * T::TN);
    return true;
}

template <bool I8>
struct PvAcc {
    typedef pv_f32x4 type;
};
template <>
struct PvAcc<true> {
    typedef pv_i32x4 type;
};

// 16-byte pieces of a 128-byte row are kept at piece ^ key(row) in LDS: the rows that
// eight neighbouring lanes read differ in it (rows of a: consecutive; rows of b: 16
// (r >> 2) + 4 j + (r & 3), which leaves a lane 16 consecutive columns of the result).
__device__ __forceinline__ int pv_key_a(int row) { return row & 7; }
__device__ __forceinline__ int pv_key_b(int row) { return (row & 3) | ((row >> 2) & 4); }

// The epilogue gets acc[j][i][e]: row mw + 16 i + r, column nw + 16 h + 4 j + e (r =
// lane & 15, h = lane >> 4), and LDS of 4 KB a wave once nothing reads it.
template <bool I8, class T, class Epi>
__global__ __launch_bounds__(T::kThreads, 2) void pv_product_kernel(PvProduct p, Epi epi) {
    // two stages, arrays of their own: the loads into one are then seen not to
    // touch what is read of the other, and are not waited for
    __shared__ __align__(16) uint8_t la0[T::TM * kSlice], la1[T::TM * kSlice];
    __shared__ __align__(16) uint8_t lb0[T::TN * kSlice], lb1[T::TN * kSlice];
    typedef typename PvAcc<I8>::type Acc;
    constexpr int MI = T::MI, QA = T::TM * 8 / T::kThreads, QB = T::TN * 8 / T::kThreads;
    int split, m0, n0;
    if (!pv_tile_of<T>(p, split, m0, n0)) return;
    const int t0 = split * p.per, t1 = min(t0 + p.per, p.slices * p.pairs);
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, r = lane & 15, h = lane >> 4;
    const int wm = wave % T::WM * (16 * MI), wn = wave / T::WM * 64;

    const uint8_t* ga[QA];
    const uint8_t* gb[QB];
#pragma unroll
    for (int q = 0; q < QA; q++) {
        const int piece = (wave * QA + q) * 64 + lane, row = piece >> 3, c = piece & 7;
        ga[q] = p.a.p + (size_t)min(m0 + row, p.M - 1) * p.a.pitch + (c ^ pv_key_a(row)) * 16;
    }
#pragma unroll
    for (int q = 0; q < QB; q++) {
        const int piece = (wave * QB + q) * 64 + lane, row = piece >> 3, c = piece & 7;
        gb[q] = p.b.p + (size_t)min(n0 + row, p.N - 1) * p.b.pitch + (c ^ pv_key_b(row)) * 16;
    }
    int pair = t0 / max(p.slices, 1), k = t0 - pair * p.slices;
    auto fetch = [&](uint8_t* la, uint8_t* lb) {
        const size_t oa = ((p.pa >> (4 * pair)) & 15) * p.a.part_bytes + (size_t)k * kSlice;
        const size_t ob = ((p.pb >> (4 * pair)) & 15) * p.b.part_bytes + (size_t)k * kSlice;
#pragma unroll
        for (int q = 0; q < QA; q++)
            __builtin_amdgcn_global_load_lds(
                (const void __attribute__((address_space(1)))*)(ga[q] + oa),
                (void __attribute__((address_space(3)))*)(la + (wave * QA + q) * 1024), 16, 0, 0);
#pragma unroll
        for (int q = 0; q < QB; q++)
            __builtin_amdgcn_global_load_lds(
                (const void __attribute__((address_space(1)))*)(gb[q] + ob),
                (void __attribute__((address_space(3)))*)(lb + (wave * QB + q) * 1024), 16, 0, 0);
        if (++k == p.slices) {
            k = 0;
            pair++;
        }
    };
    Acc acc[4][MI];
#pragma unroll
    for (int j = 0; j < 4; j++)
#pragma unroll
        for (int i = 0; i < MI; i++) acc[j][i] = Acc{0, 0, 0, 0};

    auto slice = [&](int t, const uint8_t* la, const uint8_t* lb, uint8_t* na, uint8_t* nb) {
        __builtin_amdgcn_s_waitcnt(0);  // this wave's part of the slices has landed
        __syncthreads();
        if (t + 1 < t1) fetch(na, nb);
#pragma unroll
        for (int half = 0; half < 2; half++) {
            pv_u32x4 fa[MI], fb[4];
#pragma unroll
            for (int j = 0; j < 4; j++) {
                const int row = wn + 16 * (r >> 2) + 4 * j + (r & 3);
                fb[j] = *(const pv_u32x4*)(lb + row * kSlice +
                                           ((h + 4 * half) ^ pv_key_b(row)) * 16);
            }
#pragma unroll
            for (int i = 0; i < MI; i++) {
                const int row = wm + 16 * i + r;
                fa[i] = *(const pv_u32x4*)(la + row * kSlice +
                                           ((h + 4 * half) ^ pv_key_a(row)) * 16);
            }
#pragma unroll
            for (int i = 0; i < MI; i++)
#pragma unroll
                for (int j = 0; j < 4; j++) {
                    if constexpr (I8) {
                        acc[j][i] = __builtin_amdgcn_mfma_i32_16x16x64_i8(
                            (pv_i32x4)fb[j], (pv_i32x4)fa[i], acc[j][i], 0, 0, 0);
                    } else {
                        pv_b16x8 va, vb;
                        __builtin_memcpy(&va, &fa[i], 16);
                        __builtin_memcpy(&vb, &fb[j], 16);
                        acc[j][i] =
                            __builtin_amdgcn_mfma_f32_16x16x32_bf16(vb, va, acc[j][i], 0, 0, 0);
                    }
                }
        }
    };
    if (t0 < t1) fetch(la0, lb0);
    for (int t = t0; t < t1; t += 2) {
        slice(t, la0, lb0, la1, lb1);
        if (t + 1 < t1) slice(t + 1, la1, lb1, la0, lb0);
    }
    if (p.splits > 1) {
        uint32_t* part = p.partial + (size_t)split * p.M * p.N;
#pragma unroll
        for (int i = 0; i < MI; i++) {
            const int m = m0 + wm + 16 * i + r, n = n0 + wn + 16 * h;
            if (m >= p.M) continue;
            uint32_t* o = part + (size_t)m * p.N + n;
#pragma unroll
            for (int j = 0; j < 4; j++) {
                pv_u32x4 v;
                __builtin_memcpy(&v, &acc[j][i], 16);
                if (n + 4 * j + 4 <= p.N)
                    *(pv_u32x4_any*)(o + 4 * j) = v;
                else
#pragma unroll
                    for (int e = 0; e < 4; e++)
                        if (n + 4 * j + e < p.N) o[4 * j + e] = v[e];
            }
        }
        return;
    }
    if constexpr (Epi::kLds) __syncthreads();
    epi.template tile<MI>(p, m0 + wm, n0 + wn, lane, acc, la0 + wave * 4096);
}

// W (4 or 16) consecutive values of a row from column n on, wherever the row begins.
template <int W>
__device__ __forceinline__ void pv_store_run(const PvRows& out, int m, int n, int N,
                                             const float (&v)[W]) {
    const size_t at = (size_t)m * out.ld + n;
    const bool whole = n + W <= N;
    if (out.bf16) {
        uint16_t* o = (uint16_t*)out.p + at;
        if (whole) {
            uint32_t w[W / 2];
#pragma unroll
            for (int i = 0; i < W / 2; i++) w[i] = pv_pack_bf16x2(v[2 * i], v[2 * i + 1]);
#pragma unroll
            for (int i = 0; i < W / 8; i++)
                *(pv_u32x4_any*)(o + 8 * i) =
                    pv_u32x4{w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]};
        } else {
#pragma unroll
            for (int i = 0; i < W; i++)
                if (n + i < N) o[i] = pv_f32_to_bf16(v[i]);
        }
    } else {
        float* o = (float*)out.p + at;
        if (whole) {
#pragma unroll
            for (int i = 0; i < W / 4; i++)
                *(pv_u32x4_any*)(o + 4 * i) =
                    pv_u32x4{__float_as_uint(v[4 * i]), __float_as_uint(v[4 * i + 1]),
                             __float_as_uint(v[4 * i + 2]), __float_as_uint(v[4 * i + 3])};
        } else {
#pragma unroll
            for (int i = 0; i < W; i++)
                if (n + i < N) o[i] = v[i];
        }
    }
}

// ---- splits ----------------------------------------------------------------
// How many ways a product's slices are split: one where its tiles fill the chip,
// else enough for two workgroups a CU at most, of `least` slices or more.
static inline void pv_plan_splits(PvProduct& p, int tm, int tn, int least) {
    const size_t tiles = (size_t)((p.M + tm - 1) / tm) * ((p.N + tn - 1) / tn);
    const int all = p.slices * p.pairs;
    p.per = all;
    if (tiles > 0 && tiles < 256 && all >= 2 * least) {
        const int most = all / least;
        int n = (int)(512 / tiles);
        n = n < 1 ? 1 : (n > most ? most : n);
        p.per = (all + n - 1) / n;
    }
    p.splits = p.per ? (all + p.per - 1) / p.per : 1;
}
static inline size_t pv_partial_bytes(const PvProduct& p) {
    return p.splits > 1 ? (size_t)p.splits * p.M * p.N * 4 : 0;
}

// The splits' sums in order, then epi.one(m, n, sum).
template <bool I8, class Epi>
__global__ __launch_bounds__(256) void pv_join_kernel(PvProduct p, Epi epi) {
    constexpr int kAhead = 8;  // splits in flight
    const size_t total = (size_t)p.M * p.N;
    for (size_t at = (size_t)blockIdx.x * 256 + threadIdx.x; at < total;
         at += (size_t)gridDim.x * 256) {
        float s = 0.f;
        int si = 0;
        for (int k = 0; k < p.splits; k += kAhead) {
            uint32_t v[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; u++)
                v[u] = p.partial[(size_t)min(k + u, p.splits - 1) * total + at];
#pragma unroll
            for (int u = 0; u < kAhead; u++)
                if (k + u < p.splits) {
                    if constexpr (I8)
                        si += (int)v[u];
                    else
                        s += __uint_as_float(v[u]);
                }
        }
        const int m = (int)(at / p.N), n = (int)(at - (size_t)m * p.N);
        if constexpr (I8)
            epi.one(m, n, si);
        else
            epi.one(m, n, s);
    }
}
static inline unsigned pv_blocks(size_t items, int per) {
    const size_t b = (items + per - 1) / per;
    return (unsigned)(b < 1 ? 1 : (b < (1u << 16) ? b : 1u << 16));
}

constexpr size_t kPvTilesALaunch = 1u << 22;  // a launch has fewer than 2^32 threads
template <bool I8, class T, class Epi>
static void pv_run_tiles(PvProduct p, const Epi& epi, hipStream_t s) {
    const size_t tiles =
        (size_t)((p.M + T::TM - 1) / T::TM) * ((p.N + T::TN - 1) / T::TN) * p.splits;
    for (size_t t = 0; t < tiles; t += kPvTilesALaunch) {
        p.first = (uint32_t)t;
        p.count = (uint32_t)(tiles - t < kPvTilesALaunch ? tiles - t : kPvTilesALaunch);
        hipLaunchKernelGGL((pv_product_kernel<I8, T, Epi>), dim3((p.count + 7) / 8 * 8),
                           dim3(T::kThreads), 0, s, p, epi);
    }
    if (p.splits > 1)
        hipLaunchKernelGGL((pv_join_kernel<I8, Epi>), dim3(pv_blocks((size_t)p.M * p.N, 256)),
                           dim3(256), 0, s, p, epi);
}

// ---- operands (product.hip) ------------------------------------------------
enum PvKind { kPvF32, kPvBf16, kPvInt8 };
struct PvPack {
    const void* src;
    PvKind kind;
    size_t ld;               // elements
    int R, C;                // the source's rows and columns
    const float* row_scale;  // or NULL
    const float* col_scale;  // or NULL
    int parts;
    uint8_t* dst;
    size_t pitch;            // bytes; padded with zeros up to it
    size_t part_bytes;
};
// The source as rows of bf16 parts, and its transpose as such (dst's rows: columns).
void pv_launch_pack(const PvPack& k, hipStream_t s);
void pv_launch_pack_transposed(const PvPack& k, hipStream_t s);

// out (+)= a b^T in bf16 parts: out = sum + add (dense [M][N] fp32, or NULL)
struct PvPlain {
    PvRows out;
    const float* add;
};
void pv_plan_plain(PvProduct& p);
void pv_launch_plain(const PvProduct& p, const PvPlain& e, hipStream_t s);

// Pieces of a workspace, one behind another.
struct PvCarve {
    char* base;
    size_t off;
    void* take(size_t bytes) {
        void* p = base ? base + off : nullptr;
        off += pv_align256(bytes);
        return p;
    }
};
static inline PvPanel pv_take_panel(PvCarve& c, size_t rows, size_t cols, int parts) {
    PvPanel p;
    p.pitch = pv_up(cols, 64) * 2;
    p.part_bytes = pv_align256(rows * p.pitch);
    p.parts = parts;
    p.p = (const uint8_t*)c.take(p.part_bytes * parts);
    return p;
}
static inline PvPack pv_pack_of(const void* src, PvKind kind, size_t ld, int R, int C,
                                const PvPanel& to) {
    return PvPack{src, kind, ld, R, C, nullptr, nullptr, to.parts, (uint8_t*)to.p, to.pitch,
                  to.part_bytes};
}

// Sums [parts][N] joined in a fixed order, and column sums of rows of channels (a linear
// layer's bias gradient).
void pv_launch_sum_parts(const float* partial, int parts, int N, float* out, hipStream_t s);
size_t pv_column_sum_bytes(int M, int N);
void pv_launch_column_sum(const PvRows& x, int M, int N, float* partial, float* out,
                          hipStream_t s);
