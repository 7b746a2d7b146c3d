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

#include <type_traits>
#include <utility>

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
    int size;            // PvSize
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

// Tiles: WM x WN waves of 16 MI rows by 64 columns each; ST stages of slices in LDS, ST -
// 1 of them under way while one is multiplied.
template <int WM_, int WN_, int MI_, int ST_, int PER_CU_, int KB_ = 128>
struct PvTile {
    static constexpr int WM = WM_, WN = WN_, MI = MI_, ST = ST_;
    static constexpr int KB = KB_;  // bytes of a row that a stage holds
    static constexpr int TM = WM * MI * 16, TN = WN * 64, kThreads = 64 * WM * WN;
    static constexpr int kWorkgroups = 256 * PER_CU_;  // that the chip holds at once
};
typedef PvTile<2, 4, 8, 2, 1> PvTileL;  // 256 x 256
typedef PvTile<4, 2, 4, 3, 1> PvTileG;  // 256 x 128: half the sums in registers
typedef PvTile<2, 2, 4, 4, 1> PvTileM;  // 128 x 128
typedef PvTile<4, 1, 2, 4, 1> PvTileN;  // 128 x 64: few columns
typedef PvTile<2, 1, 2, 4, 2> PvTileS;  // 64 x 64: few tiles

// The tile of index idx: eight tiles of rows by the columns in turn, so that an XCD,
// which works on neighbours at a time, has both operands in its L2.
template <class T>
__device__ __forceinline__ void pv_tile_of(const PvProduct& p, uint32_t idx, int& split, int& m0,
                                           int& n0) {
    const uint32_t mt = (uint32_t)(p.M + T::TM - 1) / T::TM, nt = (uint32_t)(p.N + T::TN - 1) / T::TN;
    split = (int)(idx / (mt * nt));
    const uint32_t t = idx % (mt * nt), g = t / (8 * nt), r = t - g * 8 * nt;
    const uint32_t gm = min(8u, mt - g * 8);
    m0 = (int)((g * 8 + r % gm) * T::TM);
    n0 = (int)(r / gm * T::TN);
}

template <bool I8>
struct PvAcc {
    typedef pv_f32x4 type;
};
template <>
struct PvAcc<true> {
    typedef pv_i32x4 type;
};

// 16-byte pieces of a stage's row are kept at piece ^ key(row) in LDS, so that the rows
// which eight neighbouring lanes read lie in different banks (rows of a: consecutive; rows
// of b: 16 (r >> 2) + 4 j + (r & 3), which leaves a lane 16 consecutive columns of the
// result).
template <int KB>
__device__ __forceinline__ int pv_key_a(int row) {
    return KB == 128 ? row & 7 : (row >> 1) & 3;
}
template <int KB>
__device__ __forceinline__ int pv_key_b(int row) {
    return KB == 128 ? (row & 3) | ((row >> 2) & 4) : ((row >> 1) & 1) | ((row >> 3) & 2);
}

// f(0), .. f(N - 1) with the index as a constant: arrays that it indexes stay in registers
template <class F, int... I>
__device__ __forceinline__ void pv_each(std::integer_sequence<int, I...>, const F& f) {
    (f(std::integral_constant<int, I>()), ...);
}
template <int N, class F>
__device__ __forceinline__ void pv_each(const F& f) {
    pv_each(std::make_integer_sequence<int, N>(), f);
}

// s_waitcnt of at most VM loads under way, and none of LDS
template <int VM>
__device__ __forceinline__ void pv_wait_loads() {
    static_assert(VM < 64, "six bits");
    __builtin_amdgcn_s_waitcnt((VM & 15) | (7 << 4) | ((VM >> 4) << 14));
}

// The epilogue gets acc[j][i][e]: row mw + 16 i + r, column nw + 16 h + 4 j + e (r =
// lane & 15, h = lane >> 4), and 4 KB of LDS a wave that nothing else uses then. A
// workgroup takes several tiles in turn: the first slices of the next one are under way
// during the epilogue.
template <bool I8, class T, class Epi>
__global__ __launch_bounds__(T::kThreads, T::kThreads* T::kWorkgroups / 256 / 256) void
pv_product_kernel(PvProduct p, Epi epi) {
    // stages, arrays of their own: the loads into one are then seen not to touch what is
    // read of another, and are not waited for
    constexpr int KB = T::KB, SA = T::TM * KB, SB = T::TN * KB, ST = T::ST;
    constexpr int PR = KB / 16;  // pieces of a row
    __shared__ __align__(16) uint8_t la0[SA], la1[SA], la2[ST > 2 ? SA : 16], la3[ST > 3 ? SA : 16];
    __shared__ __align__(16) uint8_t lb0[SB], lb1[SB], lb2[ST > 2 ? SB : 16], lb3[ST > 3 ? SB : 16];
    constexpr int kPer = kSlice / KB;  // stages of a slice
    typedef typename PvAcc<I8>::type Acc;
    constexpr int MI = T::MI, QA = T::TM * PR / T::kThreads, QB = T::TN * PR / T::kThreads;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, r = lane & 15, h = lane >> 4;
    const int wm = wave % T::WM * (16 * MI), wn = wave / T::WM * 64;
    // each XCD (workgroups go round them) takes a run of the launch's tiles
    const uint32_t run = (p.count + 7) / 8, step = gridDim.x >> 3;
    const uint32_t end = min(run * ((blockIdx.x & 7) + 1), p.count);
    uint32_t idx = run * (blockIdx.x & 7) + (blockIdx.x >> 3);
    if (idx >= end) return;

    int split, m0, n0, t0, t1, pair, k;
    const uint8_t* ga[QA];
    const uint8_t* gb[QB];
    auto enter = [&]() {
        pv_tile_of<T>(p, p.first + idx, split, m0, n0);
        t0 = split * p.per;
        t1 = min(t0 + p.per, p.slices * p.pairs) * kPer;
        pair = t0 / max(p.slices, 1);
        k = (t0 - pair * p.slices) * kPer;
        t0 *= kPer;
#pragma unroll
        for (int q = 0; q < QA; q++) {
            const int piece = (wave * QA + q) * 64 + lane, row = piece / PR, c = piece % PR;
            ga[q] = p.a.p + (size_t)min(m0 + row, p.M - 1) * p.a.pitch + (c ^ pv_key_a<KB>(row)) * 16;
        }
#pragma unroll
        for (int q = 0; q < QB; q++) {
            const int piece = (wave * QB + q) * 64 + lane, row = piece / PR, c = piece % PR;
            gb[q] = p.b.p + (size_t)min(n0 + row, p.N - 1) * p.b.pitch + (c ^ pv_key_b<KB>(row)) * 16;
        }
    };
    // load q of the QA + QB of a slice; the last one moves on to the next slice
    auto fetch_one = [&](int q, uint8_t* la, uint8_t* lb) {
        if (q < QA) {
            const size_t oa = ((p.pa >> (4 * pair)) & 15) * p.a.part_bytes + (size_t)k * KB;
            __builtin_amdgcn_global_load_lds(
                (const void __attribute__((address_space(1)))*)(ga[q < QA ? q : 0] + oa),
                (void __attribute__((address_space(3)))*)(la + (wave * QA + q) * 1024), 16, 0, 0);
        } else {
            const size_t ob = ((p.pb >> (4 * pair)) & 15) * p.b.part_bytes + (size_t)k * KB;
            __builtin_amdgcn_global_load_lds(
                (const void __attribute__((address_space(1)))*)(gb[q < QA ? 0 : q - QA] + ob),
                (void __attribute__((address_space(3)))*)(lb + (wave * QB + q - QA) * 1024), 16, 0,
                0);
        }
        if (q == QA + QB - 1 && ++k == p.slices * kPer) {
            k = 0;
            pair++;
        }
    };
    auto fetch = [&](uint8_t* la, uint8_t* lb) {
#pragma unroll
        for (int q = 0; q < QA + QB; q++) fetch_one(q, la, lb);
    };
    auto first = [&]() {  // the first ST - 1 slices of a tile
        if (t0 < t1) fetch(la0, lb0);
        if (ST > 2 && t0 + 1 < t1) fetch(la1, lb1);
        if (ST > 3 && t0 + 2 < t1) fetch(la2, lb2);
    };
    enter();
    first();
    for (;;) {
        Acc acc[4][MI];
#pragma unroll
        for (int j = 0; j < 4; j++)
#pragma unroll
            for (int i = 0; i < MI; i++) acc[j][i] = Acc{0, 0, 0, 0};
        auto load_a = [&](const uint8_t* la, int i, int half) {
            const int row = wm + 16 * i + r;
            return *(const pv_u32x4*)(la + row * KB + ((h + 4 * half) ^ pv_key_a<KB>(row)) * 16);
        };
        auto load_b = [&](const uint8_t* lb, int j, int half) {
            const int row = wn + 16 * (r >> 2) + 4 * j + (r & 3);
            return *(const pv_u32x4*)(lb + row * KB + ((h + 4 * half) ^ pv_key_b<KB>(row)) * 16);
        };
        // The products of a slice in la, lb. The loads of a later one go between them: at
        // once, they would hold every wave up for the time that they take to be issued.
        auto multiply = [&](const uint8_t* la, const uint8_t* lb, uint8_t* na, uint8_t* nb,
                            bool fetching) {
            constexpr int Q = QA + QB;
            pv_u32x4 fa[MI], fb[4];
            pv_each<4>([&](auto j) { fb[j] = load_b(lb, j, 0); });
            pv_each<MI>([&](auto i) { fa[i] = load_a(la, i, 0); });
            pv_each<KB / 64>([&](auto half) {
                pv_each<MI>([&](auto i) {
                    pv_each<4>([&](auto j) {
                        if constexpr (I8) {
                            acc[j][i] = __builtin_amdgcn_mfma_i32_16x16x64_i8(
                                (pv_i32x4)fb[j], (pv_i32x4)fa[i], acc[j][i], 0, 0, 0);
                        } else {
                            pv_b16x8 va, vb;
                            __builtin_memcpy(&va, &fa[i], 16);
                            __builtin_memcpy(&vb, &fb[j], 16);
                            acc[j][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vb, va, acc[j][i],
                                                                                0, 0, 0);
                        }
                    });
                    if constexpr (half == 0) {
                        if constexpr (KB == 128) {
                            if constexpr (i == MI - 1)
                                pv_each<4>([&](auto j) { fb[j] = load_b(lb, j, 1); });
                            fa[i] = load_a(la, i, 1);
                        }
                        constexpr int q0 = i * Q / MI, q1 = (i + 1) * Q / MI;
                        if (fetching) pv_each<q1 - q0>([&](auto q) { fetch_one(q + q0, na, nb); });
                    }
                    __builtin_amdgcn_sched_barrier(0);
                });
            });
        };
        // one slice, in la, lb; na, nb, read before this barrier, take the one ST - 1 on
        auto slice = [&](int t, const uint8_t* la, const uint8_t* lb, uint8_t* na, uint8_t* nb) {
            if (t + ST - 2 < t1)  // this wave's part of it has landed
                pv_wait_loads<(ST - 2) * (QA + QB)>();
            else
                pv_wait_loads<0>();
            pv_lds_barrier();
            multiply(la, lb, na, nb, t + ST - 1 < t1);
        };
        for (int t = t0; t < t1; t += ST) {
            if constexpr (ST == 2) {
                slice(t, la0, lb0, la1, lb1);
                if (t + 1 < t1) slice(t + 1, la1, lb1, la0, lb0);
            } else if constexpr (ST == 3) {
                slice(t, la0, lb0, la2, lb2);
                if (t + 1 < t1) slice(t + 1, la1, lb1, la0, lb0);
                if (t + 2 < t1) slice(t + 2, la2, lb2, la1, lb1);
            } else {
                slice(t, la0, lb0, la3, lb3);
                if (t + 1 < t1) slice(t + 1, la1, lb1, la0, lb0);
                if (t + 2 < t1) slice(t + 2, la2, lb2, la1, lb1);
                if (t + 3 < t1) slice(t + 3, la3, lb3, la2, lb2);
            }
        }
        const int em = m0 + wm, en = n0 + wn, es = split;
        idx += step;
        const bool more = idx < end;
        pv_lds_barrier();  // nothing reads the stages any more
        if (more) {
            enter();
            first();
        }
        if (p.splits > 1) {
            uint32_t* part = p.partial + (size_t)es * p.M * p.N;
#pragma unroll
            for (int i = 0; i < MI; i++) {
                const int m = em + 16 * i + r, n = en + 16 * h;
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
        } else {
            epi.template tile<MI>(p, em, en, lane, acc, (ST == 2 ? la1 : ST == 3 ? la2 : la3) + wave * 4096);
        }
        if (!more) return;
    }
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
// How many ways a product's slices are split, and into which tiles: unsplit where its
// tiles fill the chip, else enough for a workgroup a CU at most, of `least` slices or
// more.
enum PvSize { kPvS, kPvN, kPvM, kPvG, kPvL };
static inline size_t pv_tiles_of(int M, int N, int tm, int tn) {
    return (size_t)((M + tm - 1) / tm) * ((N + tn - 1) / tn);
}
static inline void pv_plan_splits(PvProduct& p, int least) {
    const int all = p.slices * p.pairs;
    PvSize size = kPvS;
    size_t tiles = pv_tiles_of(p.M, p.N, 64, 64);
    if (p.N > 128 && pv_tiles_of(p.M, p.N, 256, 256) * (all / 32 + 1) >= 192) {
        size = kPvL;
        tiles = pv_tiles_of(p.M, p.N, 256, 256);
    } else if (p.N > 64 && pv_tiles_of(p.M, p.N, 128, 128) * (all / 16 + 1) >= 128) {
        size = kPvM;
        tiles = pv_tiles_of(p.M, p.N, 128, 128);
    } else if (p.N <= 64 && pv_tiles_of(p.M, p.N, 128, 64) * (all / 16 + 1) >= 128) {
        size = kPvN;
        tiles = pv_tiles_of(p.M, p.N, 128, 64);
    }
    p.per = all;
    if (tiles > 0 && tiles <= 128 && all >= 2 * least) {
        const int most = all / least;
        int n = (int)(256 / tiles);
        n = n < 1 ? 1 : (n > most ? most : n);
        p.per = (all + n - 1) / n;
    }
    p.splits = p.per ? (all + p.per - 1) / p.per : 1;
    p.size = size;
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

constexpr size_t kPvTilesALaunch = (size_t)1 << 30;
template <class T>
static inline size_t pv_tiles(const PvProduct& p) {
    return (size_t)((p.M + T::TM - 1) / T::TM) * ((p.N + T::TN - 1) / T::TN) * p.splits;
}
template <bool I8, class T, class Epi>
static void pv_run_tiles(PvProduct p, const Epi& epi, hipStream_t s) {
    const size_t tiles = pv_tiles<T>(p);
    for (size_t t = 0; t < tiles; t += kPvTilesALaunch) {
        p.first = (uint32_t)t;
        p.count = (uint32_t)(tiles - t < kPvTilesALaunch ? tiles - t : kPvTilesALaunch);
        const unsigned most = (p.count + 7) / 8 * 8;
        hipLaunchKernelGGL((pv_product_kernel<I8, T, Epi>),
                           dim3(most < T::kWorkgroups ? most : T::kWorkgroups), dim3(T::kThreads),
                           0, s, p, epi);
    }
    if (p.splits > 1)
        hipLaunchKernelGGL((pv_join_kernel<I8, Epi>), dim3(pv_blocks((size_t)p.M * p.N, 256)),
                           dim3(256), 0, s, p, epi);
}

// The tiles of a product that is never split: large ones where they fill the chip, and
// smaller the fewer there are of them.
static inline PvSize pv_size_of(int M, int N) {
    if (N > 128 && pv_tiles_of(M, N, 256, 256) >= 192) return kPvL;
    if (N > 64 && pv_tiles_of(M, N, 128, 128) >= 128) return kPvM;
    return N <= 64 && pv_tiles_of(M, N, 128, 64) >= 128 ? kPvN : kPvS;
}
template <bool I8, class Epi>
static void pv_run_product(const PvProduct& p, const Epi& epi, hipStream_t s) {
    switch (p.size) {
        case kPvL: pv_run_tiles<I8, PvTileL>(p, epi, s); break;
        case kPvG: pv_run_tiles<I8, PvTileG>(p, epi, s); break;
        case kPvM: pv_run_tiles<I8, PvTileM>(p, epi, s); break;
        case kPvN: pv_run_tiles<I8, PvTileN>(p, epi, s); break;
        default: pv_run_tiles<I8, PvTileS>(p, epi, s);
    }
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
