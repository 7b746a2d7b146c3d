// Products on the matrix cores, out[m][n] = sum_k a(m, k) b(n, k), of 64 bf16 values
// (fp32 sums) or 128 8-bit integers (32-bit integer sums) a slice. The 8-bit integer
// layer and the linear cross entropy give it their operands and epilogues.
//
// An operand lies along k (a row of memory is a row of the operand, whole slices of 128
// bytes, zeros behind its end) or across it (bf16 only: a row of memory is one k, as x and
// dy are for x^T dy; the LDS loads transpose). Of an operand across k the rows past its
// last are read as that one, so that the other operand's have to be zero there.
//
// A 32-bit value can be an operand in up to three bf16 parts, h = bf16(v), m =
// bf16(v - h), l = bf16(v - h - m): 24 bits in all. The product of such operands
// is a sum of products of parts (a pair of parts is a run of slices like any
// other); hh + hm + mh + mm + hl + lh leaves out ml and lm, up to 2^-24 of a product
// together (a second part is up to 2^-8 of its value, a third 2^-17), and ll. Two parts are
// 16 bits: hh + hm + mh. What lies below 2^-133, the smallest bf16 number, is in no part.
#pragma once

#include <type_traits>
#include <utility>

#include "pv_train.h"

typedef int pv_i32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t pv_u32x4 __attribute__((ext_vector_type(4)));
typedef pv_u32x4 pv_u32x4_any __attribute__((aligned(2)));
typedef __bf16 pv_b16x8 __attribute__((ext_vector_type(8)));
typedef short pv_s16x4 __attribute__((ext_vector_type(4)));

constexpr int kSlice = 128;  // bytes of a row along k
constexpr int kDeep = 64;    // k of a slice of bf16

static inline int pv_slices(int n, int per) { return (n + per - 1) / per; }
static inline size_t pv_up(size_t n, size_t to) { return (n + to - 1) / to * to; }

struct PvPanel {  // rows at p + part * part_bytes + row * pitch
    const uint8_t* p;
    size_t pitch, part_bytes;
    int parts;
    int rows;  // that may be read (used across k)
    size_t slice_bytes;  // from one slice to the next (along k)
};
struct PvProduct {
    PvPanel a, b;
    int M, N, slices;
    int pairs;
    uint32_t pa, pb;     // pair t multiplies part (pa >> 4t) & 15 of a by that of b
    int size;            // PvSize
    int splits, per;     // slices (of all pairs) a split; partial sums where splits > 1
    float us;            // that the plan is expected to take
    uint32_t* partial;   // [splits][M][N], 32-bit words
    uint32_t first, count;  // the tiles of this launch (pv_run_tiles)
};

// The pairs of parts of two operands that a product needs: to 24 bits, or to 16 where
// neither has three parts. The smallest products come first, the first parts' last: their
// sum alone is rounded at its size.
static inline void pv_pairs(PvProduct& p, int parts_a, int parts_b) {
    p.pairs = 0;
    p.pa = p.pb = 0;
    const int orders = parts_a < 3 && parts_b < 3 ? 2 : 3;
    for (int order = orders - 1; order >= 0; order--)
        for (int i = 0; i <= order; i++) {
            const int j = order - i;
            if (i >= parts_a || j >= parts_b) continue;
            p.pa |= (uint32_t)i << (4 * p.pairs);
            p.pb |= (uint32_t)j << (4 * p.pairs);
            p.pairs++;
        }
}

// Tiles: WM x WN waves of 16 MI rows by 64 columns each; ST stages of slices in LDS, ST -
// 1 of them under way while one is multiplied. What a slice takes, beside what the matrix
// cores need for it, is the way of 32 to 64 KB from the L2 into LDS and a barrier: the more
// products a byte feeds, the nearer to their rate (bf16, us: 8192 x 5003 -> 2048 129 in
// tiles of 256 x 256, 1.3 PFLOP/s, 152, 221 and 358 in the smaller ones); few tiles need
// the small ones to fill the chip (1024 x 1024 x 1024: 27, 17, 13 and 9.6). 128 x 64 would
// never be faster than 64 x 64, of which two fit a CU: 0.43 us a slice for 0.42.
template <int WM_, int WN_, int MI_, int ST_, int PER_CU_>
struct PvTile {
    static constexpr int WM = WM_, WN = WN_, MI = MI_, ST = ST_;
    static constexpr int TM = WM * MI * 16, TN = WN * 64, kThreads = 64 * WM * WN;
    static constexpr int kWorkgroups = 256 * PER_CU_;  // that the chip holds at once
};
typedef PvTile<2, 4, 8, 2, 1> PvTileL;  // 256 x 256
typedef PvTile<4, 2, 4, 3, 1> PvTileG;  // 256 x 128
typedef PvTile<2, 2, 4, 4, 1> PvTileM;  // 128 x 128
typedef PvTile<2, 1, 2, 4, 2> PvTileS;  // 64 x 64
typedef PvTile<4, 1, 1, 3, 1> PvTileP;  // 64 x 64, all parts of a slice in a stage
enum PvSize { kPvS, kPvM, kPvG, kPvL, kPvP };
constexpr unsigned kPvAnySize = 31;  // 1 << each

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

// LDS holds an operand along k as [row][128 bytes], its 16-byte pieces at piece ^
// key(row): the rows that eight neighbouring lanes read lie in different banks. (Of a
// those are consecutive, of b the rows 32 (j >> 1) + 8 (r >> 2) + 4 (j & 1) + (r & 3),
// which leaves a lane two runs of eight columns of the result.) An operand across k is
// [k][columns], its 32-byte chunks (sixteen columns) at chunk ^ key(k): a transposing load
// takes 32 bytes of sixteen k's.
__device__ __forceinline__ int pv_key_a(int row) { return row & 7; }
__device__ __forceinline__ int pv_key_b(int row) { return (row & 3) | ((row >> 1) & 4); }
template <int COLS>
__device__ __forceinline__ int pv_key_across(int k) {
    return COLS >= 128 ? (k & 3) | ((k >> 1) & 4) : ((k >> 1) & 1) | ((k >> 2) & 2);
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

// Workgroup barrier between the stages' uses: what it orders has been waited for (by
// pv_wait_loads), so that it waits for nothing itself. (A fence would wait for every load
// into LDS under way, whichever stage it fills.)
__device__ __forceinline__ void pv_stage_barrier() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("" ::: "memory");
}

// Where the loads of an operand's slices come from: SIZE rows (columns, across k) from
// `at` on of the `limit` that it has, Q loads of 16 bytes a lane.
// Every address is one of the workgroup's and 32 bits of a lane's (kPvMostPitch), which
// costs no vector instruction a load.
constexpr size_t kPvMostPitch = ((size_t)1 << 32) / 256 - 256;
template <bool ACROSS, bool B, int SIZE, int THREADS>
struct PvSource {
    static constexpr int Q = SIZE * 8 / THREADS;
    static constexpr int kPieces = ACROSS ? SIZE / 8 : 8;  // of a row in LDS
    const uint8_t* base;
    uint32_t off[Q];
    __device__ __forceinline__ static int row_of(int q, int wave, int lane) {
        return ((wave * Q + q) * 64 + lane) / kPieces;
    }
    __device__ __forceinline__ void enter(const PvPanel& p, int at, int limit, int wave,
                                          int lane) {
        base = p.p + (ACROSS ? (size_t)at * 2 : (size_t)at * p.pitch);
#pragma unroll
        for (int q = 0; q < Q; q++) {
            const int row = row_of(q, wave, lane), c = lane % kPieces;
            if constexpr (ACROSS) {
                const int col = ((((c >> 1) ^ pv_key_across<SIZE>(row)) << 1) + (c & 1)) * 8;
                off[q] = (uint32_t)row * (uint32_t)p.pitch +
                         (uint32_t)min(col, ((limit + 7) & ~7) - 8 - at) * 2;
            } else {
                const int key = B ? pv_key_b(row) : pv_key_a(row);
                off[q] = (uint32_t)min(row, limit - 1 - at) * (uint32_t)p.pitch + (c ^ key) * 16;
            }
        }
    }
    // where a slice lies
    __device__ __forceinline__ const uint8_t* slice(const PvPanel& p, int part, int k) const {
        return base + part * p.part_bytes +
               (size_t)k * (ACROSS ? kDeep * p.pitch : p.slice_bytes);
    }
    // where load q of slice k lies in it
    __device__ __forceinline__ uint32_t offset(const PvPanel& p, int k, int q, int wave,
                                               int lane) const {
        uint32_t o = off[q];
        if constexpr (ACROSS) {  // rows past the last are read as that one
            const int past = k * kDeep + row_of(q, wave, lane) - (p.rows - 1);
            if ((k + 1) * kDeep > p.rows) o -= (uint32_t)max(past, 0) * (uint32_t)p.pitch;
        }
        return o;
    }
    __device__ __forceinline__ static void load(const uint8_t* from, uint32_t o, int q, int wave,
                                                uint8_t* lds) {
        __builtin_amdgcn_global_load_lds(
            (const void __attribute__((address_space(1)))*)(from + o),
            (void __attribute__((address_space(3)))*)(lds + (wave * Q + q) * 1024), 16, 0, 0);
    }
};

// The matrix operand of a lane out of an operand across k: eight k's of one of sixteen
// columns, whose four groups of four begin at the columns `col` of the lanes 0 .. 3.
template <int COLS>
__device__ __forceinline__ int pv_across_at(int k, int col) {
    return k * (COLS * 2) + (((col >> 4) ^ pv_key_across<COLS>(k)) << 5) + (col & 15) * 2;
}
template <int COLS>
__device__ __forceinline__ pv_u32x4 pv_load_across_at(const uint8_t* lds, const int (&at)[2]) {
    pv_u32x4 v;
#pragma unroll
    for (int s = 0; s < 2; s++) {
        const pv_s16x4 t = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (pv_s16x4 __attribute__((address_space(3)))*)(lds + at[s]));
        uint32_t u[2];
        __builtin_memcpy(u, &t, 8);
        v[2 * s] = u[0];
        v[2 * s + 1] = u[1];
    }
    return v;
}
template <int COLS>
__device__ __forceinline__ pv_u32x4 pv_load_across(const uint8_t* lds, int k0, int col, int lane) {
    const int k = k0 + 8 * (lane >> 4) + ((lane >> 2) & 3);
    const int at[2] = {pv_across_at<COLS>(k, col), pv_across_at<COLS>(k + 4, col)};
    return pv_load_across_at<COLS>(lds, at);
}

// a split's sums of a wave's tile
template <int MI, class Acc>
__device__ __forceinline__ void pv_store_partial(const PvProduct& p, int split, int mw, int nw,
                                                 int lane, const Acc (&acc)[4][MI]) {
    uint32_t* part = p.partial + (size_t)split * p.M * p.N;
    const int r = lane & 15, h = lane >> 4;
#pragma unroll
    for (int i = 0; i < MI; i++) {
        const int m = mw + 16 * i + r;
        if (m >= p.M) continue;
#pragma unroll
        for (int j = 0; j < 4; j++) {
            const int n = nw + 32 * (j >> 1) + 8 * h + 4 * (j & 1);
            uint32_t* o = part + (size_t)m * p.N + n;
            pv_u32x4 v;
            __builtin_memcpy(&v, &acc[j][i], 16);
            if (n + 4 <= p.N)
                *(pv_u32x4_any*)o = v;
            else
#pragma unroll
                for (int e = 0; e < 4; e++)
                    if (n + e < p.N) o[e] = v[e];
        }
    }
}

// Stages, arrays of their own in LDS: the loads into one are then seen not to touch what is
// read of another, and are not waited for.
struct PvStages {
    uint8_t *a0, *a1, *a2, *a3, *b0, *b1, *b2, *b3;
};

// The epilogue gets acc[j][i][e]: row mw + 16 i + r, column nw + 32 (j >> 1) + 8 h + 4
// (j & 1) + e (r = lane & 15, h = lane >> 4). A workgroup takes several tiles in turn: the
// first slices of the next one are under way during the epilogue.
template <bool I8, bool TA, bool TB, class T, class Epi>
__device__ __forceinline__ void pv_product_tiles(const PvProduct& p, const Epi& epi,
                                                 uint32_t block, uint32_t blocks,
                                                 const PvStages& lds) {
    static_assert(!I8 || (!TA && !TB), "the transposing loads are of 16 bits");
    constexpr int ST = T::ST;
    uint8_t *const la0 = lds.a0, *const la1 = lds.a1, *const la2 = lds.a2, *const la3 = lds.a3;
    uint8_t *const lb0 = lds.b0, *const lb1 = lds.b1, *const lb2 = lds.b2, *const lb3 = lds.b3;
    typedef typename PvAcc<I8>::type Acc;
    constexpr int MI = T::MI;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lane = threadIdx.x & 63, r = lane & 15, h = lane >> 4;
    const int wm = wave % T::WM * (16 * MI), wn = wave / T::WM * 64;
    // each XCD (workgroups go round them) takes a run of the launch's tiles
    const uint32_t run = (p.count + 7) / 8, step = blocks >> 3;
    const uint32_t end = min(run * ((block & 7) + 1), p.count);
    uint32_t idx = run * (block & 7) + (block >> 3);
    if (idx >= end) return;

    int split, m0, n0, t0, t1, pair, k;
    PvSource<TA, false, T::TM, T::kThreads> from_a;
    PvSource<TB, true, T::TN, T::kThreads> from_b;
    constexpr int QA = decltype(from_a)::Q, QB = decltype(from_b)::Q, Q = QA + QB;
    auto enter = [&]() {
        pv_tile_of<T>(p, p.first + idx, split, m0, n0);
        t0 = split * p.per;
        t1 = min(t0 + p.per, p.slices * p.pairs);
        pair = t0 / max(p.slices, 1);
        k = t0 - pair * p.slices;
        from_a.enter(p.a, m0, p.M, wave, lane);
        from_b.enter(p.b, n0, p.N, wave, lane);
    };
    // The loads of a slice, one at a time: where it lies, load q of Q, on to the next one.
    const uint8_t *slice_a, *slice_b;
    auto fetch_begin = [&]() {
        slice_a = from_a.slice(p.a, (p.pa >> (4 * pair)) & 15, k);
        slice_b = from_b.slice(p.b, (p.pb >> (4 * pair)) & 15, k);
    };
    auto fetch_one = [&](auto q, uint8_t* la, uint8_t* lb) {
        if constexpr (q < QA)
            from_a.load(slice_a, from_a.offset(p.a, k, q, wave, lane), q, wave, la);
        else
            from_b.load(slice_b, from_b.offset(p.b, k, q - QA, wave, lane), q - QA, wave, lb);
    };
    auto fetch_end = [&]() {
        if (++k == p.slices) {
            k = 0;
            pair = pair + 1 < p.pairs ? pair + 1 : 0;
        }
    };
    auto fetch = [&](uint8_t* la, uint8_t* lb) {
        fetch_begin();
        pv_each<Q>([&](auto q) { fetch_one(q, la, lb); });
        fetch_end();
        __builtin_amdgcn_sched_barrier(0);  // in this order: they are waited for by count
    };
    // The first ST - 1 slices of a tile. (Some of other slices, where it has fewer: loads
    // that may not have been issued would be waited for with all others.)
    auto first = [&]() {
        if (t0 >= t1) return;
        fetch(la0, lb0);
        if constexpr (ST > 2) fetch(la1, lb1);
        if constexpr (ST > 3) fetch(la2, lb2);
    };
    auto load_a = [&](const uint8_t* la, int i, int half) {
        if constexpr (TA) {
            return pv_load_across<T::TM>(la, 32 * half, wm + 16 * i + 4 * (lane & 3), lane);
        } else {
            const int row = wm + 16 * i + r;
            return *(const pv_u32x4*)(la + row * kSlice + ((h + 4 * half) ^ pv_key_a(row)) * 16);
        }
    };
    auto load_b = [&](const uint8_t* lb, int j, int half) {
        if constexpr (TB) {
            return pv_load_across<T::TN>(
                lb, 32 * half, wn + 32 * (j >> 1) + 8 * (lane & 3) + 4 * (j & 1), lane);
        } else {
            const int row = wn + 32 * (j >> 1) + 8 * (r >> 2) + 4 * (j & 1) + (r & 3);
            return *(const pv_u32x4*)(lb + row * kSlice + ((h + 4 * half) ^ pv_key_b(row)) * 16);
        }
    };
    enter();
    first();
    for (;;) {
        Acc acc[4][MI];
#pragma unroll
        for (int j = 0; j < 4; j++)
#pragma unroll
            for (int i = 0; i < MI; i++) acc[j][i] = Acc{0, 0, 0, 0};
        // The products of a slice in la, lb; `between` goes between them.
        auto multiply = [&](const uint8_t* la, const uint8_t* lb, auto between) {
            pv_u32x4 fa[MI], fb[4];
            pv_each<4>([&](auto j) { fb[j] = load_b(lb, j, 0); });
            pv_each<MI>([&](auto i) { fa[i] = load_a(la, i, 0); });
            pv_each<2>([&](auto half) {
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
                        if constexpr (i == MI - 1)
                            pv_each<4>([&](auto j) { fb[j] = load_b(lb, j, 1); });
                        fa[i] = load_a(la, i, 1);
                        between(i);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                });
            });
        };
        // A slice in la, lb, while na, nb, read before the barrier, take the one ST - 1 on.
        // Its loads go between the products: at once, they would hold every wave up for the
        // time that they take to be issued.
        auto steady = [&](const uint8_t* la, const uint8_t* lb, uint8_t* na, uint8_t* nb) {
            pv_wait_loads<(ST - 2) * Q>();  // this wave's part of the slice has landed
            pv_stage_barrier();
            fetch_begin();
            multiply(la, lb, [&](auto i) {
                constexpr int q0 = i * Q / MI, q1 = (i + 1) * Q / MI;
                pv_each<q1 - q0>([&](auto q) {
                    fetch_one(std::integral_constant<int, q0 + q>(), na, nb);
                });
            });
            fetch_end();
        };
        // one of the last slices of a tile, which may have no later one to load
        auto last = [&](int t, const uint8_t* la, const uint8_t* lb, uint8_t* na, uint8_t* nb) {
            if (t >= t1) return;
            pv_wait_loads<0>();
            pv_stage_barrier();
            if (t + ST - 1 < t1) fetch(na, nb);
            multiply(la, lb, [](auto) {});
        };
        // either, where the sums leave no registers for two forms of the loop
        auto any = [&](int t, const uint8_t* la, const uint8_t* lb, uint8_t* na, uint8_t* nb) {
            if (t >= t1) return;
            pv_wait_loads<0>();
            pv_stage_barrier();
            const bool more = t + 1 < t1;
            if (more) fetch_begin();
            multiply(la, lb, [&](auto i) {
                constexpr int q0 = i * Q / MI, q1 = (i + 1) * Q / MI;
                if (more)
                    pv_each<q1 - q0>([&](auto q) {
                        fetch_one(std::integral_constant<int, q0 + q>(), na, nb);
                    });
            });
            if (more) fetch_end();
        };
        int t = t0;
        if constexpr (ST == 2) {
            for (; t < t1; t += 2) {
                any(t, la0, lb0, la1, lb1);
                any(t + 1, la1, lb1, la0, lb0);
            }
        } else if constexpr (ST == 3) {
            for (; t + 4 < t1; t += 3) {
                steady(la0, lb0, la2, lb2);
                steady(la1, lb1, la0, lb0);
                steady(la2, lb2, la1, lb1);
            }
            last(t, la0, lb0, la2, lb2);
            last(t + 1, la1, lb1, la0, lb0);
            last(t + 2, la2, lb2, la1, lb1);
            last(t + 3, la0, lb0, la2, lb2);
        } else {
            for (; t + 6 < t1; t += 4) {
                steady(la0, lb0, la3, lb3);
                steady(la1, lb1, la0, lb0);
                steady(la2, lb2, la1, lb1);
                steady(la3, lb3, la2, lb2);
            }
            for (; t < t1; t += 4) {
                last(t, la0, lb0, la3, lb3);
                last(t + 1, la1, lb1, la0, lb0);
                last(t + 2, la2, lb2, la1, lb1);
                last(t + 3, la3, lb3, la2, lb2);
            }
        }
        const int em = m0 + wm, en = n0 + wn, es = split;
        idx += step;
        const bool more = idx < end;
        if (more) {
            pv_wait_loads<63>();
            pv_stage_barrier();  // nothing reads the stages any more
            enter();
            first();
        }
        if (p.splits > 1) {
            pv_store_partial<MI>(p, es, em, en, lane, acc);
        } else {
            epi.template tile<MI>(p, em, en, lane, acc);
        }
        if (!more) return;
    }
}
template <bool I8, bool TA, bool TB, class T, class Epi>
__global__ __launch_bounds__(T::kThreads, T::kThreads* T::kWorkgroups / 256 / 256) void
pv_product_kernel(PvProduct p, Epi epi) {
    constexpr int SA = T::TM * kSlice, SB = T::TN * kSlice, ST = T::ST;
    __shared__ __align__(16) uint8_t la0[SA], la1[SA], la2[ST > 2 ? SA : 16], la3[ST > 3 ? SA : 16];
    __shared__ __align__(16) uint8_t lb0[SB], lb1[SB], lb2[ST > 2 ? SB : 16], lb3[ST > 3 ? SB : 16];
    pv_product_tiles<I8, TA, TB, T>(p, epi, blockIdx.x, gridDim.x,
                                    PvStages{la0, la1, la2, la3, lb0, lb1, lb2, lb3});
}

// The same product in tiles of 64 x 64 whose stages hold every part of a slice: a step of
// 64 k's is one barrier for all pairs of parts (999 x 323 x 1003 in 32 bits: 36 steps of a
// pair each took 16 us), and a part is loaded once for all pairs that it is in. A step
// of three by three parts takes 1.2 us, its products 0.3: 48 KB go into LDS for it, and
// 120 KB out of it.
template <bool TA, bool TB, int PA, int PB, class Epi>
__device__ __forceinline__ void pv_parts_tiles(const PvProduct& p, const Epi& epi, uint32_t block,
                                               uint32_t blocks, const PvStages& lds) {
    typedef PvTileP T;
    uint8_t *const la0 = lds.a0, *const la1 = lds.a1, *const la2 = lds.a2;
    uint8_t *const lb0 = lds.b0, *const lb1 = lds.b1, *const lb2 = lds.b2;
    constexpr int SA = T::TM * kSlice, SB = T::TN * kSlice, MI = T::MI;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lane = threadIdx.x & 63, r = lane & 15, h = lane >> 4;
    const int wm = wave * 16;
    const uint32_t run = (p.count + 7) / 8, step = blocks >> 3;
    const uint32_t end = min(run * ((block & 7) + 1), p.count);
    uint32_t idx = run * (block & 7) + (block >> 3);
    if (idx >= end) return;
    int split, m0, n0, k, k1;
    PvSource<TA, false, T::TM, T::kThreads> from_a;
    PvSource<TB, true, T::TN, T::kThreads> from_b;
    constexpr int QA = decltype(from_a)::Q, QB = decltype(from_b)::Q;
    auto enter = [&]() {
        pv_tile_of<T>(p, p.first + idx, split, m0, n0);
        k = split * p.per / p.pairs;  // (whole steps)
        k1 = min(k + p.per / p.pairs, p.slices);
        from_a.enter(p.a, m0, p.M, wave, lane);
        from_b.enter(p.b, n0, p.N, wave, lane);
    };
    auto fetch = [&](int at, uint8_t* la, uint8_t* lb) {
        pv_each<QA>([&](auto q) {
            const uint32_t o = from_a.offset(p.a, at, q, wave, lane);
            pv_each<PA>([&](auto part) {
                from_a.load(from_a.slice(p.a, part, at), o, q, wave, la + part * SA);
            });
        });
        pv_each<QB>([&](auto q) {
            const uint32_t o = from_b.offset(p.b, at, q, wave, lane);
            pv_each<PB>([&](auto part) {
                from_b.load(from_b.slice(p.b, part, at), o, q, wave, lb + part * SB);
            });
        });
    };
    // Where a lane's values of either half of a slice lie, as numbers that the compiler does
    // not take apart: behind a chain of more than four sums it no longer sees which array is
    // read, and waits for the loads into every other one.
    static_assert(T::TM == 64 && T::TN == 64, "keys of k's bits 1 and 3");
    auto whole = [](int at) {
        asm("" : "+v"(at));
        return at;
    };
    auto across = [&](int half, int col) {
        return whole(pv_across_at<64>(32 * half + 8 * h + ((lane >> 2) & 3), col));
    };
    auto along = [&](int half, int row, int key) {
        return whole(row * kSlice + ((h + 4 * half) ^ key) * 16);
    };
    int at_a[2], at_b[2][4];
    pv_each<2>([&](auto half) {
        const int row = wm + r;
        at_a[half] = TA ? across(half, wm + 4 * (lane & 3)) : along(half, row, pv_key_a(row));
        pv_each<4>([&](auto j) {
            const int row = 32 * (j >> 1) + 8 * (r >> 2) + 4 * (j & 1) + (r & 3);
            at_b[half][j] = TB ? across(half, 32 * (j >> 1) + 8 * (lane & 3) + 4 * (j & 1))
                               : along(half, row, pv_key_b(row));
        });
    });
    auto load_operand = [](auto is_across, const uint8_t* lds, int at) {
        if constexpr (is_across) {
            const int four[2] = {at, at + 4 * 128};
            return pv_load_across_at<64>(lds, four);
        } else {
            return *(const pv_u32x4*)(lds + at);
        }
    };
    auto load_a = [&](const uint8_t* la, int half) {
        return load_operand(std::integral_constant<bool, TA>(), la, at_a[half]);
    };
    auto load_b = [&](const uint8_t* lb, int j, int half) {
        return load_operand(std::integral_constant<bool, TB>(), lb, at_b[half][j]);
    };
    // (of a single step, a second one: see pv_product_tiles)
    auto first = [&]() {
        if (k >= k1) return;
        fetch(k, la0, lb0);
        __builtin_amdgcn_sched_barrier(0);  // in this order: they are waited for by count
        fetch(min(k + 1, p.slices - 1), la1, lb1);
    };
    enter();
    first();
    for (;;) {
        // the sums of first parts, and of the others, whose digits would be lost in them
        pv_f32x4 acc[4][MI], rest[4];
#pragma unroll
        for (int j = 0; j < 4; j++) acc[j][0] = rest[j] = pv_f32x4{0.f, 0.f, 0.f, 0.f};
        constexpr int kOrders = PA < 3 && PB < 3 ? 2 : 3;  // as pv_pairs
        auto multiply = [&](const uint8_t* la, const uint8_t* lb) {
            pv_each<2>([&](auto half) {
                pv_u32x4 fa[PA], fb[PB][4];
                pv_each<PA>([&](auto i) { fa[i] = load_a(la + i * SA, half); });
                pv_each<PB>([&](auto i) {
                    pv_each<4>([&](auto j) { fb[i][j] = load_b(lb + i * SB, j, half); });
                });
                pv_each<PA>([&](auto x) {
                    pv_each<PB>([&](auto y) {
                        if constexpr (x + y < kOrders)
                            pv_each<4>([&](auto j) {
                                pv_b16x8 va, vb;
                                __builtin_memcpy(&va, &fa[x], 16);
                                __builtin_memcpy(&vb, &fb[y][j], 16);
                                pv_f32x4& to = x + y == 0 ? acc[j][0] : rest[j];
                                to = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vb, va, to, 0, 0, 0);
                            });
                    });
                });
            });
            k++;
        };
        auto steady = [&](const uint8_t* la, const uint8_t* lb, uint8_t* na, uint8_t* nb) {
            pv_wait_loads<PA * QA + PB * QB>();  // all but those of the next step
            pv_stage_barrier();
            fetch(k + 2, na, nb);
            multiply(la, lb);
        };
        auto last = [&](const uint8_t* la, const uint8_t* lb, uint8_t* na, uint8_t* nb) {
            if (k >= k1) return;
            pv_wait_loads<0>();
            pv_stage_barrier();
            if (k + 2 < k1) fetch(k + 2, na, nb);
            multiply(la, lb);
        };
        while (k + 4 < k1) {
            steady(la0, lb0, la2, lb2);
            steady(la1, lb1, la0, lb0);
            steady(la2, lb2, la1, lb1);
        }
        last(la0, lb0, la2, lb2);
        last(la1, lb1, la0, lb0);
        last(la2, lb2, la1, lb1);
        last(la0, lb0, la2, lb2);
#pragma unroll
        for (int j = 0; j < 4; j++) acc[j][0] += rest[j];
        const int em = m0 + wm, en = n0, es = split;
        idx += step;
        const bool more = idx < end;
        if (more) {
            pv_wait_loads<0>();  // (none is: for the compiler's count of them)
            pv_stage_barrier();  // nothing reads the stages any more
            enter();
            first();
        }
        if (p.splits > 1)
            pv_store_partial<MI>(p, es, em, en, lane, acc);
        else
            epi.template tile<MI>(p, em, en, lane, acc);
        if (!more) return;
    }
}

template <bool TA, bool TB, int PA, int PB, class Epi>
__global__ __launch_bounds__(PvTileP::kThreads, 1) void pv_parts_kernel(PvProduct p, Epi epi) {
    constexpr int SA = PA * PvTileP::TM * kSlice, SB = PB * PvTileP::TN * kSlice;
    __shared__ __align__(16) uint8_t la0[SA], la1[SA], la2[SA], lb0[SB], lb1[SB], lb2[SB];
    pv_parts_tiles<TA, TB, PA, PB>(p, epi, blockIdx.x, gridDim.x,
                                   PvStages{la0, la1, la2, nullptr, lb0, lb1, lb2, nullptr});
}

// Sixteen values of columns, as a lane has them: `none` from N on, or where there are none.
__device__ __forceinline__ void pv_load_columns(const float* from, int nb, int N, float none,
                                                float (&v)[16]) {
#pragma unroll
    for (int a = 0; a < 2; a++) {
        const int n = nb + 32 * a;
        if (from && n + 8 <= N) {
            const pv_u32x4 x = *(const pv_u32x4_any*)(from + n),
                           y = *(const pv_u32x4_any*)(from + n + 4);
#pragma unroll
            for (int i = 0; i < 8; i++) v[8 * a + i] = __uint_as_float(i < 4 ? x[i] : y[i - 4]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; i++)
                v[8 * a + i] = n + i < N ? (from ? from[n + i] : 0.f) : none;
        }
    }
}
// The column of value q (of sixteen) of a lane whose first one is nb = nw + 8 h: acc[q >>
// 2][i][q & 3].
__device__ __forceinline__ int pv_col(int nb, int q) { return nb + 32 * (q >> 3) + (q & 7); }

// A lane's sixteen values of a row, two runs of eight, wherever the row begins.
__device__ __forceinline__ void pv_store_runs(const PvRows& out, int m, int nb, int N,
                                              const float (&v)[16]) {
#pragma unroll
    for (int a = 0; a < 2; a++) {
        const int n = nb + 32 * a;
        const size_t at = (size_t)m * out.ld + n;
        const bool whole = n + 8 <= N;
        if (out.bf16) {
            uint16_t* o = (uint16_t*)out.p + at;
            if (whole) {
                pv_u32x4 w;
#pragma unroll
                for (int i = 0; i < 4; i++)
                    w[i] = pv_pack_bf16x2(v[8 * a + 2 * i], v[8 * a + 2 * i + 1]);
                *(pv_u32x4_any*)o = w;
            } else {
#pragma unroll
                for (int i = 0; i < 8; i++)
                    if (n + i < N) o[i] = pv_f32_to_bf16(v[8 * a + i]);
            }
        } else {
            float* o = (float*)out.p + at;
            if (whole) {
#pragma unroll
                for (int i = 0; i < 8; i += 4)
                    *(pv_u32x4_any*)(o + i) = pv_u32x4{
                        __float_as_uint(v[8 * a + i]), __float_as_uint(v[8 * a + i + 1]),
                        __float_as_uint(v[8 * a + i + 2]), __float_as_uint(v[8 * a + i + 3])};
            } else {
#pragma unroll
                for (int i = 0; i < 8; i++)
                    if (n + i < N) o[i] = v[8 * a + i];
            }
        }
    }
}

// ---- tiles and splits ------------------------------------------------------
static inline size_t pv_tiles_of(int M, int N, int tm, int tn) {
    return (size_t)((M + tm - 1) / tm) * ((N + tn - 1) / tn);
}
// The tiles that a product takes and how many ways its slices are split, by the time that
// each choice is expected to take: rounds of workgroups, each its slices and an epilogue,
// and the splits' sums written, read and joined. The times a slice and the rest are fitted
// to unsplit products in every size of tile. (512 x 2304 by 32768 deep, us: 256 x 128 in
// seven 85, 256 x 256 in twelve 90, unsplit 242 to 724; 4096 x 512 by 49999: 256 x 256 in
// eight 202, unsplit 404 to 1230; 8192 x 5003 -> 2048: unsplit 129, in two 212.)
struct PvSizeCost {
    int size, tm, tn, slots;
    float slice, rest;  // us
};
static constexpr PvSizeCost kPvCosts[] = {
    {kPvL, PvTileL::TM, PvTileL::TN, PvTileL::kWorkgroups, 1.4f, 6.f},
    {kPvG, PvTileG::TM, PvTileG::TN, PvTileG::kWorkgroups, 0.82f, 4.5f},
    {kPvM, PvTileM::TM, PvTileM::TN, PvTileM::kWorkgroups, 0.62f, 3.5f},
    {kPvS, PvTileS::TM, PvTileS::TN, PvTileS::kWorkgroups, 0.42f, 3.f},
};
// The pairs of operands that PvTileP is built for.
static constexpr bool pv_all_parts(int a, int b) {
    return (a == 3 && (b == 3 || b == 1)) || (a == 1 && b == 3);
}
static inline PvSizeCost pv_parts_cost(int pairs) {
    return PvSizeCost{kPvP, PvTileP::TM, PvTileP::TN, PvTileP::kWorkgroups,
                      pairs > 3 ? 0.18f : 0.22f, 3.f};
}
static inline void pv_plan(PvProduct& p, bool may_split, unsigned sizes = kPvAnySize) {
    const int all = p.slices * p.pairs;
    float best = 0.f;
    auto choose = [&](const PvSizeCost& c) {
        const size_t tiles = pv_tiles_of(p.M, p.N, c.tm, c.tn);
        // (split no further than one round of workgroups, and into runs of four slices)
        for (int n = 1; n == 1 || (may_split && tiles * (size_t)(n - 1) < (size_t)c.slots &&
                                   all / n >= 4);
             n += n < 8 ? 1 : n / 4) {
            int per = n == 1 ? all : (all + n - 1) / n;
            if (c.size == kPvP) per = (per + p.pairs - 1) / p.pairs * p.pairs;  // whole steps
            const int splits = per ? (all + per - 1) / per : 1;
            const size_t rounds = (tiles * splits + c.slots - 1) / c.slots;
            float us = (float)rounds * ((float)per * c.slice + c.rest);
            if (splits > 1) us += 4.f + (float)splits * (float)p.M * (float)p.N * (8.f / 4e6f);
            if (best == 0.f || us < best) {
                best = us;
                p.size = c.size;
                p.per = per;
                p.splits = splits;
                p.us = us;
            }
        }
    };
    for (const PvSizeCost& c : kPvCosts)
        if (sizes >> c.size & 1) choose(c);
    if ((sizes >> kPvP & 1) && pv_all_parts(p.a.parts, p.b.parts) && p.pairs > 1)
        choose(pv_parts_cost(p.pairs));
}
static inline size_t pv_partial_bytes(const PvProduct& p) {
    return p.splits > 1 ? (size_t)p.splits * p.M * p.N * 4 : 0;
}

// The splits' sums in a fixed order, then epi.one(m, n, sum): 64 results a workgroup, whose
// four waves take a quarter of the splits each, eight loads in flight. (50 x 128 results of
// 103 splits, one thread a result: 15.8 us.)
template <bool I8, class Epi>
__device__ __forceinline__ void pv_join(const PvProduct& p, const Epi& epi, size_t block,
                                        size_t blocks) {
    constexpr int kAhead = 8;
    typedef typename std::conditional<I8, int, float>::type Sum;
    __shared__ Sum part[4][64];
    const size_t total = (size_t)p.M * p.N;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, quarter = (p.splits + 3) / 4;
    const int k0 = wave * quarter, k1 = min(k0 + quarter, p.splits);
    for (size_t at0 = block * 64; at0 < total; at0 += blocks * 64) {
        const size_t at = min(at0 + lane, total - 1);
        Sum s = 0;
        for (int k = k0; k < k1; k += kAhead) {
            uint32_t v[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; u++)
                v[u] = p.partial[(size_t)min(k + u, k1 - 1) * total + at];
#pragma unroll
            for (int u = 0; u < kAhead; u++)
                if (k + u < k1) {
                    if constexpr (I8)
                        s += (int)v[u];
                    else
                        s += __uint_as_float(v[u]);
                }
        }
        part[wave][lane] = s;
        __syncthreads();
        if (wave == 0 && at0 + lane < total) {
            const int m = (int)(at / p.N), n = (int)(at - (size_t)m * p.N);
            epi.one(m, n, ((part[0][lane] + part[1][lane]) + part[2][lane]) + part[3][lane]);
        }
        __syncthreads();
    }
}
template <bool I8, class Epi>
__global__ __launch_bounds__(256) void pv_join_kernel(PvProduct p, Epi epi) {
    pv_join<I8>(p, epi, blockIdx.x, gridDim.x);
}
static inline bool pv_join_narrow(const PvProduct& p) {
    return p.splits > 16 || (size_t)p.M * p.N < (1u << 18);
}
// The same where there are many results of few splits: four neighbours a thread.
template <bool I8, class Epi>
__global__ __launch_bounds__(256) void pv_join_wide_kernel(PvProduct p, Epi epi) {
    typedef typename std::conditional<I8, int, float>::type Sum;
    const size_t total = (size_t)p.M * p.N;
    for (size_t at = ((size_t)blockIdx.x * 256 + threadIdx.x) * 4; at < total;
         at += (size_t)gridDim.x * 1024) {
        const int n = (int)min((size_t)4, total - at);
        Sum s[4] = {0, 0, 0, 0};
#pragma unroll 4
        for (int k = 0; k < p.splits; k++) {
            const uint32_t* from = p.partial + (size_t)k * total + at;
            pv_u32x4 v = {0, 0, 0, 0};
            if (n == 4)
                v = *(const pv_u32x4_any*)from;
            else
                for (int u = 0; u < 3; u++)
                    if (u < n) v[u] = from[u];
#pragma unroll
            for (int u = 0; u < 4; u++) {
                if constexpr (I8)
                    s[u] += (int)v[u];
                else
                    s[u] += __uint_as_float(v[u]);
            }
        }
        int m = (int)(at / p.N), c = (int)(at - (size_t)m * p.N);
#pragma unroll
        for (int u = 0; u < 4; u++) {
            if (u >= n) break;
            epi.one(m, c, s[u]);
            if (++c == p.N) {
                c = 0;
                m++;
            }
        }
    }
}
static inline unsigned pv_blocks(size_t items, int per) {
    const size_t b = (items + per - 1) / per;
    return (unsigned)(b < 1 ? 1 : (b < (1u << 16) ? b : 1u << 16));
}

constexpr size_t kPvTilesALaunch = (size_t)1 << 30;
template <class T, class Kernel, class Epi>
static void pv_launch_tiles(Kernel kernel, PvProduct p, const Epi& epi, hipStream_t s) {
    const size_t tiles = pv_tiles_of(p.M, p.N, T::TM, T::TN) * p.splits;
    for (size_t t = 0; t < tiles; t += kPvTilesALaunch) {
        p.first = (uint32_t)t;
        p.count = (uint32_t)(tiles - t < kPvTilesALaunch ? tiles - t : kPvTilesALaunch);
        const unsigned most = (p.count + 7) / 8 * 8;
        hipLaunchKernelGGL(kernel, dim3(most < T::kWorkgroups ? most : T::kWorkgroups),
                           dim3(T::kThreads), 0, s, p, epi);
    }
}
template <bool I8, bool TA, bool TB, class T, class Epi>
static void pv_run_tiles(const PvProduct& p, const Epi& epi, hipStream_t s) {
    pv_launch_tiles<T>(pv_product_kernel<I8, TA, TB, T, Epi>, p, epi, s);
}
template <bool TA, bool TB, class Epi>
static void pv_run_parts(const PvProduct& p, const Epi& epi, hipStream_t s) {
    if (p.a.parts == 3 && p.b.parts == 3)
        pv_launch_tiles<PvTileP>(pv_parts_kernel<TA, TB, 3, 3, Epi>, p, epi, s);
    else if (p.a.parts == 3)
        pv_launch_tiles<PvTileP>(pv_parts_kernel<TA, TB, 3, 1, Epi>, p, epi, s);
    else if constexpr (!TB)  // (what lies across the sum as b follows an a of several parts)
        pv_launch_tiles<PvTileP>(pv_parts_kernel<TA, TB, 1, 3, Epi>, p, epi, s);
}

// SIZES: the tiles (1 << PvSize) that the plan may have chosen
template <bool I8, bool TA, bool TB, unsigned SIZES = kPvAnySize, class Epi>
static void pv_run_product(const PvProduct& p, const Epi& epi, hipStream_t s) {
    if constexpr (SIZES >> kPvL & 1)
        if (p.size == kPvL) pv_run_tiles<I8, TA, TB, PvTileL>(p, epi, s);
    if constexpr (SIZES >> kPvG & 1)
        if (p.size == kPvG) pv_run_tiles<I8, TA, TB, PvTileG>(p, epi, s);
    if constexpr (SIZES >> kPvM & 1)
        if (p.size == kPvM) pv_run_tiles<I8, TA, TB, PvTileM>(p, epi, s);
    if constexpr (SIZES >> kPvS & 1)
        if (p.size == kPvS) pv_run_tiles<I8, TA, TB, PvTileS>(p, epi, s);
    if constexpr (!I8 && (SIZES >> kPvP & 1))
        if (p.size == kPvP) pv_run_parts<TA, TB>(p, epi, s);
}
// The splits' sums of a product that has some.
template <bool I8, class Epi>
static void pv_run_join(const PvProduct& p, const Epi& epi, hipStream_t s) {
    if (p.splits <= 1) return;
    const size_t results = (size_t)p.M * p.N;
    if (pv_join_narrow(p))
        hipLaunchKernelGGL((pv_join_kernel<I8, Epi>), dim3(pv_blocks(results, 64)), dim3(256), 0, s,
                           p, epi);
    else
        hipLaunchKernelGGL((pv_join_wide_kernel<I8, Epi>), dim3(pv_blocks(results, 1024)),
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
    uint8_t* dst;            // [part][rows][pitch bytes], zeros from R and C on
    size_t pitch, part_bytes;
    int rows;
    float* sums;             // set: no rows of parts, but the sums of the source's columns
                             // over runs of `rows` rows, [runs][C]
};
// rows of a run, and how many there are (one: the sums are whole)
__host__ __device__ static inline int pv_sum_rows(int M) { return M <= 1024 ? 1024 : 256; }
__host__ __device__ static inline int pv_sum_runs(int M) { return (M + pv_sum_rows(M) - 1) / pv_sum_rows(M); }
// Up to five at once.
struct PvPacks {
    PvPack job[5];
    unsigned begin[6];  // the first workgroup of each
    int n;
    void add(const PvPack& k) { job[n++] = k; }
};
void pv_launch_packs(PvPacks& k, hipStream_t s);
// out (+)= the product of bf16 parts: out = sum + add (dense [M][N] fp32, or NULL); a along
// k or across it, b across it
struct PvPlain {
    PvRows out;
    const float* add;
};
// `sums`: column sums to be joined too, in the launch that joins the splits' sums if there
// is one.
struct PvSums {
    const float* runs;
    int n, N;
    float* out;  // or NULL: none
};
void pv_launch_plain(const PvProduct& p, bool a_across, const PvPlain& e, const PvSums& sums,
                     hipStream_t s);
// Two of them that do not depend on each other, x's a along k, y's across it, as one launch:
// the size of tile in which they are that (-1: none), and its plan, which either has when
// it is run alone too, so that its bits are the same.
int pv_pair_size(const PvProduct& x, const PvProduct& y);
void pv_take_pair(PvProduct& p, int size);
void pv_launch_pair(const PvProduct& x, const PvPlain& ex, const PvProduct& y, const PvPlain& ey,
                    const PvSums& sums, hipStream_t s);

// Sums [n][N] of runs joined in a fixed order.
void pv_launch_sum_runs(const PvSums& sums, hipStream_t s);

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
static inline PvPanel pv_take_panel(PvCarve& c, int rows, int cols, int parts) {
    PvPanel p;
    p.pitch = pv_up(cols, 64) * 2;
    p.part_bytes = pv_align256((size_t)rows * p.pitch);
    p.parts = parts;
    p.rows = rows;
    p.slice_bytes = kSlice;
    p.p = (const uint8_t*)c.take(p.part_bytes * parts);
    return p;
}
// Whether rows of C channels are an operand as they lie, and the operand that they are.
static inline bool pv_in_place(const PvRows& r, int C) {
    return r.bf16 && C % kDeep == 0 && r.ld % 8 == 0 && pv_aligned16(r.p) &&
           (size_t)r.ld * 2 <= kPvMostPitch;
}
static inline PvPanel pv_panel_of(const PvRows& r, int rows) {
    return PvPanel{(const uint8_t*)r.p, (size_t)r.ld * 2, 0, 1, rows, kSlice};
}
static inline PvPack pv_pack_of(const void* src, PvKind kind, size_t ld, int R, int C,
                                const PvPanel& to) {
    return PvPack{src, kind, ld, R, C, nullptr, nullptr, to.parts, (uint8_t*)to.p, to.pitch,
                  to.part_bytes, to.rows, nullptr};
}
static inline PvPack pv_sums_of(const PvRows& x, int R, int C, float* sums) {
    return PvPack{x.p, x.bf16 ? kPvBf16 : kPvF32, (size_t)x.ld, R, C, nullptr, nullptr, 0, nullptr,
                  0, 0, pv_sum_rows(R), sums};
}
