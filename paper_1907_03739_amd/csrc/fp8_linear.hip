// Linear layer in 8-bit floating point, a power-of-two scale for each block of
// 128 values, and its gradients (pvconv_train.h).
//
// With s_b = 2^e_b the scale of a block of 128 values and q = round(v / s_b) in
// e4m3: out[m][n] = act( sum over blocks b of s_b(m) s_b(n) q(m) . q(n) + bias_n ).
// The scaled matrix instruction of gfx950 (16x16x128) spans one block: it takes the
// blocks' two scales as they are, adds the block's products on a grid of the largest
// of them, and the blocks in fp32 (pv_fp8_tile_kernel has what that means for which
// outputs).
//
// A layer's forward and the gradient of its input quantise the rows of x or dy on
// their way into the product (pv_fp8_few_, _resident_, _fused_kernel: path_of has
// the rule); the weight's gradient, whose blocks run along the rows, takes them
// transposed out of the workspace (pv_fp8_quantise_, _tile_kernel).
#include <initializer_list>
#include <type_traits>

#include "pv_train.h"
#include "pv_wave.h"

namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));
constexpr int kThreads = 256;
constexpr int kB = PVCONV_FP8_BLOCK;

// The exponent e of a block whose largest finite magnitude has these bits:
// the smallest e >= -126 with top <= 448 * 2^e (448 = 1.75 * 2^8), 0 for 0.
__device__ __forceinline__ int block_exponent(uint32_t top) {
    if (top == 0) return 0;
    const int e = (int)(top >> 23) - 135 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0);
    return max(e, -126);
}
__device__ __forceinline__ float two_to(int e) { return __uint_as_float((uint32_t)(127 + e) << 23); }

// |v| for the block's largest: 0 for a value that is not finite
__device__ __forceinline__ uint32_t finite_bits(float v) {
    const uint32_t u = __float_as_uint(v) & 0x7fffffffu;
    return u < 0x7f800000u ? u : 0u;
}
// Four values of v / scale, a power of two, as e4m3 bytes: nearest, ties to even;
// what is not finite gives NaN.
typedef short i16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t pack_scaled(float a, float b, float c, float d, float scale) {
    i16x2 q = {0, 0};
    q = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(q, a, b, scale, false);
    q = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(q, c, d, scale, true);
    uint32_t r;
    __builtin_memcpy(&r, &q, 4);
    return r;
}

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
template <bool XB>
struct XVec {  // eight consecutive values of a row
    typedef u32x4 at_any __attribute__((aligned(2)));
    u32x4 w[XB ? 1 : 2];
    __device__ __forceinline__ float get(int i) const {
        if constexpr (XB)
            return __uint_as_float(i & 1 ? w[0][i / 2] & 0xffff0000u : w[0][i / 2] << 16);
        else
            return __uint_as_float(w[i / 4][i % 4]);
    }
    // The vector at column c0, or the row's last eight columns where it reaches
    // past them (K >= 8): no branch parts a block's loads.
    __device__ __forceinline__ void load(const PvRows& x, size_t row, int c0, int K) {
        const char* p = (const char*)x.p + (row * x.ld + min(c0, K - 8)) * (XB ? 2 : 4);
        w[0] = *(const at_any*)p;
        if constexpr (!XB) w[1] = *(const at_any*)(p + 16);
    }
    __device__ __forceinline__ void set(const uint32_t (&e)[8]) {  // bits of floats
#pragma unroll
        for (int i = 0; i < 8; i++) {
            if constexpr (!XB)
                w[i / 4][i % 4] = e[i];
            else
                w[0][i / 2] = i & 1 ? w[0][i / 2] | e[i] : e[i] >> 16;
        }
    }
    __device__ __forceinline__ void clear() {
        w[0] = u32x4{0, 0, 0, 0};
        if constexpr (!XB) w[1] = u32x4{0, 0, 0, 0};
    }
    // Values loaded `by` columns early: moved into place, zeros after the row's end.
    __device__ __forceinline__ void move_down(int by) {
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; i++) x[i] = get(i);
#pragma unroll
        for (int s = 4; s; s >>= 1) {
#pragma unroll
            for (int i = 0; i < 8; i++) x[i] = by & s ? (i + s < 8 ? x[i + s] : 0.f) : x[i];
        }
        uint32_t e[8];
#pragma unroll
        for (int i = 0; i < 8; i++) e[i] = by >= 8 ? 0u : __float_as_uint(x[i]);
        set(e);
    }
    // The largest magnitude's bits; at least infinity's where a value may not be
    // finite.
    __device__ __forceinline__ uint32_t top() const {
        if constexpr (XB) {
            typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
            u16x2 m = {0, 0};
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const uint32_t u = w[0][i] & 0x7fff7fffu;
                u16x2 v;
                __builtin_memcpy(&v, &u, 4);
                m = __builtin_elementwise_max(m, v);
            }
            return (uint32_t)(m[0] > m[1] ? m[0] : m[1]) << 16;
        } else {
            float m = 0.f;  // a NaN is passed over
#pragma unroll
            for (int i = 0; i < 8; i++) m = fmaxf(m, fabsf(get(i)));
            return __float_as_uint(m);
        }
    }
    __device__ __forceinline__ uint32_t finite_top() const {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 8; i++) m = max(m, finite_bits(get(i)));
        return m;
    }
    // The eight as e4m3 of v / scale, a power of two: nearest, ties to even; what
    // is not finite gives NaN.
    __device__ __forceinline__ uint2 bytes(float scale) const {
        i16x2 q[2] = {{0, 0}, {0, 0}};
#pragma unroll
        for (int i = 0; i < 2; i++) {
            if constexpr (XB) {
                bf16x2 a, b;
                const uint32_t u = w[0][2 * i], v = w[0][2 * i + 1];
                __builtin_memcpy(&a, &u, 4);
                __builtin_memcpy(&b, &v, 4);
                q[i] = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(q[i], a, scale, false);
                q[i] = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(q[i], b, scale, true);
            } else {
                q[i] = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(q[i], get(4 * i), get(4 * i + 1),
                                                                scale, false);
                q[i] = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(q[i], get(4 * i + 2),
                                                                get(4 * i + 3), scale, true);
            }
        }
        uint2 r;
        __builtin_memcpy(&r, q, 8);
        return r;
    }
};

// max over 16 consecutive lanes
template <int CTRL>
__device__ __forceinline__ uint32_t max_dpp(uint32_t v) {
    return max(v, dpp_u32<CTRL, 0xf>(v));
}

// The quantisers: a workgroup takes a tile of 128 x 128 into registers, eight
// columns by eight rows a thread, and writes it in any of
//   kRows    q[cb][r][128], scales per row and 128 columns: scale[cb][r]
//   kCols    qt[rb][c][128], scales per column and 128 rows: scale_t[rb][c]
//   kBlock   both as the weight's layouts, q[r][cb * 128 ..], qt[c][rb * 128 ..],
//            one scale for the tile: scale[rb][cb], scale_t[cb][rb]
//   kSum     sum[rb][c]: the tile's plain column sums
// (Block by block, a product's slices are whole: by rows, they would lie a
// power of two apart where M is one, on few of the memory's channels.)
// Bound by HBM: one read of x, a byte a value out; the transposed bytes turn
// around in LDS so that their stores are rows of 128 bytes. The columns of 32768 x
// 512 and 32768 x 2304 bf16: 184 MB read and 92 MB written in 57 us, 4.8 TB/s.
enum { kRows = 1, kCols = 2, kBlock = 4, kSum = 8 };  // kSum: where `sum` is set
struct Quantise {
    PvRows x;
    int M, C;      // rows, columns
    uint8_t* q;
    uint8_t* scale;
    uint8_t* qt;
    uint8_t* scale_t;
    float* sum;
};
// One launch quantises a's tiles, then b's (of b.x.p set).
struct QuantiseJobs {
    Quantise a, b;
    int tiles_a;
};
constexpr int kPitch = 33;  // dwords a transposed column in LDS (32 and one to spread the banks)

__device__ __forceinline__ uint32_t max_over_row16(uint32_t v) {  // 16 consecutive lanes
#pragma unroll
    for (int m = 1; m < 16; m <<= 1) v = max(v, (uint32_t)__shfl_xor((int)v, m));
    return v;
}

template <bool XB, bool NARROW, int WHAT>
__global__ __launch_bounds__(kThreads) void pv_fp8_quantise_kernel(QuantiseJobs jobs) {
    constexpr bool kT = (WHAT & (kCols | kBlock)) != 0;
    __shared__ uint32_t turn[kT ? kB * kPitch : 1];
    __shared__ uint32_t tops[4][kB];
    __shared__ float sums[(WHAT & kSum) ? 4 : 1][kB];
    const bool second = (int)blockIdx.x >= jobs.tiles_a;
    const Quantise z = second ? jobs.b : jobs.a;
    const int tile = (int)blockIdx.x - (second ? jobs.tiles_a : 0);
    const int cbs = pv_fp8_blocks(z.C), rbs = pv_fp8_blocks(z.M);
    const int rb = tile / cbs, cb = tile % cbs;
    const int wave = threadIdx.x >> 6, cg = threadIdx.x & 15, rg = threadIdx.x >> 4;
    const int c0 = cb * kB + cg * 8;
    // row of the tile: half * 64 + rg * 4 + j
    XVec<XB> x[8];
#pragma unroll
    for (int r = 0; r < 8; r++) {
        const int row = rb * kB + (r >> 2) * 64 + rg * 4 + (r & 3);
        const size_t from = min(row, z.M - 1);
        if constexpr (NARROW) {  // rows of fewer channels than a vector
            uint32_t e[8];
#pragma unroll
            for (int i = 0; i < 8; i++) {
                const float f = pv_load_one(z.x.p, XB, from * z.x.ld + min(c0 + i, z.C - 1));
                e[i] = c0 + i < z.C ? __float_as_uint(f) : 0u;
            }
            x[r].set(e);
        } else {
            x[r].load(z.x, from, c0, z.C);
        }
    }
    if (!NARROW && (cb + 1) * kB > z.C) {  // the row's last block
#pragma unroll
        for (int r = 0; r < 8; r++) x[r].move_down(max(c0 - (z.C - 8), 0));
    }
    if ((rb + 1) * kB > z.M) {  // rows past the last: zeros
#pragma unroll
        for (int r = 0; r < 8; r++)
            if (rb * kB + (r >> 2) * 64 + rg * 4 + (r & 3) >= z.M) x[r].clear();
    }
    if ((WHAT & kSum) && z.sum) {
        float t[8];
#pragma unroll
        for (int i = 0; i < 8; i++) {
            t[i] = 0.f;
#pragma unroll
            for (int r = 0; r < 8; r++) t[i] += x[r].get(i);
            t[i] += __shfl_xor(t[i], 16);
            t[i] += __shfl_xor(t[i], 32);
            if ((threadIdx.x & 48) == 0) sums[wave][cg * 8 + i] = t[i];
        }
    }
    if constexpr (WHAT & kRows) {
#pragma unroll
        for (int r = 0; r < 8; r++) {
            const int e = block_exponent(max_over_row16(x[r].finite_top()));
            const int row = rb * kB + (r >> 2) * 64 + rg * 4 + (r & 3);
            const uint2 w = x[r].bytes(two_to(e));
            if (row < z.M) {
                *(uint2*)(z.q + ((size_t)cb * z.M + row) * kB + cg * 8) = w;
                if (cg == 0) z.scale[(size_t)cb * z.M + row] = (uint8_t)(e + 127);
            }
        }
    }
    if constexpr (kT) {
#pragma unroll
        for (int i = 0; i < 8; i++) {
            uint32_t top = 0;
#pragma unroll
            for (int r = 0; r < 8; r++) top = max(top, finite_bits(x[r].get(i)));
            top = max(top, (uint32_t)__shfl_xor((int)top, 16));
            top = max(top, (uint32_t)__shfl_xor((int)top, 32));
            if ((threadIdx.x & 48) == 0) tops[wave][cg * 8 + i] = top;
        }
        __syncthreads();
        uint32_t all = 0;
        if constexpr (WHAT & kBlock) {
            const int l = threadIdx.x & 63;
#pragma unroll
            for (int w = 0; w < 4; w++) all = max(all, max(tops[w][l], tops[w][64 + l]));
#pragma unroll
            for (int m = 1; m < 64; m <<= 1) all = max(all, (uint32_t)__shfl_xor((int)all, m));
        }
        const int tile_e = block_exponent(all);
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const int c = cg * 8 + i;
            const int e = (WHAT & kBlock)
                              ? tile_e
                              : block_exponent(max(max(tops[0][c], tops[1][c]),
                                                   max(tops[2][c], tops[3][c])));
            const float f = two_to(e);
            turn[c * kPitch + rg] =
                pack_scaled(x[0].get(i), x[1].get(i), x[2].get(i), x[3].get(i), f);
            turn[c * kPitch + 16 + rg] =
                pack_scaled(x[4].get(i), x[5].get(i), x[6].get(i), x[7].get(i), f);
            if (!(WHAT & kBlock) && rg == 0 && cb * kB + c < z.C)
                z.scale_t[(size_t)rb * z.C + cb * kB + c] = (uint8_t)(e + 127);
        }
        if constexpr (WHAT & kBlock) {
#pragma unroll
            for (int r = 0; r < 8; r++) {
                const int row = rb * kB + (r >> 2) * 64 + rg * 4 + (r & 3);
                const uint2 w = x[r].bytes(two_to(tile_e));
                if (row < z.M) *(uint2*)(z.q + ((size_t)row * cbs + cb) * kB + cg * 8) = w;
            }
            if (threadIdx.x == 0) {
                z.scale[(size_t)rb * cbs + cb] = (uint8_t)(tile_e + 127);
                if (z.qt) z.scale_t[(size_t)cb * rbs + rb] = (uint8_t)(tile_e + 127);
            }
        }
        __syncthreads();
        const int c = threadIdx.x >> 1, h = (threadIdx.x & 1) * 16;
        if (z.qt && cb * kB + c < z.C) {
            const size_t piece = (WHAT & kBlock) ? (size_t)(cb * kB + c) * rbs + rb
                                                 : (size_t)rb * z.C + cb * kB + c;
            uint4* to = (uint4*)(z.qt + piece * kB + h * 4);
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const uint32_t* t = turn + c * kPitch + h + 4 * i;
                to[i] = make_uint4(t[0], t[1], t[2], t[3]);
            }
        }
    }
    if ((WHAT & kSum) && z.sum) {
        __syncthreads();
        const int c = threadIdx.x;
        if (c < kB && cb * kB + c < z.C)
            z.sum[(size_t)rb * z.C + cb * kB + c] = sums[0][c] + sums[1][c] + sums[2][c] + sums[3][c];
    }
}

// The product: out[m][n] = act( sum over blocks of a[m] . b[n] + bias_n ).
//
// A workgroup of four waves (2 x 2) owns a tile of 128 x 128 and walks the
// blocks: the next block's two slices of 128 x 128 bytes go straight into LDS
// while the present one is multiplied, a wave 64 x 64 of it on the matrix
// instruction, b as its first operand: a lane then holds 4 x 4 consecutive
// columns of a row, and stores 32 or 64 bytes of it.
//
// EXACT: the fp8 instruction adds a block's products on a grid set by the
// largest of them: about 5e-5 of a sum of values spread over e4m3's range.
// bf16 outputs, which round 40 times coarser, take it (their error against 64 bits
// is that of one rounding; with exact sums 16384 x 4928 -> 256 would take 65 us for
// 48, 16384 x 512 -> 2048 55 for 38, 32768 x 2304 -> 512 93 for 65); fp32 outputs turn
// the bytes, with their scales, into bf16 (four digits and a power of two: exact from
// 2^-133 up) and use the bf16 instruction, whose sums are good to fp32, at half the
// rate.
//
// LDS rows are 128 bytes, in 16-byte pieces exchanged by a key of the row
// (a_key, b_key), so that the lanes of a fragment read fall on all the banks.
//
// The weight's gradient of 32768 rows, 2304 x 512: 77 Gflop in bf16 in 87 us, 0.89
// PFLOP/s of the 1.88 that a loop of these instructions alone reaches and of a
// library product's 1.1; 58 % of the waves' cycles issue matrix instructions. (The
// conversions are not its bound: 89 us without them; on the fp8 instruction it would
// take 63.) Bound by the latency of a slice at two workgroups a CU.
struct Product {
    const uint8_t* a;   // [blocks][M][128]
    const uint8_t* sa;  // [blocks][M]
    int M;
    const uint8_t* b;   // block k of row n at n * b_row + k * b_blk
    size_t b_row, b_blk;
    const uint8_t* sb;  // at (n / step) * sb_row + block * sb_blk
    int step;
    size_t sb_row, sb_blk;
    int N, blocks, K;
    int per, splits;    // blocks a split takes
    const float* bias;
    int act;
    float slope;
    PvRows out;
    float* partial;     // [splits][M][N] where splits > 1
    // extra workgroups of the tiled product: dbias [bias_n] from the blocks' column
    // sums [bias_blocks][bias_n]
    const float* sum;
    int bias_n, bias_blocks;
    float* dbias;
};
constexpr int kTile = 128;

__device__ __forceinline__ int a_key(int row) { return row & 7; }
__device__ __forceinline__ int b_key(int row) { return (row & 3) | ((row >> 2) & 4); }
// of J fragments that take rows 4 J (r >> 2) + 4 j + (r & 3)
template <int J>
__device__ __forceinline__ int w_key(int row) {
    return (row & 3) | ((row >> (J == 2 ? 1 : 2)) & 4);
}

// Eight e4m3 bytes times 2^(byte - 127), as bf16 (which ends at 2^-133: a byte of 1 and
// less than 2^-7 times its scale is rounded to that grid).
__device__ __forceinline__ bf16x8 to_bf16(uint32_t lo, uint32_t hi, uint32_t byte) {
    const float f = __uint_as_float(byte << 23);
    union {
        bf16x2 p[4];
        bf16x8 v;
    } u;
    u.p[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, f, false);
    u.p[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, f, true);
    u.p[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, f, false);
    u.p[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, f, true);
    return u.v;
}

// the bias of W consecutive columns from n on (splits get it when they join)
template <int W>
__device__ __forceinline__ void load_bias(const Product& p, int n, float (&b)[W]) {
    const bool have = p.bias && p.splits == 1;
#pragma unroll
    for (int i = 0; i < W; i++) b[i] = have ? p.bias[min(n + i, p.N - 1)] : 0.f;
}

// W (8 or 16) consecutive outputs of a row, their bias added, from column n on: 16
// bytes a store wherever the row begins (an odd number of columns leaves most rows
// on no boundary: 26421 x 77 -> 1298 took 90 us by single elements).
typedef u32x4 u32x4_any __attribute__((aligned(2)));
template <int W>
__device__ __forceinline__ void store_run(const Product& p, int split, int m, int n,
                                          const float (&v)[W]) {
    const bool whole = n + W <= p.N;
    auto floats = [&](float* o, const float (&f)[W]) {
        if (whole) {
#pragma unroll
            for (int i = 0; i < W / 4; i++)
                *(u32x4_any*)(o + 4 * i) =
                    u32x4{__float_as_uint(f[4 * i]), __float_as_uint(f[4 * i + 1]),
                          __float_as_uint(f[4 * i + 2]), __float_as_uint(f[4 * i + 3])};
        } else {
#pragma unroll
            for (int i = 0; i < W; i++)
                if (n + i < p.N) o[i] = f[i];
        }
    };
    if (p.splits > 1) {
        floats(p.partial + ((size_t)split * p.M + m) * p.N + n, v);
        return;
    }
    float r[W];
#pragma unroll
    for (int i = 0; i < W; i++) r[i] = pv_activate(v[i], p.act, p.slope);
    const size_t at = (size_t)m * p.out.ld + n;
    if (!p.out.bf16) {
        floats((float*)p.out.p + at, r);
        return;
    }
    uint16_t* o = (uint16_t*)p.out.p + at;
    if (whole) {
        uint32_t w[W / 2];
#pragma unroll
        for (int i = 0; i < W / 2; i++) w[i] = pv_pack_bf16x2(r[2 * i], r[2 * i + 1]);
#pragma unroll
        for (int i = 0; i < W / 8; i++)
            *(u32x4_any*)(o + 8 * i) = u32x4{w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]};
    } else {
#pragma unroll
        for (int i = 0; i < W; i++)
            if (n + i < p.N) o[i] = pv_f32_to_bf16(r[i]);
    }
}

// dbias from the blocks' column sums, in a fixed order: 16 columns a workgroup,
// 16 threads a column.
constexpr int kBiasColumns = 16;
__device__ __forceinline__ void sum_bias(const Product& p, int group, double* part) {
    const int c = group * kBiasColumns + (threadIdx.x & 15);
    double s = 0.;
    if (c < p.bias_n)
        for (int i = threadIdx.x >> 4; i < p.bias_blocks; i += 16)
            s += (double)p.sum[(size_t)i * p.bias_n + c];
    part[threadIdx.x] = s;
    __syncthreads();
    if (threadIdx.x < 16 && c < p.bias_n) {
        for (int w = 1; w < 16; w++) s += part[threadIdx.x + 16 * w];
        p.dbias[c] = (float)s;
    }
}

template <bool EXACT>
__global__ __launch_bounds__(kThreads, 2) void pv_fp8_tile_kernel(Product p, int tiles) {
    // two stages, arrays of their own: the loads into one are then seen not to
    // touch what is read of the other, and are not waited for
    __shared__ __align__(16) uint8_t la0[kTile * kB], la1[kTile * kB];
    __shared__ __align__(16) uint8_t lb0[kTile * kB], lb1[kTile * kB];
    // scale bytes, as the fragments take them: dword r of a wave's 64 rows
    // holds the bytes of the four fragments' row r
    __shared__ __align__(16) uint8_t ls0[2 * kTile], ls1[2 * kTile];
    const int mt = (p.M + kTile - 1) / kTile, nt = (p.N + kTile - 1) / kTile;
    if ((int)blockIdx.x >= tiles) {
        sum_bias(p, (int)blockIdx.x - tiles, (double*)la0);
        return;
    }
    // Workgroups go round the XCDs; each XCD takes a run of tiles, the columns
    // of a row of tiles next to one another, so that its L2 serves a's rows.
    const size_t total = (size_t)mt * nt * p.splits, run = (total + 7) / 8;
    const size_t idx = (size_t)(blockIdx.x & 7) * run + (blockIdx.x >> 3);
    if ((blockIdx.x >> 3) >= run || idx >= total) return;
    const int split = (int)(idx / ((size_t)mt * nt));
    const int t = (int)(idx % ((size_t)mt * nt));
    const int m0 = t / nt * kTile, n0 = t % nt * kTile;
    const int k0 = split * p.per, k1 = min(k0 + p.per, p.blocks);

    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, r = lane & 15, h = lane >> 4;
    const int wm = (wave & 1) * 64, wn = (wave >> 1) * 64;
    // this lane's pieces of the two slices: four 1 KB rows of LDS a wave
    const uint8_t* ga[4];
    const uint8_t* gb[4];
#pragma unroll
    for (int q = 0; q < 4; q++) {
        const int piece = (wave * 4 + q) * 64 + lane, row = piece >> 3, c = piece & 7;
        ga[q] = p.a + ((size_t)k0 * p.M + min(m0 + row, p.M - 1)) * kB + (c ^ a_key(row)) * 16;
        gb[q] = p.b + (size_t)min(n0 + row, p.N - 1) * p.b_row + k0 * p.b_blk +
                (c ^ b_key(row)) * 16;
    }
    const uint8_t* gs;
    size_t gs_step;
    int gs_to;
    {
        const int row = threadIdx.x & 127;
        if (threadIdx.x < kTile) {
            gs = p.sa + (size_t)k0 * p.M + min(m0 + row, p.M - 1);
            gs_step = p.M;
            // row = 64 w + 16 i + r
            gs_to = (row & 64) + (row & 15) * 4 + ((row >> 4) & 3);
        } else {
            gs = p.sb + (size_t)(min(n0 + row, p.N - 1) / p.step) * p.sb_row +
                 (size_t)k0 * p.sb_blk;
            gs_step = p.sb_blk;
            // row = 64 w + 16 (r >> 2) + 4 j + (r & 3)
            gs_to = kTile + (row & 64) + ((row >> 4) & 3) * 16 + (row & 3) * 4 + ((row >> 2) & 3);
        }
    }
    auto fetch = [&](uint8_t* la, uint8_t* lb) {
#pragma unroll
        for (int q = 0; q < 4; q++) {
            __builtin_amdgcn_global_load_lds(
                (const void __attribute__((address_space(1)))*)ga[q],
                (void __attribute__((address_space(3)))*)(la + (wave * 4 + q) * 1024), 16, 0,
                0);
            __builtin_amdgcn_global_load_lds(
                (const void __attribute__((address_space(1)))*)gb[q],
                (void __attribute__((address_space(3)))*)(lb + (wave * 4 + q) * 1024), 16, 0,
                0);
            ga[q] += (size_t)p.M * kB;
            gb[q] += p.b_blk;
        }
    };
    pv_f32x4 acc[4][4];  // [fragment of b][fragment of a]
#pragma unroll
    for (int j = 0; j < 4; j++)
#pragma unroll
        for (int i = 0; i < 4; i++) acc[j][i] = pv_f32x4{0.f, 0.f, 0.f, 0.f};

    fetch(la0, lb0);
    uint8_t byte = *gs;
    // one block: `la`, `lb`, `ls` hold it, the others take the next
    auto block = [&](int k, const uint8_t* la, const uint8_t* lb, uint8_t* ls, uint8_t* na,
                     uint8_t* nb) {
        ls[gs_to] = byte;
        __builtin_amdgcn_s_waitcnt(0);  // this wave's part of the slices has landed
        __syncthreads();
        if (k + 1 < k1) {
            fetch(na, nb);
            gs += gs_step;
            byte = *gs;
        }
        i32x8 fa[4], fb[4];
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const int ra = wm + 16 * i + r, rb = wn + 16 * (r >> 2) + 4 * i + (r & 3);
            union {
                uint4 u[2];
                i32x8 v;
            } f, g;
            f.u[0] = *(const uint4*)(la + ra * kB + (h ^ a_key(ra)) * 16);
            f.u[1] = *(const uint4*)(la + ra * kB + ((h + 4) ^ a_key(ra)) * 16);
            g.u[0] = *(const uint4*)(lb + rb * kB + (h ^ b_key(rb)) * 16);
            g.u[1] = *(const uint4*)(lb + rb * kB + ((h + 4) ^ b_key(rb)) * 16);
            fa[i] = f.v;
            fb[i] = g.v;
        }
        const uint32_t sa = *(const uint32_t*)(ls + wm + 4 * r);
        const uint32_t sb = *(const uint32_t*)(ls + kTile + wn + 4 * r);
        if constexpr (!EXACT) {
#pragma unroll
            for (int j = 0; j < 4; j++)
#pragma unroll
                for (int i = 0; i < 4; i++)
                    acc[j][i] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(
                        fb[j], fa[i], acc[j][i], 0, 0, 0, (int)(sb >> (8 * j)), 0,
                        (int)(sa >> (8 * i)));
        } else {
#pragma unroll
            for (int q = 0; q < 4; q++) {
                bf16x8 va[4];
#pragma unroll
                for (int i = 0; i < 4; i++)
                    va[i] = to_bf16(fa[i][2 * q], fa[i][2 * q + 1], sa >> (8 * i) & 255u);
#pragma unroll
                for (int j = 0; j < 4; j++) {
                    const bf16x8 vb = to_bf16(fb[j][2 * q], fb[j][2 * q + 1], sb >> (8 * j) & 255u);
#pragma unroll
                    for (int i = 0; i < 4; i++)
                        acc[j][i] =
                            __builtin_amdgcn_mfma_f32_16x16x32_bf16(vb, va[i], acc[j][i], 0, 0, 0);
                }
            }
        }
    };
    for (int k = k0; k < k1; k += 2) {
        block(k, la0, lb0, ls0, la1, lb1);
        if (k + 1 < k1) block(k + 1, la1, lb1, ls1, la0, lb0);
    }
    float bias[16];
    load_bias<16>(p, n0 + wn + 16 * h, bias);
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const int m = m0 + wm + 16 * i + r;
        float v[16];
#pragma unroll
        for (int j = 0; j < 4; j++)
#pragma unroll
            for (int e = 0; e < 4; e++) v[4 * j + e] = acc[j][i][e] + bias[4 * j + e];
        if (m < p.M) store_run<16>(p, split, m, n0 + wn + 16 * h, v);
    }
}

// The product of rows that are quantised on the way in: x is read once from
// memory as it is, and no quantised copy of it exists.
//
// Eight waves: side by side, 64 rows by 32 columns each, or two by four of 64 by 64
// (MW = 2, where such tiles fill the chip: the same LDS reads feed twice the
// products). Two a SIMD, one's quantising beside the other's products; waves beyond
// the last column quantise only. A block's slices of x and of the weight come into
// registers two blocks ahead. 16 lanes hold a row's 128 values, take their
// largest by DPP moves, and put the bytes into LDS with the row's scale; the
// weight goes through LDS as it is, loaded by whole rows of 128 bytes (as
// fragments straight from the L2, 16 bytes of 64 rows a load, it took 25 us of 64
// at 16384 x 4928 -> 256). The barrier of a block waits for LDS alone, never for
// the loads under way.
// 16384 x 4928 -> 256, bf16: 47 us, 0.88 PFLOP/s, x at 3.5 TB/s beside 320 MB of
// the weight from the L2. 32768 x 2304 -> 512: 79 us in tiles of 128 rows, 0.98
// PFLOP/s (97 in tiles of 64). Bound by LDS reads and a barrier a block.
struct Fused {
    PvRows x;
    int M, K;
    const uint8_t* w;   // [N][blocks * 128]
    const uint8_t* sw;  // [N / 128][blocks]
};

// A block's rows of x, from registers (THREADS threads, 16 of them a row, V rows a
// thread) into LDS as bytes with their scales.
template <int THREADS, int V, bool XB>
__device__ __forceinline__ void quantise_slice(const XVec<XB> (&from)[V], int k, int K,
                                               uint8_t* to, uint8_t* scales) {
    const int xr = threadIdx.x >> 4, xc = (threadIdx.x & 15) * 8;
    XVec<XB> x[V];
    uint32_t top[V], all = 0;
#pragma unroll
    for (int v = 0; v < V; v++) x[v] = from[v];
    if ((k + 1) * kB > K) {  // the row's last block
#pragma unroll
        for (int v = 0; v < V; v++) x[v].move_down(max(k * kB + xc - (K - 8), 0));
    }
#pragma unroll
    for (int v = 0; v < V; v++) {
        top[v] = x[v].top();
        all = max(all, top[v]);
    }
    if (__builtin_expect(__any(all >= 0x7f800000u), 0)) {
#pragma unroll
        for (int v = 0; v < V; v++) top[v] = x[v].finite_top();
    }
#pragma unroll
    for (int v = 0; v < V; v++) top[v] = max_dpp<0xB1>(top[v]);  // quad_perm [1,0,3,2]
#pragma unroll
    for (int v = 0; v < V; v++) top[v] = max_dpp<0x4E>(top[v]);  // quad_perm [2,3,0,1]
#pragma unroll
    for (int v = 0; v < V; v++) top[v] = max_dpp<0x141>(top[v]);  // row_half_mirror
#pragma unroll
    for (int v = 0; v < V; v++) top[v] = max_dpp<0x140>(top[v]);  // row_mirror
#pragma unroll
    for (int v = 0; v < V; v++) {
        // block_exponent + 127, but that zeros may take any scale here
        const int byte = max((int)((top[v] + 0x1fffffu) >> 23) - 8, 1);
        const int row = xr + (THREADS / 16) * v;
        *(uint2*)(to + row * kB + ((xc >> 4) ^ a_key(row)) * 16 + (xc & 8)) =
            x[v].bytes(__uint_as_float((uint32_t)byte << 23));
        // row = 64 w + 16 i + r: byte i of dword r of the 64
        if (xc == 0) scales[(row & ~63) + (row & 15) * 4 + ((row >> 4) & 3)] = (uint8_t)byte;
    }
}

union Frag {
    u32x4 u[2];
    i32x8 v;
};
// acc += the wave's 16 J columns of the weight (rows wn + 4 J (r >> 2) + 4 j +
// (r & 3) of its slice lw, keyed by w_key) times the 64 rows of x (lx, scales
// lsx), sw the weight's scale.
template <int J, bool EXACT>
__device__ __forceinline__ void multiply_slices(pv_f32x4 (&acc)[J][4], const uint8_t* lw, int wn,
                                                const uint8_t* lx, const uint8_t* lsx, int sw) {
    const int r = threadIdx.x & 15, h = (threadIdx.x & 63) >> 4;
    Frag fa[4], fw[J];
#pragma unroll
    for (int j = 0; j < J; j++) {
        const int row = wn + 4 * J * (r >> 2) + 4 * j + (r & 3);
        fw[j].u[0] = *(const u32x4*)(lw + row * kB + (h ^ w_key<J>(row)) * 16);
        fw[j].u[1] = *(const u32x4*)(lw + row * kB + ((h + 4) ^ w_key<J>(row)) * 16);
    }
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const int row = 16 * i + r;
        fa[i].u[0] = *(const u32x4*)(lx + row * kB + (h ^ a_key(row)) * 16);
        fa[i].u[1] = *(const u32x4*)(lx + row * kB + ((h + 4) ^ a_key(row)) * 16);
    }
    const uint32_t sa = *(const uint32_t*)(lsx + 4 * r);
    if constexpr (!EXACT) {
#pragma unroll
        for (int j = 0; j < J; j++)
#pragma unroll
            for (int i = 0; i < 4; i++)
                acc[j][i] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(
                    fw[j].v, fa[i].v, acc[j][i], 0, 0, 0, sw, 0, (int)(sa >> (8 * i)));
    } else {
#pragma unroll
        for (int q = 0; q < 4; q++) {
            bf16x8 va[4];
#pragma unroll
            for (int i = 0; i < 4; i++)
                va[i] = to_bf16(fa[i].v[2 * q], fa[i].v[2 * q + 1], sa >> (8 * i) & 255u);
#pragma unroll
            for (int j = 0; j < J; j++) {
                const bf16x8 vb = to_bf16(fw[j].v[2 * q], fw[j].v[2 * q + 1], sw);
#pragma unroll
                for (int i = 0; i < 4; i++)
                    acc[j][i] =
                        __builtin_amdgcn_mfma_f32_16x16x32_bf16(vb, va[i], acc[j][i], 0, 0, 0);
            }
        }
    }
}

constexpr int kFusedM = 64, kFusedTileN = 256, kFusedThreads = 512, kFusedWaves = 2;

template <int MW, bool XB, bool EXACT>
__global__ __launch_bounds__(kFusedThreads, kFusedWaves) void pv_fp8_fused_kernel(Fused f,
                                                                                 Product p) {
    constexpr int BM = kFusedM * MW, BN = kFusedTileN;
    // vectors of x a thread; fragments of the weight a wave; its loads a wave
    constexpr int V = BM * 16 / kFusedThreads, J = 2 * MW, W = BN * kB / 16 / kFusedThreads;
    __shared__ __align__(16) uint8_t lw[2][BN * kB];
    __shared__ __align__(16) uint8_t la[2][BM * kB];
    __shared__ __align__(16) uint8_t ls[2][BM];
    __shared__ uint8_t lsw[BN / kB][PVCONV_FP8_MAX_CHANNELS / kB];  // the weight's scales
    const int mt = (f.M + BM - 1) / BM, nt = (p.N + BN - 1) / BN;
    // tiles of one row of tiles run side by side on one XCD, as above
    const size_t total = (size_t)mt * nt * p.splits, run = (total + 7) / 8;
    const size_t idx = (size_t)(blockIdx.x & 7) * run + (blockIdx.x >> 3);
    if ((blockIdx.x >> 3) >= run || idx >= total) return;
    const int split = (int)(idx / ((size_t)mt * nt));
    const int t = (int)(idx % ((size_t)mt * nt));
    const int m0 = t / nt * BM, n0 = t % nt * BN;
    const int k0 = split * p.per, k1 = min(k0 + p.per, p.blocks);

    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, r = lane & 15, h = lane >> 4;
    // the wave's rows and columns of the tile
    const int wm = wave % MW * 64, wn = wave / MW * (32 * MW);
    const bool multiplies = n0 + wn < p.N;
    const int xr = threadIdx.x >> 4, xc = (threadIdx.x & 15) * 8;  // row (+ 32 v), column
    for (int i = threadIdx.x; i < BN / kB * (k1 - k0); i += kFusedThreads) {
        const int row = i / (k1 - k0), k = i - row * (k1 - k0);
        lsw[row][k] = f.sw[(size_t)min(n0 / kB + row, (p.N - 1) / kB) * p.blocks + k0 + k];
    }
    XVec<XB> xs[2][V];
    auto fetch_x = [&](XVec<XB>(&to)[V], int k) {
#pragma unroll
        for (int v = 0; v < V; v++)
            to[v].load(f.x, (size_t)min(m0 + xr + (kFusedThreads / 16) * v, f.M - 1), k * kB + xc, f.K);
    };
    auto quantise = [&](const XVec<XB>(&from)[V], int k, uint8_t* to, uint8_t* scales) {
        quantise_slice<kFusedThreads, V>(from, k, f.K, to, scales);
    };
    // this thread's pieces of the weight's slice: eight threads a row
    const int wr = threadIdx.x >> 3, wc = threadIdx.x & 7;
    const uint8_t* gw[W];
#pragma unroll
    for (int q = 0; q < W; q++)
        gw[q] = f.w + (size_t)min(n0 + wr + kFusedThreads / 8 * q, p.N - 1) * p.blocks * kB + wc * 16;
    u32x4 ws[2][W];
    auto fetch_w = [&](u32x4(&to)[W], int k) {
#pragma unroll
        for (int q = 0; q < W; q++) to[q] = *(const u32x4*)(gw[q] + (size_t)k * kB);
    };
    auto put_w = [&](const u32x4(&from)[W], uint8_t* to) {
#pragma unroll
        for (int q = 0; q < W; q++) {
            const int row = wr + kFusedThreads / 8 * q;
            *(u32x4*)(to + row * kB + (wc ^ w_key<J>(row)) * 16) = from[q];
        }
    };
    pv_f32x4 acc[J][4];  // [fragment of the weight][fragment of x]
#pragma unroll
    for (int j = 0; j < J; j++)
#pragma unroll
        for (int i = 0; i < 4; i++) acc[j][i] = pv_f32x4{0.f, 0.f, 0.f, 0.f};
    // Block k. Its loads are not under conditions (past the last block they fetch
    // that one again): the waits then count the loads under way exactly. Loads
    // return in order, and x, the slower one, is asked for last.
    auto block = [&](int k, int st, XVec<XB>(&x_free)[V], u32x4(&w_free)[W]) {
        pv_lds_barrier();
        fetch_w(w_free, min(k + 2, k1 - 1));
        fetch_x(x_free, min(k + 2, k1 - 1));
        if (multiplies && k < k1)
            multiply_slices<J, EXACT>(acc, lw[st], wn, la[st] + wm * kB, ls[st] + wm,
                                      lsw[wn / kB][k - k0]);
    };
    fetch_w(ws[0], k0);
    fetch_x(xs[0], k0);
    fetch_w(ws[1], min(k0 + 1, k1 - 1));
    fetch_x(xs[1], min(k0 + 1, k1 - 1));
    put_w(ws[0], lw[0]);
    quantise(xs[0], k0, la[0], ls[0]);
    // (one way out: where blocks are odd in number, the last half multiplies
    // nothing)
    for (int k = k0; k < k1; k += 2) {
        block(k, 0, xs[0], ws[0]);
        put_w(ws[1], lw[1]);
        quantise(xs[1], k + 1, la[1], ls[1]);
        block(k + 1, 1, xs[1], ws[1]);
        put_w(ws[0], lw[0]);
        quantise(xs[0], k + 2, la[0], ls[0]);
    }
    float bias[4 * J];
    load_bias<4 * J>(p, n0 + wn + 4 * J * h, bias);
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const int m = m0 + wm + 16 * i + r;
        float v[4 * J];
#pragma unroll
        for (int j = 0; j < J; j++)
#pragma unroll
            for (int e = 0; e < 4; e++) v[4 * j + e] = acc[j][i][e] + bias[4 * j + e];
        if (m < f.M && multiplies) store_run<4 * J>(p, split, m, n0 + wn + 4 * J * h, v);
    }
}

// The same for rows short enough to stay: a workgroup quantises its 64 rows
// whole into LDS once (up to kResidentBlocks blocks of 8 KB) and goes over a
// share of the columns, 128 at a time, the weight's slices flowing through two
// stages without a stop from one tile of columns to the next. x is read once
// for all of the share, the outputs are the traffic. Four waves side by side, 64
// rows by 32 columns each.
// 16384 x 512 -> 2048, bf16: 39 us, 0.88 PFLOP/s, bound by LDS: a wave reads 12 KB
// for 64 x 32 x 128. (Rows' fragments kept in registers over the tiles of columns
// would read a third of that, but four blocks of them spill.)
constexpr int kResidentThreads = 256, kResidentN = 128, kResidentBlocks = 8;
constexpr int kResidentShare = 16;  // tiles of columns a workgroup at most: their bias lies in LDS

template <bool XB, bool EXACT>
__global__ __launch_bounds__(kResidentThreads, 2) void pv_fp8_resident_kernel(Fused f, Product p,
                                                                             int share) {
    constexpr int BM = kFusedM, BN = kResidentN, T = kResidentThreads;
    constexpr int V = BM * 16 / T, J = 2, W = BN * kB / 16 / T;
    __shared__ __align__(16) uint8_t lw[2][BN * kB];
    __shared__ __align__(16) uint8_t ls[kResidentBlocks][BM];
    __shared__ uint8_t lsw[kResidentShare * kResidentBlocks];  // a scale a step
    __shared__ __align__(16) float lbias[kResidentShare * BN];
    extern __shared__ __align__(16) uint8_t la[];  // [blocks][BM * 128]
    const int nt = (p.N + BN - 1) / BN, shares = (nt + share - 1) / share;
    const int m0 = (int)(blockIdx.x / shares) * BM, t0 = (int)(blockIdx.x % shares) * share;
    const int steps = (min(t0 + share, nt) - t0) * p.blocks;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, r = lane & 15, h = lane >> 4;
    const int wn = wave * 32;

    const int wr = threadIdx.x >> 3, wc = threadIdx.x & 7;
    u32x4 ws[2][W];
    // The steps in order: the blocks of a tile of columns, then the next tile's
    // (past the last step, that one again).
    const uint8_t* gw[W];
    auto rows_of = [&](int t) {
#pragma unroll
        for (int q = 0; q < W; q++)
            gw[q] = f.w + (size_t)min(t * BN + wr + T / 8 * q, p.N - 1) * p.blocks * kB + wc * 16;
    };
    int fs = 0, ft = t0, fk = 0;
    auto fetch_w = [&](u32x4(&to)[W]) {
#pragma unroll
        for (int q = 0; q < W; q++) to[q] = *(const u32x4*)(gw[q] + (size_t)fk * kB);
        if (++fs < steps) {
            if (++fk == p.blocks) {
                fk = 0;
                rows_of(++ft);
            }
        }
    };
    rows_of(t0);
    auto put_w = [&](const u32x4(&from)[W], uint8_t* to) {
#pragma unroll
        for (int q = 0; q < W; q++) {
            const int row = wr + T / 8 * q;
            *(u32x4*)(to + row * kB + (wc ^ w_key<J>(row)) * 16) = from[q];
        }
    };
    fetch_w(ws[0]);
    fetch_w(ws[1]);
    for (int i = threadIdx.x; i < steps; i += T) lsw[i] = f.sw[(size_t)t0 * p.blocks + i];
    for (int i = threadIdx.x; i < share * BN; i += T)
        lbias[i] = p.bias ? p.bias[min(t0 * BN + i, p.N - 1)] : 0.f;
    XVec<XB> xs[2][V];
    auto fetch_x = [&](XVec<XB>(&to)[V], int k) {
#pragma unroll
        for (int v = 0; v < V; v++)
            to[v].load(f.x, (size_t)min(m0 + (int)(threadIdx.x >> 4) + (T / 16) * v, f.M - 1),
                       min(k, p.blocks - 1) * kB + (threadIdx.x & 15) * 8, f.K);
    };
    fetch_x(xs[0], 0);
    fetch_x(xs[1], 1);
    for (int k = 0; k < p.blocks; k += 2) {
        quantise_slice<T, V>(xs[0], k, f.K, la + (size_t)k * BM * kB, ls[k]);
        fetch_x(xs[0], k + 2);
        if (k + 1 < p.blocks)
            quantise_slice<T, V>(xs[1], k + 1, f.K, la + (size_t)(k + 1) * BM * kB, ls[k + 1]);
        fetch_x(xs[1], k + 3);
    }
    pv_f32x4 acc[J][4];
    int t = t0, k = 0;
    auto step = [&](int s, const uint8_t* lws, u32x4(&w_free)[W], const u32x4(&w_next)[W],
                    uint8_t* lw_next) {
        pv_lds_barrier();
        fetch_w(w_free);
        if (k == 0) {
#pragma unroll
            for (int j = 0; j < J; j++)
#pragma unroll
                for (int i = 0; i < 4; i++) acc[j][i] = pv_f32x4{0.f, 0.f, 0.f, 0.f};
        }
        if (s < steps && t * BN + wn < p.N)
            multiply_slices<J, EXACT>(acc, lws, wn, la + (size_t)k * BM * kB, ls[k],
                                      lsw[s]);
        put_w(w_next, lw_next);
        if (++k < p.blocks) return;
        if (s < steps && t * BN + wn < p.N) {
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const int m = m0 + 16 * i + r;
                float v[4 * J];
#pragma unroll
                for (int j = 0; j < J; j++)
#pragma unroll
                    for (int e = 0; e < 4; e++)
                        v[4 * j + e] = acc[j][i][e] +
                                       lbias[(t - t0) * BN + wn + 8 * h + 4 * j + e];
                if (m < f.M) store_run<8>(p, 0, m, t * BN + wn + 8 * h, v);
            }
        }
        k = 0;
        t++;
    };
    put_w(ws[0], lw[0]);
    for (int s = 0; s < steps; s += 2) {
        step(s, lw[0], ws[0], ws[1], lw[1]);
        step(s + 1, lw[1], ws[1], ws[0], lw[0]);
    }
}

// Few rows: a workgroup takes 16 rows by 16 columns, its eight waves a share of
// the blocks each, whose sums meet in LDS in wave order: one launch, and the
// weight's bytes spread over as many workgroups as there are 16 columns. A wave
// quantises its blocks of x in registers, where they are its matrix operand:
// lane (r, h) holds row r's values 16 h .. and 64 + 16 h .. of the block. It ends
// after the latency of a wave's few blocks: 2.6 to 4.2 us for one row of 128 to
// 2048 channels, 7.7 of 4928.
constexpr int kFewThreads = 512;

template <bool XB, bool EXACT>
__global__ __launch_bounds__(kFewThreads) void pv_fp8_few_kernel(Fused f, Product p) {
    constexpr int kWaves = kFewThreads / 64;
    __shared__ float part[kWaves][256];
    const int nt = (p.N + 15) / 16;
    const int m0 = (int)(blockIdx.x / nt) * 16, n0 = (int)(blockIdx.x % nt) * 16;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, r = lane & 15, h = lane >> 4;
    const size_t row = min(m0 + r, f.M - 1);
    const int n = min(n0 + r, p.N - 1);
    const uint8_t* gw = f.w + (size_t)n * p.blocks * kB + h * 16;
    const uint8_t* gs = f.sw + (size_t)(n / kB) * p.blocks;
    struct Block {
        XVec<XB> x[4];
        Frag w;
        int sw;
    };
    auto fetch = [&](Block& b, int k) {
        k = min(k, p.blocks - 1);
        b.w.u[0] = *(const u32x4*)(gw + (size_t)k * kB);
        b.w.u[1] = *(const u32x4*)(gw + (size_t)k * kB + 64);
        b.sw = gs[k];
#pragma unroll
        for (int v = 0; v < 4; v++)
            b.x[v].load(f.x, row, k * kB + (v >> 1) * 64 + h * 16 + (v & 1) * 8, f.K);
    };
    pv_f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    auto multiply = [&](Block& b, int k) {
        if ((k + 1) * kB > f.K) {
#pragma unroll
            for (int v = 0; v < 4; v++)
                b.x[v].move_down(
                    max(k * kB + (v >> 1) * 64 + h * 16 + (v & 1) * 8 - (f.K - 8), 0));
        }
        uint32_t top = 0;
#pragma unroll
        for (int v = 0; v < 4; v++) top = max(top, b.x[v].finite_top());
        top = max(top, (uint32_t)__shfl_xor((int)top, 16));
        top = max(top, (uint32_t)__shfl_xor((int)top, 32));
        const int byte = block_exponent(top) + 127;
        Frag a;
#pragma unroll
        for (int v = 0; v < 4; v++) {
            const uint2 q = b.x[v].bytes(__uint_as_float((uint32_t)byte << 23));
            a.v[2 * v] = (int)q.x;
            a.v[2 * v + 1] = (int)q.y;
        }
        if constexpr (!EXACT) {
            acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b.w.v, a.v, acc, 0, 0, 0, b.sw,
                                                                   0, byte);
        } else {
#pragma unroll
            for (int q = 0; q < 4; q++)
                acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                    to_bf16(b.w.v[2 * q], b.w.v[2 * q + 1], b.sw),
                    to_bf16(a.v[2 * q], a.v[2 * q + 1], byte), acc, 0, 0, 0);
        }
    };
    Block b0, b1;
    fetch(b0, wave);
    for (int k = wave; k < p.blocks; k += 2 * kWaves) {
        fetch(b1, k + kWaves);
        multiply(b0, k);
        fetch(b0, k + 2 * kWaves);
        if (k + kWaves < p.blocks) multiply(b1, k + kWaves);
    }
#pragma unroll
    for (int i = 0; i < 4; i++) part[wave][r * 16 + 4 * h + i] = acc[i];
    __syncthreads();
    const int m = m0 + (int)(threadIdx.x >> 4), c = n0 + (int)(threadIdx.x & 15);
    if (threadIdx.x < 256 && m < f.M && c < p.N) {
        float v = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; w++) v += part[w][threadIdx.x];
        if (p.bias) v += p.bias[c];
        pv_store_one(p.out.p, p.out.bf16, (size_t)m * p.out.ld + c,
                     pv_activate(v, p.act, p.slope));
    }
}

// out = act( the splits' sums in order + bias ). Bound by memory: 7 sums of 2304 x
// 512, 33 MB, mostly from the caches, in 8.6 us (10.6 with one load in flight).
__global__ __launch_bounds__(kThreads) void pv_fp8_join_kernel(Product p) {
    constexpr int kAhead = 8;  // splits in flight
    const size_t total = (size_t)p.M * p.N;
    for (size_t i = (size_t)blockIdx.x * kThreads + threadIdx.x; i < total;
         i += (size_t)gridDim.x * kThreads) {
        float s = 0.f;
        for (int k = 0; k < p.splits; k += kAhead) {
            float v[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; u++)
                v[u] = p.partial[(size_t)min(k + u, p.splits - 1) * total + i];
#pragma unroll
            for (int u = 0; u < kAhead; u++)
                if (k + u < p.splits) s += v[u];
        }
        const size_t m = i / p.N;
        const int n = (int)(i - m * p.N);
        pv_store_one(p.out.p, p.out.bf16, m * p.out.ld + n,
                     pv_activate(s + (p.bias ? p.bias[n] : 0.f), p.act, p.slope));
    }
}

// dbias alone
__global__ __launch_bounds__(kThreads) void pv_fp8_bias_kernel(Product p) {
    __shared__ double part[kThreads];
    sum_bias(p, blockIdx.x, part);
}

// the weight's gradient of no rows
__global__ __launch_bounds__(kThreads) void pv_fp8_zero_kernel(float* p, size_t n) {
    for (size_t i = (size_t)blockIdx.x * kThreads + threadIdx.x; i < n;
         i += (size_t)gridDim.x * kThreads)
        p[i] = 0.f;
}

unsigned grid_of(size_t blocks) {
    return (unsigned)(blocks < 1 ? 1 : (blocks < (1u << 20) ? blocks : 1u << 20));
}

// The quantised rows and columns in a workspace.
struct Quantised {
    uint8_t *q, *scale;
};
struct Carve {
    char* base;
    size_t off;
    void* take(size_t bytes) {
        void* p = base ? base + off : nullptr;
        off += pv_align256(bytes);
        return p;
    }
    Quantised rows(int rows, int cols) {
        Quantised r;
        r.q = (uint8_t*)take((size_t)rows * pv_fp8_blocks(cols) * kB);
        r.scale = (uint8_t*)take((size_t)rows * pv_fp8_blocks(cols));
        return r;
    }
};
// How many ways a product's blocks are split: one where its tiles fill the chip,
// else enough for kWanted workgroups at most (two a CU: more would wait for a second
// round, 108 us with 1024 for 87 at 32768 rows, 2304 x 512), of kLeast blocks or
// more (joining costs a launch, a block some half a microsecond).
constexpr int kWanted = 512, kLeast = 6;
constexpr int kFusedN = 1024;
void plan_splits(int M, int N, int bm, int bn, int blocks, int* per, int* splits) {
    const size_t tiles = (size_t)((M + bm - 1) / bm) * ((N + bn - 1) / bn);
    *per = blocks;
    if (tiles > 0 && tiles < kWanted / 2 && blocks >= 2 * kLeast) {
        const int most = blocks / kLeast;
        int n = (int)(kWanted / tiles);
        n = n < 1 ? 1 : (n > most ? most : n);
        *per = (blocks + n - 1) / n;
    }
    *splits = *per ? (blocks + *per - 1) / *per : 1;
}
size_t partial_bytes(int M, int N, int bm, int bn, int blocks) {
    int per, splits;
    plan_splits(M, N, bm, bn, blocks, &per, &splits);
    return splits > 1 ? (size_t)splits * M * N * 4 : 0;
}

// How a product of rows by a weight runs: few rows, rows that stay in LDS, rows
// quantised on the way in, or the quantiser and the product apart (also rows of
// fewer channels than a vector). Few: as long as each of its workgroups has a CU
// to itself (bf16, few / else, us: 256 x 2048 -> 256, 256 workgroups, 6.0 / 13.9;
// 512 rows 10.0 / 14.1; 512 x 4928 -> 256 20.3 / 15.5; 128 x 512 -> 2048, 1024
// workgroups, 10.1 / 6.6).
constexpr int kFewTiles = 256;
enum Path { kFew, kResident, kFused, kApart };
Path path_of(int M, int K, int N) {
    if (K < 8) return kApart;
    if ((size_t)((M + 15) / 16) * ((N + 15) / 16) <= kFewTiles) return kFew;
    if (N > kFusedTileN && pv_fp8_blocks(K) <= kResidentBlocks) return kResident;
    return N <= kFusedN ? kFused : kApart;
}

struct RowsWs {  // of a product of rows by a weight
    Quantised x;
    float* partial;
};
RowsWs carve_rows(Carve& c, int M, int K, int N) {
    const Path path = path_of(M, K, N);
    RowsWs w{{nullptr, nullptr}, nullptr};
    if (path == kApart) w.x = c.rows(M, K);
    if (path == kFused || path == kApart)
        w.partial = (float*)c.take(
            path == kFused ? partial_bytes(M, N, kFusedM, kFusedTileN, pv_fp8_blocks(K))
                           : partial_bytes(M, N, kTile, kTile, pv_fp8_blocks(K)));
    return w;
}
struct BwdWs {
    RowsWs dx;
    Quantised dyt, xt;
    float* sum;
    float* partial;  // dw's
    size_t total;
};
BwdWs carve_bwd(void* base, int M, int K, int N) {
    Carve c{(char*)base, 0};
    BwdWs w;
    w.dx = carve_rows(c, M, N, K);
    w.dyt = c.rows(N, M);
    w.xt = c.rows(K, M);
    w.sum = (float*)c.take((size_t)pv_fp8_blocks(M) * N * 4);
    w.partial = (float*)c.take(partial_bytes(N, K, kTile, kTile, pv_fp8_blocks(M)));
    w.total = c.off;
    return w;
}

template <typename F>
void with_bool(bool b, F f) {
    if (b)
        f(std::true_type());
    else
        f(std::false_type());
}

int tiles_of(const Quantise& z) { return pv_fp8_blocks(z.M) * pv_fp8_blocks(z.C); }

template <int WHAT>
void launch_quantise(const Quantise& a, hipStream_t s, const Quantise* b = nullptr) {
    if (b && (a.x.bf16 != b->x.bf16 || (a.C < 8) != (b->C < 8))) {
        launch_quantise<WHAT>(a, s);
        launch_quantise<WHAT>(*b, s);
        return;
    }
    const QuantiseJobs jobs{a, b ? *b : a, tiles_of(a)};
    const unsigned grid = (unsigned)(tiles_of(a) + (b ? tiles_of(*b) : 0));
    with_bool(a.x.bf16, [&](auto XB) {
        with_bool(a.C < 8, [&](auto NARROW) {
            pv_fp8_quantise_kernel<decltype(XB)::value, decltype(NARROW)::value, WHAT>
                <<<grid, kThreads, 0, s>>>(jobs);
        });
    });
}

// HIP takes fewer than 2^32 threads a launch: what would need more than kMostThreads
// runs in parts, rows after rows.
constexpr size_t kMostThreads = (size_t)1 << 31;

// The columns of a (and b), in blocks along the rows, or their sums.
template <int WHAT>
void launch_columns(const Quantise& a, hipStream_t s, const Quantise* b = nullptr) {
    static_assert((WHAT & (kRows | kBlock)) == 0, "a part's rows lie on their own");
    const size_t tiles = (size_t)tiles_of(a) + (b ? tiles_of(*b) : 0);
    if (tiles * kThreads <= kMostThreads) {
        launch_quantise<WHAT>(a, s, b);
        return;
    }
    for (const Quantise* z : {&a, b}) {
        if (!z) continue;
        const int cbs = pv_fp8_blocks(z->C), rbs = pv_fp8_blocks(z->M);
        const int run = (int)(kMostThreads / kThreads / cbs);
        for (int rb = 0; rb < rbs; rb += run) {
            Quantise part = *z;
            part.x.p = (char*)z->x.p + (size_t)rb * kB * z->x.ld * (z->x.bf16 ? 2 : 4);
            part.M = (rb + run < rbs ? (rb + run) * kB : z->M) - rb * kB;
            if (z->qt) part.qt = z->qt + (size_t)rb * z->C * kB;
            if (z->scale_t) part.scale_t = z->scale_t + (size_t)rb * z->C;
            if (z->sum) part.sum = z->sum + (size_t)rb * z->C;
            launch_quantise<WHAT>(part, s);
        }
    }
}

void launch_product(Product p, hipStream_t s) {
    plan_splits(p.M, p.N, kTile, kTile, p.blocks, &p.per, &p.splits);
    const size_t total = (size_t)((p.M + kTile - 1) / kTile) * ((p.N + kTile - 1) / kTile) * p.splits;
    const unsigned grid = (unsigned)((total + 7) / 8 * 8);
    const unsigned more = p.dbias ? (unsigned)((p.bias_n + kBiasColumns - 1) / kBiasColumns) : 0;
    if (p.out.bf16)
        pv_fp8_tile_kernel<false><<<grid + more, kThreads, 0, s>>>(p, (int)grid);
    else
        pv_fp8_tile_kernel<true><<<grid + more, kThreads, 0, s>>>(p, (int)grid);
    if (p.splits > 1)
        pv_fp8_join_kernel<<<grid_of(((size_t)p.M * p.N + kThreads - 1) / kThreads), kThreads, 0,
                             s>>>(p);
}

// 128 rows a workgroup where those fill the chip (and bf16 x: the slices of fp32
// need the registers of 64).
bool fused_wide(const PvRows& x, int M, int N) {
    return x.bf16 && (size_t)(M / (2 * kFusedM)) * ((N + kFusedTileN - 1) / kFusedTileN) >=
                         kWanted / 2;
}

void launch_fused(const PvRows& x, Product p, hipStream_t s) {
    const bool wide = fused_wide(x, p.M, p.N);
    const int bm = wide ? 2 * kFusedM : kFusedM;
    plan_splits(p.M, p.N, kFusedM, kFusedTileN, p.blocks, &p.per, &p.splits);
    const size_t total =
        (size_t)((p.M + bm - 1) / bm) * ((p.N + kFusedTileN - 1) / kFusedTileN) * p.splits;
    const unsigned grid = (unsigned)((total + 7) / 8 * 8);
    const Fused f{x, p.M, p.K, p.b, p.sb};
    with_bool(x.bf16, [&](auto XB) {
        with_bool(!p.out.bf16, [&](auto EXACT) {
            constexpr bool kXB = decltype(XB)::value, kExact = decltype(EXACT)::value;
            if constexpr (kXB) {
                if (wide) {
                    pv_fp8_fused_kernel<2, kXB, kExact><<<grid, kFusedThreads, 0, s>>>(f, p);
                    return;
                }
            }
            pv_fp8_fused_kernel<1, kXB, kExact><<<grid, kFusedThreads, 0, s>>>(f, p);
        });
    });
    if (p.splits > 1)
        pv_fp8_join_kernel<<<grid_of(((size_t)p.M * p.N + kThreads - 1) / kThreads), kThreads, 0,
                             s>>>(p);
}

void launch_few(const PvRows& x, const Product& p, hipStream_t s) {
    const Fused f{x, p.M, p.K, p.b, p.sb};
    const unsigned grid = (unsigned)(((p.M + 15) / 16) * ((p.N + 15) / 16));
    with_bool(x.bf16, [&](auto XB) {
        with_bool(!p.out.bf16, [&](auto EXACT) {
            pv_fp8_few_kernel<decltype(XB)::value, decltype(EXACT)::value>
                <<<grid, kFewThreads, 0, s>>>(f, p);
        });
    });
}

void launch_resident(const PvRows& x, const Product& p, hipStream_t s) {
    // shares of the columns: enough workgroups for the chip, few rows quantised twice
    const int mt = (p.M + kFusedM - 1) / kFusedM, nt = (p.N + kResidentN - 1) / kResidentN;
    const int least = (nt + kResidentShare - 1) / kResidentShare;
    int shares = kWanted / mt;
    shares = shares < least ? least : (shares > nt ? nt : shares);
    const int share = (nt + shares - 1) / shares;
    shares = (nt + share - 1) / share;
    const Fused f{x, p.M, p.K, p.b, p.sb};
    with_bool(x.bf16, [&](auto XB) {
        with_bool(!p.out.bf16, [&](auto EXACT) {
            pv_fp8_resident_kernel<decltype(XB)::value, decltype(EXACT)::value>
                <<<(unsigned)((size_t)mt * shares), kResidentThreads,
                   (size_t)p.blocks * kFusedM * kB, s>>>(f, p, share);
        });
    });
}

// The weight (or its transpose) as the product's second operand.
Product with_weight(const Quantised& a, int M, const uint8_t* w, const uint8_t* sw, int N,
                    int blocks, const PvRows& out, float* partial) {
    Product p{};
    p.a = a.q;
    p.sa = a.scale;
    p.M = M;
    p.b = w;
    p.b_row = (size_t)blocks * kB;
    p.b_blk = kB;
    p.sb = sw;
    p.step = kB;
    p.sb_row = blocks;
    p.sb_blk = 1;
    p.N = N;
    p.blocks = blocks;
    p.act = PVCONV_ACT_NONE;
    p.out = out;
    p.partial = partial;
    return p;
}

// Rows a part of a product takes: all of them unless its launches might need more
// than kMostThreads (512 threads for 64 rows x 128 columns of x or y at most). Parts
// are then alike, far larger than what any rule below or path_of looks at.
int rows_a_part(int M, int K, int N) {
    const size_t threads =
        ((size_t)M + kFusedM - 1) / kFusedM * pv_fp8_blocks(K > N ? K : N) * kFusedThreads;
    const size_t parts = (threads + kMostThreads - 1) / kMostThreads;
    return parts <= 1 ? M : pv_fp8_blocks((int)(((size_t)M + parts - 1) / parts)) * kB;
}

// out = act( Q(x) W^T + bias )
void launch_rows_product(const PvRows& x, int M, int K, int N, const uint8_t* weight,
                         const uint8_t* scale, const float* bias, int act, float slope,
                         const PvRows& out, const RowsWs& w, hipStream_t s) {
    const Path path = path_of(M, K, N);
    const int rows = rows_a_part(M, K, N);
    for (int m = 0; m < M; m += rows) {
        const int n = rows < M - m ? rows : M - m;
        PvRows xm = x, ym = out;
        xm.p = (char*)x.p + (size_t)m * x.ld * (x.bf16 ? 2 : 4);
        ym.p = (char*)out.p + (size_t)m * out.ld * (out.bf16 ? 2 : 4);
        Product p = with_weight(w.x, n, weight, scale, N, pv_fp8_blocks(K), ym, w.partial);
        p.K = K;
        p.bias = bias;
        p.act = act;
        p.slope = slope;
        p.splits = 1;
        switch (path) {
            case kFew: launch_few(xm, p, s); break;
            case kResident: launch_resident(xm, p, s); break;
            case kFused: launch_fused(xm, p, s); break;
            case kApart:
                launch_quantise<kRows>(
                    Quantise{xm, n, K, w.x.q, w.x.scale, nullptr, nullptr, nullptr}, s);
                launch_product(p, s);
                break;
        }
    }
}

}  // namespace

pvconv_status pv_launch_fp8_quantize_weight(const PvRows& w, int N, int K, uint8_t* q,
                                            uint8_t* scale, uint8_t* qt, uint8_t* scale_t,
                                            hipStream_t s) {
    launch_quantise<kBlock>(Quantise{w, N, K, q, scale, qt, scale_t, nullptr}, s);
    return pv_launch_status();
}

size_t pv_fp8_linear_ws_bytes(int M, int K, int N) {
    Carve c{nullptr, 0};
    carve_rows(c, M, K, N);
    return c.off;
}

pvconv_status pv_launch_fp8_linear(const PvRows& x, int M, int K, int N, const uint8_t* weight,
                                   const uint8_t* scale, const float* bias, int act, float slope,
                                   const PvRows& y, void* ws, hipStream_t s) {
    Carve c{(char*)ws, 0};
    launch_rows_product(x, M, K, N, weight, scale, bias, act, slope, y, carve_rows(c, M, K, N), s);
    return pv_launch_status();
}

size_t pv_fp8_linear_bwd_ws_bytes(int M, int K, int N) { return carve_bwd(nullptr, M, K, N).total; }

pvconv_status pv_launch_fp8_linear_bwd(const PvRows& dy, const PvRows& x, int M, int K, int N,
                                       const uint8_t* weight_t, const uint8_t* scale_t,
                                       const PvRows& dx, float* dw, float* dbias, void* ws,
                                       hipStream_t s) {
    const BwdWs w = carve_bwd(ws, M, K, N);
    const int mb = pv_fp8_blocks(M);
    if (dx.p && M)
        launch_rows_product(dy, M, N, K, weight_t, scale_t, nullptr, PVCONV_ACT_NONE, 0.f, dx, w.dx,
                            s);
    const Quantise zy{dy, M, N, nullptr, nullptr, w.dyt.q, w.dyt.scale, dbias ? w.sum : nullptr};
    const Quantise zx{x, M, K, nullptr, nullptr, w.xt.q, w.xt.scale, nullptr};
    if (dw && M)
        launch_columns<kCols | kSum>(zy, s, &zx);
    else if (dbias && M)
        launch_columns<kSum>(zy, s);
    if (dw && M) {
        Product p{};
        p.a = w.dyt.q;
        p.sa = w.dyt.scale;
        p.M = N;
        p.b = w.xt.q;
        p.b_row = kB;
        p.b_blk = (size_t)K * kB;
        p.sb = w.xt.scale;
        p.step = 1;
        p.sb_row = 1;
        p.sb_blk = K;
        p.N = K;
        p.blocks = mb;
        p.act = PVCONV_ACT_NONE;
        p.out = PvRows{dw, false, K};
        p.partial = w.partial;
        p.sum = w.sum;
        p.bias_n = N;
        p.bias_blocks = mb;
        p.dbias = dbias;
        launch_product(p, s);
    } else if (dw) {
        pv_fp8_zero_kernel<<<grid_of(((size_t)N * K + kThreads - 1) / kThreads), kThreads, 0, s>>>(
            dw, (size_t)N * K);
    }
    if (dbias && !(dw && M)) {
        Product p{};
        p.sum = w.sum;
        p.bias_n = N;
        p.bias_blocks = mb;
        p.dbias = dbias;
        pv_fp8_bias_kernel<<<(N + kBiasColumns - 1) / kBiasColumns, kThreads, 0, s>>>(p);
    }
    return pv_launch_status();
}
