// Linear layer in 8-bit floating point, a power-of-two scale for each block of
// 128 values, and its gradients (pvconv_train.h).
//
// Activations are quantised into the workspace, then multiplied on the scaled
// matrix instruction of gfx950 (16x16x128: one instruction spans one block of
// 128, so it takes the blocks' two scales as they are and its sums stay fp32).
#include <type_traits>

#include "pv_train.h"

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
// a value that is not finite becomes NaN
__device__ __forceinline__ float nan_unless_finite(float v) {
    return (__float_as_uint(v) & 0x7fffffffu) < 0x7f800000u ? v : __uint_as_float(0x7fc00000u);
}

// Four values, already scaled, as e4m3 bytes (round to nearest even).
__device__ __forceinline__ uint32_t pack_e4m3(float a, float b, float c, float d) {
    int r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    r = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true);
    return (uint32_t)r;
}

// The same of values still to be scaled by f; not finite: NaN.
__device__ __forceinline__ uint32_t pack_scaled(float a, float b, float c, float d, float f) {
    return pack_e4m3(nan_unless_finite(a) * f, nan_unless_finite(b) * f, nan_unless_finite(c) * f,
                     nan_unless_finite(d) * f);
}

// The quantisers: a workgroup takes a tile of 128 x 128 into registers, eight
// columns by eight rows a thread, and writes it in any of
//   kRows    q[r][cb * 128 ..], scales per row and 128 columns: scale[cb][r]
//   kCols    qt[c][rb * 128 ..], scales per column and 128 rows: scale_t[rb][c]
//   kBlock   both, one scale for the tile: scale[rb][cb], scale_t[cb][rb]
//   kSum     sum[rb][c]: the tile's plain column sums
// Bound by HBM: one read of x, a byte a value out; the transposed bytes turn
// around in LDS so that their stores are rows of 128 bytes.
enum { kRows = 1, kCols = 2, kBlock = 4, kSum = 8 };
struct Quantise {
    PvRows x;
    int M, C;      // rows, columns
    uint8_t* q;
    uint8_t* scale;
    uint8_t* qt;
    uint8_t* scale_t;
    float* sum;
};
constexpr int kPitch = 33;  // dwords a transposed column in LDS (32 and one to spread the banks)

__device__ __forceinline__ uint32_t max_over_row16(uint32_t v) {  // 16 consecutive lanes
#pragma unroll
    for (int m = 1; m < 16; m <<= 1) v = max(v, (uint32_t)__shfl_xor((int)v, m));
    return v;
}

template <bool XB, bool VEC, int WHAT>
__global__ __launch_bounds__(kThreads) void pv_fp8_quantise_kernel(Quantise z) {
    constexpr bool kT = (WHAT & (kCols | kBlock)) != 0;
    __shared__ uint32_t turn[kT ? kB * kPitch : 1];
    __shared__ uint32_t tops[4][kB];
    __shared__ float sums[(WHAT & kSum) ? 4 : 1][kB];
    const int cbs = pv_fp8_blocks(z.C), rbs = pv_fp8_blocks(z.M);
    const int rb = blockIdx.x / cbs, cb = blockIdx.x % cbs;
    const int wave = threadIdx.x >> 6, cg = threadIdx.x & 15, rg = threadIdx.x >> 4;
    const int c0 = cb * kB + cg * 8;
    // row of the tile: half * 64 + rg * 4 + j
    float v[8][8];
#pragma unroll
    for (int r = 0; r < 8; r++) {
        const int row = rb * kB + (r >> 2) * 64 + rg * 4 + (r & 3);
        const size_t at = (size_t)row * z.x.ld + c0;
        if (row < z.M && VEC && c0 + 8 <= z.C) {
            pv_load_vec<XB, 8>(z.x.p, at, v[r]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; i++)
                v[r][i] = row < z.M && c0 + i < z.C ? pv_load_one(z.x.p, XB, at + i) : 0.f;
        }
    }
    if constexpr (WHAT & kSum) {
        float t[8];
#pragma unroll
        for (int i = 0; i < 8; i++) {
            t[i] = 0.f;
#pragma unroll
            for (int r = 0; r < 8; r++) t[i] += v[r][i];
            t[i] += __shfl_xor(t[i], 16);
            t[i] += __shfl_xor(t[i], 32);
            if ((threadIdx.x & 48) == 0) sums[wave][cg * 8 + i] = t[i];
        }
    }
    if constexpr (WHAT & kRows) {
#pragma unroll
        for (int r = 0; r < 8; r++) {
            uint32_t top = 0;
#pragma unroll
            for (int i = 0; i < 8; i++) top = max(top, finite_bits(v[r][i]));
            const int e = block_exponent(max_over_row16(top));
            const float f = two_to(-e);
            const int row = rb * kB + (r >> 2) * 64 + rg * 4 + (r & 3);
            uint2 w;
            w.x = pack_scaled(v[r][0], v[r][1], v[r][2], v[r][3], f);
            w.y = pack_scaled(v[r][4], v[r][5], v[r][6], v[r][7], f);
            if (row < z.M) {
                *(uint2*)(z.q + ((size_t)row * cbs + cb) * kB + cg * 8) = w;
                if (cg == 0) z.scale[(size_t)cb * z.M + row] = (uint8_t)(e + 127);
            }
        }
    }
    if constexpr (kT) {
#pragma unroll
        for (int i = 0; i < 8; i++) {
            uint32_t top = 0;
#pragma unroll
            for (int r = 0; r < 8; r++) top = max(top, finite_bits(v[r][i]));
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
            const float f = two_to(-e);
            turn[c * kPitch + rg] = pack_scaled(v[0][i], v[1][i], v[2][i], v[3][i], f);
            turn[c * kPitch + 16 + rg] = pack_scaled(v[4][i], v[5][i], v[6][i], v[7][i], f);
            if (!(WHAT & kBlock) && rg == 0 && cb * kB + c < z.C)
                z.scale_t[(size_t)rb * z.C + cb * kB + c] = (uint8_t)(e + 127);
        }
        if constexpr (WHAT & kBlock) {
            const float f = two_to(-tile_e);
#pragma unroll
            for (int r = 0; r < 8; r++) {
                const int row = rb * kB + (r >> 2) * 64 + rg * 4 + (r & 3);
                uint2 w;
                w.x = pack_scaled(v[r][0], v[r][1], v[r][2], v[r][3], f);
                w.y = pack_scaled(v[r][4], v[r][5], v[r][6], v[r][7], f);
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
            uint4* to = (uint4*)(z.qt + ((size_t)(cb * kB + c) * rbs + rb) * kB + h * 4);
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const uint32_t* t = turn + c * kPitch + h + 4 * i;
                to[i] = make_uint4(t[0], t[1], t[2], t[3]);
            }
        }
    }
    if constexpr (WHAT & kSum) {
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
// bf16 outputs, which round 40 times coarser, take it; fp32 outputs turn the
// bytes, with their scales, into bf16 (exact: four digits and a power of two)
// and use the bf16 instruction, whose sums are good to fp32, at half the rate.
//
// LDS rows are 128 bytes, in 16-byte pieces exchanged by a key of the row
// (a_key, b_key), so that the lanes of a fragment read fall on all the banks.
struct Product {
    const uint8_t* a;   // [M][blocks * 128]
    const uint8_t* sa;  // [blocks][M]
    int M;
    const uint8_t* b;   // [N][blocks * 128]
    const uint8_t* sb;  // at (n / step) * sb_row + block * sb_blk
    int step;
    size_t sb_row, sb_blk;
    int N, blocks;
    int per, splits;    // blocks a split takes
    const float* bias;
    int act;
    float slope;
    PvRows out;
    float* partial;     // [splits][M][N] where splits > 1
};
constexpr int kTile = 128;

__device__ __forceinline__ int a_key(int row) { return row & 7; }
__device__ __forceinline__ int b_key(int row) { return (row & 3) | ((row >> 2) & 4); }

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// Eight e4m3 bytes times 2^(byte - 127), as bf16.
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

// 16 consecutive outputs of a row from column n on
__device__ __forceinline__ void store16(const Product& p, int split, int m, int n,
                                        const float (&v)[16], bool vec) {
    if (p.splits > 1) {
        float* o = p.partial + ((size_t)split * p.M + m) * p.N + n;
        if (vec && n + 16 <= p.N) {
#pragma unroll
            for (int i = 0; i < 4; i++)
                *(float4*)(o + 4 * i) = make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2],
                                                    v[4 * i + 3]);
        } else {
#pragma unroll
            for (int i = 0; i < 16; i++)
                if (n + i < p.N) o[i] = v[i];
        }
        return;
    }
    float r[16];
#pragma unroll
    for (int i = 0; i < 16; i++) {
        const float add = p.bias && n + i < p.N ? p.bias[n + i] : 0.f;
        r[i] = pv_activate(v[i] + add, p.act, p.slope);
    }
    const size_t at = (size_t)m * p.out.ld + n;
    if (vec && n + 16 <= p.N) {
        if (p.out.bf16) {
            uint32_t w[8];
#pragma unroll
            for (int i = 0; i < 8; i++) w[i] = pv_pack_bf16x2(r[2 * i], r[2 * i + 1]);
            uint4* o = (uint4*)((uint16_t*)p.out.p + at);
            o[0] = make_uint4(w[0], w[1], w[2], w[3]);
            o[1] = make_uint4(w[4], w[5], w[6], w[7]);
        } else {
            float4* o = (float4*)((float*)p.out.p + at);
#pragma unroll
            for (int i = 0; i < 4; i++)
                o[i] = make_float4(r[4 * i], r[4 * i + 1], r[4 * i + 2], r[4 * i + 3]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 16; i++)
            if (n + i < p.N) pv_store_one(p.out.p, p.out.bf16, at + i, r[i]);
    }
}

template <bool EXACT>
__global__ __launch_bounds__(kThreads, 2) void pv_fp8_tile_kernel(Product p, bool vec) {
    // two stages, arrays of their own: the loads into one are then seen not to
    // touch what is read of the other, and are not waited for
    __shared__ __align__(16) uint8_t la0[kTile * kB], la1[kTile * kB];
    __shared__ __align__(16) uint8_t lb0[kTile * kB], lb1[kTile * kB];
    // scale bytes, as the fragments take them: dword r of a wave's 64 rows
    // holds the bytes of the four fragments' row r
    __shared__ __align__(16) uint8_t ls0[2 * kTile], ls1[2 * kTile];
    const int mt = (p.M + kTile - 1) / kTile, nt = (p.N + kTile - 1) / kTile;
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
        ga[q] = p.a + (size_t)min(m0 + row, p.M - 1) * p.blocks * kB + (size_t)k0 * kB +
                (c ^ a_key(row)) * 16;
        gb[q] = p.b + (size_t)min(n0 + row, p.N - 1) * p.blocks * kB + (size_t)k0 * kB +
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
            ga[q] += kB;
            gb[q] += kB;
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
            f.u[0] = *(const uint4*)(la + ra * kB + ((2 * h) ^ a_key(ra)) * 16);
            f.u[1] = *(const uint4*)(la + ra * kB + ((2 * h + 1) ^ a_key(ra)) * 16);
            g.u[0] = *(const uint4*)(lb + rb * kB + ((2 * h) ^ b_key(rb)) * 16);
            g.u[1] = *(const uint4*)(lb + rb * kB + ((2 * h + 1) ^ b_key(rb)) * 16);
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
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const int m = m0 + wm + 16 * i + r;
        float v[16];
#pragma unroll
        for (int j = 0; j < 4; j++)
#pragma unroll
            for (int e = 0; e < 4; e++) v[4 * j + e] = acc[j][i][e];
        if (m < p.M) store16(p, split, m, n0 + wn + 16 * h, v, vec);
    }
}

// out = act( the splits' sums in order + bias )
__global__ __launch_bounds__(kThreads) void pv_fp8_join_kernel(Product p) {
    const size_t total = (size_t)p.M * p.N;
    for (size_t i = (size_t)blockIdx.x * kThreads + threadIdx.x; i < total;
         i += (size_t)gridDim.x * kThreads) {
        float s = 0.f;
        for (int k = 0; k < p.splits; k++) s += p.partial[(size_t)k * total + i];
        const size_t m = i / p.N;
        const int n = (int)(i - m * p.N);
        pv_store_one(p.out.p, p.out.bf16, m * p.out.ld + n,
                     pv_activate(s + (p.bias ? p.bias[n] : 0.f), p.act, p.slope));
    }
}

// dbias from the blocks' column sums, in block order
__global__ __launch_bounds__(kThreads) void pv_fp8_bias_kernel(const float* sum, int blocks, int N,
                                                               float* dbias) {
    const int c = blockIdx.x * kThreads + threadIdx.x;
    if (c >= N) return;
    double s = 0.;
    for (int i = 0; i < blocks; i++) s += (double)sum[(size_t)i * N + c];
    dbias[c] = (float)s;
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
// How many ways a product's blocks are split: one where its tiles fill the
// chip, else enough for about kWanted workgroups of two blocks or more.
constexpr int kWanted = 512;
void plan_splits(int M, int N, int blocks, int* per, int* splits) {
    const size_t tiles = (size_t)((M + kTile - 1) / kTile) * ((N + kTile - 1) / kTile);
    *per = blocks;
    if (tiles > 0 && tiles < kWanted / 2 && blocks > 1) {
        const int most = (blocks + 1) / 2;
        int n = (int)((kWanted + tiles - 1) / tiles);
        n = n < 1 ? 1 : (n > most ? most : n);
        *per = (blocks + n - 1) / n;
    }
    *splits = blocks > 1 ? (blocks + *per - 1) / *per : 1;
}
size_t partial_bytes(int M, int N, int blocks) {
    int per, splits;
    plan_splits(M, N, blocks, &per, &splits);
    return splits > 1 ? (size_t)splits * M * N * 4 : 0;
}

struct FwdWs {
    Quantised x;
    float* partial;
    size_t total;
};
FwdWs carve_fwd(void* base, int M, int K, int N) {
    Carve c{(char*)base, 0};
    FwdWs w;
    w.x = c.rows(M, K);
    w.partial = (float*)c.take(partial_bytes(M, N, pv_fp8_blocks(K)));
    w.total = c.off;
    return w;
}
struct BwdWs {
    Quantised dy, dyt, xt;
    float* sum;
    float* partial;  // dx's, then dw's
    size_t total;
};
BwdWs carve_bwd(void* base, int M, int K, int N) {
    Carve c{(char*)base, 0};
    BwdWs w;
    w.dy = c.rows(M, N);
    w.dyt = c.rows(N, M);
    w.xt = c.rows(K, M);
    w.sum = (float*)c.take((size_t)pv_fp8_blocks(M) * N * 4);
    const size_t px = partial_bytes(M, K, pv_fp8_blocks(N)), pw = partial_bytes(N, K, pv_fp8_blocks(M));
    w.partial = (float*)c.take(px > pw ? px : pw);
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

template <int WHAT>
void launch_quantise(const Quantise& z, hipStream_t s) {
    const size_t tiles = (size_t)pv_fp8_blocks(z.M) * pv_fp8_blocks(z.C);
    with_bool(z.x.bf16, [&](auto XB) {
        with_bool(pv_vec_width(8, z.x.bf16 ? 2 : 4, z.x.p, 8, z.x.ld) == 8, [&](auto VEC) {
            pv_fp8_quantise_kernel<decltype(XB)::value, decltype(VEC)::value, WHAT>
                <<<(unsigned)tiles, kThreads, 0, s>>>(z);
        });
    });
}

void launch_product(Product p, hipStream_t s) {
    plan_splits(p.M, p.N, p.blocks, &p.per, &p.splits);
    const size_t total = (size_t)((p.M + kTile - 1) / kTile) * ((p.N + kTile - 1) / kTile) * p.splits;
    const unsigned grid = (unsigned)((total + 7) / 8 * 8);
    const bool vec = p.splits > 1 ? p.N % 4 == 0
                                  : pv_aligned16(p.out.p) && p.out.ld % (p.out.bf16 ? 8 : 4) == 0;
    if (p.out.bf16)
        pv_fp8_tile_kernel<false><<<grid, kThreads, 0, s>>>(p, vec);
    else
        pv_fp8_tile_kernel<true><<<grid, kThreads, 0, s>>>(p, vec);
    if (p.splits > 1)
        pv_fp8_join_kernel<<<grid_of(((size_t)p.M * p.N + kThreads - 1) / kThreads), kThreads, 0,
                             s>>>(p);
}

// The weight (or its transpose) as the product's second operand.
Product with_weight(const Quantised& a, int M, const uint8_t* w, const uint8_t* sw, int N,
                    int blocks, const PvRows& out, float* partial) {
    Product p{};
    p.a = a.q;
    p.sa = a.scale;
    p.M = M;
    p.b = w;
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

}  // namespace

pvconv_status pv_launch_fp8_quantize_weight(const PvRows& w, int N, int K, uint8_t* q,
                                            uint8_t* scale, uint8_t* qt, uint8_t* scale_t,
                                            hipStream_t s) {
    launch_quantise<kBlock>(Quantise{w, N, K, q, scale, qt, scale_t, nullptr}, s);
    return pv_launch_status();
}

size_t pv_fp8_linear_ws_bytes(int M, int K, int N) { return carve_fwd(nullptr, M, K, N).total; }

pvconv_status pv_launch_fp8_linear(const PvRows& x, int M, int K, int N, const uint8_t* weight,
                                   const uint8_t* scale, const float* bias, int act, float slope,
                                   const PvRows& y, void* ws, hipStream_t s) {
    const FwdWs w = carve_fwd(ws, M, K, N);
    launch_quantise<kRows>(Quantise{x, M, K, w.x.q, w.x.scale, nullptr, nullptr, nullptr}, s);
    Product p = with_weight(w.x, M, weight, scale, N, pv_fp8_blocks(K), y, w.partial);
    p.bias = bias;
    p.act = act;
    p.slope = slope;
    launch_product(p, s);
    return pv_launch_status();
}

size_t pv_fp8_linear_bwd_ws_bytes(int M, int K, int N) { return carve_bwd(nullptr, M, K, N).total; }

pvconv_status pv_launch_fp8_linear_bwd(const PvRows& dy, const PvRows& x, int M, int K, int N,
                                       const uint8_t* weight_t, const uint8_t* scale_t,
                                       const PvRows& dx, float* dw, float* dbias, void* ws,
                                       hipStream_t s) {
    const BwdWs w = carve_bwd(ws, M, K, N);
    const int mb = pv_fp8_blocks(M);
    if (M) {
        const Quantise z{dy, M, N, w.dy.q, w.dy.scale, w.dyt.q, w.dyt.scale, w.sum};
        if (dx.p && dw && dbias)
            launch_quantise<kRows | kCols | kSum>(z, s);
        else {
            if (dx.p) launch_quantise<kRows>(z, s);
            if (dw) launch_quantise<kCols>(z, s);
            if (dbias) launch_quantise<kSum>(z, s);
        }
    }
    if (dx.p && M)
        launch_product(with_weight(w.dy, M, weight_t, scale_t, K, pv_fp8_blocks(N), dx, w.partial),
                       s);
    if (dw && M) {
        launch_quantise<kCols>(Quantise{x, M, K, nullptr, nullptr, w.xt.q, w.xt.scale, nullptr}, s);
        Product p{};
        p.a = w.dyt.q;
        p.sa = w.dyt.scale;
        p.M = N;
        p.b = w.xt.q;
        p.sb = w.xt.scale;
        p.step = 1;
        p.sb_row = 1;
        p.sb_blk = K;
        p.N = K;
        p.blocks = mb;
        p.act = PVCONV_ACT_NONE;
        p.out = PvRows{dw, false, K};
        p.partial = w.partial;
        launch_product(p, s);
    } else if (dw) {
        pv_fp8_zero_kernel<<<grid_of(((size_t)N * K + kThreads - 1) / kThreads), kThreads, 0, s>>>(
            dw, (size_t)N * K);
    }
    if (dbias)
        pv_fp8_bias_kernel<<<(N + kThreads - 1) / kThreads, kThreads, 0, s>>>(w.sum, mb, N, dbias);
    return pv_launch_status();
}
