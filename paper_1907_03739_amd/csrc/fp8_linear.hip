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

// q[r][blocks * 128] and scale[r][blocks] of rows; a wave per block of 128
// consecutive channels, two a lane.
__global__ __launch_bounds__(kThreads) void pv_fp8_rows_kernel(PvRows x, int M, int K, int blocks,
                                                               uint8_t* q, uint8_t* scale) {
    const int lane = threadIdx.x & 63;
    const size_t total = (size_t)M * blocks;
    for (size_t i = (size_t)blockIdx.x * 4 + (threadIdx.x >> 6); i < total;
         i += (size_t)gridDim.x * 4) {
        const size_t row = i / blocks;
        const int kb = (int)(i % blocks), c = kb * kB + 2 * lane;
        const float a = c < K ? pv_load_one(x.p, x.bf16, row * x.ld + c) : 0.f;
        const float b = c + 1 < K ? pv_load_one(x.p, x.bf16, row * x.ld + c + 1) : 0.f;
        uint32_t top = max(finite_bits(a), finite_bits(b));
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, m));
        const int e = block_exponent(top);
        const float f = two_to(-e);
        const uint32_t w = pack_e4m3(nan_unless_finite(a) * f, nan_unless_finite(b) * f, 0.f, 0.f);
        *(uint16_t*)(q + (row * blocks + kb) * kB + 2 * lane) = (uint16_t)w;
        if (lane == 0) scale[i] = (uint8_t)(e + 127);
    }
}

// qt[c][blocks * 128] and scale[c][blocks] of columns, in blocks of 128
// consecutive rows; a thread per (column, block). sum: the columns' plain sums
// over the block, [blocks][K], or NULL.
__global__ __launch_bounds__(kThreads) void pv_fp8_columns_kernel(PvRows x, int M, int K,
                                                                  int blocks, uint8_t* qt,
                                                                  uint8_t* scale, float* sum) {
    const size_t total = (size_t)K * blocks;
    for (size_t i = (size_t)blockIdx.x * kThreads + threadIdx.x; i < total;
         i += (size_t)gridDim.x * kThreads) {
        const int c = (int)(i % K);
        const size_t mb = i / K;
        uint32_t top = 0;
        float s = 0.f;
        for (int r = 0; r < kB; r++) {
            const size_t m = mb * kB + r;
            if (m >= (size_t)M) break;
            const float v = pv_load_one(x.p, x.bf16, m * x.ld + c);
            top = max(top, finite_bits(v));
            s += v;
        }
        if (sum) sum[mb * K + c] = s;
        if (!qt) continue;
        const int e = block_exponent(top);
        const float f = two_to(-e);
        for (int r = 0; r < kB; r += 4) {
            float v[4];
#pragma unroll
            for (int j = 0; j < 4; j++) {
                const size_t m = mb * kB + r + j;
                v[j] = m < (size_t)M
                           ? nan_unless_finite(pv_load_one(x.p, x.bf16, m * x.ld + c)) * f
                           : 0.f;
            }
            *(uint32_t*)(qt + ((size_t)c * blocks + mb) * kB + r) =
                pack_e4m3(v[0], v[1], v[2], v[3]);
        }
        scale[(size_t)c * blocks + mb] = (uint8_t)(e + 127);
    }
}

// A block of 128 x 128 of the weight a workgroup, and its transpose.
__global__ __launch_bounds__(kThreads) void pv_fp8_weight_kernel(PvRows w, int N, int K,
                                                                 uint8_t* q, uint8_t* scale,
                                                                 uint8_t* qt, uint8_t* scale_t) {
    __shared__ uint32_t tops[kThreads];
    const int nb = pv_fp8_blocks(N), kb = pv_fp8_blocks(K);
    const int bn = blockIdx.x / kb, bk = blockIdx.x % kb;
    const int n1 = min(N - bn * kB, kB), k1 = min(K - bk * kB, kB);
    uint32_t top = 0;
    for (int i = threadIdx.x; i < kB * kB; i += kThreads) {
        const int n = i / kB, k = i % kB;
        if (n < n1 && k < k1)
            top = max(top, finite_bits(pv_load_one(w.p, w.bf16, (size_t)(bn * kB + n) * w.ld +
                                                                    bk * kB + k)));
    }
    tops[threadIdx.x] = top;
    __syncthreads();
    for (int m = kThreads / 2; m; m >>= 1) {
        if (threadIdx.x < m) tops[threadIdx.x] = max(tops[threadIdx.x], tops[threadIdx.x + m]);
        __syncthreads();
    }
    const int e = block_exponent(tops[0]);
    const float f = two_to(-e);
    if (threadIdx.x == 0) {
        scale[bn * kb + bk] = (uint8_t)(e + 127);
        if (scale_t) scale_t[bk * nb + bn] = (uint8_t)(e + 127);
    }
    for (int i = threadIdx.x; i < kB * kB; i += kThreads) {
        const int n = i / kB, k = i % kB;
        float v = 0.f;
        if (n < n1 && k < k1)
            v = nan_unless_finite(
                    pv_load_one(w.p, w.bf16, (size_t)(bn * kB + n) * w.ld + bk * kB + k)) *
                f;
        const uint8_t b = (uint8_t)pack_e4m3(v, 0.f, 0.f, 0.f);
        if (n < n1) q[(size_t)(bn * kB + n) * kb * kB + bk * kB + k] = b;
        if (qt && k < k1) qt[(size_t)(bk * kB + k) * nb * kB + bn * kB + n] = b;
    }
}

// out[m][n] = act( sum over blocks of a[m] . b[n] + bias_n ): a wave per tile
// of 16 x 16. a [M][blocks*128], sa [M][blocks]; b [N][blocks*128], its scales
// one per row (step 1) or per 128 rows (step 128).
__global__ __launch_bounds__(kThreads) void pv_fp8_product_kernel(
    const uint8_t* a, const uint8_t* sa, int M, const uint8_t* b, const uint8_t* sb, int step,
    int N, int blocks, const float* bias, int act, float slope, PvRows out) {
    const int lane = threadIdx.x & 63, r = lane & 15, h = lane >> 4;
    const size_t nt = (N + 15) / 16, total = (size_t)((M + 15) / 16) * nt;
    for (size_t t = (size_t)blockIdx.x * 4 + (threadIdx.x >> 6); t < total;
         t += (size_t)gridDim.x * 4) {
        const int m0 = (int)(t / nt) * 16, n0 = (int)(t % nt) * 16;
        const size_t m = min(m0 + r, M - 1), n = min(n0 + r, N - 1);
        const uint8_t* pa = a + m * blocks * kB + h * 32;
        const uint8_t* pb = b + n * blocks * kB + h * 32;
        const uint8_t* qa = sa + m * blocks;
        const uint8_t* qb = sb + n / step * blocks;
        pv_f32x4 acc = {0.f, 0.f, 0.f, 0.f};
        for (int k = 0; k < blocks; k++) {
            i32x8 va, vb;
            __builtin_memcpy(&va, __builtin_assume_aligned(pa + (size_t)k * kB, 16), 32);
            __builtin_memcpy(&vb, __builtin_assume_aligned(pb + (size_t)k * kB, 16), 32);
            acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(va, vb, acc, 0, 0, 0, qa[k], 0,
                                                                   qb[k]);
        }
        const int c = n0 + r;
        if (c < N) {
            const float add = bias ? bias[c] : 0.f;
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const int row = m0 + h * 4 + i;
                if (row < M)
                    pv_store_one(out.p, out.bf16, (size_t)row * out.ld + c,
                                 pv_activate(acc[i] + add, act, slope));
            }
        }
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
struct BwdWs {
    Quantised dy, dyt, xt;
    float* sum;
    size_t total;
};
BwdWs carve_bwd(void* base, int M, int K, int N) {
    Carve c{(char*)base, 0};
    BwdWs w;
    w.dy = c.rows(M, N);
    w.dyt = c.rows(N, M);
    w.xt = c.rows(K, M);
    w.sum = (float*)c.take((size_t)pv_fp8_blocks(M) * N * 4);
    w.total = c.off;
    return w;
}

void launch_rows(const PvRows& x, int M, int K, const Quantised& q, hipStream_t s) {
    const int blocks = pv_fp8_blocks(K);
    pv_fp8_rows_kernel<<<grid_of(((size_t)M * blocks + 3) / 4), kThreads, 0, s>>>(
        x, M, K, blocks, q.q, q.scale);
}

void launch_product(const Quantised& a, int M, const uint8_t* b, const uint8_t* sb, int step,
                    int N, int blocks, const float* bias, int act, float slope, const PvRows& out,
                    hipStream_t s) {
    const size_t tiles = (size_t)((M + 15) / 16) * ((N + 15) / 16);
    pv_fp8_product_kernel<<<grid_of((tiles + 3) / 4), kThreads, 0, s>>>(
        a.q, a.scale, M, b, sb, step, N, blocks, bias, act, slope, out);
}

}  // namespace

pvconv_status pv_launch_fp8_quantize_weight(const PvRows& w, int N, int K, uint8_t* q,
                                            uint8_t* scale, uint8_t* qt, uint8_t* scale_t,
                                            hipStream_t s) {
    pv_fp8_weight_kernel<<<pv_fp8_blocks(N) * pv_fp8_blocks(K), kThreads, 0, s>>>(w, N, K, q, scale,
                                                                                qt, scale_t);
    return pv_launch_status();
}

size_t pv_fp8_linear_ws_bytes(int M, int K, int N) {
    (void)N;
    Carve c{nullptr, 0};
    c.rows(M, K);
    return c.off;
}

pvconv_status pv_launch_fp8_linear(const PvRows& x, int M, int K, int N, const uint8_t* weight,
                                   const uint8_t* scale, const float* bias, int act, float slope,
                                   const PvRows& y, void* ws, hipStream_t s) {
    Carve c{(char*)ws, 0};
    const Quantised q = c.rows(M, K);
    launch_rows(x, M, K, q, s);
    launch_product(q, M, weight, scale, kB, N, pv_fp8_blocks(K), bias, act, slope, y, s);
    return pv_launch_status();
}

size_t pv_fp8_linear_bwd_ws_bytes(int M, int K, int N) { return carve_bwd(nullptr, M, K, N).total; }

pvconv_status pv_launch_fp8_linear_bwd(const PvRows& dy, const PvRows& x, int M, int K, int N,
                                       const uint8_t* weight_t, const uint8_t* scale_t,
                                       const PvRows& dx, float* dw, float* dbias, void* ws,
                                       hipStream_t s) {
    const BwdWs w = carve_bwd(ws, M, K, N);
    const int mb = pv_fp8_blocks(M);
    if (dx.p && M) {
        launch_rows(dy, M, N, w.dy, s);
        launch_product(w.dy, M, weight_t, scale_t, kB, K, pv_fp8_blocks(N), nullptr,
                       PVCONV_ACT_NONE, 0.f, dx, s);
    }
    if ((dw || dbias) && M)
        pv_fp8_columns_kernel<<<grid_of(((size_t)N * mb + kThreads - 1) / kThreads), kThreads, 0,
                                s>>>(dy, M, N, mb, dw ? w.dyt.q : nullptr, w.dyt.scale,
                                     dbias ? w.sum : nullptr);
    if (dw) {
        if (M)
            pv_fp8_columns_kernel<<<grid_of(((size_t)K * mb + kThreads - 1) / kThreads), kThreads,
                                    0, s>>>(x, M, K, mb, w.xt.q, w.xt.scale, nullptr);
        launch_product(w.dyt, N, w.xt.q, w.xt.scale, 1, K, mb, nullptr, PVCONV_ACT_NONE, 0.f,
                       PvRows{dw, false, K}, s);
    }
    if (dbias)
        pv_fp8_bias_kernel<<<(N + kThreads - 1) / kThreads, kThreads, 0, s>>>(w.sum, mb, N, dbias);
    return pv_launch_status();
}
