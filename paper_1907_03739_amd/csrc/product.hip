// Operands of the products in pv_product.h, plain products and column sums.
#include "pv_product.h"

namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ float load_kind(const void* src, PvKind kind, size_t at) {
    if (kind == kPvF32) return ((const float*)src)[at];
    if (kind == kPvBf16) return pv_bf16_to_f32(((const uint16_t*)src)[at]);
    return (float)((const int8_t*)src)[at];
}

// The next bf16 part of v, which leaves v - part. The largest finite values would
// round to infinity: they are cut off instead.
__device__ __forceinline__ uint16_t next_part(float& v) {
    uint16_t h = pv_f32_to_bf16(v);
    const uint32_t u = __float_as_uint(v);
    const bool finite = (u & 0x7fffffffu) < 0x7f800000u;
    if (finite && (h & 0x7fffu) == 0x7f80u) h = (uint16_t)(u >> 16);
    v = finite ? v - pv_bf16_to_f32(h) : 0.f;
    return h;
}

// Eight consecutive columns a thread.
__global__ __launch_bounds__(kThreads) void pv_pack_kernel(PvPack k) {
    const size_t per = k.pitch / 16, total = per * k.R;
    for (size_t at = (size_t)blockIdx.x * kThreads + threadIdx.x; at < total;
         at += (size_t)gridDim.x * kThreads) {
        const size_t row = at / per;
        const int c0 = (int)(at - row * per) * 8;
        const float rs = k.row_scale ? k.row_scale[row] : 1.f;
        float v[8];
        const size_t from = row * k.ld + c0;
        if (c0 + 8 <= k.C && k.kind == kPvBf16) {
            const pv_u32x4 w = *(const pv_u32x4_any*)((const uint16_t*)k.src + from);
#pragma unroll
            for (int i = 0; i < 8; i++)
                v[i] = __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
        } else if (c0 + 8 <= k.C && k.kind == kPvF32) {
            const pv_u32x4 w = *(const pv_u32x4_any*)((const float*)k.src + from);
            const pv_u32x4 y = *(const pv_u32x4_any*)((const float*)k.src + from + 4);
#pragma unroll
            for (int i = 0; i < 8; i++) v[i] = __uint_as_float(i < 4 ? w[i] : y[i - 4]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; i++)
                v[i] = c0 + i < k.C ? load_kind(k.src, k.kind, from + i) : 0.f;
        }
        if (k.row_scale) {
#pragma unroll
            for (int i = 0; i < 8; i++) v[i] *= rs;
        }
        if (k.col_scale) {
#pragma unroll
            for (int i = 0; i < 8; i++)
                if (c0 + i < k.C) v[i] *= k.col_scale[c0 + i];
        }
        for (int part = 0; part < k.parts; part++) {
            uint16_t q[8];
#pragma unroll
            for (int i = 0; i < 8; i++) q[i] = c0 + i < k.C ? next_part(v[i]) : (uint16_t)0;
            pv_u32x4 w;
#pragma unroll
            for (int i = 0; i < 4; i++) w[i] = (uint32_t)q[2 * i] | ((uint32_t)q[2 * i + 1] << 16);
            *(pv_u32x4*)(k.dst + part * k.part_bytes + row * k.pitch + (size_t)c0 * 2) = w;
        }
    }
}

// Tiles of 64 x 64 through LDS.
__global__ __launch_bounds__(kThreads) void pv_pack_transposed_kernel(PvPack k) {
    __shared__ float tile[64][65];
    const size_t rt = k.pitch / 128, total = rt * ((k.C + 63) / 64);
    for (size_t t = blockIdx.x; t < total; t += gridDim.x) {
        const size_t r0 = t % rt * 64;
        const int c0 = (int)(t / rt) * 64;
        const int c = threadIdx.x & 63;
        const float cs = k.col_scale && c0 + c < k.C ? k.col_scale[c0 + c] : 1.f;
        for (int i = threadIdx.x >> 6; i < 64; i += 4) {
            float v = 0.f;
            if (r0 + i < (size_t)k.R && c0 + c < k.C) {
                v = load_kind(k.src, k.kind, (r0 + i) * k.ld + c0 + c);
                if (k.row_scale) v *= k.row_scale[r0 + i];
                if (k.col_scale) v *= cs;
            }
            tile[i][c] = v;
        }
        __syncthreads();
        for (int q = threadIdx.x; q < 512; q += kThreads) {  // eight rows of a column
            const int col = q >> 3, i0 = (q & 7) * 8;
            if (c0 + col >= k.C) continue;
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; i++) v[i] = tile[i0 + i][col];
            for (int part = 0; part < k.parts; part++) {
                pv_u32x4 w;
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    const uint32_t lo = next_part(v[2 * i]), hi = next_part(v[2 * i + 1]);
                    w[i] = lo | (hi << 16);
                }
                *(pv_u32x4*)(k.dst + part * k.part_bytes + (size_t)(c0 + col) * k.pitch +
                             (r0 + i0) * 2) = w;
            }
        }
        __syncthreads();
    }
}

struct PlainEpi {
    PvPlain e;
    template <int MI>
    __device__ __forceinline__ void tile(const PvProduct& p, int mw, int nw, int lane,
                                         const pv_f32x4 (&acc)[4][MI], uint8_t*) const {
        const int r = lane & 15, n = nw + 16 * (lane >> 4);
#pragma unroll
        for (int i = 0; i < MI; i++) {
            const int m = mw + 16 * i + r;
            if (m >= p.M) continue;
            float v[16];
#pragma unroll
            for (int c = 0; c < 16; c++) v[c] = acc[c >> 2][i][c & 3];
            if (e.add) {
                const float* from = e.add + (size_t)m * p.N + n;
#pragma unroll
                for (int c = 0; c < 16; c += 4) {
                    if (n + c + 4 <= p.N) {
                        const pv_u32x4 w = *(const pv_u32x4_any*)(from + c);
#pragma unroll
                        for (int u = 0; u < 4; u++) v[c + u] += __uint_as_float(w[u]);
                    } else {
#pragma unroll
                        for (int u = 0; u < 4; u++)
                            if (n + c + u < p.N) v[c + u] += from[c + u];
                    }
                }
            }
            pv_store_run<16>(e.out, m, n, p.N, v);
        }
    }
    int N;
    __device__ __forceinline__ void one(int m, int n, float v) const {
        if (e.add) v += e.add[(size_t)m * N + n];
        pv_store_one(e.out.p, e.out.bf16, (size_t)m * e.out.ld + n, v);
    }
};

// Sums of columns over a run of rows: 64 columns a workgroup, four rows at a time.
constexpr int kSumRows = 256;
__global__ __launch_bounds__(kThreads) void pv_column_sum_kernel(PvRows x, int M, int N,
                                                                 float* partial) {
    __shared__ double part[4][64];
    const size_t nb = (N + 63) / 64, total = nb * ((M + kSumRows - 1) / kSumRows);
    const int w = threadIdx.x >> 6, lane = threadIdx.x & 63;
    for (size_t t = blockIdx.x; t < total; t += gridDim.x) {
        const int c = (int)(t % nb) * 64 + lane;
        const size_t r0 = t / nb * kSumRows;
        const int rows = (int)min((size_t)kSumRows, (size_t)M - r0);
        double s = 0.;
        if (c < N)
#pragma unroll 8
            for (int i = w; i < rows; i += 4)
                s += (double)pv_load_one(x.p, x.bf16, (r0 + i) * x.ld + c);
        part[w][lane] = s;
        __syncthreads();
        if (w == 0 && c < N)
            partial[t / nb * N + c] =
                (float)(((part[0][lane] + part[1][lane]) + part[2][lane]) + part[3][lane]);
        __syncthreads();
    }
}

// 16 columns a workgroup, 16 threads a column, in a fixed order.
__global__ __launch_bounds__(kThreads) void pv_sum_parts_kernel(const float* partial, int parts,
                                                                int N, float* out) {
    __shared__ double part[kThreads];
    const int c = (int)blockIdx.x * 16 + (threadIdx.x & 15);
    double s = 0.;
    if (c < N)
        for (int i = threadIdx.x >> 4; i < parts; i += 16) s += (double)partial[(size_t)i * N + c];
    part[threadIdx.x] = s;
    __syncthreads();
    if (threadIdx.x < 16 && c < N) {
        for (int w = 1; w < 16; w++) s += part[threadIdx.x + 16 * w];
        out[c] = (float)s;
    }
}

}  // namespace

void pv_launch_pack(const PvPack& k, hipStream_t s) {
    if (k.R <= 0) return;
    hipLaunchKernelGGL(pv_pack_kernel, dim3(pv_blocks(k.pitch / 16 * k.R, kThreads)),
                       dim3(kThreads), 0, s, k);
}
void pv_launch_pack_transposed(const PvPack& k, hipStream_t s) {
    if (k.C <= 0 || k.pitch == 0) return;
    hipLaunchKernelGGL(pv_pack_transposed_kernel,
                       dim3(pv_blocks(k.pitch / 128 * ((k.C + 63) / 64), 1)), dim3(kThreads), 0, s,
                       k);
}

void pv_launch_plain(const PvProduct& p, const PvPlain& e, hipStream_t s) {
    pv_run_product<false>(p, PlainEpi{e, p.N}, s);
}

void pv_launch_sum_parts(const float* partial, int parts, int N, float* out, hipStream_t s) {
    hipLaunchKernelGGL(pv_sum_parts_kernel, dim3((N + 15) / 16), dim3(kThreads), 0, s, partial,
                       parts, N, out);
}
size_t pv_column_sum_bytes(int M, int N) { return (size_t)((M + kSumRows - 1) / kSumRows) * N * 4; }
void pv_launch_column_sum(const PvRows& x, int M, int N, float* partial, float* out,
                          hipStream_t s) {
    const int parts = (M + kSumRows - 1) / kSumRows;
    if (parts)
        hipLaunchKernelGGL(pv_column_sum_kernel, dim3(pv_blocks((size_t)parts * ((N + 63) / 64), 1)),
                           dim3(kThreads), 0, s, x, M, N, partial);
    pv_launch_sum_parts(partial, parts, N, out, s);
}
