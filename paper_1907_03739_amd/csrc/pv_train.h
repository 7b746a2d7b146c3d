// Internal interface and device helpers of the operators declared in
// pvconv_train.h: group norm, the 8-bit linear layer, the distillation loss.
#pragma once

#include "pv_common.h"
#include "pvconv_train.h"

// VEC consecutive elements of a row as floats: one aligned load of VEC * 2
// (bf16) or VEC * 4 bytes. VEC = 8 of fp32 is two 16-byte loads.
template <bool BF16, int VEC>
__device__ __forceinline__ void pv_load_vec(const void* base, size_t at, float (&v)[VEC]) {
    if constexpr (BF16) {
        const uint16_t* p = (const uint16_t*)base + at;
        if constexpr (VEC == 1) {
            v[0] = pv_bf16_to_f32(*p);
        } else {
            uint32_t w[VEC / 2];
            __builtin_memcpy(w, __builtin_assume_aligned(p, VEC * 2), VEC * 2);
#pragma unroll
            for (int i = 0; i < VEC / 2; i++) {
                v[2 * i] = __uint_as_float(w[i] << 16);
                v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
            }
        }
    } else {
        const float* p = (const float*)base + at;
        __builtin_memcpy(v, __builtin_assume_aligned(p, VEC >= 4 ? 16 : VEC * 4), VEC * 4);
    }
}

template <bool BF16, int VEC>
__device__ __forceinline__ void pv_store_vec(void* base, size_t at, const float (&v)[VEC]) {
    if constexpr (BF16) {
        uint16_t* p = (uint16_t*)base + at;
        if constexpr (VEC == 1) {
            *p = pv_f32_to_bf16(v[0]);
        } else {
            uint32_t w[VEC / 2];
#pragma unroll
            for (int i = 0; i < VEC / 2; i++) w[i] = pv_pack_bf16x2(v[2 * i], v[2 * i + 1]);
            __builtin_memcpy(__builtin_assume_aligned(p, VEC * 2), w, VEC * 2);
        }
    } else {
        float* p = (float*)base + at;
        __builtin_memcpy(__builtin_assume_aligned(p, VEC >= 4 ? 16 : VEC * 4), v, VEC * 4);
    }
}

__device__ __forceinline__ float pv_load_one(const void* base, bool bf16, size_t at) {
    return bf16 ? pv_bf16_to_f32(((const uint16_t*)base)[at]) : ((const float*)base)[at];
}
__device__ __forceinline__ void pv_store_one(void* base, bool bf16, size_t at, float v) {
    if (bf16)
        ((uint16_t*)base)[at] = pv_f32_to_bf16(v);
    else
        ((float*)base)[at] = v;
}

// The largest power of two up to `most` that divides every n and by which the
// pointer is aligned (elements of es bytes).
static inline int pv_vec_width(int most, int es, const void* p, int n0, int n1) {
    int v = most;
    while (v > 1 && (n0 % v || n1 % v || ((uintptr_t)p & (uintptr_t)(v * es > 16 ? 15 : v * es - 1))))
        v >>= 1;
    return v;
}

// ---- group norm (group_norm.hip) -------------------------------------------
size_t pv_group_norm_ws_bytes(int B, int N, int C, int groups);
size_t pv_group_norm_bwd_ws_bytes(int B, int N, int C, int groups);
struct PvRows {  // rows of channels: an array, its type, its row stride
    void* p;
    bool bf16;
    int ld;
};
struct PvNorm {
    int B, N, C, groups;
    const int32_t* lengths;
    const float* gamma;
    const float* beta;
    float eps;
    int act;
    float slope;
};
pvconv_status pv_launch_group_norm(const PvNorm& n, const PvRows& x, const PvRows& y,
                                   float* stats, void* ws, hipStream_t s);
pvconv_status pv_launch_group_norm_bwd(const PvNorm& n, const PvRows& dy, const PvRows& x,
                                       const PvRows& dx, const float* stats, float* dgamma,
                                       float* dbeta, void* ws, hipStream_t s);

// ---- 8-bit linear layer (fp8_linear.hip) -----------------------------------
__host__ __device__ static inline int pv_fp8_blocks(int n) {
    return (n + PVCONV_FP8_BLOCK - 1) / PVCONV_FP8_BLOCK;
}
pvconv_status pv_launch_fp8_quantize_weight(const PvRows& w, int N, int K, uint8_t* q,
                                            uint8_t* scale, uint8_t* qt, uint8_t* scale_t,
                                            hipStream_t s);
size_t pv_fp8_linear_ws_bytes(int M, int K, int N);
pvconv_status pv_launch_fp8_linear(const PvRows& x, int M, int K, int N, const uint8_t* weight,
                                   const uint8_t* scale, const float* bias, int act, float slope,
                                   const PvRows& y, void* ws, hipStream_t s);
size_t pv_fp8_linear_bwd_ws_bytes(int M, int K, int N);
pvconv_status pv_launch_fp8_linear_bwd(const PvRows& dy, const PvRows& x, int M, int K, int N,
                                       const uint8_t* weight_t, const uint8_t* scale_t,
                                       const PvRows& dx, float* dw, float* dbias, void* ws,
                                       hipStream_t s);

// ---- distillation loss (distill.hip) ---------------------------------------
struct PvDistill {
    PvRows z;
    int M, V;
    const float* t_val;
    const int32_t* t_class;
    int top;
    const int32_t* labels;
    float temperature, alpha;
};
// loss (and lse) and, where dz.p is set, the gradient of row_weight
pvconv_status pv_launch_distill(const PvDistill& d, const float* row_weight, float* loss,
                                float* lse, const PvRows& dz, hipStream_t s);
pvconv_status pv_launch_distill_bwd(const PvDistill& d, const float* lse, const float* dloss,
                                    const PvRows& dz, hipStream_t s);
