// Argument checks shared by the C ABI's files (host only).
#pragma once

#include "pv_common.h"

namespace {

inline bool dtype_ok(pvconv_dtype d) { return d == PVCONV_F32 || d == PVCONV_BF16; }
inline size_t esize(pvconv_dtype d) { return d == PVCONV_BF16 ? 2 : 4; }
inline bool act_ok(pvconv_act a) {
    return a == PVCONV_ACT_NONE || a == PVCONV_ACT_RELU || a == PVCONV_ACT_LEAKY;
}
inline bool bn_ok(const pvconv_bn* bn) {
    if (!bn || !bn->gamma) return true;
    return bn->beta && bn->mean && bn->var && bn->eps >= 0.f;
}
inline hipStream_t as_stream(void* s) { return (hipStream_t)s; }

// Elements must fit the int32 voxel ids and list offsets the kernels use.
inline bool sizes_fit(long long B, long long N) { return B * N <= (1LL << 30); }

// Two row-major arrays of `rows` rows share at least one byte: array a has
// rows of ca elements of dtype ta at a stride of lda elements, b likewise.
// Column slices of one wider array (the same row pitch, disjoint column
// ranges, as the segmentation networks use them) do not overlap.
inline bool overlap(const void* a, long long rows, int ca, int lda, pvconv_dtype ta,
                    const void* b, int cb, int ldb, pvconv_dtype tb) {
    if (rows <= 0) return false;
    const long long pa = (long long)lda * esize(ta), pb = (long long)ldb * esize(tb);
    const long long wa = (long long)ca * esize(ta), wb = (long long)cb * esize(tb);
    const long long a0 = (long long)(uintptr_t)a, b0 = (long long)(uintptr_t)b;
    if (a0 + (rows - 1) * pa + wa <= b0 || b0 + (rows - 1) * pb + wb <= a0) return false;
    if (pa != pb) return true;
    // the same pitch: b's rows start e bytes into a's rows (or a's into b's)
    const long long e = ((b0 - a0) % pa + pa) % pa;
    return !(e >= wa && e + wb <= pa);
}

// Two byte ranges [a, a + na) and [b, b + nb) intersect.
inline bool bytes_overlap(const void* a, size_t na, const void* b, size_t nb) {
    const uintptr_t a0 = (uintptr_t)a, b0 = (uintptr_t)b;
    return na && nb && a0 < b0 + nb && b0 < a0 + na;
}

}  // namespace
