// e4m3 codes of the paged cache and their power-of-two scales.
#pragma once

#include "common.h"

namespace msparse {

namespace {

// smallest power of two s >= 2^-126 with amax <= 448 s (448 = 0.875 * 2^9)
__device__ __forceinline__ float code_scale(float amax) {
    int e;
    const float m = frexpf(amax, &e);
    e = m <= 0.875f ? e - 9 : e - 8;
    return amax > 0.f ? ldexpf(1.f, max(e, -126)) : 0x1p-126f;
}
__device__ __forceinline__ float finite_abs(float x) {
    const float a = fabsf(x);
    return a < INFINITY ? a : 0.f;
}
// e4m3 of x * inv, to nearest even; what is not finite becomes NaN
__device__ __forceinline__ float code_input(float x, float inv) {
    return fabsf(x) < INFINITY ? x * inv : __builtin_nanf("");
}
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d, float inv) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(code_input(a, inv), code_input(b, inv), 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(code_input(c, inv), code_input(d, inv), w, true);
    return uint32_t(w);
}
// codes moved to a scale 1 / ratio times larger
__device__ __forceinline__ uint32_t rescale4(uint32_t w, float ratio) {
    int r = __builtin_amdgcn_cvt_pk_fp8_f32(__builtin_amdgcn_cvt_f32_fp8(w, 0) * ratio,
                                            __builtin_amdgcn_cvt_f32_fp8(w, 1) * ratio, 0, false);
    r = __builtin_amdgcn_cvt_pk_fp8_f32(__builtin_amdgcn_cvt_f32_fp8(w, 2) * ratio,
                                        __builtin_amdgcn_cvt_f32_fp8(w, 3) * ratio, r, true);
    return uint32_t(r);
}

}  // namespace

}  // namespace msparse
