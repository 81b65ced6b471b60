// Rounding into 8-bit floating point: a block's scale from its largest magnitude,
// and values within the scaled range.
#pragma once

#include "model_internal.h"

#include <hip/hip_bf16.h>
#include <hip/hip_fp16.h>

namespace o2m {

__device__ inline float as_float(float x) { return x; }
__device__ inline float as_float(__half x) { return __half2float(x); }
__device__ inline float as_float(__hip_bfloat16 x) { return __bfloat162float(x); }

__device__ inline bool finite(float x) { return fabsf(x) <= 3.402823466e38f; }
// |x|, and 0 in the place of Inf and NaN
__device__ inline float magnitude(float x) { return finite(x) ? fabsf(x) : 0.0f; }

// A block's scale: its inverse in fp32, and what the operand holds (the float's
// bits, or exponent + 127).
struct Scale {
    float inv;
    uint32_t held;
};
__device__ inline Scale scale_of(float amax, int format, int scale_type) {
    if (scale_type == O2M_SCALES_F32) {
        const float top = format == O2M_FP8_E4M3 ? 448.0f : 57344.0f;
        const float s = amax > 0.0f ? fmaxf(__fdiv_rn(amax, top), 1.17549435e-38f) : 1.0f;
        return {__fdiv_rn(1.0f, s), __float_as_uint(s)};
    }
    // F = 1.75 2^p: the exponent of amax less p, and one more past 1.75
    const uint32_t bits = __float_as_uint(amax);
    const int p = format == O2M_FP8_E4M3 ? 8 : 15;
    int e = (int)(bits >> 23) - 127 - p + ((bits & 0x7FFFFFu) > 0x600000u);
    e = amax > 0.0f ? max(e, -126) : 0;
    return {__uint_as_float((uint32_t)(127 - e) << 23), (uint32_t)(e + 127)};
}

// x inv within the format's range; Inf and NaN become NaN.
__device__ inline float scaled(float x, float inv, float top) {
    const float y = fminf(fmaxf(x * inv, -top), top);
    return finite(x) ? y : __uint_as_float(0x7FC00000u);
}

// Four values in 8 bits, rounded to nearest, ties to even.
__device__ inline uint32_t pack_fp8(const float (&y)[4], int format) {
    int r = 0;
    if (format == O2M_FP8_E4M3) {
        r = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], r, false);
        r = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], r, true);
    } else {
        r = __builtin_amdgcn_cvt_pk_bf8_f32(y[0], y[1], r, false);
        r = __builtin_amdgcn_cvt_pk_bf8_f32(y[2], y[3], r, true);
    }
    return (uint32_t)r;
}

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;

// Eight entries of one line from `x0`, of which `n` exist; zeros after them.  (The
// loads need no alignment but the entries' own.)
template <class T>
__device__ inline void load8(const T *x0, int n, float (&v)[8]) {
    if (n >= 8) {
        u32x4 w[sizeof(T) / 2];
        __builtin_memcpy(w, x0, sizeof w);
        T t[8];
        __builtin_memcpy(t, w, sizeof w);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = as_float(t[j]);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = j < n ? as_float(x0[j]) : 0.0f;
    }
}

}  // namespace o2m
