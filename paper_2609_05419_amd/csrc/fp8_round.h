// Rounding into 8-bit floating point: a block's scale from its largest magnitude,
// and values within the scaled range.
#pragma once

#include "model_internal.h"

#include <hip/hip_bf16.h>
#include <hip/hip_fp16.h>
#include <type_traits>

namespace o2m {

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

// Eight entries of one line as they lie in memory, two to a word or one.
template <class T>
struct Run8 {
    static constexpr int kWords = 2 * sizeof(T);
    static constexpr bool kHalves = sizeof(T) == 2;
    uint32_t w[kWords];
};

// Eight entries from `x0`, of which `n` exist; zeros after them.  (The loads need no
// alignment but the entries' own.)
template <class T>
__device__ inline Run8<T> load_run(const T *x0, int n) {
    Run8<T> r;
    if (n >= 8) {
        __builtin_memcpy(&r, x0, sizeof r);
    } else {
        T t[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) t[j] = j < n ? x0[j] : T(0.0f);
        __builtin_memcpy(&r, t, sizeof r);
    }
    return r;
}
template <class T>
__device__ inline float entry(const Run8<T> &r, int j) {
    if constexpr (sizeof(T) == 4) return __uint_as_float(r.w[j]);
    const uint32_t h = j & 1 ? r.w[j / 2] >> 16 : r.w[j / 2] & 0xFFFFu;
    if constexpr (std::is_same<T, __half>::value) return __half2float(__ushort_as_half((unsigned short)h));
    return __uint_as_float(h << 16);
}
template <class T>
__device__ inline void load8(const T *x0, int n, float (&v)[8]) {
    const Run8<T> r = load_run(x0, n);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = entry(r, j);
}

// Magnitudes are compared as bits, which order as the numbers do, with Inf and NaN
// above all of them: words of two 16-bit magnitudes, or of one.
template <class T>
__device__ inline uint32_t magnitude_bits(uint32_t w) { return w & (sizeof(T) == 2 ? 0x7FFF7FFFu : 0x7FFFFFFFu); }
template <class T>
__device__ inline uint32_t larger(uint32_t x, uint32_t y) {
    if constexpr (sizeof(T) == 4) return max(x, y);
    typedef unsigned short v2u16 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(v2u16, x), __builtin_bit_cast(v2u16, y)));
}
// The larger one of a word's.
template <class T>
__device__ inline uint32_t largest_in(uint32_t w) { return sizeof(T) == 4 ? w : max(w >> 16, w & 0xFFFFu); }
template <class T>
__device__ inline bool bits_finite(uint32_t bits) {
    return bits < (sizeof(T) == 4 ? 0x7F800000u : std::is_same<T, __half>::value ? 0x7C00u : 0x7F80u);
}
template <class T>
__device__ inline float bits_value(uint32_t bits) {
    if constexpr (sizeof(T) == 4) return __uint_as_float(bits);
    if constexpr (std::is_same<T, __half>::value) return __half2float(__ushort_as_half((unsigned short)bits));
    return __uint_as_float(bits << 16);
}
template <class T>
__device__ inline uint32_t largest_of(const Run8<T> &r) {
    uint32_t m = magnitude_bits<T>(r.w[0]);
#pragma unroll
    for (int i = 1; i < Run8<T>::kWords; ++i) m = larger<T>(m, magnitude_bits<T>(r.w[i]));
    return largest_in<T>(m);
}

// The largest over the 16 lanes of a row of a wave, in all of them.
__device__ inline uint32_t largest_of_16(uint32_t x) {
    x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0xB1, 0xF, 0xF, true));    // lanes 1 apart
    x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x4E, 0xF, 0xF, true));    // 2 apart
    x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x141, 0xF, 0xF, true));   // the halves of 8, mirrored
    return max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x140, 0xF, 0xF, true));   // of 16
}
// Over the four rows of a wave, word for word, in all of them.
template <class T>
__device__ inline uint32_t larger_of_rows(uint32_t x) {
    auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    x = larger<T>(r[0], r[1]);
    auto q = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    return larger<T>(q[0], q[1]);
}

// Eight entries in 8 bits.  FINITE: none is Inf or NaN, and none is past the block's
// largest, so that none leaves the format's range.
template <bool FINITE, class T>
__device__ inline uint2 round_run(const Run8<T> &r, float inv, int format) {
    const float top = format == O2M_FP8_E4M3 ? 448.0f : 57344.0f;
    float y[4], z[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        y[j] = FINITE ? entry(r, j) * inv : scaled(entry(r, j), inv, top);
        z[j] = FINITE ? entry(r, 4 + j) * inv : scaled(entry(r, 4 + j), inv, top);
    }
    return uint2{pack_fp8(y, format), pack_fp8(z, format)};
}

}  // namespace o2m
