// What the kernels of 8-bit block-scaled products share: an operand as they see
// it, its scales, its values in fp16, and outputs of either type.
#pragma once

#include "mfma_tiles.h"
#include "model_internal.h"

#include <hip/hip_bf16.h>
#include <hip/hip_fp16.h>

namespace o2m {

struct Side {
    const uint8_t *values;
    int64_t ld;
    const void *scales;
    int64_t s_row, s_blk;
    int rows;
    int by_row;   // 1: a scale per row, 0: per 128 rows
    int pow2;
};

typedef _Float16 v2f16 __attribute__((ext_vector_type(2)));
typedef _Float16 v8f16 __attribute__((ext_vector_type(8)));
typedef __bf16 v2bf16 __attribute__((ext_vector_type(2)));
typedef __bf16 v8bf16 __attribute__((ext_vector_type(8)));

// Eight 8-bit values (two dwords) in fp16, exactly.
template <int F>
__device__ inline v8f16 widen(int x, int y) {
    v2f16 r[4];
    const uint32_t w[2] = {(uint32_t)x, (uint32_t)y};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        r[2 * i] = F == O2M_FP8_E4M3 ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w[i], 1.0f, false)
                                     : __builtin_amdgcn_cvt_scalef32_pk_f16_bf8(w[i], 1.0f, false);
        r[2 * i + 1] = F == O2M_FP8_E4M3 ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w[i], 1.0f, true)
                                         : __builtin_amdgcn_cvt_scalef32_pk_f16_bf8(w[i], 1.0f, true);
    }
    return v8f16{r[0][0], r[0][1], r[1][0], r[1][1], r[2][0], r[2][1], r[3][0], r[3][1]};
}

// The same with a power-of-two scale, in bf16: exactly where the products lie within
// its normal range.
template <int F>
__device__ inline v8bf16 widen_scaled(int x, int y, float scale) {
    v2bf16 r[4];
    const uint32_t w[2] = {(uint32_t)x, (uint32_t)y};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        r[2 * i] = F == O2M_FP8_E4M3 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], scale, false)
                                     : __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(w[i], scale, false);
        r[2 * i + 1] = F == O2M_FP8_E4M3 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], scale, true)
                                         : __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(w[i], scale, true);
    }
    return v8bf16{r[0][0], r[0][1], r[1][0], r[1][1], r[2][0], r[2][1], r[3][0], r[3][1]};
}

__device__ inline float load_out(const void *C, int64_t i, int type) {
    if (type == O2M_TYPE_F32) return static_cast<const float *>(C)[i];
    if (type == O2M_TYPE_F16) return __half2float(static_cast<const __half *>(C)[i]);
    return __bfloat162float(static_cast<const __hip_bfloat16 *>(C)[i]);
}
__device__ inline void store_out(void *C, int64_t i, int type, float v) {
    if (type == O2M_TYPE_F32) static_cast<float *>(C)[i] = v;
    else if (type == O2M_TYPE_F16) static_cast<__half *>(C)[i] = __float2half(v);
    else static_cast<__hip_bfloat16 *>(C)[i] = __float2bfloat16(v);
}

// The scale of `row` in block kb, as an e8m0 byte or a float.  Rows past the last
// one take its scale (their values are zeros).
__device__ inline int64_t scale_index(const Side &s, int row, int kb) {
    row = min(row, s.rows - 1);
    return (s.by_row ? row : row >> 7) * s.s_row + kb * s.s_blk;
}
__device__ inline int scale_code(const Side &s, int row, int kb) {
    return static_cast<const uint8_t *>(s.scales)[scale_index(s, row, kb)];
}
// 2^(code - 127); 2^-127 (code 0) is half the smallest normal number, 255 is NaN
__device__ inline float code_value(uint32_t code) {
    return code == 255 ? __uint_as_float(0x7FC00000u) : __uint_as_float(code ? code << 23 : 0x00400000u);
}
// ANY: of either kind; otherwise a float
template <bool ANY>
__device__ inline float scale_value(const Side &s, int row, int kb) {
    const int64_t i = scale_index(s, row, kb);
    if (ANY && s.pow2) return code_value(static_cast<const uint8_t *>(s.scales)[i]);
    return static_cast<const float *>(s.scales)[i];
}

inline Side side_of(const o2m_fp8_operand &o, int rows) {
    return {static_cast<const uint8_t *>(o.values), o.ld, o.scales, o.s_row, o.s_blk, rows, o.block == 1,
            o.scale_type == O2M_SCALES_POW2};
}

}  // namespace o2m
