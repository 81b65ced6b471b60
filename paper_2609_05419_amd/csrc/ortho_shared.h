// What the kernels of the orthogonalised update share.
#pragma once

#include "fp8_round.h"
#include "mfma_pipe.h"
#include "model_internal.h"

#include <hip/hip_bf16.h>
#include <hip/hip_fp16.h>

namespace o2m {

typedef _Float16 f16;
typedef f16 v8f16 __attribute__((ext_vector_type(8)));

constexpr int kScaleX = 14, kScaleA = 11, kScaleB = 6;   // k_ortho.hip says why

__device__ inline void store_any(void *p, int64_t i, int type, float v) {
    if (type == O2M_TYPE_F32) static_cast<float *>(p)[i] = v;
    else if (type == O2M_TYPE_F16) static_cast<__half *>(p)[i] = __float2half(v);
    else static_cast<__hip_bfloat16 *>(p)[i] = __float2bfloat16(v);
}

// Eight neighbouring entries, of which the first n exist, zeros after them.
__device__ inline v8f load_some(const void *p, int64_t i, int n, int type) {
    float v[8];
    if (type == O2M_TYPE_F32) load8(static_cast<const float *>(p) + i, n, v);
    else if (type == O2M_TYPE_F16) load8(static_cast<const __half *>(p) + i, n, v);
    else load8(static_cast<const __hip_bfloat16 *>(p) + i, n, v);
    return v8f{v[0], v[1], v[2], v[3], v[4], v[5], v[6], v[7]};
}

// G of a batch as lines of contiguous entries.
struct Lines {
    const void *G;
    int64_t line, batch;   // strides
    int lines, len, type;
};

// The whole update of matrices that fit into LDS, one workgroup each
// (k_ortho_small.hip).
bool ortho_fits_lds(int r, int c, bool split);
hipError_t launch_ortho_small(const OrthoArgs &o, bool split, hipStream_t st);

}  // namespace o2m
