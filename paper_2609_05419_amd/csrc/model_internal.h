// Internal definitions of the products of trained models: 8-bit block-scaled
// operands (o2m_fp8_operand, include/o2m.h) and the orthogonalised update.
// What the product kernels share (staging of operand rows through LDS, the
// MFMA fragments) is in mfma_tiles.h.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "blocks.h"
#include "o2m.h"

namespace o2m {

// The runtime counts a launch's threads in 32 bits.
inline bool launch_fits(int64_t groups, int threads) { return groups * threads <= 0xFFFFFFFFLL; }

// Quantize the matrix of `lines` x `len` entries, entry (p, q) at X[p ld + q]:
// along its lines into `along` and across them into `across` (rows of an
// operand are lines, or entry positions q); either may be null.
hipError_t launch_quantize(int lines, int len, const void *X, int type, int64_t ld, const o2m_fp8_operand *along,
                           const o2m_fp8_operand *across, hipStream_t st);

// C = A B^T, entry (i, j) at C[i ldc + j].
hipError_t launch_gemm_fp8(int m, int n, int k, const o2m_fp8_operand &A, const o2m_fp8_operand &B, void *C, int type,
                           int64_t ldc, bool accumulate, void *ws, hipStream_t st);
size_t gemm_fp8_workspace(int m, int n, int k);
// Whether one launch covers the product.
bool gemm_fp8_fits(int m, int n, int k, int scale_type, int type);

// The same with few tokens, W the operand with the many rows; entry (t, r) of Y at
// t y_tok + r y_row.
hipError_t launch_few(int tokens, int n, int k, const o2m_fp8_operand &X, const o2m_fp8_operand &W, void *Y, int type,
                      int64_t y_tok, int64_t y_row, bool accumulate, hipStream_t st);
// The linear layer in one launch, where linear_is_fused.
bool linear_is_fused(int tokens, int k);
hipError_t launch_linear_fused(int tokens, int n, int k, const void *X, int x_type, int64_t ldx, const o2m_fp8_operand &W,
                               void *Y, int64_t ldy, hipStream_t st);

struct OrthoArgs {
    int batch, rows, cols;          // of the work matrix: rows <= cols
    const void *G;
    int64_t g_row, g_col, g_batch;  // strides in elements
    void *O;
    int64_t o_row, o_col, o_batch;
    int type;
    int steps;
    const double *coef;
    double eps;
};
size_t ortho_workspace(int batch, int rows, int cols, int type);
// Whether the whole update is one launch, of a workgroup per matrix.
bool ortho_is_small(int rows, int cols, int type);
hipError_t launch_ortho(const OrthoArgs &g, void *ws, hipStream_t st);

// Zero entries (i, j) of C at i + j ldc, of `size` bytes.
hipError_t launch_zero_out(void *C, int64_t m, int64_t n, int64_t ldc, int size, hipStream_t st);

}  // namespace o2m
