// Products of 8-bit block-scaled operands (include/o2m.h: o2m_gemm_fp8).
//
//   C[i, j] = sum_b sa[i, b] sb[j, b] sum_{k in block b} qa[i, k] qb[j, k]
//
// A block of 128 along k is one v_mfma_f32_16x16x128_f8f6f4, so a scale belongs
// to one MFMA: power-of-two scales go into the scaled form of the instruction,
// fp32 ones multiply the partial sum of the block as it is added up.
//
// That instruction adds 8 neighbouring products at a time with 13 bits below
// the largest of them, and such groups in fp32 (measured: of two products of a
// group the smaller one is lost below 2^-13 of the larger, of different groups
// below 2^-24).  On normal data in blocks a sum is 1.5e-5 to 3e-5 off in the
// 2-norm: far below the rounding of a bf16 (1.7e-3) or fp16 (2.1e-4) result,
// which therefore take it, and far above that of an fp32 one.  Products with an
// fp32 result turn the values to 16 bits in registers and add up with
// v_mfma_f32_16x16x32 (6e-8), at half the rate: to fp16, which holds both formats
// exactly, and scale a block's sum, or, where scales are powers of two, to bf16
// times the scale, which is exact as well and leaves nothing to do after the
// MFMAs (4096^3 140 -> 124 us).
//
// Bound: 8-bit (fp32 results: 16-bit) MFMA for large products.
//
// Which kernel runs (plan_fp8):
//   up to 32 rows on one side          k_fp8_few.hip, bound by reading the other
//   fp32 results                       k_fp8_wide.hip
//   power-of-two scales                k_fp8_scaled.hip
//   fp32 scales                        k_fp8_partial.hip
// Products with too few tiles to fill the part are split along k, and join_parts
// adds the fp32 sums up in a fixed order.
#include "fp8_plan.h"
#include "fp8_tile.h"

#include <algorithm>

namespace o2m {
namespace {

// The sums of a split launch, 4 neighbouring outputs a thread.
__global__ __launch_bounds__(256) void join_parts(Fp8Args g) {
    const int per_row = g.pitch / 4;
    const int64_t total = (int64_t)g.a.rows * per_row, plane = (int64_t)g.a.rows * g.pitch;
    for (int64_t t = blockIdx.x * 256LL + threadIdx.x; t < total; t += gridDim.x * 256LL) {
        const int row = (int)(t / per_row), col = (int)(t % per_row) * 4;
        const float *p = g.parts + row * (int64_t)g.pitch + col;
        v4f v = *reinterpret_cast<const v4f *>(p);
        for (int z = 1; z < g.splits; ++z) v += *reinterpret_cast<const v4f *>(p + z * plane);
        store_run<4>(g, row, col, v);
    }
}

template <class T>
__global__ __launch_bounds__(256) void zero_out(T *C, int64_t m, int64_t total, int64_t ldc) {
    for (int64_t t = blockIdx.x * 256LL + threadIdx.x; t < total; t += gridDim.x * 256LL)
        C[t % m + t / m * ldc] = T(0);
}

}  // namespace

hipError_t launch_zero_out(void *C, int64_t m, int64_t n, int64_t ldc, int size, hipStream_t st) {
    const int64_t total = m * n;
    if (total <= 0) return hipSuccess;
    const unsigned grid = (unsigned)(ceil_div(total, 256) < 2048 ? ceil_div(total, 256) : 2048);
    if (size == 4) zero_out<uint32_t><<<grid, 256, 0, st>>>(static_cast<uint32_t *>(C), m, total, ldc);
    else zero_out<uint16_t><<<grid, 256, 0, st>>>(static_cast<uint16_t *>(C), m, total, ldc);
    return hipGetLastError();
}

size_t gemm_fp8_workspace(int m, int n, int k) {
    // either order of the result: its rows are those of one operand or the other
    int splits = 1;
    for (const Sum sum : {kScaled, kPartial, kWide, kWideScaled})
        splits = std::max({splits, plan_fp8(m, n, k, sum).splits, plan_fp8(n, m, k, sum).splits});
    if (splits == 1) return 0;
    return sizeof(float) * (size_t)splits * (size_t)std::max(m * round_up64(n, 4), n * round_up64(m, 4));
}

bool gemm_fp8_fits(int m, int n, int k, int scale_type, int type) {
    const Sum sum = sum_of(scale_type, type);
    const Fp8Plan p = plan_fp8(m, n, k, sum);
    if (p.few) return launch_fits(ceil_div(std::max(m, n), 16), 256);
    const TileCost &s = kCosts[sum][p.size];
    return launch_fits(round_up64(ceil_div(m, s.rows) * ceil_div(n, s.cols), kXcds) * p.splits,
                       sum == kPartial && p.size == k256 ? 512 : 256);
}

hipError_t launch_gemm_fp8(int m, int n, int k, const o2m_fp8_operand &A, const o2m_fp8_operand &B, void *C, int type,
                           int64_t ldc, bool accumulate, void *ws, hipStream_t st) {
    const bool wide = type == O2M_TYPE_F32;
    const Fp8Plan p = plan_fp8(m, n, k, sum_of(A.scale_type, type));
    if (p.few)
        return n <= m ? launch_few(n, m, k, B, A, C, type, 1, ldc, accumulate, st)
                      : launch_few(m, n, k, A, B, C, type, ldc, 1, accumulate, st);
    Fp8Args g = {};
    g.a = side_of(A, m);
    g.b = side_of(B, n);
    g.k = k;
    g.kblocks = (int)ceil_div(k, kBlockK);
    g.C = C;
    g.ldc = ldc;
    g.type = type;
    g.accumulate = accumulate;
    g.parts = static_cast<float *>(ws);
    g.pitch = (int)round_up64(n, 4);
    g.splits = p.splits;
    g.per = p.per;
    const int format = A.format * 2 + B.format;
    // the large kernel of power-of-two scales reads those of 8 rows at once
    auto fits = [](const Side &s) { return !s.by_row || (s.s_row == 1 && s.rows >= 8); };
    const TileSize size = p.size <= k256x128 && g.a.pow2 && !(fits(g.a) && fits(g.b)) ? k128 : p.size;
    const hipError_t e = wide       ? launch_fp8_wide(g, format, size, st)
                         : g.a.pow2 ? launch_fp8_scaled(g, format, size, st)
                                    : launch_fp8_partial(g, format, size, st);
    if (e != hipSuccess || p.splits == 1) return e;
    const int64_t threads = (int64_t)m * (g.pitch / 4);
    join_parts<<<(unsigned)std::min<int64_t>(ceil_div(threads, 256), 2048), 256, 0, st>>>(g);
    return hipGetLastError();
}

}  // namespace o2m
