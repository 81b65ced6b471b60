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

constexpr int kFewRows = 32;

// Tiles and splits of a launch: those with the least estimated time (us), a round of
// workgroups after the other.  A size has `fixed` per round (its first copies and
// its results), and per stage `one` while a CU has one workgroup, `full` with all
// of `resident` (of one resident: while few CUs work, and when all do, which
// lowers the clock).  Fitted to 100 products of 20 shapes, of which the measured
// best or one within 3% of it is taken.  Measured (us; tiles of 256 x 256, 256 x 128,
// 128 x 128, 64 x 64):
//   power-of-two scales      4096 x 4096 x 4096     56    71    80
//                            3000 x 3000 x 3000     42    56    52    58
//                            2048 x 4096 x 8192     81    63    73
//                            2048 x 2048 x 2048     29    21    18    18
//                            1000 x 1000 x 1000     22    16    11     7
//   fp32 scales              4096 x 4096 x 4096     75          86
//                            2048 x 4096 x 8192    124          87
//                            2048 x 2048 x 2048     39          20    19
//   fp32 scales and results  3000 x 3000 x 3000                 80    86
//                            1537 x 1283 x 2051                 32    26
//                            512 x 2048 x 2048                  25    14
//   powers of two, fp32 res. 3000 x 3000 x 3000                 72    79
// (fp32 results: the widened fragments leave no registers for tiles of 256 x 256,
// which took 151 us with spilled ones.)  Tiles of 64 x 64 that leave CUs idle are
// split along k, from 4 stages each: 300 x 300 x 8000 (25 tiles) 30 us in one piece,
// 11.5 in 8; 64 x 4096 x 4096 (64) 16, and 10.7 in 4; 1000 x 1000 x 1000 (256) 6.9, and
// 12.1 in 2.  (Near the edge the launch of its own that the joining takes decides:
// 333 x 1283 x 2051 with 126 tiles takes the GPU 12.1 us, in 2 splits 10.8, but a linear
// layer of it, launch by launch, 16 and 18.)
struct Plan {
    bool few;
    TileSize size;
    int splits, per;
};
struct TileCost {
    TileSize size;
    int rows, cols, resident;
    double fixed, one, full;
};
constexpr TileCost kCosts[4][4] = {
    {{k256, 256, 256, 1, 13.0, 1.00, 1.33}, {k256x128, 256, 128, 1, 9.5, 0.69, 0.82},
     {k128, 128, 128, 2, 6.5, 0.70, 1.03}, {k64, 64, 64, 4, 3.5, 0.40, 0.88}},
    {{k256, 256, 256, 1, 11.0, 1.70, 2.00}, {}, {k128, 128, 128, 2, 6.5, 0.84, 1.24}, {k64, 64, 64, 4, 3.5, 0.45, 0.98}},
    {{}, {}, {k128, 128, 128, 2, 8.0, 1.22, 1.98}, {k64, 64, 64, 4, 4.0, 0.60, 1.55}},
    {{}, {}, {k128, 128, 128, 2, 7.5, 1.15, 1.80}, {k64, 64, 64, 4, 4.1, 0.55, 1.42}}};

Plan plan_fp8(int m, int n, int k, Sum sum) {
    const int kblocks = (int)ceil_div(k, kBlockK);
    Plan best = {};
    best.splits = 1;
    best.per = kblocks;
    best.few = std::min(m, n) <= kFewRows;
    if (best.few) return best;
    double least = 0.0;
    for (const TileCost &s : kCosts[sum]) {
        if (!s.rows) continue;
        for (int want = 1; want <= 16; want *= 2) {
            if (want > 1 && (s.size != k64 || kblocks < 4 * want)) break;
            Plan p = {};
            p.size = s.size;
            p.per = (int)ceil_div(kblocks, want);
            p.splits = (int)ceil_div(kblocks, p.per);
            const int64_t groups = ceil_div(m, s.rows) * ceil_div(n, s.cols) * p.splits;
            const int64_t round = (int64_t)kCus * s.resident, rest = groups % round;
            double t = (double)(groups / round) * (s.fixed + p.per * s.full);
            if (rest > 0) {
                const double fill = s.resident == 1 ? (double)rest / kCus
                                                    : (double)(ceil_div(rest, kCus) - 1) / (s.resident - 1);
                t += s.fixed + p.per * (s.one + (s.full - s.one) * fill);
            }
            if (p.splits > 1) t += 3.0 + p.splits * (0.15 + 0.8e-6 * m * n);   // join_parts
            if (least == 0.0 || t < least) {
                least = t;
                best = p;
            }
        }
    }
    return best;
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

static Sum sum_of(int scale_type, int type) {
    const bool wide = type == O2M_TYPE_F32;
    return scale_type == O2M_SCALES_POW2 ? (wide ? kWideScaled : kScaled) : wide ? kWide : kPartial;
}

bool gemm_fp8_fits(int m, int n, int k, int scale_type, int type) {
    const Sum sum = sum_of(scale_type, type);
    const Plan p = plan_fp8(m, n, k, sum);
    if (p.few) return launch_fits(ceil_div(std::max(m, n), 16), 256);
    const TileCost &s = kCosts[sum][p.size];
    return launch_fits(round_up64(ceil_div(m, s.rows) * ceil_div(n, s.cols), kXcds) * p.splits,
                       sum == kPartial && p.size == k256 ? 512 : 256);
}

hipError_t launch_gemm_fp8(int m, int n, int k, const o2m_fp8_operand &A, const o2m_fp8_operand &B, void *C, int type,
                           int64_t ldc, bool accumulate, void *ws, hipStream_t st) {
    const bool wide = type == O2M_TYPE_F32;
    const Plan p = plan_fp8(m, n, k, sum_of(A.scale_type, type));
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
