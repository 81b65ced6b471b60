// Which kernel, tiles and splits a product of 8-bit block-scaled operands takes
// (k_fp8.hip).  Shared by the launches and the host-compiled test of them.
#pragma once

#include "blocks.h"
#include "o2m.h"
#include "tile_schedule.h"

#include <algorithm>

namespace o2m {

// How a block's products are added up.
enum Sum {
    kScaled,       // 8-bit MFMA with power-of-two scales
    kPartial,      // 8-bit MFMA, then fp32 scales
    kWide,         // fp16 MFMA, then fp32 scales
    kWideScaled,   // bf16 MFMA of values scaled by powers of two as they are widened
};

inline Sum sum_of(int scale_type, int type) {
    const bool wide = type == O2M_TYPE_F32;
    return scale_type == O2M_SCALES_POW2 ? (wide ? kWideScaled : kScaled) : wide ? kWide : kPartial;
}

enum TileSize { k256, k256x128, k128, k64 };

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
// layer of it, launch by launch, 16 and 18.)  16 splits are the most, a bound that
// no measurement set: 128 x 128 x 131072 takes 42 us in 16, on 64 workgroups.
struct Fp8Plan {
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

inline Fp8Plan plan_fp8(int m, int n, int k, Sum sum) {
    const int kblocks = (int)ceil_div(k, kBlockK);
    Fp8Plan best = {};
    best.splits = 1;
    best.per = kblocks;
    best.few = std::min(m, n) <= kFewRows;
    if (best.few) return best;
    double least = 0.0;
    for (const TileCost &s : kCosts[sum]) {
        if (!s.rows) continue;
        for (int want = 1; want <= 16; want *= 2) {
            if (want > 1 && (s.size != k64 || kblocks < 4 * want)) break;
            Fp8Plan p = {};
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

}  // namespace o2m
