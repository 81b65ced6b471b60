// 8-bit block-scaled products with fp32 results: the values are turned to 16 bits as
// they come from LDS, and their exact products are summed by 16-bit MFMAs, a
// block's sum being scaled afterwards or its values before (k_fp8.hip says why).  A
// wave widens its 4 fragments of B once a stage and
// each of A once for 4 of B.
#include "fp8_tile.h"

namespace o2m {

namespace {
template <Sum SUM>
hipError_t launch(Fp8Args &g, int format, TileSize size, hipStream_t st) {
    switch (format) {
    case 0: return launch_sizes<SUM, 0, 0, false>(g, size, st);
    case 1: return launch_sizes<SUM, 0, 1, false>(g, size, st);
    case 2: return launch_sizes<SUM, 1, 0, false>(g, size, st);
    default: return launch_sizes<SUM, 1, 1, false>(g, size, st);
    }
}
}  // namespace

hipError_t launch_fp8_wide(Fp8Args &g, int format, TileSize size, hipStream_t st) {
    return g.a.pow2 ? launch<kWideScaled>(g, format, size, st) : launch<kWide>(g, format, size, st);
}

}  // namespace o2m
