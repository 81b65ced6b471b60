// 8-bit block-scaled products with fp32 results: the values are turned to fp16 as
// they come from LDS, and a block's exact products are summed by fp16 MFMAs, then
// scaled (k_fp8.hip says why).  A wave widens its 4 fragments of B once a stage and
// each of A once for 4 of B.
#include "fp8_tile.h"

namespace o2m {

hipError_t launch_fp8_wide(Fp8Args &g, int format, TileSize size, hipStream_t st) {
    switch (format) {
    case 0: return launch_sizes<kWide, 0, 0, false>(g, size, st);
    case 1: return launch_sizes<kWide, 0, 1, false>(g, size, st);
    case 2: return launch_sizes<kWide, 1, 0, false>(g, size, st);
    default: return launch_sizes<kWide, 1, 1, false>(g, size, st);
    }
}

}  // namespace o2m
