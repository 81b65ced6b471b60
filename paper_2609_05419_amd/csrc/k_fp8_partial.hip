// 8-bit block-scaled products with fp32 scales and 16-bit results: each block's sum
// comes from the 8-bit MFMA and is scaled as it is added up, 4 multiply-adds a
// lane per MFMA (8 where both operands have a scale per row), beside which the
// other wave of the SIMD keeps the MFMA pipe busy.
#include "fp8_tile.h"

namespace o2m {

template <int FA, int FB>
static hipError_t launch(Fp8Args &g, TileSize size, hipStream_t st) {
    return g.b.by_row ? launch_sizes<kPartial, FA, FB, false>(g, size, st) : launch_sizes<kPartial, FA, FB, true>(g, size, st);
}

hipError_t launch_fp8_partial(Fp8Args &g, int format, TileSize size, hipStream_t st) {
    switch (format) {
    case 0: return launch<0, 0>(g, size, st);
    case 1: return launch<0, 1>(g, size, st);
    case 2: return launch<1, 0>(g, size, st);
    default: return launch<1, 1>(g, size, st);
    }
}

}  // namespace o2m
