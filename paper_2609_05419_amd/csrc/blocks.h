// Blocks of 8-bit operands, and quotients that are rounded up.
#pragma once

#include <stdint.h>

namespace o2m {

constexpr int kBlockK = 128;   // entries of a block along the inner dimension

inline int64_t ceil_div(int64_t x, int64_t q) { return (x + q - 1) / q; }
inline int64_t round_up64(int64_t x, int64_t q) { return ceil_div(x, q) * q; }

}  // namespace o2m
