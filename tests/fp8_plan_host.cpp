// Host build of the 8-bit products' plan, for tests/test_fp8_plan.py.
#define O2M_HD
#include "../paper_2609_05419_amd/csrc/fp8_plan.h"

extern "C" {
// few, rows and columns of a tile, splits, stages of a split
void t_plan_fp8(int m, int n, int k, int scale_type, int type, int *out) {
    const o2m::Sum sum = o2m::sum_of(scale_type, type);
    const o2m::Fp8Plan p = o2m::plan_fp8(m, n, k, sum);
    const o2m::TileCost &s = o2m::kCosts[sum][p.size];
    const int v[5] = {p.few, s.rows, s.cols, p.splits, p.per};
    for (int i = 0; i < 5; ++i) out[i] = v[i];
}
}
