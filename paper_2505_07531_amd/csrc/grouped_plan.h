// Block shapes of the products grouped by expert of the uniform, codebook and Q4X kinds, and the choice
// between them. Plain C++.
#pragma once

#include "mx4_plan.h"

namespace qx {
namespace grouped {

// The first four are those of grouped.hip, ks chunks a stage; the last one is shape C of gemm_tile.hip
// (128 x 192). Costs as in mx4_plan.h, fitted to 1170 times (8 and 32 experts of 1376x4096, 4096x1408 and
// 2816x2048, 2 to 350 rows each, unevenly shared), half of them within 5 to 12 %: of uniform-4 g128 and
// uniform-3 g64, and of codebook-4 g64, whose table reads fill LDS. The shapes that they choose take 1.3 %
// and 3.7 % more than the best in the mean. us of the five with uniform-4 g128: 32 experts of 1376x4096,
// m = 64 24 / 33 / 56 / 50 / 67, m = 960 54 / 44 / 59 / 56 / 71, m = 11200 490 / 310 / 253 / 238 / 201; 8 of
// 2816x2048, m = 512 31 / 23 / 18 / 21 / 37; 32 of 2816x2048, m = 4160 212 / 122 / 115 / 98 / 111.
constexpr int kShapes = 5, kTile = 4;
using mx4::ShapeCost;
inline constexpr ShapeCost shapes[2][kShapes] = {
    {
        {1, 2, 1, 1, 4, 4, false, {1.56f, 0.266f, 0.703f, 0.103f}},
        {2, 2, 1, 2, 2, 2, false, {2.69f, 0.478f, 0.803f, 0.261f}},
        {4, 2, 1, 4, 2, 2, true, {3.f, 0.809f, 2.8f, 0.939f}},
        {4, 2, 1, 4, 1, 1, false, {3.8f, 1.02f, 0.274f, 1.f}},
        {8, 3, 1, 4, 2, 2, true, {8.43f, 1.7f, 14.9f, 0.943f}},
    },
    {
        {1, 2, 1, 1, 4, 4, false, {3.5f, 0.285f, 1.15f, 0.141f}},
        {2, 2, 1, 2, 2, 2, false, {3.37f, 0.615f, 1.5f, 0.338f}},
        {4, 2, 1, 4, 2, 2, true, {3.f, 1.02f, 4.85f, 0.976f}},
        {4, 2, 1, 4, 1, 1, false, {6.14f, 1.15f, 2.17f, 1.16f}},
        {8, 3, 1, 4, 2, 2, true, {10.5f, 2.08f, 24.f, 0.885f}},
    },
};

inline int pick_shape(const qx_desc* d, int m, int experts) {
  const ShapeCost* const all = shapes[d->kind == QX_CODEBOOK && d->bits == 4];
  int best = 0;
  float least = 1e30f;
  for (int i = 0; i < kShapes; ++i) {
    const float us = mx4::shape_us(all[i], mx4::expert_tiles(m, experts, 16 * all[i].mt * all[i].wm), d->n, d->k, true);
    if (us < least) least = us, best = i;
  }
  return best;
}

}  // namespace grouped
}  // namespace qx
