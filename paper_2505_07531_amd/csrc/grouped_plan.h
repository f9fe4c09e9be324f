// Block shapes of the products grouped by expert of the uniform, codebook and Q4X kinds, and the choice
// between them. Plain C++.
#pragma once

#include "mx4_plan.h"

namespace qx {
namespace grouped {

// The last shape is C of gemm_tile.hip (128 x 192), the others are those of grouped.hip, ks chunks a stage.
// Costs as in mx4_plan.h, fitted to the times of 181 sizes (4 to 128 experts, n = 256 to 6000, k = 512 to 5120,
// 1 to 300 rows each, unevenly shared): of uniform-4 g128, uniform-3 g64 and codebook-3 g128, and of codebook-4
// g64, whose table reads fill LDS; before the rows of X were read a step ahead. With the present kernels and
// 1.2 GB of weights read in turn the shapes that they choose take 2.4 to 3.7 % more than the best of all in the
// mean, in each of the 13 formats (uniform-4 g64 the most, codebook-4 g64 the least, Q4X 3.5; at most 53 %); where
// a shape is within 30 % of the best, 96 of 100 costs are within 23 to 32 % of its time, 40 % with codebooks of
// groups of 32. us in the order of the list, uniform-4 g128: 8 experts of 576x3584, m = 108 9.3 / 14.5 / 15.6 /
// 26 / 31 / 61; 66 of 694x1024, m = 940 18.5 / 14.8 / 17.6 / 23 / 18.3 / 33; 5 of 916x3840, m = 361 18.1 / 19.6 /
// 17.2 / 28 / 33 / 66; 7 of 2057x2688, m = 402 30 / 28 / 26 / 25 / 27 / 50; 78 of 3398x768, m = 3471 204 / 107 /
// 85 / 103 / 65 / 87; 5 of 5205x3712, m = 808 139 / 130 / 94 / 93 / 96 / 70.
constexpr int kShapes = 6, kTile = 5;
using mx4::ShapeCost;
inline constexpr ShapeCost shapes[2][kShapes] = {
    {
        {1, 2, 1, 1, 4, 4, false, {3.62f, 0.193f, 0.486f, 0.139f}},
        {1, 2, 1, 2, 2, 2, false, {3.21f, 0.404f, 0.2f, 0.293f}},
        {2, 2, 1, 2, 2, 2, false, {3.67f, 0.434f, 0.439f, 0.345f}},
        {4, 2, 1, 4, 2, 2, true, {4.15f, 0.93f, 3.38f, 1.03f}},
        {4, 2, 1, 4, 1, 1, true, {3.07f, 1.14f, 0.2f, 0.953f}},
        {8, 3, 1, 4, 2, 2, true, {5.78f, 2.12f, 0.2f, 2.06f}},
    },
    {
        {1, 2, 1, 1, 4, 4, true, {3.54f, 0.216f, 0.704f, 0.201f}},
        {1, 2, 1, 2, 2, 2, true, {3.3f, 0.453f, 0.2f, 0.438f}},
        {2, 2, 1, 2, 2, 2, true, {3.72f, 0.483f, 0.657f, 0.47f}},
        {4, 2, 1, 4, 2, 2, true, {4.62f, 1.14f, 4.32f, 1.22f}},
        {4, 2, 1, 4, 1, 1, true, {2.89f, 1.36f, 0.386f, 1.33f}},
        {8, 3, 1, 4, 2, 2, true, {5.85f, 2.61f, 1.71f, 2.61f}},
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
