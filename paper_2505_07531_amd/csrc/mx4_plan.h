// Block shapes of the MX4 products (mx4_tile.h) and the choice between them. Plain C++.
#pragma once

#include <cmath>

#include "qx_internal.h"

namespace qx {
namespace mx4 {

// A block of wm x wn x wk waves, each with mt x nt tiles of 16 x 16 (activation rows x weight rows);
// the wk waves take different k, ks units of it (128 with MX4 rows, 64 with fp16) a stage.
// Cost in us at k = 128 K of up to 256 blocks, one a compute unit: us[0] + us[1] K; of every 256 more:
// us[2] + us[3] K. One block of a shape with `one` set fills a compute unit, so that those are whole
// rounds. Fitted to 2577 times (170 sizes with n = 256 to 22016, k = 512 to 11264, m = 1 to 4096), of which
// 96 of 100 are within 13 % (fp16 rows; MX4 rows within 30 %); the shapes that they choose take 0.7 % and
// 3 % more than the best of the measured ones in the mean.
struct ShapeCost {
  int mt, nt, wm, wn, wk, ks;
  bool one;
  float us[4];
};
constexpr int kShapes = 9;
template <bool A4>
inline constexpr ShapeCost shapes[kShapes] = {
    {1, 1, 1, 1, 8, 2, true, {2.92f, 0.0693f, 1.54f, 0.0845f}},
    {1, 2, 1, 1, 4, 2, false, {2.7f, 0.149f, 0.374f, 0.0869f}},
    {2, 2, 1, 1, 8, 1, true, {3.16f, 0.136f, 1.8f, 0.162f}},
    {2, 4, 1, 1, 4, 1, false, {3.2f, 0.281f, 1.27f, 0.15f}},
    {4, 2, 1, 1, 8, 1, true, {3.63f, 0.211f, 2.41f, 0.253f}},
    {4, 2, 1, 2, 4, 1, true, {3.65f, 0.323f, 2.67f, 0.366f}},
    {4, 4, 1, 2, 2, 1, false, {4.14f, 0.711f, 2.11f, 0.499f}},
    {4, 4, 2, 4, 1, 1, true, {4.33f, 1.6f, 4.51f, 1.62f}},
    {8, 4, 2, 4, 1, 1, true, {5.73f, 2.61f, 11.3f, 2.62f}},
};
template <>
inline constexpr ShapeCost shapes<true>[kShapes] = {
    {1, 1, 1, 1, 8, 2, false, {3.04f, 0.0253f, 0.792f, 0.0301f}},
    {1, 2, 1, 1, 4, 2, false, {2.85f, 0.0567f, 0.353f, 0.0504f}},
    {2, 2, 1, 1, 8, 1, false, {3.35f, 0.05f, 0.826f, 0.0711f}},
    {2, 4, 1, 1, 4, 1, false, {3.35f, 0.104f, 0.258f, 0.113f}},
    {4, 2, 1, 1, 8, 1, true, {3.85f, 0.068f, 2.15f, 0.0984f}},
    {4, 4, 1, 1, 4, 1, false, {4.1f, 0.144f, 1.68f, 0.123f}},
    {4, 4, 1, 1, 8, 1, true, {4.31f, 0.107f, 3.25f, 0.133f}},
    {4, 4, 2, 2, 1, 2, false, {4.43f, 0.411f, 2.28f, 0.333f}},
    {8, 4, 2, 4, 1, 2, true, {5.39f, 0.827f, 9.66f, 0.971f}},
};

// Cost of `tiles` row tiles of 16 * mt * wm rows by n columns; `ragged`: their number is a guess.
inline float shape_us(const ShapeCost& s, float tiles, int n, int k, bool ragged) {
  const long nx = ((long)n + 16 * s.nt * s.wn - 1) / (16 * s.nt * s.wn);
  const float rounds = tiles * (float)nx / 256.f, K = (float)(k / 128);
  float more = rounds <= 1.f ? 0.f : rounds - 1.f;
  if (s.one && more > 0.f) more = ragged ? more + 0.4f : (float)(long)(rounds + 0.999f) - 1.f;
  return s.us[0] + s.us[1] * K + more * (s.us[2] + s.us[3] * K);
}

// Row tiles of bm rows that m rows of `experts` experts take. Only the device knows their sizes: the rows
// are taken as shared by as many experts as there can be, with shares that differ by a factor of two or
// so. Then an expert has half a tile more than its rows fill, and few have less than one (32 experts of
// 4096x1408, 4001 MX4 rows: 36 us in tiles of 128 x 128, 51 in 256 x 256, which counted as one tile
// an expert).
inline float expert_tiles(int m, int experts, int bm) {
  const float used = (float)(experts < m ? experts : m), full = (float)m / (used * (float)bm);
  return used * (0.5f + full + 0.5f * std::exp(-2.f * full));
}

// experts: of a grouped product (0: none).
template <bool A4>
inline int pick_shape(int n, int k, int m, int experts) {
  int best = 0;
  float least = 1e30f;
  for (int i = 0; i < kShapes; ++i) {
    const ShapeCost& s = shapes<A4>[i];
    const int bm = 16 * s.mt * s.wm;
    const float tiles = experts > 0 ? expert_tiles(m, experts, bm) : (float)((m + bm - 1) / bm);
    const float us = shape_us(s, tiles, n, k, experts > 0);
    if (us < least) least = us, best = i;
  }
  return best;
}

}  // namespace mx4
}  // namespace qx
