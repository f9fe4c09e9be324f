// Block shapes of the MX4 products (mx4_tile.h) and the choice between them. Plain C++.
#pragma once

#include <cmath>

#include "qx_internal.h"

namespace qx {
namespace mx4 {

// A block of wm x wn x wk waves, each with mt x nt tiles of 16 x 16 (activation rows x weight rows);
// the wk waves take different k, ks units of it (128 with MX4 rows, 64 with fp16) a stage.
// Cost in us at k = 128 K of up to 256 blocks, one a compute unit: us[0] + us[1] K; of every 256 more:
// us[2] + us[3] K. One block of a shape with `one` set fills a compute unit, or nearly: those come in
// whole rounds. Fitted to the times of 384 products (168 of one matrix, n = 256 to 22016, k = 512 to 11264,
// m = 2 to 4096, and 216 of 4 to 128 experts) before the reads of a unit were held together ahead of its
// products. With the present kernels, on the same products (but those of two fp16 rows that take no tiles)
// with 1.2 GB of weights read in turn, the shapes that the costs choose take 0.6 % (fp16 rows) and 1.6 % (MX4
// rows) more than the best of all shapes in the mean, 3.6 and 2.3 % grouped by expert, where the rows of an
// expert are a guess; at most 20 and 21 %, grouped 40 and 32 %. Where a shape is within 30 % of the best, 96
// of 100 costs are within 21 to 31 % of its time.
// The last shape has several blocks a compute unit, for experts with few rows (in the same run, 32 experts of
// 2816x4096, 32 fp16 rows: 25.2 us, 31.4 in the best of the others; 64 of 2816x2048, 48 MX4 rows: 20.5, 21.7).
struct ShapeCost {
  int mt, nt, wm, wn, wk, ks;
  bool one;
  float us[4];
};
constexpr int kShapes = 10;
template <bool A4>
inline constexpr ShapeCost shapes[kShapes] = {
    {1, 1, 1, 1, 8, 2, true, {3.33f, 0.0665f, 1.44f, 0.102f}},
    {1, 2, 1, 1, 4, 2, false, {2.89f, 0.159f, 0.519f, 0.102f}},
    {2, 2, 1, 1, 8, 1, true, {3.46f, 0.137f, 1.82f, 0.194f}},
    {2, 4, 1, 1, 4, 1, false, {3.19f, 0.314f, 0.733f, 0.215f}},
    {4, 2, 1, 1, 8, 1, true, {3.8f, 0.229f, 2.35f, 0.288f}},
    {4, 2, 1, 2, 4, 1, true, {3.79f, 0.35f, 2.76f, 0.409f}},
    {4, 4, 1, 2, 2, 1, false, {4.41f, 0.787f, 1.87f, 0.539f}},
    {4, 4, 2, 4, 1, 1, true, {5.15f, 1.73f, 5.32f, 1.79f}},
    {8, 4, 2, 4, 1, 1, true, {8.29f, 2.66f, 4.93f, 2.95f}},
    {1, 4, 1, 1, 4, 1, false, {2.8f, 0.273f, 0.459f, 0.169f}},
};
template <>
inline constexpr ShapeCost shapes<true>[kShapes] = {
    {1, 1, 1, 1, 8, 2, false, {3.17f, 0.0293f, 0.906f, 0.0424f}},
    {1, 2, 1, 1, 4, 2, false, {2.96f, 0.0658f, 0.535f, 0.0673f}},
    {2, 2, 1, 1, 8, 1, false, {3.47f, 0.06f, 0.963f, 0.0944f}},
    {2, 4, 1, 1, 4, 1, true, {3.27f, 0.132f, 0.683f, 0.138f}},
    {4, 2, 1, 1, 8, 1, true, {3.75f, 0.084f, 2.14f, 0.144f}},
    {4, 4, 1, 1, 4, 1, true, {4.07f, 0.169f, 1.58f, 0.154f}},
    {4, 4, 1, 1, 8, 1, true, {4.5f, 0.129f, 3.31f, 0.198f}},
    {4, 4, 2, 2, 1, 2, true, {5.1f, 0.437f, 2.1f, 0.317f}},
    {8, 4, 2, 4, 1, 2, true, {6.73f, 0.981f, 5.95f, 1.15f}},
    {1, 2, 1, 1, 4, 1, true, {2.66f, 0.0883f, 0.285f, 0.0631f}},
};
// fp16 rows of one matrix do without the last shape: it is the best for 4 of the 165 products, by 3 to 11 %,
// but a cost is too coarse to tell them from those where its blocks come out uneven over the compute units: it
// would be chosen for 4, of which 3 then take 8 to 15 % more (13242x512, m = 3: 4.3 us, 3.8 in 16 x 32).
template <bool A4>
constexpr bool built(int shape, bool grouped) { return A4 || grouped || shape < kShapes - 1; }

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
// 4096x1408, 4001 MX4 rows: 42 us in tiles of 128 x 128, 51 in 256 x 256, which would count as one tile
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
    if (!built<A4>(i, experts > 0)) continue;
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
