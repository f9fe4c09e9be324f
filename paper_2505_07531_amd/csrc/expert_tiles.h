// Tiles of products grouped by expert: which rows and columns a block multiplies, found on the
// device from the offsets alone.
#pragma once

#include <hip/hip_runtime.h>

#include "qx_internal.h"

namespace qx {

struct ExpertTile {
  int expert, row0, rows, nt;  // rows 0: nothing to do for the block
};

// The tile of block `block`: row tiles of bm rows of every expert that has rows, times nx column
// tiles. Experts follow each other, within one the row tiles of a column tile, so that neighbours
// read the same weights; blocks of one XCD (block % 8) take a contiguous run of all tiles.
// Uniform over the wave, and every wave of a block finds the same. Offsets are held to [0, m] and
// an expert that ends before it begins has no rows, so none lead outside of X or Y.
__device__ __forceinline__ ExpertTile expert_tile(const Experts& ex, int m, int bm, int nx, int block) {
  const int lane = threadIdx.x & 63;
  int begin, rows, own, sum;
  auto scan = [&](int e0) {  // this lane's expert, and the row tiles of it and those before
    const int e = e0 + lane;
    begin = min(max(ex.offsets[min(e, ex.count)], 0), m);
    const int end = min(max(ex.offsets[min(e + 1, ex.count)], 0), m);
    rows = max(end - begin, 0);  // past the last expert both are its end
    sum = own = (rows + bm - 1) / bm;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int v = __shfl_up(sum, d);
      sum += lane >= d ? v : 0;
    }
  };
  int total = 0;
  for (int e0 = 0; e0 < ex.count; e0 += 64) {
    scan(e0);
    total += __builtin_amdgcn_readlane(sum, 63);
  }
  total = min(total, (1 << 30) / nx);  // more than any launch has: overlapping offsets
  const int share = (total * nx + 7) >> 3, at = (block & 7) * share + (block >> 3);
  ExpertTile r = {0, 0, 0, 0};
  if ((block >> 3) >= share || at >= total * nx) return r;
  int before = 0;
  for (int e0 = 0; e0 < ex.count; e0 += 64) {
    if (ex.count > 64) scan(e0);
    const unsigned long long past = __ballot(before + sum > at / nx);
    if (past != 0) {
      const int f = __builtin_ctzll(past), tiles = __builtin_amdgcn_readlane(own, f);
      const int in = at - (before + __builtin_amdgcn_readlane(sum, f) - tiles) * nx, mt = in % tiles;
      r.nt = in / tiles;
      r.expert = e0 + f;
      r.row0 = __builtin_amdgcn_readlane(begin, f) + mt * bm;
      r.rows = min(__builtin_amdgcn_readlane(rows, f) - mt * bm, bm);
      return r;
    }
    before += __builtin_amdgcn_readlane(sum, 63);
  }
  return r;
}

// Blocks that cover the tiles of any offsets that do not decrease: every expert with rows can
// have one tile that is not full. 0: more than a launch takes.
inline unsigned expert_blocks(const Experts& ex, int m, int bm, int nx) {
  const long tiles = m / bm + (ex.count < m ? ex.count : m), blocks = (tiles * nx + 7) / 8 * 8;
  return blocks < (1 << 22) ? (unsigned)blocks : 0u;
}

}  // namespace qx
