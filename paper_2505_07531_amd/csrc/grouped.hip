// Products grouped by expert, fp16 rows, for the uniform, codebook and Q4X kinds: Y[r] = X[r] W'[e]^T for
// the rows r of expert e, in tiles (expert_tiles.h finds a block's expert and rows from the offsets).
//
// W' are the fp16 weights that qx_dequant writes: uniform s (q - z), the difference exact, the product
// rounded once; codebooks two byte lookups a code; Q4X a lookup times s, rounded once. Codes are decoded in
// registers in the order of k, 8 a lane, so that rows of X go to LDS as they are; the products are
// v_mfma_f32_16x16x32_f16 with fp32 sums, weights first: a lane ends with four columns of Y.
//
// The rounding of uniform levels to fp16 is that of W' itself, as on the matrix cores of qx_gemm. Y is then as
// far from 64-bit products of W' as its own rounding takes it (2.07e-4 in the norm, uniform-4 g128, k = 4096),
// and 2.68e-4 from products of the unrounded levels. To multiply with q - z and scale the sums of every group
// instead would take four multiply-adds a lane and tile of 16 x 16 for each group, at g32 beside every single
// product instruction.
//
// Experts have few rows each, so a tile is small and its time is that of one block's chain over k: codes,
// tables and rows go straight to LDS a stage ahead, one barrier a stage, and k is split over the waves of a
// block, whose sums are added in their order. A piece of codes is 16 bytes of a chunk and slice; the chunks of
// a stage lie beside each other, 32 to 64 bytes a slice, which is what the loads cost most by: 8 experts of
// 1376x4096, uniform-4 g128, m = 999, in 64 x 128 take 28.3 us (398 TFLOP/s), the loads alone 27.3, decoding and
// products alone 21.6 (blobs in the last-level cache; read from memory 31.1, 29.2 and 21.6). 32 experts of that
// size, m = 64, from memory: 25 us.
#include "expert_tiles.h"
#include "grouped_plan.h"
#include "lds_loads.h"
#include "qx_device.h"

namespace qx {
namespace {

// A block of wm x wn x wk waves, each with mt x nt tiles of 16 x 16 (activation rows x weight rows); the wk
// waves take different chunks of a stage.
template <int BITS, int KIND, int G, int I>
struct Grouped {
  static constexpr grouped::ShapeCost S = grouped::shapes[0][I];
  static constexpr int MT = S.mt, NT = S.nt, WM = S.wm, WN = S.wn, WK = S.wk, NG = 128 / G;
  static constexpr int kWaves = WM * WN * WK, kThreads = 64 * kWaves, BM = 16 * MT * WM, BN = 16 * NT * WN;
  static constexpr int KU = S.ks;  // chunks in a stage, one a wave
  static_assert(KU == WK, "chunks");
  // 16-byte pieces: of activations; of codes, [slice][row][chunk]; of codebooks, [chunk][part][row]
  static constexpr int kXPieces = BM * 16 * KU, kWPieces = BN * BITS * KU;
  static constexpr int kParts = KIND == QX_CODEBOOK ? NG * (2 << BITS) / 16 : 0, kTPieces = BN * kParts * KU;
  // dwords of tables: uniform words [chunk][group][row], Q4X scales and selectors [chunk][2][row]
  static constexpr int kWords = KIND == QX_UNIFORM ? NG : KIND == QX_Q4X ? 2 : 0, kMWords = BN * kWords * KU;
  static constexpr int loads(int items) { return (items + kThreads - 1) / kThreads; }
  static constexpr int kX = 0, kW = kX + loads(kXPieces) * kThreads * 16, kT = kW + loads(kWPieces) * kThreads * 16;
  static constexpr int kM = kT + loads(kTPieces) * kThreads * 16, kAll = kM + loads(kMWords) * kThreads * 4;
  static constexpr int kSums = WK > 1 ? (kWaves * MT * NT + 1) / 2 * 1024 : 0;  // the waves' sums, half in each buffer
  static constexpr int kStage = kAll > kSums ? kAll : kSums, kLds = 2 * kStage + (KIND == QX_Q4X ? 128 : 0);
};

// What decodes the codes of one group: uniform (s, s) and -(1024 + z), tables, Q4X both.
template <int BITS, int KIND>
struct Levels {
  uint32_t sp, z;
  LutGroup<BITS> lut;
};

// The weights of 8 codes in natural order, their 4 + 4 bytes in q0 and q1.
template <int BITS, int KIND>
__device__ __forceinline__ void four_weights(uint32_t q, const Levels<BITS, KIND>& l, uint32_t& w01, uint32_t& w23) {
  if constexpr (KIND == QX_UNIFORM) {
    // code bytes under the exponent of 1024: 1024 + q; q - z is exact, its product with s rounded once
    w01 = hmul2(hadd2(perm(0x64646464u, q, 0x04010400u), l.z), l.sp);
    w23 = hmul2(hadd2(perm(0x64646464u, q, 0x04030402u), l.z), l.sp);
  } else {
    uint32_t lo, hi;
    if constexpr (BITS == 3) {
      lo = perm(l.lut.lo[1], l.lut.lo[0], q);
      hi = perm(l.lut.hi[1], l.lut.hi[0], q);
    } else {
      lut4_bytes(l.lut, q, lo, hi);
    }
    w01 = perm(hi, lo, 0x05010400u);
    w23 = perm(hi, lo, 0x07030602u);
    if constexpr (KIND == QX_Q4X) w01 = hmul2(w01, l.sp), w23 = hmul2(w23, l.sp);
  }
}
template <int BITS, int KIND>
__device__ __forceinline__ h8_t eight_weights(uint32_t q0, uint32_t q1, const Levels<BITS, KIND>& l) {
  uint32_t w[4];
  four_weights<BITS, KIND>(q0, l, w[0], w[1]);
  four_weights<BITS, KIND>(q1, l, w[2], w[3]);
  return frag(w[0], w[1], w[2], w[3]);
}

template <int BITS, int KIND, int G, int I, int THREADS = Grouped<BITS, KIND, G, I>::kThreads>
__global__ __launch_bounds__(THREADS, THREADS / 256) void grouped_kernel(const char* __restrict__ packed,
                                                                         const char* __restrict__ X, uint16_t* __restrict__ Y,
                                                                         int n, int k, int m, int nx, Experts ex) {
  using S = Grouped<BITS, KIND, G, I>;
  constexpr int MT = S::MT, NT = S::NT, KU = S::KU, BN = S::BN, NTH = S::kThreads, NG = S::NG;
  // one variable a buffer: the compiler then knows that loads into one do not concern reads of the other
  __shared__ __align__(1024) char lds0[S::kStage];
  __shared__ __align__(1024) char lds1[S::kStage];
  __shared__ __align__(16) uint32_t q4lut[KIND == QX_Q4X ? 32 : 4];
  const ExpertTile own = expert_tile(ex, m, S::BM, nx, blockIdx.x);
  if (own.rows == 0) return;  // whole block, before any barrier
  packed += (size_t)own.expert * ex.stride;
  X += (size_t)own.row0 * k * 2;
  const int n0 = own.nt * BN, wlast = min(n - n0, BN) - 1, xlast = own.rows - 1;
  const int t = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(t >> 6), lane = t & 63, g = lane >> 4, li = lane & 15;
  const int wk = wave % S::WK, wn = wave / S::WK % S::WN, wm = wave / (S::WK * S::WN);
  const int C = k >> 7, G_row = k / G, stages = (C + KU - 1) / KU;
  const size_t meta = (size_t)n * k * BITS / 8;
  const char* const codes = packed + (size_t)n0 * BITS * C * 16;
  const char* const tables = packed + meta + (size_t)n0 * G_row * (KIND == QX_UNIFORM ? 4 : KIND == QX_Q4X ? 2 : 2 << BITS);
  const int words = (G_row + 15) / 16;  // Q4X selector words of a row
  const char* const sels = packed + meta + (size_t)n * G_row * 2 + (size_t)n0 * words * 4;
  if constexpr (KIND == QX_Q4X) stage_q4x_tables(packed + q4x_offsets(n, k).codebook, q4lut);

  // Stage st holds chunks first(st) .. + KU - 1: the last one ends with the row; rows shorter than a
  // stage repeat their last chunk, which is never multiplied.
  auto first = [&](int st) { return max(min(st * KU, C - KU), 0); };
  unsigned xat[S::loads(S::kXPieces)], wat[S::loads(S::kWPieces)], tat[S::loads(S::kTPieces) + 1], mat[S::loads(S::kMWords) + 1];
#pragma unroll
  for (int i = 0; i < S::loads(S::kXPieces); ++i) {
    const int q = i * NTH + t, row = min(q / (16 * KU), xlast);
    int p = (q % (16 * KU)) ^ (q / (16 * KU) & 15);
    if (BITS == 4) p = (p & ~15) | (p & 3) << 2 | (p >> 2 & 3);  // place 4 T + g holds piece 4 g + T
    xat[i] = row * k * 2 + min(p * 16, k * 2 - 16);
  }
#pragma unroll
  for (int i = 0; i < S::loads(S::kWPieces); ++i) {
    const int q = i * NTH + t, row = q / KU % BN, s = min(q / (KU * BN), BITS - 1);
    const int cc = (q % KU) ^ (row * KU / 16 & (KU - 1));  // 16 rows of a chunk lie in 16 different places mod 256 bytes
    wat[i] = ((min(row, wlast) * BITS + s) * C + min(cc, C - 1)) * 16;
  }
  // where a format has none of them the loop runs no turn, but is compiled: divisors of 1 then
  constexpr int kParts = S::kParts + !S::kParts, kWords = S::kWords + !S::kWords;
#pragma unroll
  for (int i = 0; i < S::loads(S::kTPieces); ++i) {
    const int q = i * NTH + t, row = q % BN, part = q / BN % kParts, cc = min(q / (BN * kParts), KU - 1);
    tat[i] = (min(row, wlast) * C + min(cc, C - 1)) * kParts * 16 + part * 16;
  }
#pragma unroll
  for (int i = 0; i < S::loads(S::kMWords); ++i) {
    const int q = i * NTH + t, row = q % BN, w = q / BN % kWords, cc = min(min(q / (BN * kWords), KU - 1), C - 1);
    if (KIND == QX_UNIFORM) mat[i] = (min(row, wlast) * G_row + cc * NG + w) * 4;
    else mat[i] = w == 0 ? (min(row, wlast) * G_row + cc * 2) * 2 : min(row, wlast) * words * 4;  // selectors: of the row
  }
  // of a block with few rows a wave leaves out the loads past the last one: what LDS holds there enters
  // columns of products that are not stored
  const int xloads = (own.rows * 16 * KU - wave * 64 + NTH - 1) / NTH;
  auto load = [&](int st, char* buf) {
    const int c = first(st);
    // kept apart from the lanes' offsets: summed before the loop they would take two registers each
    const char *xb = X + c * 256, *wb = codes + c * 16, *tb = tables + c * (KIND == QX_UNIFORM ? NG * 4 : KIND == QX_Q4X ? 4 : S::kParts * 16);
    asm volatile("" : "+s"(xb), "+s"(wb), "+s"(tb));
#pragma unroll
    for (int i = 0; i < S::loads(S::kXPieces); ++i)
      if (S::BM > 32 || i < xloads) load_lds<16>(xb + xat[i], buf + S::kX + (i * NTH + wave * 64) * 16);
#pragma unroll
    for (int i = 0; i < S::loads(S::kWPieces); ++i) load_lds<16>(wb + wat[i], buf + S::kW + (i * NTH + wave * 64) * 16);
#pragma unroll
    for (int i = 0; i < S::loads(S::kTPieces); ++i) load_lds<16>(tb + tat[i], buf + S::kT + (i * NTH + wave * 64) * 16);
#pragma unroll
    for (int i = 0; i < S::loads(S::kMWords); ++i) {
      const char* src = tb + mat[i];
      if constexpr (KIND == QX_Q4X) {
        const int q = i * NTH + t, cc = min(min(q / (BN * 2), KU - 1), C - 1);
        if (q / BN % 2 == 1) src = sels + mat[i] + (c + cc) / 8 * 4;
      }
      load_lds<4>(src, buf + S::kM + (i * NTH + wave * 64) * 4);
    }
  };

  f4_t acc[MT][NT];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[i][j] = f4_t{0.f, 0.f, 0.f, 0.f};

  // Group grp of chunk cc of the weight row (in the tile) `row`.
  auto levels = [&](const char* buf, int cc, int grp, int row, int c) {
    Levels<BITS, KIND> l;
    if constexpr (KIND == QX_UNIFORM) {
      const uint32_t w = *reinterpret_cast<const uint32_t*>(buf + in_vgpr(S::kM + ((cc * NG + grp) * BN + row) * 4));
      l.sp = perm(w, w, 0x01000100u);
      // z is an integer-valued fp16: the bits of -(1024 + z) are those of -1024 plus z
      l.z = (0xE400u + (uint32_t)(unsigned short)__builtin_bit_cast(_Float16, (uint16_t)(w >> 16))) * 0x00010001u;
    } else if constexpr (KIND == QX_Q4X) {
      const uint32_t at = in_vgpr(S::kM + (cc * 2 * BN + row) * 4);
      const uint32_t w = *reinterpret_cast<const uint32_t*>(buf + at), sel = *reinterpret_cast<const uint32_t*>(buf + (at + BN * 4));
      l.sp = perm(w, w, grp == 0 ? 0x01000100u : 0x03020302u);
      const uint32_t* const tp = q4lut + 8 * (sel >> (4 * (c & 7) + 2 * grp) & 3u);
      const u32x4 tl = *reinterpret_cast<const u32x4*>(tp), th = *reinterpret_cast<const u32x4*>(tp + 4);
      l.lut = LutGroup<BITS>{{tl.x, tl.y, tl.z, tl.w}, {th.x, th.y, th.z, th.w}};
    } else {
      constexpr int U = (2 << BITS) / 16;  // pieces of a table
      const uint32_t at = in_vgpr(S::kT + ((cc * S::kParts + grp * U) * BN + row) * 16);
      uint32_t w[4 * U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const u32x4 v = *reinterpret_cast<const u32x4*>(buf + (at + u * BN * 16));
        w[4 * u] = v.x, w[4 * u + 1] = v.y, w[4 * u + 2] = v.z, w[4 * u + 3] = v.w;
      }
      l.lut = lut_group<BITS>(w);
    }
    return l;
  };
  // The products of chunk c, in place cc of the buffer: in step T lane group g takes the 8 codes from 8 f
  // on, f = 4 g + T with 4-bit codes (a slice a lane group) and 4 T + g with 3-bit codes:
  //   T = 0: bits 0-2 of dwords 2g, 2g+1; T = 1: bits 0-2 of dwords 8+2g, 9+2g (g < 2) or bits 3-5 of
  //   dwords 2(g-2), 2(g-2)+1; T = 2: bits 3-5 of dwords 4+2g, 5+2g; T = 3: the spare codes of dwords 2g, 2g+1.
  auto chunk = [&](const char* buf, int cc, int c) {
    u32x4 d4[BITS == 4 ? NT : 1];
    Levels<BITS, KIND> l4[BITS == 4 ? NT : 1];
    const uint32_t wat0 = in_vgpr(S::kW + (wn * NT * 16 + li) * KU * 16 + (cc ^ (li * KU / 16 & (KU - 1))) * 16);
    constexpr int kSlice = BN * KU * 16;
    if constexpr (BITS == 4) {
      const uint32_t at = in_vgpr(wat0 + g * kSlice);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        d4[nt] = *reinterpret_cast<const u32x4*>(buf + (at + nt * KU * 256));
        l4[nt] = levels(buf, cc, 32 * g / G, wn * NT * 16 + nt * 16 + li, c);
      }
    }
    // the rows of X are read a step ahead and stay there (64 x 128 tiles: 3 to 5 % less time than beside
    // their products, where the compiler puts them)
    h8_t x[2][MT];
    auto read_x = [&](int T) {
      const uint32_t xr = in_vgpr(S::kX + (wm * MT * 16 + li) * KU * 256 + ((cc * 16 + 4 * T + g) ^ li) * 16);
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) x[T & 1][mt] = *reinterpret_cast<const h8_t*>(buf + (xr + mt * KU * 4096));
    };
    read_x(0);
#pragma unroll
    for (int T = 0; T < 4; ++T) {
      if (T < 3) read_x(T + 1);
      __builtin_amdgcn_sched_barrier(0);
      h8_t w[NT];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        if constexpr (BITS == 4) {
          const uint32_t D = d4[nt][T], e = D & 0x0F0F0F0Fu, o = D >> 4 & 0x0F0F0F0Fu;
          w[nt] = eight_weights<BITS, KIND>(perm(o, e, 0x05010400u), perm(o, e, 0x07030602u), l4[nt]);
        } else {
          const int sl = T == 0 || T == 3 ? g >> 1 : T == 1 ? (g < 2 ? 2 : 0) : g < 2 ? 1 : 2;
          const u32x2 L = *reinterpret_cast<const u32x2*>(buf + (in_vgpr(wat0 + sl * kSlice + 8 * (g & 1)) + nt * KU * 256));
          uint32_t q[2] = {L.x, L.y};
          u32x2 H = {0u, 0u};
          if (T == 3) H = *reinterpret_cast<const u32x2*>(buf + (in_vgpr(wat0 + 2 * kSlice + 8 * (g & 1)) + nt * KU * 256));
          const uint32_t h[2] = {H.x, H.y};
#pragma unroll
          for (int i = 0; i < 2; ++i)
            q[i] = T == 0   ? q[i] & 0x07070707u
                   : T == 1 ? q[i] >> (g < 2 ? 0 : 3) & 0x07070707u
                   : T == 2 ? q[i] >> 3 & 0x07070707u
                            : (q[i] >> 6 & 0x03030303u) | (h[i] >> (g < 2 ? 4 : 5) & 0x04040404u);
          w[nt] = eight_weights<BITS, KIND>(q[0], q[1], levels(buf, cc, 32 * T / G, wn * NT * 16 + nt * 16 + li, c));
        }
      }
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) acc[mt][nt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(w[nt], x[T & 1][mt], acc[mt][nt], 0, 0, 0);
    }
  };
  auto compute = [&](int st, const char* buf) {
    const int c = st * KU + wk;
    if (c < C) chunk(buf, c - first(st), c);
  };
  load(0, lds0);
  lds_loaded();
  int st = 0;
  for (; st + 1 < stages; st += 2) {
    load(st + 1, lds1);
    compute(st, lds0);
    lds_loaded();
    if (st + 2 < stages) load(st + 2, lds0);
    compute(st + 1, lds1);
    lds_loaded();
  }
  if (st < stages) compute(st, lds0);

  // the partial sums of waves on different k, added in their order: tile i by wave i % WK
  if constexpr (S::WK > 1) {
    __syncthreads();
    constexpr int kPer = S::kStage / 1024;  // tiles of 1 KB in each buffer
    const int base = (wave - wk) * MT * NT;
    auto at = [&](int i) { return (i < kPer ? lds0 + i * 1024 : lds1 + (i - kPer) * 1024) + lane * 16; };
#pragma unroll
    for (int i = 0; i < MT * NT; ++i) *reinterpret_cast<f4_t*>(at(base + wk * MT * NT + i)) = acc[i / NT][i % NT];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < MT * NT; ++i) {
      if (i % S::WK != wk) continue;
      f4_t sum = *reinterpret_cast<const f4_t*>(at(base + i));
#pragma unroll
      for (int w = 1; w < S::WK; ++w) sum += *reinterpret_cast<const f4_t*>(at(base + w * MT * NT + i));
      acc[i / NT][i % NT] = sum;
    }
  }
#pragma unroll
  for (int i = 0; i < MT * NT; ++i) {
    if (S::WK > 1 && i % S::WK != wk) continue;
    const int row = (wm * MT + i / NT) * 16 + li, col = n0 + (wn * NT + i % NT) * 16 + 4 * g;
    if (row < own.rows && col < n) store4(Y + (size_t)(own.row0 + row) * n + col, acc[i / NT][i % NT], n - col);
  }
}

template <int BITS, int KIND, int G, int I>
int launch_shape(const qx_desc* d, const void* packed, const Experts& ex, int m, const uint16_t* X, uint16_t* Y, hipStream_t s) {
  using S = Grouped<BITS, KIND, G, I>;
  static_assert(S::kLds <= 160 * 1024, "LDS");
  const int nx = (int)(((long)d->n + S::BN - 1) / S::BN);
  const unsigned blocks = expert_blocks(ex, m, S::BM, nx);
  if (blocks == 0) return QX_E_UNSUPPORTED;
  hipLaunchKernelGGL((grouped_kernel<BITS, KIND, G, I>), dim3(blocks), dim3(S::kThreads), 0, s,
                     static_cast<const char*>(packed), reinterpret_cast<const char*>(X), Y, d->n, d->k, m, nx, ex);
  return hipGetLastError() == hipSuccess ? QX_OK : QX_E_HIP;
}

}  // namespace

int launch_gemm_grouped(const qx_desc* d, const void* packed, const Experts& ex, int m, const uint16_t* X, uint16_t* Y,
                        hipStream_t s) {
  const int shape = grouped::pick_shape(d, m, ex.count);
  if (shape == grouped::kTile) return launch_gemm_tile_grouped(d, packed, ex, m, X, Y, s);
#define QX_GROUPED(B, K, G)                                                          \
  if (d->bits == B && d->kind == K && d->group == G)                                 \
    return shape == 0   ? launch_shape<B, K, G, 0>(d, packed, ex, m, X, Y, s)        \
           : shape == 1 ? launch_shape<B, K, G, 1>(d, packed, ex, m, X, Y, s)        \
           : shape == 2 ? launch_shape<B, K, G, 2>(d, packed, ex, m, X, Y, s)        \
           : shape == 3 ? launch_shape<B, K, G, 3>(d, packed, ex, m, X, Y, s)        \
                        : launch_shape<B, K, G, 4>(d, packed, ex, m, X, Y, s);
  QX_GROUPED(3, 0, 32) QX_GROUPED(3, 0, 64) QX_GROUPED(3, 0, 128) QX_GROUPED(3, 1, 32) QX_GROUPED(3, 1, 64)
  QX_GROUPED(3, 1, 128) QX_GROUPED(4, 0, 32) QX_GROUPED(4, 0, 64) QX_GROUPED(4, 0, 128) QX_GROUPED(4, 1, 32)
  QX_GROUPED(4, 1, 64) QX_GROUPED(4, 1, 128) QX_GROUPED(4, 2, 64)
#undef QX_GROUPED
  return QX_E_UNSUPPORTED;
}

}  // namespace qx
