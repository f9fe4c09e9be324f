// Products with microscaled 4-bit weights, Y[m][n] = sum_k X[m][k] W'[n][k], of fp16 rows X or of rows
// of the same format, of one matrix or grouped by expert: the kernel for all sizes, in tiles.
//
// Products. A wave multiplies 16 NT weight rows with 16 MT activation rows. With MX4 rows a lane holds
// one block of 32 codes of a row (16 bytes) and the four lane groups four neighbouring blocks: both
// sides go as they are into v_mfma_scale_f32_16x16x128_f8f6f4, their scale bytes beside them, 128 k an
// instruction. With fp16 rows the codes become fp16 times their scale, two a
// v_cvt_scalef32_pk_f16_fp4 (exact for every blob that was quantized from fp16), and two
// v_mfma_f32_16x16x32_f16 take 64 k; a decoded fragment serves MT products. Weights are the first
// operand, so that a lane ends with four neighbouring columns of Y. Sums are fp32 throughout.
//
// Memory. Codes, rows and scales travel from memory straight into LDS (16 bytes a lane, no registers),
// a stage ahead of their use, one barrier a stage. What this costs is requests, not bytes: 16 pieces of
// 64 bytes took as long as 16 of 128 (16384x4096, m = 4096, MX4 rows in 256 x 256 tiles: 289 us with
// stages of 128 k, 183 with 256), and scales a dword a row and stage were a fifth of the time; hence 16
// bytes of scales a row, every 512 k.
//
// k is split over WK waves of a block where tiles are few; their sums are added through LDS in the
// order of the waves. The outputs of large tiles pass through LDS, so that stores write whole rows of
// the tile (32-byte pieces: 9 us more of 183). The order of the sums is fixed: the same bits every time.
//
// Measured (kernel trace, card warm; us, and TFLOP/s): MX4 rows 22016x4096, m = 4096: 242 (3050); fp16
// rows 11008x4096, m = 2001: 180 (1000), where a library product of fp16 matrices of 8192^3 reaches 1140; 32
// experts of 2816x4096, 32 fp16 rows: 20.9 (5.0 TB/s). The matrix cores are busy two fifths of the largest
// tiles' time, the rest is the start and end of a tile (all compute units store at once) and loads.
//
// The pairs of times here and below are those of the step that chose between them, both sides in turn on one
// card; later steps moved both. Deeper rings of smaller stages in the largest tiles, and halves of a block's
// waves multiplying and loading in turn, were not faster (285 to 320 us on the MX4 product above, 265
// without). Three buffers of small tiles gain a tenth where blocks are few and k is long (4096x11008, 64 fp16
// rows: 20.2 to 18.1 us) and lose far more where several share a compute unit (22016x4096, 8 rows: 13.2 to
// 20.7): two buffers.
#pragma once

#include <type_traits>

#include "gemm_tile_plan.h"
#include "lds_loads.h"
#include "mx4_device.h"
#include "mx4_plan.h"

namespace qx {
namespace mx4 {

template <bool A4_, int I>
struct Mx4Shape {
  static constexpr bool A4 = A4_;
  static constexpr ShapeCost cost = shapes<A4>[I];
  static constexpr int MT = cost.mt, NT = cost.nt, WM = cost.wm, WN = cost.wn, WK = cost.wk, KS = cost.ks;
  static constexpr int kWaves = WM * WN * WK, kThreads = 64 * kWaves;
  static constexpr int BM = 16 * MT * WM, BN = 16 * NT * WN;
  static constexpr int UK = A4 ? 128 : 64;          // k of a unit: what a wave reads of a row at once
  static constexpr int KU = WK * KS;                // units in a stage
  static constexpr int WP = UK / 32 * KU, XP = (A4 ? 4 : 8) * KU;  // 16-byte pieces of a row
  static constexpr int WL = (BN * WP + kThreads - 1) / kThreads, XL = (BM * XP + kThreads - 1) / kThreads;  // loads of a thread
  static constexpr int kW = WL * kThreads * 16, kX = XL * kThreads * 16;  // the last loads' surplus repeats a row
  // waves on different k leave their sums in the buffers, 1 KB a tile of 16 x 16
  static constexpr int kSums = WK > 1 ? (kWaves * MT * NT + 1) / 2 * 1024 : 0;
  // large tiles go out through the buffers, half of the rows in each
  static constexpr bool kLdsOut = WK == 1 && BN >= 128;
  static constexpr int kOut = kLdsOut ? BM * BN : 0, kLeast = kSums > kOut ? kSums : kOut;
  static constexpr int kStage = kW + kX > kLeast ? kW + kX : kLeast;
  // Scales, 16 bytes of a row at once (512 k): SR stages share them, or a stage has SN of them.
  static constexpr int kSRows = BN + (A4 ? BM : 0), kUnitBytes = UK / 32;
  static constexpr int SR = KU * kUnitBytes < 16 ? 16 / (KU * kUnitBytes) : 1, SN = SR > 1 ? 1 : KU * kUnitBytes / 16;
  static constexpr int kScales = SN * kSRows * 16, kLds = 2 * (kStage + kScales);
  static_assert(SR > 1 ? 16 % (KU * kUnitBytes) == 0 : KU * kUnitBytes % 16 == 0, "scales of whole stages");
};

// Piece p of a row of P pieces lies at position p ^ swizzle(row) of the row. A read of 16 bytes a
// lane is served in four steps, each of lanes 0-3 and 12-15 of one lane group and 4-11 of its
// neighbour: their pieces have to lie in 16 different places mod 256 bytes.
template <int P>
__device__ __forceinline__ int swizzle(int row) {
  return P >= 16 ? row & 15 : P == 8 ? row >> 1 & 7 : P == 4 ? -(row >> 2) & 3 : row >> 3 & 1;
}

// The rows and columns of a block, and its loads.
struct Mx4Block {
  int n0, m0, rows, expert;
};
template <class S, bool GROUPED>
__device__ __forceinline__ Mx4Block find_block(const Experts& ex, int m, int nx, int my, int groups) {
  if constexpr (GROUPED) {
    const ExpertTile t = expert_tile(ex, m, S::BM, nx, blockIdx.x);
    return {t.nt * S::BN, t.row0, t.rows, t.expert};
  } else {
    const int total = nx * my, share = (total + 7) >> 3, at = blockIdx.x >> 3;
    const int tile = (int)(blockIdx.x & 7) * share + at;
    if (at >= share || tile >= total) return {0, 0, 0, 0};
    const tile::TileAt b = tile::tile_at(tile, nx, my, groups);
    return {b.bn * S::BN, b.bm * S::BM, min(m - b.bm * S::BM, S::BM), 0};
  }
}

template <class S>
struct Mx4Loads {
  const char *W, *Wsc, *X, *Xsc;  // the block's first rows: codes (or fp16) and scales
  unsigned wat[S::WL], xat[S::XL];  // this thread's loads, from there
  int C, G, wave, t, wlast, xlast, xloads;

  __device__ __forceinline__ Mx4Loads(const char* packed, const char* Xall, const Mx4Block& b, int n, int k, int m) {
    const int wbytes = k >> 1, xbytes = S::A4 ? k >> 1 : k * 2;  // of a row
    G = k >> 5;
    W = packed + (size_t)b.n0 * wbytes;
    Wsc = packed + (size_t)n * wbytes + (size_t)b.n0 * G;
    X = Xall + (size_t)b.m0 * xbytes;
    Xsc = S::A4 ? Xall + (size_t)m * xbytes + (size_t)b.m0 * G : nullptr;
    C = k / S::UK, t = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(t >> 6);
    wlast = min(n - b.n0, S::BN) - 1, xlast = b.rows - 1;
    // Of a block with few rows a wave leaves out the loads past the last one: what LDS holds there enters
    // columns of products that are not stored (32 experts, 32 fp16 rows: 28.4 to 25.8 us; of the blocks
    // of 64 rows and more none was faster for it, 11008x4096 m = 2001 183.5 to 192).
    xloads = (b.rows * S::XP - wave * 64 + S::kThreads - 1) / S::kThreads;
#pragma unroll
    for (int i = 0; i < S::WL; ++i) {
      const int q = i * S::kThreads + t, row = q / S::WP, p = (q % S::WP) ^ swizzle<S::WP>(row);
      wat[i] = min(row, wlast) * wbytes + min(p * 16, wbytes - 16);
    }
#pragma unroll
    for (int i = 0; i < S::XL; ++i) {
      const int q = i * S::kThreads + t, row = q / S::XP;
      int p = (q % S::XP) ^ swizzle<S::XP>(row);
      if (!S::A4) p = (p & ~7) | ((p & 3) << 1) | ((p >> 2) & 1);  // place 4 j + g holds piece 2 g + j
      xat[i] = min(row, xlast) * xbytes + min(p * 16, xbytes - 16);
    }
  }

  // Stage st holds units first(st) .. first(st) + KU - 1: the last one ends with the row, so that no
  // load passes it; rows shorter than a stage repeat their last piece, which is never multiplied.
  __device__ __forceinline__ int first(int st) const { return max(min(st * S::KU, C - S::KU), 0); }

  __device__ __forceinline__ void load(int st, char* buf) const {
    const int c = first(st);
    // kept apart from the lanes' offsets: summed before the loop they would take two registers each
    const char *wb = W + c * (S::UK / 2), *xb = X + c * (S::A4 ? 64 : 128);
    asm volatile("" : "+s"(wb), "+s"(xb));
#pragma unroll
    for (int i = 0; i < S::WL; ++i) load_lds<16>(wb + wat[i], buf + (i * S::kThreads + wave * 64) * 16);
#pragma unroll
    for (int i = 0; i < S::XL; ++i)
      if (S::BM > 32 || i < xloads) load_lds<16>(xb + xat[i], buf + S::kW + (i * S::kThreads + wave * 64) * 16);
  }

  // Where the 16 bytes of a row's scales numbered p begin: the last ones end with the row.
  __device__ __forceinline__ int scales_from(int p) const { return max(min(16 * p, G - 16), 0); }

  // The scales of stages st .. st + SR - 1 (st a multiple of SR), one piece of every row after the other.
  __device__ __forceinline__ void load_scales(int st, char* buf) const {
    const int first = st / S::SR * S::SN;
    if (G >= 16) {
#pragma unroll
      for (int i = 0; i < (S::SN * S::kSRows + S::kThreads - 1) / S::kThreads; ++i) {
        const int q = i * S::kThreads + t, row = q % S::kSRows;
        const char* src = row < S::BN ? Wsc + (unsigned)(min(row, wlast) * G) : Xsc + (unsigned)(min(row - S::BN, xlast) * G);
        if (q < S::SN * S::kSRows)
          load_lds<16>(src + scales_from(first + q / S::kSRows), buf + (i * S::kThreads + wave * 64) * 16);
      }
    } else {  // rows of 4, 8 or 12 scales, all in the first piece
#pragma unroll
      for (int i = 0; i < (4 * S::kSRows + S::kThreads - 1) / S::kThreads; ++i) {
        const int q = i * S::kThreads + t, row = q / 4, col = min(q % 4 * 4, G - 4);
        const char* src = row < S::BN ? Wsc + (unsigned)(min(row, wlast) * G) : Xsc + (unsigned)(min(row - S::BN, xlast) * G);
        if (q < 4 * S::kSRows) load_lds<4>(src + col, buf + (i * S::kThreads + wave * 64) * 4);
      }
    }
  }
};

// The operands of one unit of a wave, and its products.
template <class S>
struct Mx4Unit {
  static constexpr int J = S::A4 ? 1 : 2;  // products of 32 k a unit
  // MX4 rows: pieces of 32 codes. fp16 rows: 16 codes of a weight row, fragments of the rows
  typename std::conditional<S::A4, u32x4, u32x2>::type q[S::NT];
  u32x4 x[J][S::MT];
  uint32_t qs[S::NT], xs[S::A4 ? S::MT : 1];  // scales in the low byte

  // Unit u of the buffer; its scales are in the dword at `sd` of a row's 16 bytes in `sbuf`, from byte
  // `sb` of it on.
  __device__ __forceinline__ void read(const char* buf, int u, const char* sbuf, int sd, int sb, int wm, int wn) {
    const int lane = threadIdx.x & 63, g = lane >> 4, li = lane & 15;
    const int sw = swizzle<S::WP>(li), sx = swizzle<S::XP>(li);
    // one offset from the buffer's start for each kind of read, unknown to the compiler: longer
    // sums of addresses lose it which buffer a read is of, and it waits for all loads
    const int sw4 = (int)in_vgpr(sd + (wn * S::NT * 16 + li) * 16), sx4 = (int)in_vgpr(sd + (S::BN + wm * S::MT * 16 + li) * 16);
    if constexpr (S::A4) {
      const int wr = (int)in_vgpr((wn * S::NT * 16 + li) * S::WP * 16 + ((u * 4 + g) ^ sw) * 16);
      const int xr = (int)in_vgpr(S::kW + (wm * S::MT * 16 + li) * S::XP * 16 + ((u * 4 + g) ^ sx) * 16);
#pragma unroll
      for (int nt = 0; nt < S::NT; ++nt) {
        q[nt] = *reinterpret_cast<const u32x4*>(buf + (wr + nt * 256 * S::WP));
        qs[nt] = *reinterpret_cast<const uint32_t*>(sbuf + (sw4 + nt * 256)) >> (8 * g);
      }
#pragma unroll
      for (int mt = 0; mt < S::MT; ++mt) {
        x[0][mt] = *reinterpret_cast<const u32x4*>(buf + (xr + mt * 256 * S::XP));
        xs[mt] = *reinterpret_cast<const uint32_t*>(sbuf + (sx4 + mt * 256)) >> (8 * g);
      }
    } else {
      const int wr = (int)in_vgpr((wn * S::NT * 16 + li) * S::WP * 16 + ((u * 2 + (g >> 1)) ^ sw) * 16 + (g & 1) * 8);
      const int xr0 = (int)in_vgpr(S::kW + (wm * S::MT * 16 + li) * S::XP * 16 + ((u * 8 + g) ^ sx) * 16);
      const int xr1 = (int)in_vgpr(S::kW + (wm * S::MT * 16 + li) * S::XP * 16 + ((u * 8 + 4 + g) ^ sx) * 16);
#pragma unroll
      for (int nt = 0; nt < S::NT; ++nt) {
        q[nt] = *reinterpret_cast<const u32x2*>(buf + (wr + nt * 256 * S::WP));
        qs[nt] = *reinterpret_cast<const uint32_t*>(sbuf + (sw4 + nt * 256)) >> (8 * sb + 8 * (g >> 1));
      }
#pragma unroll
      for (int mt = 0; mt < S::MT; ++mt) {
        x[0][mt] = *reinterpret_cast<const u32x4*>(buf + (xr0 + mt * 256 * S::XP));
        x[1][mt] = *reinterpret_cast<const u32x4*>(buf + (xr1 + mt * 256 * S::XP));
      }
    }
  }

  __device__ __forceinline__ void multiply(f4_t (&acc)[S::MT][S::NT]) const {
    // All reads before the first product, not each beside its own as the compiler would: MX4 rows 22016x4096,
    // m = 4096 237 us, 248 without; fp16 rows, 32 experts of 2816x4096, m = 8192 in 64 x 128 232, 245. The
    // 128 x 64 wave tile has no registers for it with fp16 rows (22016x4096, m = 4096 546, 795 with it).
    if constexpr (S::A4 || S::MT < 8) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int j = 0; j < J; ++j) {
      h8_t w[S::A4 ? 1 : S::NT];
      if constexpr (!S::A4)
#pragma unroll
        for (int nt = 0; nt < S::NT; ++nt)
          w[nt] = mx4_frag(q[nt][j], __builtin_bit_cast(float, (qs[nt] & 255u) << 23));
#pragma unroll
      for (int mt = 0; mt < S::MT; ++mt)
#pragma unroll
        for (int nt = 0; nt < S::NT; ++nt) {
          if constexpr (S::A4)
            acc[mt][nt] = mfma_mx4(q[nt], qs[nt], x[0][mt], xs[mt], acc[mt][nt]);
          else
            acc[mt][nt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(w[nt], __builtin_bit_cast(h8_t, x[j][mt]), acc[mt][nt], 0, 0, 0);
        }
    }
  }
};

template <class S>
__device__ __forceinline__ void clear(f4_t (&acc)[S::MT][S::NT]) {
#pragma unroll
  for (int i = 0; i < S::MT; ++i)
#pragma unroll
    for (int j = 0; j < S::NT; ++j) acc[i][j] = f4_t{0.f, 0.f, 0.f, 0.f};
}

template <class S>
__device__ __forceinline__ void store_tile(uint16_t* Y, const f4_t (&acc)[S::MT][S::NT], const Mx4Block& b, int n, int wm,
                                           int wn, int wk) {
  const int lane = threadIdx.x & 63, g = lane >> 4, li = lane & 15;
#pragma unroll
  for (int mt = 0; mt < S::MT; ++mt) {
    const int row = (wm * S::MT + mt) * 16 + li;
    if (row >= b.rows) continue;
#pragma unroll
    for (int nt = 0; nt < S::NT; ++nt) {
      if (S::WK > 1 && (mt * S::NT + nt) % S::WK != wk) continue;
      const int col = b.n0 + (wn * S::NT + nt) * 16 + 4 * g;
      if (col < n) store4(Y + (size_t)(b.m0 + row) * n + col, acc[mt][nt], n - col);
    }
  }
}

// The same through LDS (half of the rows in each buffer), so that every store instruction writes whole
// rows of the tile's columns. Piece p of 16 bytes of a row lies at place p ^ (row % 16): the lanes
// write four columns of 16 rows at once, which then lie in different banks.
template <class S>
__device__ __forceinline__ void store_tile_lds(uint16_t* Y, const f4_t (&acc)[S::MT][S::NT], char* lds0, char* lds1,
                                               const Mx4Block& b, int n, int wm, int wn) {
  constexpr int P = S::BN / 8, kHalf = S::BM / 2;
  const int lane = threadIdx.x & 63, g = lane >> 4, li = lane & 15;
#pragma unroll
  for (int mt = 0; mt < S::MT; ++mt) {
    const int row0 = (wm * S::MT + mt) * 16;
    char* const at = (row0 < kHalf ? lds0 + row0 * S::BN * 2 : lds1 + (row0 - kHalf) * S::BN * 2) + li * S::BN * 2;
#pragma unroll
    for (int nt = 0; nt < S::NT; ++nt) {
      const f4_t v = acc[mt][nt];
      *reinterpret_cast<u32x2*>(at + (((wn * S::NT + nt) * 2 + (g >> 1)) ^ li) * 16 + (g & 1) * 8) =
          u32x2{float_to_half_bits(v[0]) | float_to_half_bits(v[1]) << 16, float_to_half_bits(v[2]) | float_to_half_bits(v[3]) << 16};
    }
  }
  __syncthreads();
  for (int q = threadIdx.x; q < b.rows * P; q += S::kThreads) {
    const int row = q / P, p = q % P, col = b.n0 + p * 8;
    const char* const at = row < kHalf ? lds0 + row * S::BN * 2 : lds1 + (row - kHalf) * S::BN * 2;
    const u32x4 v = *reinterpret_cast<const u32x4*>(at + (p ^ (row & 15)) * 16);
    uint16_t* const dst = Y + (size_t)(b.m0 + row) * n + col;
    if (col + 8 <= n) {
      *reinterpret_cast<u32x4_any*>(dst) = v;
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (col + i < n) dst[i] = (uint16_t)(v[i / 2] >> (16 * (i % 2)));
    }
  }
}

// Two buffers, one loaded while the other is multiplied.
template <class S, bool GROUPED>
__global__ __launch_bounds__(S::kThreads, (S::kWaves + 3) / 4) void mx4_tile_kernel(
    const char* __restrict__ packed, const char* __restrict__ X, uint16_t* __restrict__ Y, int n, int k, int m, int nx,
    int my, int groups, Experts ex) {
  // one variable a buffer: the compiler then knows that loads into one do not concern reads of another
  __shared__ __align__(1024) char lds0[S::kStage];
  __shared__ __align__(1024) char lds1[S::kStage];
  __shared__ __align__(1024) char scales[2 * S::kScales];
  const Mx4Block b = find_block<S, GROUPED>(ex, m, nx, my, groups);
  if (b.rows == 0) return;  // whole block, before any barrier
  const Mx4Loads<S> ld(packed + (GROUPED ? (size_t)b.expert * ex.stride : 0), X, b, n, k, m);
  const int wave = ld.wave, lane = threadIdx.x & 63;
  const int wk = wave % S::WK, wn = wave / S::WK % S::WN, wm = wave / (S::WK * S::WN);
  const int C = ld.C, stages = (C + S::KU - 1) / S::KU;
  f4_t acc[S::MT][S::NT];
  clear<S>(acc);
  // The next scales are loaded behind the stage's last read of scales, since a read waits for all loads
  // of scales before it: with MX4 rows before the stage's last products, with fp16 rows, whose operands
  // leave no registers for that, after them.
  auto next_scales = [&](int st) {
    if (st < stages && st % S::SR == 0) ld.load_scales(st, scales + (st / S::SR & 1) * S::kScales);
  };
  auto compute = [&](int st, const char* buf) {
#pragma unroll
    for (int s = 0; s < S::KS; ++s) {
      const int c = st * S::KU + wk * S::KS + s;
      Mx4Unit<S> unit;
      // MX4 rows leave room for a branch: waves whose rows are all past the expert's last multiply nothing
      // (32 experts of 2816x4096, m = 8192: 87 us, 91 without; with fp16 rows 248 and 247)
      const bool some = (S::KU == 1 || c < C) && !(S::A4 && GROUPED && S::WM > 1 && wm * S::MT * 16 >= b.rows);
      if (some) {
        const int p = S::SR > 1 ? 0 : (wk * S::KS + s) * S::kUnitBytes / 16;
        const int at = c * S::kUnitBytes - ld.scales_from(st / S::SR * S::SN + p);
        unit.read(buf, c - ld.first(st), scales, (st / S::SR & 1) * S::kScales + p * S::kSRows * 16 + (at & ~3), at & 3, wm, wn);
      }
      if (S::A4 && s == S::KS - 1) next_scales(st + 1);
      if (some) unit.multiply(acc);
    }
    if (!S::A4) next_scales(st + 1);
  };
  ld.load(0, lds0);
  ld.load_scales(0, scales);
  lds_loaded();
  int st = 0;
  for (; st + 1 < stages; st += 2) {
    ld.load(st + 1, lds1);
    compute(st, lds0);
    lds_loaded();
    if (st + 2 < stages) ld.load(st + 2, lds0);
    compute(st + 1, lds1);
    lds_loaded();
  }
  if (st < stages) compute(st, lds0);

  // the partial sums of waves on different k, added in their order: tile i by wave i % WK
  if constexpr (S::WK > 1) {
    __syncthreads();
    constexpr int kPer = S::kStage / 1024;  // tiles of 1 KB in each buffer
    const int base = (wave - wk) * S::MT * S::NT;  // of the waves of this part of the block
    auto at = [&](int i) { return (i < kPer ? lds0 + i * 1024 : lds1 + (i - kPer) * 1024) + lane * 16; };
#pragma unroll
    for (int i = 0; i < S::MT * S::NT; ++i)
      *reinterpret_cast<f4_t*>(at(base + wk * S::MT * S::NT + i)) = acc[i / S::NT][i % S::NT];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < S::MT * S::NT; ++i) {
      if (i % S::WK != wk) continue;
      f4_t sum = *reinterpret_cast<const f4_t*>(at(base + i));
#pragma unroll
      for (int w = 1; w < S::WK; ++w) sum += *reinterpret_cast<const f4_t*>(at(base + w * S::MT * S::NT + i));
      acc[i / S::NT][i % S::NT] = sum;
    }
  }
  if constexpr (S::kLdsOut) {
    __syncthreads();
    store_tile_lds<S>(Y, acc, lds0, lds1, b, n, wm, wn);
  } else {
    store_tile<S>(Y, acc, b, n, wm, wn, wk);
  }
}

template <class S, bool GROUPED>
int launch_shape(const qx_desc* d, const void* packed, const Experts& ex, int m, const void* X, uint16_t* Y, hipStream_t s) {
  static_assert(S::kLds <= tile::kLdsBytes, "LDS");
  const int nx = (int)(((long)d->n + S::BN - 1) / S::BN), my = (m + S::BM - 1) / S::BM;
  const unsigned blocks = GROUPED ? expert_blocks(ex, m, S::BM, nx)
                                  : (long)nx * my < (1 << 22) ? ((unsigned)nx * (unsigned)my + 7u) / 8u * 8u : 0u;
  if (blocks == 0) return QX_E_UNSUPPORTED;
  hipLaunchKernelGGL((mx4_tile_kernel<S, GROUPED>), dim3(blocks), dim3(S::kThreads), 0, s, static_cast<const char*>(packed),
                     static_cast<const char*>(X), Y, d->n, d->k, m, nx, my, tile::tile_groups(my), ex);
  return hipGetLastError() == hipSuccess ? QX_OK : QX_E_HIP;
}

// The shape that costs least for the product.
template <bool A4, bool GROUPED, int I = 0>
int launch(const qx_desc* d, const void* packed, const Experts& ex, int m, const void* X, uint16_t* Y, int shape,
           hipStream_t s) {
  if constexpr (I < kShapes) {
    if constexpr (built<A4>(I, GROUPED))
      if (shape == I) return launch_shape<Mx4Shape<A4, I>, GROUPED>(d, packed, ex, m, X, Y, s);
    return launch<A4, GROUPED, I + 1>(d, packed, ex, m, X, Y, shape, s);
  }
  return QX_E_UNSUPPORTED;
}

}  // namespace mx4
}  // namespace qx
