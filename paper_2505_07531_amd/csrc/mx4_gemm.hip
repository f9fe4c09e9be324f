// Products of fp16 rows with microscaled 4-bit weights: the launcher of the tiles (mx4_tile.h), and the
// kernel for one row.
#include "mx4_tile.h"

namespace qx {
namespace {

constexpr int kGemvRows = 4, kGemvWaves = 8;

// M rows, 1 or 2. A lane takes one block of 32 codes of each of kGemvRows weight rows and holds the 32
// values of each row of X that belong to it in registers; a wave takes 64 neighbouring blocks (2048 k), SEG
// waves a whole row, or more in turns. Read-bound: 17 bytes of codes and scale for 32 M products, 16
// conversions and 16 M v_dot2 (with three rows the VALU takes longer than the loads). No x in LDS and no barrier before the products: only the SEG sums of a row
// meet there.
template <int SEG, int M>
__global__ __launch_bounds__(64 * kGemvWaves) void mx4_gemv_kernel(const char* __restrict__ packed,
                                                                  const u32x4* __restrict__ x, uint16_t* __restrict__ y,
                                                                  int n, int k) {
  constexpr int kRows = kGemvRows * (kGemvWaves / SEG);  // of a block
  __shared__ float sums[M][kRows][SEG];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int seg = wave % SEG, part = wave / SEG, G = k >> 5, row0 = blockIdx.x * kRows + part * kGemvRows;
  const uint8_t* const scales = reinterpret_cast<const uint8_t*>(packed + (size_t)n * (k >> 1));
  float sum[M][kGemvRows] = {};
  for (int b0 = seg * 64; b0 < G; b0 += SEG * 64) {
    const int b = min(b0 + lane, G - 1);
    u32x4 xv[M][4], q[kGemvRows];
    uint32_t s[kGemvRows];
#pragma unroll
    for (int c = 0; c < M; ++c)
#pragma unroll
      for (int j = 0; j < 4; ++j) xv[c][j] = x[c * 4 * G + 4 * b + j];
#pragma unroll
    for (int r = 0; r < kGemvRows; ++r) {
      const size_t at = (size_t)min(row0 + r, n - 1) * G + b;
      q[r] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(packed) + at);
      s[r] = scales[at];
    }
#pragma unroll
    for (int r = 0; r < kGemvRows; ++r) {
      const float scale = __builtin_bit_cast(float, s[r] << 23);
      float v[M] = {};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const u32x4 w = __builtin_bit_cast(u32x4, mx4_frag(q[r][j], scale));
#pragma unroll
        for (int c = 0; c < M; ++c)
#pragma unroll
          for (int i = 0; i < 4; ++i) v[c] = dot2(w[i], xv[c][j][i], v[c]);
      }
#pragma unroll
      for (int c = 0; c < M; ++c) sum[c][r] += b0 + lane < G ? v[c] : 0.f;  // past the row's end: its last block again
    }
  }
#pragma unroll
  for (int c = 0; c < M; ++c)
#pragma unroll
    for (int r = 0; r < kGemvRows; ++r) {
      const float v = wave_sum(sum[c][r]);
      if (lane == 63) sums[c][part * kGemvRows + r][seg] = v;
    }
  __syncthreads();
  const int at = threadIdx.x % kRows, c = threadIdx.x / kRows, row = blockIdx.x * kRows + at;
  if (c < M && row < n) {
    float v = sums[c][at][0];
#pragma unroll
    for (int i = 1; i < SEG; ++i) v += sums[c][at][i];
    y[(size_t)c * n + row] = (uint16_t)float_to_half_bits(v);
  }
}

template <int SEG, int M>
int launch_gemv_seg(const qx_desc* d, const void* packed, const uint16_t* x, uint16_t* y, hipStream_t s) {
  constexpr int kRows = kGemvRows * (kGemvWaves / SEG);
  const long blocks = ((long)d->n + kRows - 1) / kRows;
  if (blocks >= (1 << 22)) return QX_E_UNSUPPORTED;
  hipLaunchKernelGGL((mx4_gemv_kernel<SEG, M>), dim3((unsigned)blocks), dim3(64 * kGemvWaves), 0, s,
                     static_cast<const char*>(packed), reinterpret_cast<const u32x4*>(x), y, d->n, d->k);
  return hipGetLastError() == hipSuccess ? QX_OK : QX_E_HIP;
}

template <int M>
int launch_gemv_rows(const qx_desc* d, const void* packed, const uint16_t* x, uint16_t* y, hipStream_t s) {
  if (d->k <= 2048) return launch_gemv_seg<1, M>(d, packed, x, y, s);
  if (d->k <= 4096) return launch_gemv_seg<2, M>(d, packed, x, y, s);
  if (d->k <= 8192) return launch_gemv_seg<4, M>(d, packed, x, y, s);
  return launch_gemv_seg<8, M>(d, packed, x, y, s);
}

}  // namespace

// As many waves a row as it has 2048 k, 8 at most. us with 1 / 2 / 4 / 8 waves a row, and in the tiles:
// 22016x1024 4.9 / 5.4 / 7.0 / 9.2, 5.3; 22016x4096 9.8 / 9.4 / 10.1 / 11.6, 11.9 (5.1 TB/s); 4096x4096
// 4.3 / 3.6 / 4.0 / 3.8, 5.8; 4096x8192 6.7 / 5.9 / 5.2 / 5.3, 8.8; 16384x11008 18.7 / 18.1 / 18.7 / 18.4, 25.7
// (1.2 GB of weights read in turn).
int launch_gemv_mx4(const qx_desc* d, const void* packed, const uint16_t* x, uint16_t* y, hipStream_t s) {
  return launch_gemv_rows<1>(d, packed, x, y, s);
}

// Two rows without tiles where a row of weights is long. us, and in the tiles: 22016x1024 6.2, 5.3; 4096x2048
// 3.9, 4.5; 22016x4096 12.0, 12.2; 4096x4096 4.2, 5.9; 509x8192 4.2, 8.4; 8192x8192 10.4, 15.0; 16384x11008
// 25.2, 25.8. Three rows, when that was chosen: 4096x4096 5.5, 5.0; 8192x8192 18.6, 14.0.
int launch_gemm_mx4(const qx_desc* d, const void* packed, int m, const uint16_t* X, uint16_t* Y, hipStream_t s) {
  if (m == 1) return launch_gemv_rows<1>(d, packed, X, Y, s);
  if (m == 2 && d->k >= 2048) return launch_gemv_rows<2>(d, packed, X, Y, s);
  return mx4::launch<false, false>(d, packed, Experts{}, m, X, Y, mx4::pick_shape<false>(d->n, d->k, m, 0), s);
}

int launch_gemm_mx4_grouped(const qx_desc* d, const void* packed, const Experts& ex, int m, const uint16_t* X,
                            uint16_t* Y, hipStream_t s) {
  return mx4::launch<false, true>(d, packed, ex, m, X, Y, mx4::pick_shape<false>(d->n, d->k, m, ex.count), s);
}

}  // namespace qx
