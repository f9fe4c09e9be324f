// Products with microscaled 4-bit weights, Y[m][n] = sum_k X[m][k] W'[n][k], for fp16 rows X and for
// rows of the same format, of one matrix or grouped by expert.
//
// A lane holds one block of 32 codes of a weight row (16 bytes) and the four lane groups of a wave
// four neighbouring blocks, 128 of k. For fp16 rows the codes are converted with their scale, two a
// v_cvt_scalef32_pk_f16_fp4, into the operands of four v_mfma_f32_16x16x32_f16; for rows of the same
// format both sides go to v_mfma_scale_f32_16x16x128_f8f6f4 as they are. Weights are the first
// operand, so that a lane ends with four neighbouring columns of Y.
#include "mx4_device.h"

namespace qx {
namespace {

// One wave: 16 weight rows, 16 * MT activation rows, all of k, operands straight from memory.
template <bool A4, bool GROUPED, int MT>
__global__ __launch_bounds__(256) void mx4_gemm_kernel(const char* __restrict__ packed, const char* __restrict__ X,
                                                       uint16_t* __restrict__ Y, int n, int k, int m, int nx, Experts ex) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, g = lane >> 4, li = lane & 15;
  int n0 = (int)(blockIdx.x % nx) * 64 + wave * 16, m0 = (int)(blockIdx.x / nx) * 16 * MT, rows = min(m - m0, 16 * MT);
  const char* W = packed;
  if constexpr (GROUPED) {
    const ExpertTile t = expert_tile(ex, m, 16 * MT, nx, blockIdx.x);
    if (t.rows == 0) return;
    n0 = t.nt * 64 + wave * 16, m0 = t.row0, rows = t.rows, W += (size_t)t.expert * ex.stride;
  }
  const int G = k >> 5;
  const size_t wrow = (size_t)min(n0 + li, n - 1);
  const char* wc = W + wrow * (k >> 1) + 16 * g;
  const uint8_t* ws = reinterpret_cast<const uint8_t*>(W + (size_t)n * (k >> 1)) + wrow * G + g;
  size_t xrow[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) xrow[t] = (size_t)m0 + min(16 * t + li, rows - 1);
  f4_t acc[MT] = {};
  for (int c = 0; c < k >> 7; ++c) {
    const u32x4 q = *reinterpret_cast<const u32x4*>(wc + 64 * c);
    const uint32_t s = ws[4 * c];
    if constexpr (A4) {
      const uint8_t* xs = reinterpret_cast<const uint8_t*>(X + (size_t)m * (k >> 1));
#pragma unroll
      for (int t = 0; t < MT; ++t) {
        const u32x4 x = *reinterpret_cast<const u32x4*>(X + xrow[t] * (k >> 1) + 64 * c + 16 * g);
        acc[t] = mfma_mx4(q, s, x, xs[xrow[t] * G + 4 * c + g], acc[t]);
      }
    } else {
      const float scale = __builtin_bit_cast(float, s << 23);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const h8_t w = mx4_frag(q[j], scale);
#pragma unroll
        for (int t = 0; t < MT; ++t) {
          const h8_t x = *reinterpret_cast<const h8_t*>(X + 2 * (xrow[t] * k + 128 * c + 32 * g + 8 * j));
          acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(w, x, acc[t], 0, 0, 0);
        }
      }
    }
  }
  const int col = n0 + 4 * g;
#pragma unroll
  for (int t = 0; t < MT; ++t)
    if (16 * t + li < rows && col < n) store4(Y + (size_t)(m0 + 16 * t + li) * n + col, acc[t], n - col);
}

template <bool A4, bool GROUPED>
int run(const qx_desc* d, const void* packed, const Experts& ex, int m, const void* X, uint16_t* Y, hipStream_t s) {
  constexpr int MT = 4;
  const long nx = ((long)d->n + 63) / 64, tiles = ((long)m + 16 * MT - 1) / (16 * MT);
  const unsigned blocks = GROUPED ? expert_blocks(ex, m, 16 * MT, (int)nx) : nx * tiles < (1 << 22) ? (unsigned)(nx * tiles) : 0u;
  if (blocks == 0) return QX_E_UNSUPPORTED;
  hipLaunchKernelGGL((mx4_gemm_kernel<A4, GROUPED, MT>), dim3(blocks), dim3(256), 0, s,
                     static_cast<const char*>(packed), static_cast<const char*>(X), Y, d->n, d->k, m, (int)nx, ex);
  return hipGetLastError() == hipSuccess ? QX_OK : QX_E_HIP;
}

}  // namespace

int launch_gemv_mx4(const qx_desc* d, const void* packed, const uint16_t* x, uint16_t* y, hipStream_t s) {
  return run<false, false>(d, packed, Experts{}, 1, x, y, s);
}
int launch_gemm_mx4(const qx_desc* d, const void* packed, int m, const uint16_t* X, uint16_t* Y, hipStream_t s) {
  return run<false, false>(d, packed, Experts{}, m, X, Y, s);
}
int launch_gemm_a4(const qx_desc* d, const void* packed, int m, const void* Xq, uint16_t* Y, hipStream_t s) {
  return run<true, false>(d, packed, Experts{}, m, Xq, Y, s);
}
int launch_gemm_mx4_grouped(const qx_desc* d, const void* packed, const Experts& ex, int m, const uint16_t* X,
                            uint16_t* Y, hipStream_t s) {
  return run<false, true>(d, packed, ex, m, X, Y, s);
}
int launch_gemm_a4_grouped(const qx_desc* d, const void* packed, const Experts& ex, int m, const void* Xq,
                           uint16_t* Y, hipStream_t s) {
  return run<true, true>(d, packed, ex, m, Xq, Y, s);
}

}  // namespace qx
