// Microscaled 4-bit floating point: rounding of fp16 rows to E2M1 codes with one E8M0 scale per
// 32 elements, and the expansion back. The layout is declared in include/qx.h.
//
// Mathematics. A block's scale is 2^(floor(log2 max|x|) - 2), so that its largest element lands in
// [4, 8) of a code range that ends at 6; x / scale is rounded to the nearest E2M1 value, ties to the
// even code, magnitudes above 6 to 6. Both steps are exact up to that one rounding: the exponent is
// read from the maximum's bits and the conversion instruction divides by a power of two.
#include "qx_device.h"
#include "qx_internal.h"

namespace qx {
namespace {

typedef unsigned short us2_t __attribute__((ext_vector_type(2)));

// Larger of two pairs of 16-bit magnitudes.
__device__ __forceinline__ uint32_t umax2(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(us2_t, a), __builtin_bit_cast(us2_t, b)));
}
template <int CTRL>
__device__ __forceinline__ uint32_t dpp_max2(uint32_t v) {
  return umax2(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, false));
}

// Eight elements a thread, the four threads of a block next to each other.
__global__ __launch_bounds__(256) void quantize_mx4_kernel(const u32x4* __restrict__ X, uint32_t* __restrict__ codes,
                                                           uint8_t* __restrict__ scales, size_t items) {
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < items; i += (size_t)gridDim.x * 256) {
    const u32x4 x = X[i];
    // as integers the magnitudes of fp16 order like their values, infinity and NaN above all
    uint32_t a = umax2(umax2(x.x & 0x7FFF7FFFu, x.y & 0x7FFF7FFFu), umax2(x.z & 0x7FFF7FFFu, x.w & 0x7FFF7FFFu));
    a = dpp_max2<0xB1>(a);  // quad_perm [1,0,3,2]
    a = dpp_max2<0x4E>(a);  // quad_perm [2,3,0,1]
    const uint32_t top = max(a & 0xFFFFu, a >> 16);
    // fp16 subnormals are normal in fp32, so its exponent field is floor(log2) + 127 for all but 0
    const uint32_t ex = __builtin_bit_cast(uint32_t, half_bits_to_float(top)) >> 23;
    const uint32_t s = top >= 0x7C00u ? 255u : top == 0u ? 0u : ex - 2u;
    const float scale = __builtin_bit_cast(float, s << 23);
    uint32_t q = 0;
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(q, as_h2(x.x), scale, 0);
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(q, as_h2(x.y), scale, 1);
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(q, as_h2(x.z), scale, 2);
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(q, as_h2(x.w), scale, 3);
    codes[i] = q;
    if ((threadIdx.x & 3) == 0) scales[i >> 2] = (uint8_t)s;
  }
}

// Eight codes a thread.
template <int OUT>
__global__ __launch_bounds__(256) void dequant_mx4_kernel(const uint32_t* __restrict__ codes,
                                                          const uint8_t* __restrict__ scales, void* __restrict__ out,
                                                          size_t items) {
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < items; i += (size_t)gridDim.x * 256) {
    const uint32_t q = codes[i];
    if constexpr (OUT == QX_OUT_F16) {
      const float scale = __builtin_bit_cast(float, (uint32_t)scales[i >> 2] << 23);
      static_cast<u32x4*>(out)[i] = u32x4{as_u32(__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(q, scale, 0)),
                                          as_u32(__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(q, scale, 1)),
                                          as_u32(__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(q, scale, 2)),
                                          as_u32(__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(q, scale, 3))};
    } else {
      const uint32_t e = q & 0x0F0F0F0Fu, o = (q >> 4) & 0x0F0F0F0Fu;
      static_cast<u32x2*>(out)[i] = u32x2{perm(o, e, 0x05010400u), perm(o, e, 0x07030602u)};
    }
  }
}

unsigned blocks_for(size_t items) {
  const size_t b = (items + 255) / 256;
  return (unsigned)(b < (1u << 20) ? b : (1u << 20));  // more are walked by the same blocks
}

}  // namespace

int launch_quantize_mx4(int m, int k, const uint16_t* X, void* packed, hipStream_t s) {
  const size_t items = (size_t)m * k / 8;
  char* p = static_cast<char*>(packed);
  hipLaunchKernelGGL(quantize_mx4_kernel, dim3(blocks_for(items)), dim3(256), 0, s, reinterpret_cast<const u32x4*>(X),
                     reinterpret_cast<uint32_t*>(p), reinterpret_cast<uint8_t*>(p + items * 4), items);
  return hipGetLastError() == hipSuccess ? QX_OK : QX_E_HIP;
}

int launch_dequant_mx4(const qx_desc* d, const void* packed, int out_kind, void* out, hipStream_t s) {
  const size_t items = (size_t)d->n * d->k / 8;
  const char* p = static_cast<const char*>(packed);
  const uint32_t* codes = reinterpret_cast<const uint32_t*>(p);
  const uint8_t* scales = reinterpret_cast<const uint8_t*>(p + items * 4);
  if (out_kind == QX_OUT_CODES)
    hipLaunchKernelGGL(dequant_mx4_kernel<QX_OUT_CODES>, dim3(blocks_for(items)), dim3(256), 0, s, codes, scales, out, items);
  else
    hipLaunchKernelGGL(dequant_mx4_kernel<QX_OUT_F16>, dim3(blocks_for(items)), dim3(256), 0, s, codes, scales, out, items);
  return hipGetLastError() == hipSuccess ? QX_OK : QX_E_HIP;
}

}  // namespace qx
