// Device helpers of the microscaled 4-bit format.
#pragma once

#include "expert_tiles.h"
#include "lds_loads.h"
#include "qx_device.h"

namespace qx {

typedef int i32x8 __attribute__((ext_vector_type(8)));

// Eight codes (one dword, natural order) as fp16 times the scale 2^(s - 127) given as s << 23:
// exact where the product is a value of fp16, else rounded to nearest-even; s = 255 gives NaN.
__device__ __forceinline__ h8_t mx4_frag(uint32_t q, float scale) {
  return frag(as_u32(__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(q, scale, 0)),
              as_u32(__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(q, scale, 1)),
              as_u32(__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(q, scale, 2)),
              as_u32(__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(q, scale, 3)));
}

// acc + (16 rows of a) x (16 rows of b) over 128 codes: lane l holds block l / 16 of row l % 16
// of both, 32 codes each, and that block's scale in the low byte of sa and sb.
__device__ __forceinline__ f4_t mfma_mx4(u32x4 a, uint32_t sa, u32x4 b, uint32_t sb, f4_t acc) {
  const i32x8 av = {(int)a.x, (int)a.y, (int)a.z, (int)a.w, 0, 0, 0, 0};
  const i32x8 bv = {(int)b.x, (int)b.y, (int)b.z, (int)b.w, 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(av, bv, acc, 4, 4, 0, (int)sa, 0, (int)sb);
}

}  // namespace qx
