// Loads from memory straight into LDS, and stores of a tile's columns to rows of Y.
#pragma once

#include "qx_device.h"

namespace qx {

typedef __attribute__((address_space(1))) const void GlobalVoid;
typedef __attribute__((address_space(3))) void LdsVoid;

// SIZE bytes a lane from memory straight to LDS: lane l's go to dst + SIZE * l (dst uniform).
template <int SIZE>
__device__ __forceinline__ void load_lds(const char* src, char* dst) {
  static_assert(SIZE == 16 || SIZE == 4, "sizes that the target has");
  if constexpr (SIZE == 16)
    __builtin_amdgcn_global_load_lds((GlobalVoid*)src, (LdsVoid*)dst, 16, 0, 0);
  else
    __builtin_amdgcn_global_load_lds((GlobalVoid*)src, (LdsVoid*)dst, 4, 0, 0);
}

// Between loads to LDS and their reads by any wave of the block: a wave waits for its own loads, which the
// barrier alone does not (they count as loads from memory, and __syncthreads orders LDS), then for the
// other waves. The wait is vmcnt(0) with the other counters at their maximum.
__device__ __forceinline__ void lds_loaded() {
  __builtin_amdgcn_s_waitcnt(0x0F70);
  __syncthreads();
}

// Neighbouring columns of a row of Y, which may start at any multiple of 2 bytes.
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(2)));
__device__ __forceinline__ void store4(uint16_t* dst, f4_t v, int left) {  // left: columns to the row's end
  uint32_t h[4];
#pragma unroll
  for (int r = 0; r < 4; ++r) h[r] = float_to_half_bits(v[r]);
  if (left >= 4) {
    *reinterpret_cast<u32x2_any*>(dst) = u32x2{h[0] | (h[1] << 16), h[2] | (h[3] << 16)};
  } else {
#pragma unroll
    for (int r = 0; r < 4; ++r)
      if (r < left) dst[r] = (uint16_t)h[r];
  }
}

}  // namespace qx
