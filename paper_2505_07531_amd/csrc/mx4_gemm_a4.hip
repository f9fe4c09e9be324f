// Products of MX4 rows with microscaled 4-bit weights: the launcher of the tiles (mx4_tile.h).
#include "mx4_tile.h"

namespace qx {

int launch_gemm_a4(const qx_desc* d, const void* packed, int m, const void* Xq, uint16_t* Y, hipStream_t s) {
  return mx4::launch<true, false>(d, packed, Experts{}, m, Xq, Y, mx4::pick_shape<true>(d->n, d->k, m, 0), s);
}

int launch_gemm_a4_grouped(const qx_desc* d, const void* packed, const Experts& ex, int m, const void* Xq,
                           uint16_t* Y, hipStream_t s) {
  return mx4::launch<true, true>(d, packed, ex, m, Xq, Y, mx4::pick_shape<true>(d->n, d->k, m, ex.count), s);
}

}  // namespace qx
