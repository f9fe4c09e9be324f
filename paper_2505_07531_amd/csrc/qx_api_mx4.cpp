// C entry points of the microscaled 4-bit format and of products grouped by expert: argument
// checks, the host packer, and the launchers' calls.
#include <cstring>

#include "qx_check.h"

using namespace qx;

namespace {

bool overlaps_none(const qx_desc* d, size_t stride, int32_t experts) {
  return experts <= 1 || stride >= packed_bytes(d);
}

int check_grouped(const qx_desc* d, size_t stride, int32_t experts, int32_t m) {
  const int st = check_desc(d);
  if (st != QX_OK) return st;
  if (m < 0 || m > kMaxRows || experts < 0 || experts > kMaxExperts) return QX_E_ARG;
  if (stride % 16 != 0 || !overlaps_none(d, stride, experts)) return QX_E_ARG;
  return QX_OK;
}

}  // namespace

extern "C" {

int qx_pack_mx4(const qx_desc* d, const uint8_t* codes, const uint8_t* scales, void* packed, size_t cap,
                size_t* packed_size) {
  const int st = check_desc(d);
  if (st != QX_OK) return st;
  if (packed_size == nullptr || d->kind != QX_MX4) return QX_E_ARG;
  const size_t total = packed_bytes(d), nk = (size_t)d->n * d->k;
  *packed_size = total;
  if (packed == nullptr) return QX_OK;
  if (cap < total) return QX_E_SIZE;
  if (nk == 0) return QX_OK;
  if (codes == nullptr || scales == nullptr) return QX_E_ARG;
  for (size_t i = 0; i < nk; ++i)
    if (codes[i] > 15) return QX_E_ARG;
  uint8_t* blob = static_cast<uint8_t*>(packed);
  for (size_t i = 0; i < nk / 2; ++i) blob[i] = (uint8_t)(codes[2 * i] | (codes[2 * i + 1] << 4));
  std::memcpy(blob + nk / 2, scales, nk / 32);
  return QX_OK;
}

int qx_quantize_mx4(int32_t m, int32_t k, const uint16_t* X, void* packed, hipStream_t stream) {
  if (m < 0 || k <= 0 || k % 128 != 0 || k > kMaxK) return QX_E_ARG;
  if (m == 0) return QX_OK;
  if (X == nullptr || packed == nullptr || !aligned16(X) || !aligned16(packed)) return QX_E_ARG;
  return launch_quantize_mx4(m, k, X, packed, stream);
}

int qx_gemm_a4(const qx_desc* d, const void* packed, int32_t m, const void* Xq, uint16_t* Y, hipStream_t stream) {
  const int st = check_desc(d);
  if (st != QX_OK) return st;
  if (d->kind != QX_MX4) return QX_E_UNSUPPORTED;
  if (m < 0 || m > kMaxRows) return QX_E_ARG;
  if (m == 0 || d->n == 0) return QX_OK;
  if (packed == nullptr || Xq == nullptr || Y == nullptr) return QX_E_ARG;
  if (!aligned16(packed) || !aligned16(Xq) || !aligned2(Y)) return QX_E_ARG;
  return launch_gemm_a4(d, packed, m, Xq, Y, stream);
}

int qx_gemm_grouped(const qx_desc* d, const void* packed, size_t stride, int32_t experts, int32_t m,
                    const uint16_t* X, const int32_t* offsets, uint16_t* Y, hipStream_t stream) {
  const int st = check_grouped(d, stride, experts, m);
  if (st != QX_OK) return st;
  if (m == 0 || d->n == 0 || experts == 0) return QX_OK;
  if (packed == nullptr || X == nullptr || offsets == nullptr || Y == nullptr) return QX_E_ARG;
  if (!aligned16(packed) || !aligned16(X) || !aligned4(offsets) || !aligned2(Y)) return QX_E_ARG;
  const Experts ex = {stride, experts, offsets};
  if (d->kind == QX_MX4) return launch_gemm_mx4_grouped(d, packed, ex, m, X, Y, stream);
  return launch_gemm_grouped(d, packed, ex, m, X, Y, stream);
}

int qx_gemm_a4_grouped(const qx_desc* d, const void* packed, size_t stride, int32_t experts, int32_t m,
                       const void* Xq, const int32_t* offsets, uint16_t* Y, hipStream_t stream) {
  const int st = check_grouped(d, stride, experts, m);
  if (st != QX_OK) return st;
  if (d->kind != QX_MX4) return QX_E_UNSUPPORTED;
  if (m == 0 || d->n == 0 || experts == 0) return QX_OK;
  if (packed == nullptr || Xq == nullptr || offsets == nullptr || Y == nullptr) return QX_E_ARG;
  if (!aligned16(packed) || !aligned16(Xq) || !aligned4(offsets) || !aligned2(Y)) return QX_E_ARG;
  const Experts ex = {stride, experts, offsets};
  return launch_gemm_a4_grouped(d, packed, ex, m, Xq, Y, stream);
}

}  // extern "C"
