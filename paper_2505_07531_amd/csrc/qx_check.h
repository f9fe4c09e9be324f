// Argument checks shared by the C entry points.
#pragma once

#include "qx_internal.h"

namespace qx {

constexpr int kMaxK = 1 << 20;
constexpr int kMaxRows = 65536;
constexpr int kMaxExperts = 1024;

// Well-formed: the fields make sense. Supported: a kernel instance exists.
inline int check_desc(const qx_desc* d) {
  if (d == nullptr) return QX_E_ARG;
  if (d->flags != 0 || d->n < 0 || d->k <= 0 || d->k % 128 != 0 || d->k > kMaxK) return QX_E_ARG;
  if (d->kind != QX_UNIFORM && d->kind != QX_CODEBOOK && d->kind != QX_Q4X && d->kind != QX_MX4) return QX_E_ARG;
  if (d->kind == QX_Q4X && (d->bits != 4 || d->group != 64)) return QX_E_ARG;  // fixed by the format
  if (d->kind == QX_MX4 && (d->bits != 4 || d->group != 32)) return QX_E_ARG;
  if (d->bits < 1 || d->bits > 8 || d->group <= 0 || d->k % d->group != 0) return QX_E_ARG;
  if (d->bits != 3 && d->bits != 4) return QX_E_UNSUPPORTED;
  if (d->group != 32 && d->group != 64 && d->group != 128) return QX_E_UNSUPPORTED;
  return QX_OK;
}

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }
inline bool aligned2(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 1u) == 0; }

inline size_t meta_bytes_per_group(const qx_desc* d) {
  return d->kind == QX_UNIFORM ? 4 : d->kind == QX_MX4 ? 1 : 2u * (1u << d->bits);
}

inline size_t packed_bytes(const qx_desc* d) {
  if (d->kind == QX_Q4X) return q4x_offsets(d->n, d->k).total;
  const size_t n = (size_t)d->n, k = (size_t)d->k;
  return n * k * d->bits / 8 + n * (k / d->group) * meta_bytes_per_group(d);
}

}  // namespace qx
