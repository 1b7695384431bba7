// Argument checks shared by the C entry points.
#pragma once

#include <initializer_list>

#include "../../include/omnimoe.h"
#include "internal.hpp"

namespace omnimoe {

constexpr int64_t kIntMax = 2147483647LL;

inline size_t align_up(size_t v) { return (v + 255) & ~(size_t)255; }

inline bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }

inline omnimoe_status check_desc(const omnimoe_layer_desc* d, Shape* s) {
  if (!d) return OMNIMOE_ERR_INVALID_ARG;
  if (d->T < 0 || d->T > (1LL << 23)) return OMNIMOE_ERR_INVALID_ARG;
  if (d->d < 8 || d->d > kMaxWidth || d->d % 8) return OMNIMOE_ERR_INVALID_ARG;
  if (d->n_rows < 1 || d->n_rows > 4096 || d->n_cols < 1 || d->n_cols > 4096)
    return OMNIMOE_ERR_INVALID_ARG;
  if (d->d_key < 8 || d->d_key % 8) return OMNIMOE_ERR_INVALID_ARG;
  if (d->query_mode == OMNIMOE_QUERY_SPLIT) {
    if (2LL * d->d_key > d->d) return OMNIMOE_ERR_INVALID_ARG;
  } else if (d->query_mode == OMNIMOE_QUERY_SHARED) {
    if (d->d_key > d->d) return OMNIMOE_ERR_INVALID_ARG;
  } else {
    return OMNIMOE_ERR_INVALID_ARG;
  }
  if (d->H < 1 || d->K < 1) return OMNIMOE_ERR_INVALID_ARG;
  const int64_t N = (int64_t)d->n_rows * d->n_cols;
  if (d->K > N) return OMNIMOE_ERR_INVALID_ARG;
  if (d->K > 4096) return OMNIMOE_ERR_UNSUPPORTED;
  if (d->dtype != OMNIMOE_F32 && d->dtype != OMNIMOE_BF16) return OMNIMOE_ERR_INVALID_ARG;
  if (d->dtype == OMNIMOE_F32 && d->d > kMaxWidthF32) return OMNIMOE_ERR_UNSUPPORTED;
  if (d->act != OMNIMOE_ACT_GELU && d->act != OMNIMOE_ACT_SILU) return OMNIMOE_ERR_INVALID_ARG;
  if (d->group_size < 1) return OMNIMOE_ERR_INVALID_ARG;
  const int64_t rows = d->T * d->H;
  if (rows * d->K >= kIntMax || rows * (d->n_rows + d->n_cols) >= kIntMax)
    return OMNIMOE_ERR_INVALID_ARG;
  s->T = d->T;
  s->d = d->d;
  s->nr = d->n_rows;
  s->nc = d->n_cols;
  s->dk = d->d_key;
  s->H = d->H;
  s->K = d->K;
  s->bf16 = d->dtype == OMNIMOE_BF16;
  s->act = d->act;
  s->col0 = d->query_mode == OMNIMOE_QUERY_SPLIT ? d->d_key : 0;
  s->N = N;
  s->rows = rows;
  s->M = rows * d->K;
  s->hk = d->H * d->K;
  s->B = d->group_size;
  return OMNIMOE_OK;
}

inline omnimoe_status check_ptrs(std::initializer_list<const void*> ps) {
  for (const void* p : ps) {
    if (!p) return OMNIMOE_ERR_INVALID_ARG;
    if (!aligned16(p)) return OMNIMOE_ERR_ALIGNMENT;
  }
  return OMNIMOE_OK;
}

inline omnimoe_status check_opt(const void* p) {
  return (p && !aligned16(p)) ? OMNIMOE_ERR_ALIGNMENT : OMNIMOE_OK;
}

inline omnimoe_status hip_status(hipError_t e) { return e == hipSuccess ? OMNIMOE_OK : OMNIMOE_ERR_HIP; }

// Widths of the shared branch: rows of whole 16-byte chunks.
inline bool valid_d_ff(int32_t d_ff) { return d_ff >= 8 && d_ff <= kMaxFeatures && d_ff % 8 == 0; }

}  // namespace omnimoe
