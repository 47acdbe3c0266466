// Checks of arguments that the entry points of the paged cache share; none makes a HIP call before
// all of them have passed.
#pragma once

#include <cmath>

#include "launch.hpp"

namespace slnr {
namespace paged {

constexpr int64_t kMax31 = ((int64_t)1 << 31) - 1;
constexpr int64_t kMaxPositions = ((int64_t)1 << 31) - 4096;  // of a table's row: walks look a few tiles ahead

inline int value_bytes(int32_t dtype) {
  switch (dtype) {
    case SPARSELNR_BF16:
    case SPARSELNR_FP16: return 2;
    case SPARSELNR_FP32: return 4;
    default: return 0;
  }
}

// log2 of a page size, or -1.
inline int page_shift(int64_t page_size) {
  if (page_size < 1 || page_size > SPARSELNR_MAX_PAGE || (page_size & (page_size - 1))) return -1;
  int s = 0;
  while (((int64_t)1 << s) < page_size) ++s;
  return s;
}

inline bool aligned(const void *p, int64_t bytes) { return ((uintptr_t)p % (uintptr_t)bytes) == 0; }

// Rows are read 16 bytes at a time: strides that are not multiples of them are refused.
inline bool strides16(int bytes, int64_t a, int64_t b, int64_t c = 0) {
  return a * bytes % 16 == 0 && b * bytes % 16 == 0 && c * bytes % 16 == 0;
}

// An extent of one has no next row: its stride, which may be anything, counts as 0.
inline int64_t stride_of(int64_t stride, int64_t extent) { return extent > 1 ? stride : 0; }

inline int check_dim(int64_t dim) {
  if (dim < 0) return SPARSELNR_ERR_INVALID_ARG;
  return dim >= 8 && dim <= kMaxDim && dim % 8 == 0 ? SPARSELNR_OK : SPARSELNR_ERR_UNSUPPORTED;
}

inline int check_heads(int64_t Hq, int64_t Hkv) {
  if (Hq < 1 || Hkv < 1 || Hq % Hkv) return SPARSELNR_ERR_INVALID_ARG;
  return Hq <= 65535 ? SPARSELNR_OK : SPARSELNR_ERR_UNSUPPORTED;
}

// `out` is the cache with strides that count.
inline int check_cache(const sparselnr_kv_cache *c, sparselnr_kv_cache *out) {
  if (!c || c->pages < 0 || c->heads < 1) return SPARSELNR_ERR_INVALID_ARG;
  const int e = value_bytes(c->dtype);
  if (!e) return SPARSELNR_ERR_INVALID_ARG;
  if (c->k_page < 0 || c->k_slot < 0 || c->k_head < 0 || c->v_page < 0 || c->v_slot < 0 || c->v_head < 0)
    return SPARSELNR_ERR_INVALID_ARG;
  if (c->pages > 0 && (!c->k || !c->v)) return SPARSELNR_ERR_INVALID_ARG;
  const int rc = check_dim(c->dim);
  if (rc != SPARSELNR_OK) return rc;
  if (page_shift(c->page_size) < 0 || c->pages > kMax31 || c->heads > 65535) return SPARSELNR_ERR_UNSUPPORTED;
  *out = *c;
  out->k_page = stride_of(c->k_page, c->pages), out->v_page = stride_of(c->v_page, c->pages);
  out->k_slot = stride_of(c->k_slot, c->page_size), out->v_slot = stride_of(c->v_slot, c->page_size);
  out->k_head = stride_of(c->k_head, c->heads), out->v_head = stride_of(c->v_head, c->heads);
  if (!aligned(c->k, 16) || !aligned(c->v, 16) || !strides16(e, out->k_page, out->k_slot, out->k_head) ||
      !strides16(e, out->v_page, out->v_slot, out->v_head))
    return SPARSELNR_ERR_UNSUPPORTED;
  return SPARSELNR_OK;
}

inline int check_requests(const sparselnr_requests *r, int64_t page_size) {
  if (!r || r->R < 0 || r->W < 0 || r->T < 0 || r->table_stride < 0) return SPARSELNR_ERR_INVALID_ARG;
  if (r->R > 0 && (!r->seq_len || !r->qptr || (r->W > 0 && !r->table))) return SPARSELNR_ERR_INVALID_ARG;
  if (r->R > 1 && r->table_stride < r->W) return SPARSELNR_ERR_INVALID_ARG;
  if (r->R >= ((int64_t)1 << 24) || r->T >= ((int64_t)1 << 28)) return SPARSELNR_ERR_UNSUPPORTED;
  if (page_size > 0 && r->W > kMaxPositions / page_size) return SPARSELNR_ERR_UNSUPPORTED;
  return SPARSELNR_OK;
}

// What the attention calls check of queries and result; strides become those that count.  `work`: there are tokens.
inline int check_query(const void *q, int64_t *q_token, int64_t *q_head, int64_t Hq, int64_t Hkv, int32_t dtype,
                       const sparselnr_requests *r, double scale, int64_t window, int64_t max_new, const void *out,
                       float *scale2, bool *work) {
  const int rc = check_heads(Hq, Hkv);
  if (rc != SPARSELNR_OK) return rc;
  if (*q_token < 0 || *q_head < 0 || window < 0 || max_new < 0 || !(scale > 0) || !std::isfinite(scale))
    return SPARSELNR_ERR_INVALID_ARG;
  *scale2 = (float)(scale * 1.4426950408889634);
  if (!(*scale2 > 0) || !std::isfinite(*scale2)) return SPARSELNR_ERR_INVALID_ARG;
  if (r->T > 0 && r->R > 0 && (!q || !out)) return SPARSELNR_ERR_INVALID_ARG;
  *q_token = stride_of(*q_token, r->T), *q_head = stride_of(*q_head, Hq);
  if (!aligned(q, 16) || !aligned(out, 16) || !strides16(value_bytes(dtype), *q_token, *q_head))
    return SPARSELNR_ERR_UNSUPPORTED;
  if (r->T * Hq > kMax31) return SPARSELNR_ERR_UNSUPPORTED;
  *work = r->T > 0 && r->R > 0;
  return SPARSELNR_OK;
}

inline int current(Launch *l, void *stream) {
  int rc = this_device(&l->dev);
  if (rc != SPARSELNR_OK) return rc;
  if ((rc = device_cu_count(l->dev, &l->cus)) != SPARSELNR_OK) return rc;
  l->stream = (hipStream_t)stream;
  return SPARSELNR_OK;
}

inline int launched() {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? SPARSELNR_OK : hip_error(e);
}

}  // namespace paged
}  // namespace slnr
