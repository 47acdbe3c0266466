// Entry points of the cache in 4 bits: argument checks and launches.  The C ABI is declared in
// include/sparselnr.h.
#include <cmath>

#include "attend_fp4_launch.hpp"
#include "checks.hpp"

namespace {

using namespace slnr;
using namespace slnr::paged;

// `out` is the cache with strides that count.
int check_fp4_cache(const sparselnr_fp4_cache *c, sparselnr_fp4_cache *out) {
  if (!c || c->pages < 0 || c->heads < 1 || !value_bytes(c->dtype)) return SPARSELNR_ERR_INVALID_ARG;
  if (c->pages > 0 && (!c->k || !c->v || !c->k_scale || !c->v_scale)) return SPARSELNR_ERR_INVALID_ARG;
  const int64_t strides[] = {c->k_page,  c->k_slot,  c->k_head,  c->v_page,  c->v_slot,  c->v_head,
                             c->ks_page, c->ks_slot, c->ks_head, c->vs_page, c->vs_slot, c->vs_head};
  for (const int64_t s : strides)
    if (s < 0) return SPARSELNR_ERR_INVALID_ARG;
  const int rc = check_dim(c->dim);
  if (rc != SPARSELNR_OK) return rc;
  if (page_shift(c->page_size) < 0 || c->pages > kMax31 || c->heads > 65535) return SPARSELNR_ERR_UNSUPPORTED;
  *out = *c;
  out->k_page = stride_of(c->k_page, c->pages), out->v_page = stride_of(c->v_page, c->pages);
  out->k_slot = stride_of(c->k_slot, c->page_size), out->v_slot = stride_of(c->v_slot, c->page_size);
  out->k_head = stride_of(c->k_head, c->heads), out->v_head = stride_of(c->v_head, c->heads);
  out->ks_page = stride_of(c->ks_page, c->pages), out->vs_page = stride_of(c->vs_page, c->pages);
  out->ks_slot = stride_of(c->ks_slot, c->page_size), out->vs_slot = stride_of(c->vs_slot, c->page_size);
  out->ks_head = stride_of(c->ks_head, c->heads), out->vs_head = stride_of(c->vs_head, c->heads);
  if (!aligned(c->k, 16) || !aligned(c->v, 16) || !strides16(1, out->k_page, out->k_slot, out->k_head) ||
      !strides16(1, out->v_page, out->v_slot, out->v_head))
    return SPARSELNR_ERR_UNSUPPORTED;
  return SPARSELNR_OK;
}

Fp4Args rows_args(const sparselnr_fp4_cache &c, const int64_t *slots, int64_t T) {
  Fp4Args a{};
  a.slots = slots;
  a.kc = (uint8_t *)c.k, a.vc = (uint8_t *)c.v, a.ks = (uint8_t *)c.k_scale, a.vs = (uint8_t *)c.v_scale;
  a.k_page = c.k_page, a.k_slot = c.k_slot, a.k_head = c.k_head;
  a.v_page = c.v_page, a.v_slot = c.v_slot, a.v_head = c.v_head;
  a.ks_page = c.ks_page, a.ks_slot = c.ks_slot, a.ks_head = c.ks_head;
  a.vs_page = c.vs_page, a.vs_slot = c.vs_slot, a.vs_head = c.vs_head;
  a.T = (int32_t)T, a.pages = (int32_t)c.pages, a.shift = page_shift(c.page_size);
  a.Hkv = (int32_t)c.heads, a.D = (int32_t)c.dim;
  return a;
}

// `lanes` lanes a token; a block more than the units hold at once waits for nothing.
unsigned rows_grid(const Launch &l, int64_t T, int64_t lanes) {
  const int64_t blocks = (T * lanes + kFp4Block - 1) / kFp4Block, most = (int64_t)l.cus * 32;
  return (unsigned)(blocks < most ? blocks : most);
}

}  // namespace

extern "C" {

int sparselnr_cache_append_fp4(const void *k, int64_t k_token, int64_t k_head, const void *v, int64_t v_token,
                               int64_t v_head, const int64_t *slots, const sparselnr_fp4_cache *cache, int64_t T,
                               void *stream) {
  sparselnr_fp4_cache c;
  int rc = check_fp4_cache(cache, &c);
  if (rc != SPARSELNR_OK) return rc;
  if (T < 0 || k_token < 0 || k_head < 0 || v_token < 0 || v_head < 0) return SPARSELNR_ERR_INVALID_ARG;
  if (T > 0 && (!k || !v || !slots)) return SPARSELNR_ERR_INVALID_ARG;
  const int e = value_bytes(c.dtype);
  k_token = stride_of(k_token, T), v_token = stride_of(v_token, T);
  k_head = stride_of(k_head, c.heads), v_head = stride_of(v_head, c.heads);
  if (!aligned(k, 16) || !aligned(v, 16) || !strides16(e, k_token, k_head) || !strides16(e, v_token, v_head))
    return SPARSELNR_ERR_UNSUPPORTED;
  if (T >= ((int64_t)1 << 28)) return SPARSELNR_ERR_UNSUPPORTED;
  if (T == 0 || c.pages == 0) return SPARSELNR_OK;
  Fp4Args a = rows_args(c, slots, T);
  a.k = k, a.k_token = k_token, a.k_head_in = k_head;
  a.v = v, a.v_token = v_token, a.v_head_in = v_head;
  Launch l;
  if ((rc = current(&l, stream)) != SPARSELNR_OK) return rc;
  const dim3 grid(rows_grid(l, T, 2 * c.heads * ((c.dim + kGroup - 1) / kGroup) * 4)), block(kFp4Block);
  switch (c.dtype) {
    case SPARSELNR_BF16: hipLaunchKernelGGL(fp4_append<__bf16>, grid, block, 0, l.stream, a); break;
    case SPARSELNR_FP16: hipLaunchKernelGGL(fp4_append<_Float16>, grid, block, 0, l.stream, a); break;
    default: hipLaunchKernelGGL(fp4_append<float>, grid, block, 0, l.stream, a);
  }
  return launched();
}

int sparselnr_cache_read_fp4(const int64_t *slots, const sparselnr_fp4_cache *cache, void *k, void *v, int64_t T,
                             void *stream) {
  sparselnr_fp4_cache c;
  int rc = check_fp4_cache(cache, &c);
  if (rc != SPARSELNR_OK) return rc;
  if (T < 0 || (T > 0 && (!k || !v || !slots))) return SPARSELNR_ERR_INVALID_ARG;
  if (!aligned(k, 16) || !aligned(v, 16) || T >= ((int64_t)1 << 28)) return SPARSELNR_ERR_UNSUPPORTED;
  if (T == 0) return SPARSELNR_OK;
  Fp4Args a = rows_args(c, slots, T);
  a.k = k, a.v = v;
  Launch l;
  if ((rc = current(&l, stream)) != SPARSELNR_OK) return rc;
  const dim3 grid(rows_grid(l, T, 2 * c.heads * c.dim / 8)), block(kFp4Block);
  switch (c.dtype) {
    case SPARSELNR_BF16: hipLaunchKernelGGL(fp4_read<__bf16>, grid, block, 0, l.stream, a); break;
    case SPARSELNR_FP16: hipLaunchKernelGGL(fp4_read<_Float16>, grid, block, 0, l.stream, a); break;
    default: hipLaunchKernelGGL(fp4_read<float>, grid, block, 0, l.stream, a);
  }
  return launched();
}

int sparselnr_paged_attention_fp4(const void *q, int64_t q_token, int64_t q_head, int64_t Hq,
                                  const sparselnr_fp4_cache *cache, const sparselnr_requests *r, double scale,
                                  int64_t window, int64_t max_new, void *out, float *lse, void *stream) {
  sparselnr_fp4_cache c;
  int rc = check_fp4_cache(cache, &c);
  if (rc != SPARSELNR_OK) return rc;
  if ((rc = check_requests(r, c.page_size)) != SPARSELNR_OK) return rc;
  AttendFp4Args a{};
  bool work = false;
  rc = check_query(q, &q_token, &q_head, Hq, c.heads, c.dtype, r, scale, window, max_new, out, &a.scale2, &work);
  if (rc != SPARSELNR_OK || !work) return rc;
  a.q = q;
  a.q_token = q_token;
  a.q_head = q_head;
  a.k = c.k, a.v = c.v;
  a.ks = (const uint8_t *)c.k_scale, a.vs = (const uint8_t *)c.v_scale;
  a.k_page = c.k_page, a.k_slot = c.k_slot, a.k_head = c.k_head;
  a.v_page = c.v_page, a.v_slot = c.v_slot, a.v_head = c.v_head;
  a.ks_page = c.ks_page, a.ks_slot = c.ks_slot, a.ks_head = c.ks_head;
  a.vs_page = c.vs_page, a.vs_slot = c.vs_slot, a.vs_head = c.vs_head;
  a.table = r->table;
  a.table_row = r->table_stride;
  a.seq = r->seq_len;
  a.qptr = r->qptr;
  a.out = out;
  a.lse = lse;
  a.R = (int32_t)r->R, a.T = (int32_t)r->T, a.W = (int32_t)r->W;
  a.pages = (int32_t)c.pages;
  a.shift = page_shift(c.page_size);
  a.Hq = (int32_t)Hq, a.Hkv = (int32_t)c.heads, a.G = (int32_t)(Hq / c.heads), a.D = (int32_t)c.dim;
  a.groups = (a.D + kGroup - 1) / kGroup;
  a.window = window < (r->W << a.shift) ? (int32_t)window : 0;  // 0, or wider than any request: all keys
  Launch l;
  if ((rc = current(&l, stream)) != SPARSELNR_OK) return rc;
  switch (c.dtype) {
    case SPARSELNR_BF16: return attend_fp4_bf16(l, a, max_new);
    case SPARSELNR_FP16: return attend_fp4_fp16(l, a, max_new);
    default: return attend_fp4_fp32(l, a, max_new);
  }
}

}  // extern "C"
