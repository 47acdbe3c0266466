// Entry points of the paged cache: argument checks, kernel choice and launches.
// The C ABI is declared in include/sparselnr.h.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "attend_launch.hpp"
#include "runtime.hpp"
#include "select.hpp"
#include "sparselnr.h"
#include "tables.hpp"

namespace {

using namespace slnr;
using namespace slnr::paged;

constexpr int64_t kMax31 = ((int64_t)1 << 31) - 1;
constexpr int64_t kMaxPositions = ((int64_t)1 << 31) - 4096;  // of a table's row: walks look a few tiles ahead

int value_bytes(int32_t dtype) {
  switch (dtype) {
    case SPARSELNR_BF16:
    case SPARSELNR_FP16: return 2;
    case SPARSELNR_FP32: return 4;
    default: return 0;
  }
}

// log2 of a page size, or -1.
int page_shift(int64_t page_size) {
  if (page_size < 1 || page_size > SPARSELNR_MAX_PAGE || (page_size & (page_size - 1))) return -1;
  int s = 0;
  while (((int64_t)1 << s) < page_size) ++s;
  return s;
}

bool aligned(const void *p, int64_t bytes) { return ((uintptr_t)p % (uintptr_t)bytes) == 0; }

// Rows are read 16 bytes at a time: strides that are not multiples of them are refused.
bool strides16(int bytes, int64_t a, int64_t b, int64_t c = 0) {
  return a * bytes % 16 == 0 && b * bytes % 16 == 0 && c * bytes % 16 == 0;
}

// An extent of one has no next row: its stride, which may be anything, counts as 0.
int64_t stride_of(int64_t stride, int64_t extent) { return extent > 1 ? stride : 0; }

int check_dim(int64_t dim) {
  if (dim < 0) return SPARSELNR_ERR_INVALID_ARG;
  return dim >= 8 && dim <= kMaxDim && dim % 8 == 0 ? SPARSELNR_OK : SPARSELNR_ERR_UNSUPPORTED;
}

int check_heads(int64_t Hq, int64_t Hkv) {
  if (Hq < 1 || Hkv < 1 || Hq % Hkv) return SPARSELNR_ERR_INVALID_ARG;
  return Hq <= 65535 ? SPARSELNR_OK : SPARSELNR_ERR_UNSUPPORTED;
}

// `out` is the cache with strides that count.
int check_cache(const sparselnr_kv_cache *c, sparselnr_kv_cache *out) {
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

int check_requests(const sparselnr_requests *r, int64_t page_size) {
  if (!r || r->R < 0 || r->W < 0 || r->T < 0 || r->table_stride < 0) return SPARSELNR_ERR_INVALID_ARG;
  if (r->R > 0 && (!r->seq_len || !r->qptr || (r->W > 0 && !r->table))) return SPARSELNR_ERR_INVALID_ARG;
  if (r->R > 1 && r->table_stride < r->W) return SPARSELNR_ERR_INVALID_ARG;
  if (r->R >= ((int64_t)1 << 24) || r->T >= ((int64_t)1 << 28)) return SPARSELNR_ERR_UNSUPPORTED;
  if (page_size > 0 && r->W > kMaxPositions / page_size) return SPARSELNR_ERR_UNSUPPORTED;
  return SPARSELNR_OK;
}

int current(Launch *l, void *stream) {
  int rc = this_device(&l->dev);
  if (rc != SPARSELNR_OK) return rc;
  if ((rc = device_cu_count(l->dev, &l->cus)) != SPARSELNR_OK) return rc;
  l->stream = (hipStream_t)stream;
  return SPARSELNR_OK;
}

int launched() {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? SPARSELNR_OK : hip_error(e);
}

// Common part of the two attention calls.
int attend(const void *q, int64_t q_token, int64_t q_head, int64_t Hq, const sparselnr_kv_cache *cache,
           const sparselnr_requests *r, const int32_t *sel, int64_t top, double scale, int64_t window, int64_t max_new,
           void *out, float *lse, void *stream) {
  sparselnr_kv_cache kv;
  int rc = check_cache(cache, &kv);
  if (rc != SPARSELNR_OK) return rc;
  const sparselnr_kv_cache *c = &kv;
  if ((rc = check_requests(r, c->page_size)) != SPARSELNR_OK) return rc;
  if ((rc = check_heads(Hq, c->heads)) != SPARSELNR_OK) return rc;
  if (q_token < 0 || q_head < 0 || window < 0 || max_new < 0 || !(scale > 0) || !std::isfinite(scale))
    return SPARSELNR_ERR_INVALID_ARG;
  const float scale2 = (float)(scale * 1.4426950408889634);
  if (!(scale2 > 0) || !std::isfinite(scale2)) return SPARSELNR_ERR_INVALID_ARG;
  if (r->T > 0 && r->R > 0 && (!q || !out)) return SPARSELNR_ERR_INVALID_ARG;
  const int e = value_bytes(c->dtype);
  q_token = stride_of(q_token, r->T), q_head = stride_of(q_head, Hq);
  if (!aligned(q, 16) || !aligned(out, 16) || !strides16(e, q_token, q_head)) return SPARSELNR_ERR_UNSUPPORTED;
  if (r->T * Hq > kMax31) return SPARSELNR_ERR_UNSUPPORTED;
  if (r->T == 0 || r->R == 0) return SPARSELNR_OK;
  AttendArgs a{};
  a.q = q;
  a.q_token = q_token;
  a.q_head = q_head;
  a.k = c->k;
  a.v = c->v;
  a.k_page = c->k_page, a.k_slot = c->k_slot, a.k_head = c->k_head;
  a.v_page = c->v_page, a.v_slot = c->v_slot, a.v_head = c->v_head;
  a.table = r->table;
  a.table_row = r->table_stride;
  a.seq = r->seq_len;
  a.qptr = r->qptr;
  a.sel = sel;
  a.out = out;
  a.lse = lse;
  a.R = (int32_t)r->R, a.T = (int32_t)r->T, a.W = (int32_t)r->W;
  a.pages = (int32_t)c->pages;
  a.shift = page_shift(c->page_size);
  a.Hq = (int32_t)Hq, a.Hkv = (int32_t)c->heads, a.G = (int32_t)(Hq / c->heads), a.D = (int32_t)c->dim;
  a.top = (int32_t)top;
  a.window = window < (r->W << a.shift) ? (int32_t)window : 0;  // 0, or wider than any request: all keys
  a.scale2 = scale2;
  Launch l;
  if ((rc = current(&l, stream)) != SPARSELNR_OK) return rc;
  switch (c->dtype) {
    case SPARSELNR_BF16: return attend_bf16(l, a, max_new);
    case SPARSELNR_FP16: return attend_fp16(l, a, max_new);
    default: return attend_fp32(l, a, max_new);
  }
}

// A block starts at about 3 ns after the one before, and the one with a page's last new row
// reads the page: about two blocks a unit, of up to 16 tokens, or of a share of the
// heads where the tokens are few (tokens a block x shares, 8 heads of 128 in bf16; 1024
// tokens: 8 x 4 9.9 us, 1 x 1 19, 8 x 1 17; 8192: 16 x 1 34, 8 x 1 35, 16 x 4 39, 4 x 1 50;
// 64: 1 x 8 8.7, 1 x 1 10.4, 8 x 1 31).
template <class T>
int run_append(const Launch &l, const AppendArgs &a) {
  int64_t per = a.T / (l.cus / 2 > 0 ? l.cus / 2 : 1);
  per = per < 1 ? 1 : per > 16 ? 16 : per;
  const int64_t least = (a.T + grid_limit(kAppendBlock) - 1) / grid_limit(kAppendBlock);
  per = per < least ? least : per;
  int64_t shares = 2 * (int64_t)l.cus / ((a.T + per - 1) / per);
  shares = shares < 1 ? 1 : shares > a.Hkv ? a.Hkv : shares;
  hipLaunchKernelGGL(cache_append<T>, dim3((unsigned)((a.T + per - 1) / per), (unsigned)shares), dim3(kAppendBlock), 0,
                     l.stream, a, (int)per);
  return launched();
}

// ------------------------------------------------------------ selection

template <class T, int DP, int TM, int NR>
int run_select(const Launch &l, SelectArgs a, int64_t Hkv) {
  constexpr int most = NR * kWave * (kSelectWaves / TM);
  // pages of the longest request, and the carried entries in front, if they fit
  const int64_t pages = ((int64_t)a.W + 15) / 16 * 16;
  const int64_t want = (pages < 2 * kWave ? 2 * kWave : pages) + a.top;
  // A multiple of four words: so is then the row's stride, and what lies behind the rows, the 8-bit
  // queries among it, begins at a multiple of the 16 bytes that it is read in.
  static_assert(most % 4 == 0, "a full row keeps the alignment");
  a.capacity = (int32_t)(want < most ? (want + 3) / 4 * 4 : most);
  const size_t lds = (size_t)TM * (a.capacity + 4) * 4 + ((size_t)TM * a.top + 3) / 4 * 16 + 16 * (DP + 16) +
                     2 * kSelectWaves * 4 + (TM == 1 ? kSelectWaves * 4 * kWave * 4 : 0);
  const int64_t tiles = TM == 1 ? (int64_t)a.T : (int64_t)a.T / TM + a.R;
  const int64_t once = grid_limit(kSelectBlock);
  for (int64_t first = 0; first < tiles; first += once) {  // one launch, but for millions of tiles
    a.tile0 = (int32_t)first;
    const unsigned n = (unsigned)(tiles - first < once ? tiles - first : once);
    hipLaunchKernelGGL((block_select<T, DP, TM, NR>), dim3(n, (unsigned)Hkv), dim3(kSelectBlock), lds, l.stream, a);
    const int rc = launched();
    if (rc != SPARSELNR_OK) return rc;
  }
  return SPARSELNR_OK;
}

template <class T, int DP>
int select_rows(const Launch &l, const SelectArgs &a, int64_t Hkv) {
  const int64_t entries = (int64_t)a.W + 16 + a.top;
  // Fewer than three tokens a request on average, or no more blocks than compute units: a block
  // per token; otherwise 16 tokens share a page's summary.  64 requests behind 30000 tokens in pages
  // of 64, 8 heads: of 1 token 25 us (16 to a block: 56), of 2 47 (53), of 3 69 (59), of 4 91 (53);
  // 8 requests of 4 behind 200000 37 (83), 4 of 16 behind 30000 42 (22).
  if ((int64_t)a.T < 3 * (int64_t)a.R || (int64_t)a.T * Hkv <= l.cus) {
    if (entries <= 4 * kSelectBlock) return run_select<T, DP, 1, 4>(l, a, Hkv);
    return run_select<T, DP, 1, 16>(l, a, Hkv);
  }
  if (entries <= 8 * kWave) return run_select<T, DP, 16, 8>(l, a, Hkv);
  if (entries <= 16 * kWave) return run_select<T, DP, 16, 16>(l, a, Hkv);
  return run_select<T, DP, 16, 32>(l, a, Hkv);
}

template <class T>
int select_type(const Launch &l, const SelectArgs &a, int64_t Hkv) {
  if (a.D <= 64) return select_rows<T, 64>(l, a, Hkv);
  if (a.D <= 128) return select_rows<T, 128>(l, a, Hkv);
  return select_rows<T, 256>(l, a, Hkv);
}

}  // namespace

extern "C" {

int sparselnr_page_tables(const int32_t *ctx_len, const int32_t *new_len, int32_t *table, int64_t table_stride,
                          const int32_t *free_pages, int32_t *qptr, int32_t *seq_len, int64_t *slots, int32_t *counts,
                          int64_t R, int64_t W, int64_t F, int64_t T, int64_t page_size, void *stream) {
  if (R < 0 || W < 0 || F < 0 || T < 0 || table_stride < 0) return SPARSELNR_ERR_INVALID_ARG;
  if (!qptr || !counts || (R > 0 && (!ctx_len || !new_len || !seq_len)) || (R > 0 && W > 0 && !table) ||
      (F > 0 && !free_pages) || (T > 0 && !slots) || (R > 1 && table_stride < W))
    return SPARSELNR_ERR_INVALID_ARG;
  const int shift = page_shift(page_size);
  if (shift < 0 || R >= ((int64_t)1 << 24) || T >= ((int64_t)1 << 28) || F > kMax31 || W > kMaxPositions / page_size)
    return SPARSELNR_ERR_UNSUPPORTED;
  TablesArgs a{};
  a.ctx = ctx_len;
  a.len = new_len;
  a.table = table;
  a.table_row = table_stride;
  a.free_pages = free_pages;
  a.qptr = qptr;
  a.seq = seq_len;
  a.slots = slots;
  a.counts = counts;
  a.R = (int32_t)R, a.W = (int32_t)W, a.F = (int32_t)F, a.T = (int32_t)T;
  a.shift = shift;
  int64_t blocks = (T + kTablesBlock - 1) / kTablesBlock;
  if (blocks < 1) blocks = 1;
  hipLaunchKernelGGL(page_tables, dim3((unsigned)blocks), dim3(kTablesBlock), 0, (hipStream_t)stream, a);
  return launched();
}

int sparselnr_cache_append(const void *k, int64_t k_token, int64_t k_head, const void *v, int64_t v_token,
                           int64_t v_head, const int64_t *slots, const sparselnr_kv_cache *cache, int8_t *kq,
                           float *kscale, int64_t T, void *stream) {
  sparselnr_kv_cache kv;
  int rc = check_cache(cache, &kv);
  if (rc != SPARSELNR_OK) return rc;
  if (T < 0 || k_token < 0 || k_head < 0 || v_token < 0 || v_head < 0) return SPARSELNR_ERR_INVALID_ARG;
  if (T > 0 && (!k || !v || !slots)) return SPARSELNR_ERR_INVALID_ARG;
  if ((kq == nullptr) != (kscale == nullptr)) return SPARSELNR_ERR_INVALID_ARG;
  const int e = value_bytes(kv.dtype);
  k_token = stride_of(k_token, T), v_token = stride_of(v_token, T);
  k_head = stride_of(k_head, kv.heads), v_head = stride_of(v_head, kv.heads);
  if (!aligned(k, 16) || !aligned(v, 16) || !aligned(kq, 8) || !strides16(e, k_token, k_head) ||
      !strides16(e, v_token, v_head))
    return SPARSELNR_ERR_UNSUPPORTED;
  if (T >= ((int64_t)1 << 28)) return SPARSELNR_ERR_UNSUPPORTED;
  if (T == 0 || kv.pages == 0) return SPARSELNR_OK;
  AppendArgs a{};
  a.k = k, a.k_token = k_token, a.k_head_in = k_head;
  a.v = v, a.v_token = v_token, a.v_head_in = v_head;
  a.slots = slots;
  a.kc = kv.k, a.vc = kv.v;
  a.k_page = kv.k_page, a.k_slot = kv.k_slot, a.k_head = kv.k_head;
  a.v_page = kv.v_page, a.v_slot = kv.v_slot, a.v_head = kv.v_head;
  a.kq = kq, a.kscale = kscale;
  a.T = (int32_t)T, a.pages = (int32_t)kv.pages, a.shift = page_shift(kv.page_size);
  a.Hkv = (int32_t)kv.heads, a.D = (int32_t)kv.dim;
  Launch l;
  if ((rc = current(&l, stream)) != SPARSELNR_OK) return rc;
  switch (kv.dtype) {
    case SPARSELNR_BF16: return run_append<__bf16>(l, a);
    case SPARSELNR_FP16: return run_append<_Float16>(l, a);
    default: return run_append<float>(l, a);
  }
}

int sparselnr_paged_attention(const void *q, int64_t q_token, int64_t q_head, int64_t Hq,
                              const sparselnr_kv_cache *cache, const sparselnr_requests *requests, double scale,
                              int64_t window, int64_t max_new, void *out, float *lse, void *stream) {
  return attend(q, q_token, q_head, Hq, cache, requests, nullptr, 0, scale, window, max_new, out, lse, stream);
}

int sparselnr_block_select(const void *q, int64_t q_token, int64_t q_head, int64_t Hq, int32_t dtype,
                           const int8_t *kq, const float *kscale, int64_t pages, int64_t page_size, int64_t Hkv,
                           int64_t dim, const sparselnr_requests *r, int64_t top, int64_t first, int64_t local,
                           int32_t *sel, void *stream) {
  const int e = value_bytes(dtype);
  if (!e || pages < 0 || top < 1 || first < 0 || local < 0 || q_token < 0 || q_head < 0)
    return SPARSELNR_ERR_INVALID_ARG;
  if (first > top || local > top || first + local > top) return SPARSELNR_ERR_INVALID_ARG;
  int rc = check_heads(Hq, Hkv);
  if (rc != SPARSELNR_OK) return rc;
  if ((rc = check_dim(dim)) != SPARSELNR_OK) return rc;
  if (page_shift(page_size) < 0) return SPARSELNR_ERR_UNSUPPORTED;
  if ((rc = check_requests(r, page_size)) != SPARSELNR_OK) return rc;
  if (pages > 0 && (!kq || !kscale)) return SPARSELNR_ERR_INVALID_ARG;
  if (r->T > 0 && r->R > 0 && (!q || !sel)) return SPARSELNR_ERR_INVALID_ARG;
  // a score's whole number stays exact in 32-bit floating point for any dim that check_dim admits
  if (top > kSelectMaxTop || pages > kMax31 || !aligned(kq, 8) || r->T * Hq > kMax31) return SPARSELNR_ERR_UNSUPPORTED;
  if (r->T == 0 || r->R == 0) return SPARSELNR_OK;
  SelectArgs a{};
  a.q = q, a.q_token = q_token, a.q_head = q_head;
  a.kq = kq, a.kscale = kscale;
  a.table = r->table, a.table_row = r->table_stride;
  a.seq = r->seq_len, a.qptr = r->qptr;
  a.sel = sel;
  a.R = (int32_t)r->R, a.T = (int32_t)r->T, a.W = (int32_t)r->W, a.pages = (int32_t)pages;
  a.shift = page_shift(page_size);
  a.Hkv = (int32_t)Hkv, a.G = (int32_t)(Hq / Hkv), a.D = (int32_t)dim;
  a.top = (int32_t)top, a.first = (int32_t)first, a.local = (int32_t)local;
  Launch l;
  if ((rc = current(&l, stream)) != SPARSELNR_OK) return rc;
  switch (dtype) {
    case SPARSELNR_BF16: return select_type<__bf16>(l, a, Hkv);
    case SPARSELNR_FP16: return select_type<_Float16>(l, a, Hkv);
    default: return select_type<float>(l, a, Hkv);
  }
}

int sparselnr_block_attention(const void *q, int64_t q_token, int64_t q_head, int64_t Hq,
                              const sparselnr_kv_cache *cache, const sparselnr_requests *requests, const int32_t *sel,
                              int64_t top, double scale, void *out, float *lse, void *stream) {
  if (top < 1) return SPARSELNR_ERR_INVALID_ARG;
  if (requests && requests->T > 0 && requests->R > 0 && !sel) return SPARSELNR_ERR_INVALID_ARG;
  if (cache && cache->page_size > 0 && top > (kMax31 / 4) / cache->page_size) return SPARSELNR_ERR_UNSUPPORTED;
  return attend(q, q_token, q_head, Hq, cache, requests, sel, top, scale, 0, 0, out, lse, stream);
}

}  // extern "C"
