// Launches of the attention kernels for one type.  Instantiated once per type,
// each in a translation unit of its own.
#pragma once

#include "attend.hpp"
#include "pages.hpp"
#include "runtime.hpp"
#include "sparselnr.h"

namespace slnr {
namespace paged {

// Pieces that the work is cut into, per compute unit.  Two blocks of attend_few are resident
// on one.  Pieces of a selection are all alike, so they go in one round (32 tokens over 32
// pages of 64: 69 us; at 3 a unit 87, at 4 77); contexts are ragged, and shorter pieces
// even them out (64 of 513 to 15096 keys: 259 us; at 2 a unit 291, at 4 262).  A block of attend_many fills a unit: at 2
// pieces a unit 2 of 2000 tokens behind 7000 738 us (at 1 706), 1 of 512 behind 8000 179 (133), 16 of 64 behind 4000 197
// (134), 64 of 1 to 200 behind up to 4000 417 (418).
constexpr int kFewPerCu = 3;
constexpr int kFewPerCuSparse = 2;
constexpr int kManyPerCu = 1;
// A request with more rows than this (tokens times heads of a group) goes to attend_many.
// 64 requests of 4000 keys and 32 rows, 8 heads of 128 in bf16: 292 us as few rows, 382 as many;
// of 48: 410 and 385, of 128: 1046 and 413.  256 columns cross there too; 64 columns in fp16 at
// 64 rows (111 and 118; 48: 81 and 116; 128: 171 and 123), fp32 behind them (128 columns, 64 rows:
// 396 and 478; 128: 700 and 490).
template <class T, int DP>
constexpr int kFewMostRows = sizeof(T) == 2 && DP > 64 ? 32 : 64;

struct Launch {
  int dev, cus;
  hipStream_t stream;
};

// A launch has fewer than 2^32 threads a dimension.
constexpr int64_t grid_limit(int block) { return (((int64_t)1 << 32) - 1) / block; }

template <class F>
int launch(F *fn, dim3 grid, int block, size_t lds, const Launch &l, const AttendArgs &a) {
  hipLaunchKernelGGL(fn, grid, dim3(block), lds, l.stream, a);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? SPARSELNR_OK : hip_error(e);
}

// Slots of split tiles that cutting the work into about `target` pieces takes (see split_scan):
// a tile of x caps makes at most x + 1 pieces and, if it is cut, at most 2 x.
constexpr int64_t few_slots(int64_t target) { return 2 * target; }
// With a tail: the work is `target` caps, three tenths of it (and what a tile reaches over) of
// a kTailCuts-th.
constexpr int64_t many_caps(int64_t target) { return target + target * kTailCuts * 3 / 10 + kTailCuts; }
constexpr int64_t many_slots(int64_t target) { return 2 * many_caps(target); }

// Partial results of `slots` pieces of `values` numbers, behind their records.
constexpr size_t records_bytes(int64_t slots) {
  return ((size_t)(1 + slots) * kMeta * sizeof(int32_t) + 255) / 256 * 256;
}
constexpr size_t partials_bytes(int64_t slots, int64_t values) {
  return records_bytes(slots) + (size_t)slots * values * sizeof(float);
}

// The workspace has one size for all calls on a device, the largest need there is (130 MB on 256
// units): a captured graph holds its address, so no later call of other tokens, heads, hint,
// type or dim may be one that has to grow it.
constexpr int64_t kFewValues = kFewRows * (kMaxDim + 2);
constexpr int64_t kManyValues = 256 * (128 + 2);  // eight waves of 32 rows up to 128 columns, four up to 256
inline size_t attend_bytes(int cus) {
  const size_t few = partials_bytes(few_slots((int64_t)cus * kFewPerCu), kFewValues);
  const size_t many = partials_bytes(many_slots((int64_t)cus * kManyPerCu), kManyValues);
  return few > many ? few : many;
}

inline int partials(const Launch &l, int64_t slots, AttendArgs &a, HeldWorkspace *ws) {
  const int rc = hold_workspace(l.dev, l.stream, attend_bytes(l.cus), kSlotAttend, ws);
  if (rc != SPARSELNR_OK) return rc;
  a.meta = (int32_t *)ws->ptr;
  a.part = (float *)((char *)ws->ptr + records_bytes(slots));
  return SPARSELNR_OK;
}

template <class T, int DP, bool SPARSE>
int run_few(const Launch &l, AttendArgs a, int most_rows) {
  a.target = l.cus * (SPARSE ? kFewPerCuSparse : kFewPerCu);
  const int64_t requests = a.R < a.T ? a.R : a.T;  // that have tokens, at most
  int64_t tiles = SPARSE ? (int64_t)a.T * ((a.G + kFewRows - 1) / kFewRows) : (int64_t)a.T * a.G / kFewRows + requests;
  // Beside attend_many: only what is left of a request has tiles here, often nothing, and
  // a grid for more costs its launch.
  const int64_t left = requests * ((kFewMostRows<T, DP> + kFewRows - 1) / kFewRows);
  if (!SPARSE && a.few <= kFewMostRows<T, DP> && tiles > left) tiles = left;
  const int64_t pieces = tiles * a.Hkv + a.target;
  static_assert(kFewRows * (DP + 2) <= kFewValues && kFewPerCuSparse <= kFewPerCu, "fits the workspace");
  const int64_t slots = few_slots(a.target);
  HeldWorkspace ws;
  int rc = partials(l, slots, a, &ws);
  if (rc != SPARSELNR_OK) return rc;
  const int64_t most = (int64_t)l.cus * 8;
  const unsigned grid = (unsigned)(pieces < most ? pieces : most);
  rc = launch(attend_few<T, DP, SPARSE>, dim3(grid), kFewBlock, sizeof(FewShared<T, DP>), l, a);
  if (rc != SPARSELNR_OK) return rc;
  const unsigned side = most_rows < kFewRows ? most_rows : kFewRows;  // about 8000 blocks in all
  return launch(join_few<T, DP>, dim3((unsigned)(slots < 8192 / side ? slots : 8192 / side), side), kJoinBlock, 0, l, a);
}

template <class T, int DP, int NW, bool ONE_PAGE>
int run_many(const Launch &l, AttendArgs a) {
  constexpr int ROWS = 32 * NW;
  a.target = l.cus * kManyPerCu;
  const int64_t tiles = ((int64_t)a.T * a.G / ROWS + (a.R < a.T ? a.R : a.T)) * a.Hkv;
  static_assert(ROWS * (DP + 2) <= kManyValues, "fits the workspace");
  const int64_t pieces = tiles + many_caps(a.target), most = grid_limit(NW * kWave);
  HeldWorkspace ws;
  int rc = partials(l, many_slots(a.target), a, &ws);
  if (rc != SPARSELNR_OK) return rc;
  rc = launch(attend_many<T, DP, NW, ONE_PAGE>, dim3((unsigned)(pieces < most ? pieces : most)), NW * kWave, sizeof(ManyShared<T, DP, NW>), l, a);
  if (rc != SPARSELNR_OK) return rc;
  return launch(join_many<T, DP, ROWS>, dim3((unsigned)l.cus, ROWS / kJoinRows), kJoinBlock, 0, l, a);
}

// Partial results of by_pages, at most (a call that has more is worked off by KV heads, then
// by tokens): little enough that the join finds much of them in the 256 MB cache.  us at 144 MB / at 80 / at 288, of 507 MB: 2000
// tokens over 16 of 1400 pages, 8 heads 392 / 453 / 411; 4000 over 8 of 400 381 / 416 / 409; 4000 over 16 of 1000, 2 heads
// 342 / 439 / 375; 1000 over 16, 256 columns 521 / 659 / 536; 1024 over 32 of 256 359 / 400 / 412.
constexpr int64_t kPagesWorkspace = (int64_t)144 << 20;

// By pages (pages.hpp) rather than by queries: where a page is selected by four queries and
// more on average, its keys are at least four times the heads of a group (the results
// of a page are then at most half of what is gathered by queries), and 256 MB and more are
// gathered, which take longer than the four small launches before and the join.  us by queries / by pages, 8 heads of
// 128 in bf16, 16 pages a query:
// * queries a page (pages of 64, groups of 4): 1 45 / 84, 2 85 / 108, 4 163 / 140 (of 1024 pages) and 43 / 48 (of 256), 8
//   82 / 52, 16 155 / 67;
// * keys of a page to heads (512 tokens, 256 pages): 16 to 8 92 / 165, 32 to 16 164 / 314; 16 to 4 90 / 97, 32 to 8 160 / 168, 64
//   to 16 304 / 323; 32 to 4 158 / 98, 64 to 8 302 / 173;
// * MB gathered (16 queries a page and more): 128 30 / 32, 256 43 / 38, 512 79 / 45.
// Not where one token's entries pass the lists' numbers, or its partial results of one KV head (`dp` columns)
// what is kept of them.
inline bool by_pages(const AttendArgs &a, int64_t bytes, int64_t dp) {
  const int64_t picks = (int64_t)a.T * a.top;
  return a.W > 0 && picks >= 4 * (int64_t)a.R * a.W && ((int64_t)1 << a.shift) >= 4 * (int64_t)a.G &&
         (double)picks * a.Hkv * (1 << a.shift) * a.D * 2 * bytes >= (double)((int64_t)256 << 20) &&
         (int64_t)a.R * a.W * a.Hkv < ((int64_t)1 << 30) && a.G <= kPagesRows &&
         (int64_t)a.Hkv * a.top < ((int64_t)1 << 30) &&
         (int64_t)a.top * a.G * (dp + 2) * (int64_t)sizeof(float) <= kPagesWorkspace;
}

template <class T, int DP>
int run_pages(const Launch &l, const AttendArgs &a) {
  PagesArgs p{};
  const int64_t per_token = (int64_t)a.Hkv * a.top;  // selected pages
  const int64_t bytes = (int64_t)a.top * a.G * (DP + 2) * sizeof(float);  // partial results of a token, per KV head
  int64_t most = kPagesWorkspace / bytes;
  most = most > a.T ? a.T : most;
  if (most * per_token >= ((int64_t)1 << 30)) most = (((int64_t)1 << 30) - 1) / per_token;
  int64_t heads = kPagesWorkspace / (most * bytes);  // of a launch
  heads = heads > a.Hkv ? a.Hkv : heads;
  const int64_t rows = most * heads * a.top * a.G;  // of partial results
  p.buckets = a.Hkv * a.R * a.W;
  p.per_tile = kPagesRows / a.G;
  const int64_t picks = most * per_token, tiles = picks / p.per_tile + p.buckets;
  size_t size = 0;
  auto take = [&](size_t bytes) {
    const size_t at = size;
    size += (bytes + 255) / 256 * 256;
    return at;
  };
  const size_t count = take((size_t)p.buckets * 4), begin = take((size_t)p.buckets * 4),
               tile_begin = take((size_t)p.buckets * 4), total = take(4), rank = take((size_t)picks * 4),
               list = take((size_t)picks * 4), tile = take((size_t)tiles * 4),
               part = take((size_t)rows * DP * 4), ml = take((size_t)rows * 8);
  HeldWorkspace ws;
  int rc = hold_workspace(l.dev, l.stream, size, kSlotPages, &ws);
  if (rc != SPARSELNR_OK) return rc;
  auto at = [&](size_t offset) { return (int32_t *)((char *)ws.ptr + offset); };
  p.count = at(count), p.begin = at(begin), p.tile_begin = at(tile_begin), p.total = at(total), p.rank = at(rank);
  p.list = at(list), p.tile = at(tile), p.part = (float *)at(part), p.ml = (float *)at(ml);
  auto done = [&]() {
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? SPARSELNR_OK : hip_error(e);
  };
  for (int64_t t0 = 0; t0 < a.T; t0 += most) {
    p.t0 = (int32_t)t0;
    p.tokens = (int32_t)(a.T - t0 < most ? a.T - t0 : most);
    const int64_t n = p.tokens * per_token;
    const dim3 block(kPagesBlock), each((unsigned)((n + kPagesBlock - 1) / kPagesBlock));
    hipLaunchKernelGGL(pages_clear, dim3((unsigned)((p.buckets + kPagesBlock - 1) / kPagesBlock)), block, 0, l.stream, p);
    hipLaunchKernelGGL(pages_count, each, block, 0, l.stream, a, p);
    hipLaunchKernelGGL(pages_scan, dim3(1), dim3(kScanBlock), 0, l.stream, p);
    hipLaunchKernelGGL(pages_fill, each, block, 0, l.stream, a, p);
    if ((rc = done()) != SPARSELNR_OK) return rc;
    for (p.h0 = 0; p.h0 < a.Hkv; p.h0 += p.heads) {
      p.heads = heads < a.Hkv - p.h0 ? (int)heads : a.Hkv - p.h0;
      // a page makes at most one tile more than its queries fill, and none without queries
      const int64_t m = (int64_t)p.tokens * p.heads * a.top, b = (int64_t)p.heads * a.R * a.W;
      hipLaunchKernelGGL((attend_pages<T, DP>), dim3((unsigned)(m / p.per_tile + (m < b ? m : b))), block,
                         sizeof(PagesShared<T, DP>), l.stream, a, p);
      if ((rc = done()) != SPARSELNR_OK) return rc;
      const int64_t out = (int64_t)p.tokens * p.heads * a.G;
      hipLaunchKernelGGL((join_pages<T, DP>), dim3((unsigned)((out + 3) / 4)), block, 0, l.stream, a, p);
      if ((rc = done()) != SPARSELNR_OK) return rc;
    }
  }
  return SPARSELNR_OK;
}

template <class T, int DP>
int run_attend(const Launch &l, AttendArgs a, int64_t max_new) {
  if (a.sel) {
    if (by_pages(a, sizeof(T), DP)) return run_pages<T, DP>(l, a);
    return run_few<T, DP, true>(l, a, a.G < kFewRows ? a.G : kFewRows);
  }
  // rows of the longest request, as far as the host knows
  const int64_t rows = (max_new > 0 && max_new < a.T ? max_new : a.T) * a.G;
  a.few = 0x7fffffff;
  if constexpr (!(sizeof(T) == 4 && DP > 128)) {
    if (rows > kFewMostRows<T, DP>) {
      constexpr int NW = sizeof(T) == 4 || DP > 128 ? 4 : 8;
      a.few = kFewMostRows<T, DP>;
      // a tile of keys within one page, 64 rows of it within 32 bits of bytes (4073 tokens
      // behind 6818 and 7894: 706 us, 741 without)
      const bool one_page = a.shift >= 6 && a.k_slot < (1 << 23) && a.v_slot < (1 << 23);
      const int rc = one_page ? run_many<T, DP, NW, true>(l, a) : run_many<T, DP, NW, false>(l, a);
      if (rc != SPARSELNR_OK) return rc;
    }
  }
  return run_few<T, DP, false>(l, a, rows < kFewRows ? (int)rows : kFewRows);
}

template <class T>
int attend_type(const Launch &l, const AttendArgs &a, int64_t max_new) {
  if (a.D <= 64) return run_attend<T, 64>(l, a, max_new);
  if (a.D <= 128) return run_attend<T, 128>(l, a, max_new);
  return run_attend<T, 256>(l, a, max_new);
}

int attend_bf16(const Launch &l, const AttendArgs &a, int64_t max_new);
int attend_fp16(const Launch &l, const AttendArgs &a, int64_t max_new);
int attend_fp32(const Launch &l, const AttendArgs &a, int64_t max_new);

}  // namespace paged
}  // namespace slnr
