// Launches of the attention kernels for one type.  Instantiated once per type,
// each in a translation unit of its own.
#pragma once

#include "attend.hpp"
#include "runtime.hpp"
#include "sparselnr.h"

namespace slnr {
namespace paged {

// Pieces that the work is cut into, per compute unit: what is resident at once.
constexpr int kFewPerCu = 3;
constexpr int kManyPerCu = 1;
// A request with more rows than this (tokens times heads of a group) goes to attend_many.
constexpr int kFewMostRows = 64;

struct Launch {
  int dev, cus;
  hipStream_t stream;
};

template <class F>
int launch(F *fn, dim3 grid, int block, size_t lds, const Launch &l, const AttendArgs &a) {
  hipLaunchKernelGGL(fn, grid, dim3(block), lds, l.stream, a);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? SPARSELNR_OK : hip_error(e);
}

// Partial results of `slots` pieces behind their records.
template <int ROWS, int DP>
int partials(const Launch &l, int64_t slots, AttendArgs &a) {
  const size_t head = ((size_t)(1 + slots) * kMeta * sizeof(int32_t) + 255) / 256 * 256;
  void *ws = nullptr;
  const int rc = stream_workspace(l.dev, l.stream, head + (size_t)slots * ROWS * (DP + 2) * sizeof(float), &ws,
                                  kSlotAttend);
  if (rc != SPARSELNR_OK) return rc;
  a.meta = (int32_t *)ws;
  a.part = (float *)((char *)ws + head);
  return SPARSELNR_OK;
}

template <class T, int DP, bool SPARSE>
int run_few(const Launch &l, AttendArgs a, int most_rows) {
  a.target = l.cus * kFewPerCu;
  const int64_t tiles = SPARSE ? (int64_t)a.T * ((a.G + kFewRows - 1) / kFewRows)
                               : (int64_t)a.T * a.G / kFewRows + a.R;
  const int64_t pieces = tiles * a.Hkv + a.target;
  if (pieces >= ((int64_t)1 << 31)) return SPARSELNR_ERR_UNSUPPORTED;
  const int64_t slots = 2 * (int64_t)a.target;  // of split tiles: see split_scan
  int rc = partials<kFewRows, DP>(l, slots, a);
  if (rc != SPARSELNR_OK) return rc;
  const int64_t most = (int64_t)l.cus * 8;
  const unsigned grid = (unsigned)(pieces < most ? pieces : most);
  rc = launch(attend_few<T, DP, SPARSE>, dim3(grid), kFewBlock, sizeof(FewShared<T, DP>), l, a);
  if (rc != SPARSELNR_OK) return rc;
  return launch(join_few<T, DP>, dim3((unsigned)slots, most_rows < kFewRows ? most_rows : kFewRows), kJoinBlock, 0, l,
                a);
}

template <class T, int DP, int NW, bool ONE_PAGE>
int run_many(const Launch &l, AttendArgs a) {
  constexpr int ROWS = 32 * NW;
  a.target = l.cus * kManyPerCu;
  const int64_t tiles = ((int64_t)a.T * a.G / ROWS + a.R) * a.Hkv;
  // Of split_scan: a tile of x caps makes at most x + 1 and, if it is cut, at most 2 x pieces;
  // the work is `target` caps, three tenths of it (and what a tile reaches over) of a kTailCuts-th.
  const int64_t caps = (int64_t)a.target + (int64_t)a.target * kTailCuts * 3 / 10 + kTailCuts;
  const int64_t pieces = tiles + caps;
  if (pieces >= ((int64_t)1 << 31)) return SPARSELNR_ERR_UNSUPPORTED;
  const int64_t slots = 2 * caps;
  int rc = partials<ROWS, DP>(l, slots, a);
  if (rc != SPARSELNR_OK) return rc;
  rc = launch(attend_many<T, DP, NW, ONE_PAGE>, dim3((unsigned)pieces), NW * kWave, sizeof(ManyShared<T, DP, NW>), l, a);
  if (rc != SPARSELNR_OK) return rc;
  return launch(join_many<T, DP, ROWS>, dim3((unsigned)slots, ROWS / kJoinRows), kJoinBlock, 0, l, a);
}

template <class T, int DP>
int run_attend(const Launch &l, AttendArgs a, int64_t max_new) {
  if (a.sel) return run_few<T, DP, true>(l, a, a.G < kFewRows ? a.G : kFewRows);
  // rows of the longest request, as far as the host knows
  const int64_t rows = (max_new > 0 && max_new < a.T ? max_new : a.T) * a.G;
  a.few = 0x7fffffff;
  if constexpr (!(sizeof(T) == 4 && DP > 128)) {
    if (rows > kFewMostRows) {
      constexpr int NW = sizeof(T) == 4 || DP > 128 ? 4 : 8;
      a.few = kFewMostRows;
      // a tile of keys within one page, 64 rows of it within 32 bits of bytes
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
