// Launches of the attention kernels over a cache in 4 bits, for one type.
#pragma once

#include "attend_fp4.hpp"
#include "launch.hpp"

namespace slnr {
namespace paged {

// A request with more rows than this goes to attend_many_fp4.  Time in us of few | many, bf16, 8 query heads to each of 4
// KV heads: 32 requests behind 8000 keys, 48 rows each: 74 | 112 at dim 64, 94 | 126 at 128, 189 | 196 at 256; 64 rows:
// 70 | 109, 89 | 125, 232 | 199; 128 rows: 128 | 114, 172 | 135, 461 | 213.  4 requests behind 3000, 64 rows: 27 | 36,
// 31 | 44, 32 | 58.  fp32: 83 | 169, 116 | 240 and 290 | 411 for the 32 of 64 rows.
constexpr int kFew4MostRows = 64;
// Waves of a block of attend_many_fp4: two to a SIMD, one where a wave takes the registers of two (O of 256 columns, the
// three pieces of fp32 at 128).  8 | 4 waves, 500 tokens of each of 2 requests behind 6000 keys: bf16 119 | 155 us at dim 64,
// 139 | 175 at 128; fp32 172 | 222 at 64, 429 (43 to 74 registers in memory) | 315 at 128.
template <class T, int DP>
constexpr int kMany4Waves = DP > 128 || (sizeof(T) == 4 && DP > 64) ? 4 : 8;

template <class F>
int launch_fp4(F *fn, dim3 grid, int block, size_t lds, const Launch &l, const AttendFp4Args &a) {
  hipLaunchKernelGGL(fn, grid, dim3(block), lds, l.stream, a);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? SPARSELNR_OK : hip_error(e);
}

template <class T, int DP, bool ONE_PAGE>
int run_few_fp4(const Launch &l, AttendFp4Args a, int most_rows) {
  // as many blocks as there is room for, the same for each KV head
  static_assert(kFew4PerCu<T, DP> <= kFewPerCu && kFewRows * (DP + 2) <= kFewValues, "fits the workspace");
  const int64_t room = (int64_t)l.cus * kFew4PerCu<T, DP>;
  const int64_t n = room / a.Hkv > 0 ? room / a.Hkv : 1;
  HeldWorkspace ws;
  int rc = partials(l, few_slots(room > a.Hkv ? room : a.Hkv), a, &ws);
  if (rc != SPARSELNR_OK) return rc;
  rc = launch_fp4(attend_few_fp4<T, DP, ONE_PAGE>, dim3((unsigned)(n * a.Hkv)), kFewBlock, sizeof(Few4Shared<T, DP>), l, a);
  if (rc != SPARSELNR_OK || n == 1) return rc;
  return launch(join_few_fp4<T, DP>, dim3((unsigned)(n * a.Hkv), (unsigned)(most_rows < kFewRows ? most_rows : kFewRows)),
                kJoinBlock, 0, l, a);
}

template <class T, int DP, bool ONE_PAGE, int NQ>
int run_many_fp4(const Launch &l, AttendFp4Args a) {
  constexpr int NW = kMany4Waves<T, DP>, ROWS = 32 * NW;
  a.target = l.cus * kManyPerCu;
  const int64_t tiles = ((int64_t)a.T * a.G / ROWS + (a.R < a.T ? a.R : a.T)) * a.Hkv;
  static_assert(ROWS * (DP + 2) <= kManyValues, "fits the workspace");
  const int64_t pieces = tiles + many_caps(a.target), most = grid_limit(NW * kWave);
  HeldWorkspace ws;
  int rc = partials(l, many_slots(a.target), a, &ws);
  if (rc != SPARSELNR_OK) return rc;
  rc = launch_fp4(attend_many_fp4<T, DP, NW, ONE_PAGE, NQ>, dim3((unsigned)(pieces < most ? pieces : most)), NW * kWave,
                  sizeof(Many4SharedOf<T, DP, NW>), l, a);
  if (rc != SPARSELNR_OK) return rc;
  a.scale2 = 1.0f;  // its maxima are exponents of two already
  return launch(join_many<T, DP, ROWS>, dim3((unsigned)l.cus, ROWS / kJoinRows), kJoinBlock, 0, l, a);
}

template <class T, int DP, bool ONE_PAGE>
int run_attend_fp4(const Launch &l, AttendFp4Args a, int64_t max_new) {
  // rows of the longest request, as far as the host knows
  const int64_t rows = (max_new > 0 && max_new < a.T ? max_new : a.T) * a.G;
  a.few = 0x7fffffff;
  if (rows > kFew4MostRows) {
    a.few = kFew4MostRows;
    // A fourth piece of a bf16 query, for lse: the chunk of 4010 tokens 579 us, with it 642.  fp16 has it always (2 of 2000 tokens
    // behind 9000, 32/8 heads of 128, by three 567 us, by four 619), and so have few rows: 96 single tokens 127.6 and 127.9 us.
    const int rc = a.lse ? run_many_fp4<T, DP, ONE_PAGE, Four<T>::kQ>(l, a)
                         : run_many_fp4<T, DP, ONE_PAGE, Four<T>::kQOut>(l, a);
    if (rc != SPARSELNR_OK) return rc;
  }
  return run_few_fp4<T, DP, ONE_PAGE>(l, a, rows < kFewRows ? (int)rows : kFewRows);
}

template <class T, int DP>
int attend_fp4_width(const Launch &l, const AttendFp4Args &a, int64_t max_new) {
  // a tile of 64 keys within one page, the page's bytes and the pages' strides within 32 bits: then a tile has one entry
  // of the table and scalar addresses (96 single tokens: 129 us, by entries and addresses of each key 142; the chunk of 4010 tokens 613 and 647)
  const int64_t row = 1 << 19, page = (int64_t)1 << 32;
  const bool one_page = a.shift >= 6 && a.k_slot < row && a.v_slot < row && a.ks_slot < row && a.vs_slot < row &&
                        a.k_page < page && a.v_page < page && a.ks_page < page && a.vs_page < page;
  return one_page ? run_attend_fp4<T, DP, true>(l, a, max_new) : run_attend_fp4<T, DP, false>(l, a, max_new);
}

template <class T>
int attend_fp4_type(const Launch &l, const AttendFp4Args &a, int64_t max_new) {
  if (a.D <= 64) return attend_fp4_width<T, 64>(l, a, max_new);
  if (a.D <= 128) return attend_fp4_width<T, 128>(l, a, max_new);
  return attend_fp4_width<T, 256>(l, a, max_new);
}

int attend_fp4_bf16(const Launch &l, const AttendFp4Args &a, int64_t max_new);
int attend_fp4_fp16(const Launch &l, const AttendFp4Args &a, int64_t max_new);
int attend_fp4_fp32(const Launch &l, const AttendFp4Args &a, int64_t max_new);

}  // namespace paged
}  // namespace slnr
