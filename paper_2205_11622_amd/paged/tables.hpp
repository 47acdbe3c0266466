// The cache's bookkeeping: block tables and slots from the request lengths, and
// the new tokens' rows with the summaries of their pages.
#pragma once

#include "common.hpp"

namespace slnr {
namespace paged {

struct TablesArgs {
  const int32_t *ctx, *len;  // [R] cached tokens, new tokens
  int32_t *table;            // [R][W]
  int64_t table_row;
  const int32_t *free_pages;  // [F]
  int32_t *qptr, *seq;        // [R + 1], [R]
  int64_t *slots;             // [T]
  int32_t *counts;            // [3]
  int32_t R, W, F, T, shift;
};

constexpr int kTablesBlock = 256;

// One thread per new token.  Every block takes the running sums of the new tokens
// and new pages over the requests (a share of the requests per thread, then one scan
// of the block), finds its tokens' requests in them and knows each token's page:
// an old one from the table, a new one from the free list.  The token at the
// start of a new page enters it into the table: pages of the table that some block
// reads are never written in the same call.  Latency: one scan and two dependent
// loads; blocks do not wait for one another.  64 requests of one token: 3.3 us; 1024 of
// 0 to 40: 7.2 us, four requests to a thread before the scan.
__global__ __launch_bounds__(kTablesBlock) void page_tables(TablesArgs a) {
  constexpr int NT = kTablesBlock, NW = NT / kWave;
  __shared__ int begin[NT], pages[NT];
  __shared__ int wave_a[NW], wave_b[NW], wave_c[NW];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int P = 1 << a.shift;
  const int per = (a.R + NT - 1) / NT;
  const int r0 = tid * per < a.R ? tid * per : a.R, r1 = r0 + per < a.R ? r0 + per : a.R;
  // the first block counts the tokens that find no page; its look at the list is on its way early
  int listed = 0;
  if (blockIdx.x == 0 && tid < a.F) listed = a.free_pages[tid];
  auto lengths = [&](int r, int &c, int &n, int &have, int &grow) {
    c = a.ctx[r];
    n = a.len[r];
    c = c > 0 ? c : 0;
    n = n > 0 ? n : 0;
    have = (int)(((int64_t)c + P - 1) >> a.shift);
    grow = (int)(((int64_t)c + n + P - 1) >> a.shift) - have;
  };
  int tokens = 0, fresh = 0;
  for (int r = r0; r < r1; ++r) {
    int c, n, have, grow;
    lengths(r, c, n, have, grow);
    tokens += n;
    fresh += grow;
  }
  int x = tokens, y = fresh;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int px = __shfl_up(x, o), py = __shfl_up(y, o);
    if (lane >= o) x += px, y += py;
  }
  if (lane == 63) wave_a[wave] = x, wave_b[wave] = y;
  __syncthreads();
  int all = 0, taken = 0;
#pragma unroll
  for (int i = 0; i < NW; ++i) {
    if (i < wave) x += wave_a[i], y += wave_b[i];
    all += wave_a[i];
    taken += wave_b[i];
  }
  begin[tid] = x - tokens;
  pages[tid] = y - fresh;
  __syncthreads();

  // The last thread whose requests begin at or before number i of a running sum.
  auto owner = [&](const int *sum, int i) {
    int lo = 0, hi = NT - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (sum[mid] <= i)
        lo = mid;
      else
        hi = mid - 1;
    }
    return lo;
  };

  if (blockIdx.x == 0) {
    int at = x - tokens, page = y - fresh, lost = 0;
    for (int r = r0; r < r1; ++r) {
      int c, n, have, grow;
      lengths(r, c, n, have, grow);
      a.qptr[r] = at;
      a.seq[r] = c + n;
      // tokens that find no page: past the table's row or the free list, or in
      // a page that the request has given back
      const int left = a.F > page ? a.F - page : 0;
      const int64_t got = (int64_t)have + (grow < left ? grow : left);
      const int64_t room = (got < a.W ? got : a.W) << a.shift;
      const int64_t from = room > c ? room : c;
      if ((int64_t)c + n > from) lost += (int)((int64_t)c + n - from);
      if ((c & (P - 1)) && n > 0 && have <= a.W && a.table[r * a.table_row + have - 1] < 0)
        lost += n < P - (c & (P - 1)) ? n : P - (c & (P - 1));
      at += n;
      page += grow;
    }
    // entries of the list that are no pages (a list of fixed length is filled up with them)
    for (int k = tid; k < (taken < a.F ? taken : a.F); k += NT) {
      if ((k == tid ? listed : a.free_pages[k]) >= 0) continue;
      const int o = owner(pages, k);
      int first = pages[o];
      for (int r = o * per; r < a.R; ++r) {
        int c, n, have, grow;
        lengths(r, c, n, have, grow);
        if (k < first + grow) {
          const int64_t j = (int64_t)have + (k - first), end = (int64_t)c + n;  // its tokens from j P on
          if (j < a.W) lost += (int)(end - (j << a.shift) < P ? end - (j << a.shift) : P);
          break;
        }
        first += grow;
      }
    }
#pragma unroll
    for (int o = 32; o; o >>= 1) lost += __shfl_xor(lost, o);
    if (lane == 0) wave_c[wave] = lost;
    __syncthreads();
    if (tid == 0) {
      lost = 0;
#pragma unroll
      for (int i = 0; i < NW; ++i) lost += wave_c[i];
      a.qptr[a.R] = all;
      a.counts[0] = all;
      a.counts[1] = taken;
      a.counts[2] = lost;
    }
  }

  const int t = blockIdx.x * NT + tid;
  if (t >= a.T) return;
  int64_t slot = -1;
  if (t < all) {
    const int lo = owner(begin, t);
    int at = begin[lo], page = pages[lo];
    int c = 0, n = 0, have = 0, grow = 0, r = lo * per;
    for (; r < a.R; ++r) {
      lengths(r, c, n, have, grow);
      if (t < at + n) break;
      at += n;
      page += grow;
    }
    const int64_t pos = (int64_t)c + (t - at);
    const int64_t j = pos >> a.shift;
    if (r < a.R && j < a.W) {
      int32_t *row = a.table + r * a.table_row;
      int id = -1;
      if (j < have) {
        id = row[j];
      } else {
        const int64_t k = page + (j - have);
        if (k < a.F) id = a.free_pages[k];
        if ((pos & (P - 1)) == 0) row[j] = id;
      }
      if (id >= 0) slot = ((int64_t)id << a.shift) + (pos & (P - 1));
    }
  }
  a.slots[t] = slot;
}

// ----------------------------------------------------------------- new rows

struct AppendArgs {
  const void *k, *v;  // [T][Hkv][D], strides below
  int64_t k_token, k_head_in, v_token, v_head_in;
  const int64_t *slots;  // [T]
  void *kc, *vc;
  int64_t k_page, k_slot, k_head, v_page, v_slot, v_head;
  int8_t *kq;      // [pages][Hkv][D] or null
  float *kscale;   // [pages][Hkv]
  int32_t T, pages, shift, Hkv, D;
};

// A block copies the rows of `per` adjacent new tokens, of a share of the heads.  It also
// renews the summary of every page whose last new token is among them: the mean of the
// page's K rows (sum in 64 bits, rounded once, so that it does not depend on the
// order), in 8 bits with one step per head.  Rows written in this call are taken from
// the call's input, since their blocks may not have run yet, older ones from the
// cache.
//
// Latency for a decode step (the slot, a look for the page's other new rows, then all its
// rows at once), so the heads go to different blocks there; memory for a chunk, where
// more tokens a block keep the number of blocks, which start at about 3 ns each, down.
// 64 tokens, 8 heads of 128 in bf16 (4 MB with the pages' old rows): 9 us; 7868 tokens, 4
// heads of 64 in fp16 (16 MB): 16 us.
constexpr int kAppendBlock = 256;

template <class T>
__global__ __launch_bounds__(kAppendBlock) void cache_append(AppendArgs a, int per) {
  typedef typename Type<T>::Vec Vec;
  constexpr int NT = kAppendBlock;
  __shared__ double sums[8][NT];
  __shared__ unsigned most[NT];
  __shared__ int fresh_rows;
  const int tid = threadIdx.x;
  const int t0 = blockIdx.x * per, t1 = t0 + per < a.T ? t0 + per : a.T;
  const int share = (a.Hkv + gridDim.y - 1) / gridDim.y;
  const int first = blockIdx.y * share, last = first + share < a.Hkv ? first + share : a.Hkv;
  if (first >= last) return;
  const int P = 1 << a.shift;
  const int nc = a.D / 8, chunks = (last - first) * nc;
  for (int i = tid; i < (t1 - t0) * 2 * chunks; i += NT) {
    const int t = t0 + i / (2 * chunks), e = i % (2 * chunks);
    const int64_t slot = a.slots[t], page = slot >> a.shift;
    if (slot < 0 || page >= a.pages) continue;
    const int row = (int)(slot & (P - 1));
    const bool is_v = e >= chunks;
    const int c = is_v ? e - chunks : e;
    const int h = first + c / nc, d = (c % nc) * 8;
    const T *src = is_v ? (const T *)a.v + t * a.v_token + h * a.v_head_in + d
                        : (const T *)a.k + t * a.k_token + h * a.k_head_in + d;
    T *dst = is_v ? (T *)a.vc + page * a.v_page + row * a.v_slot + h * a.v_head + d
                  : (T *)a.kc + page * a.k_page + row * a.k_slot + h * a.k_head + d;
    store8<T>(dst, load8_global<T>(src));
  }
  if (!a.kq) return;

  for (int t = t0; t < t1; ++t) {
    const int64_t slot = a.slots[t], page = slot >> a.shift;
    if (slot < 0 || page >= a.pages) continue;
    const int row = (int)(slot & (P - 1));
    if (row != P - 1 && t + 1 < a.T && a.slots[t + 1] == slot + 1) continue;  // not the page's last new row
    // the page's rows up to this one that are new: the tokens before with the slots before
    if (tid == 0) fresh_rows = row + 1;
    __syncthreads();
    for (int back = 1 + tid; back <= row; back += NT)
      if (back > t || a.slots[t - back] != slot - back) {
        atomicMin(&fresh_rows, back);
        break;
      }
    __syncthreads();
    const int fresh = fresh_rows;
    const int heads = NT / nc;  // of one pass; D <= 256: at least 8
    for (int h0 = first; h0 < last; h0 += heads) {
      const int hn = last - h0 < heads ? last - h0 : heads;
      const int n = hn * nc, sides = NT / n;  // threads of a row, rows side by side
      const int c = tid % n, side = tid / n;
      const int h = h0 + c / nc, d = (c % nc) * 8;
      double s[8] = {0, 0, 0, 0, 0, 0, 0, 0};
      if (side < sides) {
        const T *old = (const T *)a.kc + page * a.k_page + h * a.k_head + d;
        const T *now = (const T *)a.k + (int64_t)(t - row) * a.k_token + h * a.k_head_in + d;  // row 0, were it new
#pragma unroll 8
        for (int i = side; i <= row; i += sides) {
          const Vec x = load8_global<T>(row - i < fresh ? now + i * a.k_token : old + i * a.k_slot);
#pragma unroll
          for (int j = 0; j < 8; ++j) s[j] += (double)(float)x[j];
        }
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) sums[j][tid] = s[j];
      if (tid < hn) most[tid] = 0;
      __syncthreads();
      // a value a thread from here on: thread e, e + NT, ... have value e of the pass
      constexpr int E = 8;  // n * 8 values, n <= NT
      float mean[E];
#pragma unroll
      for (int k = 0; k < E; ++k) {
        const int e = tid + k * NT;
        if (e < n * 8) {
          const int at = e >> 3, j = e & 7;
          double x = 0;
          for (int i = 0; i < sides; ++i) x += sums[j][i * n + at];
          mean[k] = (float)(x / (double)(row + 1));
          const float y = fabsf(mean[k]);
          atomicMax(&most[at / nc], y <= 3.402823466e38f ? __float_as_uint(y) : 0x7f800000u);
        }
      }
      __syncthreads();
#pragma unroll
      for (int k = 0; k < E; ++k) {
        const int e = tid + k * NT;
        if (e < n * 8) {
          const int hh = (e >> 3) / nc;
          const float top = __uint_as_float(most[hh]);
          // a page with infinities or NaN gets the step inf: its score is NaN, which ranks first
          const bool fine = top < __builtin_inff();
          const float step = fine ? top * kStep127 : __builtin_inff();
          const int64_t out = page * a.Hkv + h0 + hh;
          const int d = e - hh * a.D;
          a.kq[out * a.D + d] = fine && step > 0.0f ? whole8(mean[k], step) : (int8_t)0;
          if (d == 0) a.kscale[out] = step;
        }
      }
      __syncthreads();
    }
  }
}

}  // namespace paged
}  // namespace slnr
