// What becomes of the cache's pages: rows of the block table that share pages with others, rows
// given up, pages moved to the front of the cache, and the copies that go with it.
//
// shares[p] counts the rows that hold page p beyond the first: 0 for a page of one row and
// for a free one, so that page_tables, which knows no shares, leaves them right.
#pragma once

#include "attend.hpp"

namespace slnr {
namespace paged {

constexpr int kLifeBlock = 256;

struct ForkArgs {
  const int32_t *parents, *children;  // [n]
  int32_t *table;                     // [R][W]
  int64_t table_row;
  int32_t *seq, *shares;              // [R], [pages]
  const int32_t *free_pages;          // [F]
  int32_t *pairs, *counts;            // [n][2], [2]
  int32_t n, R, W, F, pages, shift;
};

__device__ __forceinline__ bool is_page(int page, int pages) { return (unsigned)page < (unsigned)pages; }

// A row's length, as far as its table goes.
__device__ __forceinline__ int row_length(const int32_t *seq, int r, int W, int shift) {
  const int64_t room = (int64_t)W << shift;
  const int s = imax(seq[r], 0);
  return s < room ? s : (int)room;
}

struct Fork {
  int parent, child, length, last;  // child < 0: left out; last: the page that is not full, or -1
};

__device__ __forceinline__ Fork fork_of(const ForkArgs &a, int i) {
  Fork f{a.parents[i], a.children[i], 0, -1};
  if ((unsigned)f.parent >= (unsigned)a.R || (unsigned)f.child >= (unsigned)a.R || f.parent == f.child) {
    f.child = -1;
    return f;
  }
  f.length = row_length(a.seq, f.parent, a.W, a.shift);
  if (f.length & ((1 << a.shift) - 1)) {
    const int page = a.table[f.parent * a.table_row + (f.length >> a.shift)];
    if (is_page(page, a.pages)) f.last = page;
  }
  return f;
}

template <class I>
__device__ __forceinline__ I block_sum(I x, I *shared) {
#pragma unroll
  for (int o = 32; o; o >>= 1) x += __shfl_xor(x, o);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6] = x;
  __syncthreads();
  x = 0;
#pragma unroll
  for (int w = 0; w < kLifeBlock / kWave; ++w) x += shared[w];
  return x;
}

// A block takes `per` adjacent forks, and along y a part of each row.  It counts the pages that the forks before them take from the
// list by itself, so blocks do not wait for one another; then it copies one parent's row
// after the other.  Latency: a parent, its length, its last page, its row, in turn; 12 forks 4.5 us, 256 of
// rows of up to 138 pages 5.8.
__global__ __launch_bounds__(kLifeBlock) void page_fork(ForkArgs a, int per) {
  __shared__ int sums[kLifeBlock / kWave];
  const int tid = threadIdx.x, P = 1 << a.shift;
  const int first = blockIdx.x * per, last = imin(first + per, a.n);
  int taken = 0;
  for (int i = tid; i < first; i += kLifeBlock) taken += fork_of(a, i).last >= 0;
  taken = block_sum(taken, sums);
  for (int i = first; i < last; ++i) {
    const Fork f = fork_of(a, i);
    int fresh = -1;
    if (f.last >= 0) {
      if (taken < a.F) fresh = a.free_pages[taken];
      if (!is_page(fresh, a.pages)) fresh = -1;
      ++taken;
    }
    if (tid == 0 && blockIdx.y == 0) {
      a.pairs[2 * (int64_t)i] = fresh < 0 ? -1 : f.last;
      a.pairs[2 * (int64_t)i + 1] = fresh;
    }
    if (f.child < 0) continue;
    const int32_t *from = a.table + f.parent * a.table_row;
    int32_t *to = a.table + f.child * a.table_row;
    const unsigned full = f.length >> a.shift;
    const bool part = f.length & (P - 1);
    // without sign: a row of nearly 2^31 entries, and a step of up to 8192 behind it
    for (unsigned j = blockIdx.y * kLifeBlock + tid; j < (unsigned)a.W; j += gridDim.y * kLifeBlock) {
      int page = -1;
      if (j < full) {
        page = from[j];
        if (is_page(page, a.pages))
          atomicAdd(a.shares + page, 1);
        else
          page = -1;
      } else if (part && j == full) {
        page = fresh;
      }
      to[j] = page;
    }
    if (tid == 0 && blockIdx.y == 0) a.seq[f.child] = f.length;
  }
  if (blockIdx.x == gridDim.x - 1 && blockIdx.y == 0) {  // it has counted them all
    int lost = 0;
    for (int k = tid; k < taken; k += kLifeBlock) lost += k >= a.F || !is_page(a.free_pages[k], a.pages);
    lost = block_sum(lost, sums);
    if (tid == 0) a.counts[0] = taken, a.counts[1] = lost;
  }
}

// -------------------------------------------------------------- sets of pages
//
// Rows given up and rows in use mark pages in a bitmap, which is then gone through in the order of the pages: that
// order, and not the one in which blocks ran, is the order of what the calls hand out.

typedef unsigned long long Word;  // 64 pages

struct LifeArgs {
  const int32_t *rows;  // [n] (free)
  int32_t *table;       // [R][W]
  int64_t table_row;
  int32_t *seq, *shares;  // [R], [pages]
  int32_t *out, *counts;  // freed pages [most], or pairs [most][2]; counts [2]
  Word *marks;            // [words]
  int32_t *before;        // [words] (compact): marked pages before a word's
  int32_t *given;         // [blocks] (free): entries that a block of page_free_rows gave up
  int64_t words;
  int32_t n, R, W, pages, shift, most;
};

__global__ __launch_bounds__(kLifeBlock) void life_clear(LifeArgs a, int64_t outs) {
  const int64_t i0 = (int64_t)blockIdx.x * kLifeBlock + threadIdx.x, step = (int64_t)gridDim.x * kLifeBlock;
  for (int64_t i = i0; i < a.words; i += step) a.marks[i] = 0;
  for (int64_t i = i0; i < outs; i += step) a.out[i] = -1;
}

__device__ __forceinline__ void mark(Word *marks, int page) { atomicOr(marks + (page >> 6), (Word)1 << (page & 63)); }

__device__ __forceinline__ int pages_held(const LifeArgs &a, int r) {
  return (int)(((int64_t)row_length(a.seq, r, a.W, a.shift) + (1 << a.shift) - 1) >> a.shift);
}

// Takes an entry by an exchange, so a row named twice is given up once: was it a page?  The page is marked if no
// row is left that holds it.
template <class M>
__device__ __forceinline__ bool give_up(const LifeArgs &a, int r, int j, M mark_it) {
  const int page = atomicExch(a.table + r * a.table_row + j, -1);
  if (!is_page(page, a.pages)) return false;
  if (atomicSub(a.shares + page, 1) <= 0) mark_it(page);
  return true;
}

// Blocks take rows along x and their entries along y, and each writes down what it gave up.  14 us over 700 rows of
// up to 512 pages, 121796 pages in all: 5 of them are the shares' atomics, 5 the marks'; without either 4.
__global__ __launch_bounds__(kLifeBlock) void page_free_rows(LifeArgs a) {
  __shared__ int sums[kLifeBlock / kWave];
  int given = 0;
  for (int i = blockIdx.x; i < a.n; i += gridDim.x) {
    const int r = a.rows[i];
    if ((unsigned)r >= (unsigned)a.R) continue;
    const int held = pages_held(a, r);
    for (int j = blockIdx.y * kLifeBlock + threadIdx.x; j < held; j += gridDim.y * kLifeBlock)
      given += give_up(a, r, j, [&](int page) { mark(a.marks, page); });
  }
  given = block_sum(given, sums);
  if (threadIdx.x == 0) a.given[blockIdx.y * gridDim.x + blockIdx.x] = given;
}

__global__ __launch_bounds__(kLifeBlock) void page_mark_used(LifeArgs a) {
  for (int r = blockIdx.x; r < a.R; r += gridDim.x) {
    const int held = pages_held(a, r);
    for (int j = blockIdx.y * kLifeBlock + threadIdx.x; j < held; j += gridDim.y * kLifeBlock) {
      const int page = a.table[r * a.table_row + j];
      if (is_page(page, a.pages)) mark(a.marks, page);
    }
  }
}

// How many of the pages below `end` are marked, counted by the whole block with eight loads on their way: 200 rows of up
// to 480 of 4 million pages given up in 35 us, compacted in 52 (one load at a time: 101, 114).
__device__ __forceinline__ int marked_below(const LifeArgs &a, int64_t end, int *sums) {
  int x = 0;
#pragma unroll 8
  for (int64_t i = threadIdx.x; i < (end >> 6); i += kLifeBlock) x += __popcll(a.marks[i]);
  if (threadIdx.x == 0 && (end & 63)) x += __popcll(a.marks[end >> 6] & (((Word)1 << (end & 63)) - 1));
  return block_sum(x, sums);
}

// Goes through the marks of a block's share of the words: visit(page, marked, marked pages before it).  A thread
// takes a word and counts what lies before it, then a wave takes the words in turn, a lane a page.
template <class F>
__device__ __forceinline__ void for_pages(const LifeArgs &a, int64_t w0, int64_t w1, int before, F visit) {
  __shared__ Word words[kLifeBlock];
  __shared__ int starts[kLifeBlock], sums[kLifeBlock / kWave];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  for (int64_t w = w0; w < w1; w += kLifeBlock) {
    const int n = (int)(w1 - w < kLifeBlock ? w1 - w : kLifeBlock);
    const Word bits = tid < n ? a.marks[w + tid] : 0;
    int upto = __popcll(bits);
    const int mine = upto;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int x = __shfl_up(upto, o);
      if (lane >= o) upto += x;
    }
    if (lane == 63) sums[wave] = upto;
    __syncthreads();
    int all = 0;
#pragma unroll
    for (int k = 0; k < kLifeBlock / kWave; ++k) {
      if (k < wave) upto += sums[k];
      all += sums[k];
    }
    words[tid] = bits;
    starts[tid] = before + upto - mine;
    __syncthreads();
    for (int k = wave; k < n; k += kLifeBlock / kWave) {
      const Word b = words[k];
      const int64_t page = (w + k) * 64 + lane;
      if (page < a.pages) visit((int)page, (bool)((b >> lane) & 1), starts[k] + __popcll(b & (((Word)1 << lane) - 1)));
    }
    before += all;
    __syncthreads();
  }
}

// Words of a block: all blocks together take them all.
__device__ __forceinline__ void share_of(const LifeArgs &a, int64_t *w0, int64_t *w1) {
  const int64_t per = (a.words + gridDim.x - 1) / gridDim.x;
  *w0 = blockIdx.x * per < a.words ? blockIdx.x * per : a.words;
  *w1 = *w0 + per < a.words ? *w0 + per : a.words;
}

__global__ __launch_bounds__(kLifeBlock) void page_free_list(LifeArgs a, int blocks) {
  __shared__ int sums[kLifeBlock / kWave];
  int64_t w0, w1;
  share_of(a, &w0, &w1);
  const int before = marked_below(a, w0 * 64, sums);
  for_pages(a, w0, w1, before, [&](int page, bool marked, int rank) {
    if (!marked) return;
    a.shares[page] = 0;
    if (rank < a.most) a.out[rank] = page;
  });
  for (int i = blockIdx.x * kLifeBlock + threadIdx.x; i < a.n; i += gridDim.x * kLifeBlock) {
    const int r = a.rows[i];
    if ((unsigned)r < (unsigned)a.R) a.seq[r] = 0;
  }
  if (blockIdx.x == gridDim.x - 1) {
    __shared__ long long totals[kLifeBlock / kWave];
    const int all = marked_below(a, a.pages, sums);
    long long given = 0;  // tables have room for more than 2^31 entries
    for (int i = threadIdx.x; i < blocks; i += kLifeBlock) given += a.given[i];
    given = block_sum(given, totals);
    if (threadIdx.x == 0) a.counts[0] = all, a.counts[1] = given < 0x7fffffff ? (int)given : 0x7fffffff;
  }
}

// The k-th page in use at or behind the place where they would all end goes to the k-th
// hole before it.  5 us for 5500 pages, the scans first.
__global__ __launch_bounds__(kLifeBlock) void page_compact_pairs(LifeArgs a) {
  __shared__ int sums[kLifeBlock / kWave];
  int64_t w0, w1;
  share_of(a, &w0, &w1);
  const int used = marked_below(a, a.pages, sums), stay = marked_below(a, used, sums);
  const int before = marked_below(a, w0 * 64, sums);
  for_pages(a, w0, w1, before, [&](int page, bool marked, int rank) {
    if (marked && page >= used)
      a.out[2 * (int64_t)(rank - stay)] = page;
    else if (!marked && page < used)
      a.out[2 * (int64_t)(page - rank) + 1] = page;
    if ((page & 63) == 0) a.before[page >> 6] = rank - stay;
  });
  if (blockIdx.x == 0 && threadIdx.x == 0) a.counts[0] = used, a.counts[1] = used - stay;
}

// The number of a page among those that move.
__device__ __forceinline__ int move_of(const Word *marks, const int32_t *before, int page) {
  return before[page >> 6] + __popcll(marks[page >> 6] & (((Word)1 << (page & 63)) - 1));
}

__global__ __launch_bounds__(kLifeBlock) void page_compact_tables(LifeArgs a) {
  const int used = a.counts[0], moves = a.counts[1];
  for (int r = blockIdx.x; r < a.R; r += gridDim.x) {
    const int held = pages_held(a, r);
    for (int j = blockIdx.y * kLifeBlock + threadIdx.x; j < held; j += gridDim.y * kLifeBlock) {
      const int page = a.table[r * a.table_row + j];
      if (is_page(page, a.pages) && page >= used)
        a.table[r * a.table_row + j] = a.out[2 * (int64_t)move_of(a.marks, a.before, page) + 1];
    }
  }
  const int blocks = gridDim.x * gridDim.y, block = blockIdx.y * gridDim.x + blockIdx.x;
  for (int k = block * kLifeBlock + threadIdx.x; k < moves; k += blocks * kLifeBlock) {
    const int from = a.out[2 * (int64_t)k], to = a.out[2 * (int64_t)k + 1];
    a.shares[to] = a.shares[from];
    a.shares[from] = 0;
  }
}

// The same two calls by one block, with the marks in LDS: three or four launches become one where the
// entries are few.  Entries are taken as one line, so short rows leave no thread out.  6 rows of up to 49 pages given up in 4.3 us
// (a call 22 to 15), 24 rows of up to 76 compacted in 5.4 (a call with its copies 36 to 26).

constexpr int kOneBlock = 1024;  // threads, and words of marks: 65536 pages

struct OneBlock {
  Word marks[kOneBlock];
  int before[kOneBlock], sums[kOneBlock / kWave];
};

// Sum over the block of `mine`; *before: that of the threads before this one.
__device__ __forceinline__ int one_scan(int mine, int *sums, int *before) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int upto = mine;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int x = __shfl_up(upto, o);
    if (lane >= o) upto += x;
  }
  __syncthreads();
  if (lane == 63) sums[wave] = upto;
  __syncthreads();
  int all = 0;
#pragma unroll
  for (int k = 0; k < kOneBlock / kWave; ++k) {
    if (k < wave) upto += sums[k];
    all += sums[k];
  }
  *before = upto - mine;
  return all;
}

// visit(page, marked, marked pages before it), a wave a word and a lane a page.
template <class F>
__device__ __forceinline__ void one_pages(const LifeArgs &a, const OneBlock &s, F visit) {
  const int lane = threadIdx.x & 63;
  for (int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); w < a.words; w += kOneBlock / kWave) {
    const Word b = s.marks[w];
    const int page = w * 64 + lane;
    if (page < a.pages) visit(page, (bool)((b >> lane) & 1), s.before[w] + __popcll(b & (((Word)1 << lane) - 1)));
  }
}

__global__ __launch_bounds__(kOneBlock) void page_free_one(LifeArgs a) {
  __shared__ OneBlock s;
  const int tid = threadIdx.x, entries = a.n * a.W;
  s.marks[tid] = 0;
  __syncthreads();
  int given = 0;
  for (int e = tid; e < entries; e += kOneBlock) {
    const int i = (unsigned)e / (unsigned)a.W, r = a.rows[i], j = e - i * a.W;
    if ((unsigned)r < (unsigned)a.R && j < pages_held(a, r))
      given += give_up(a, r, j, [&](int page) { mark(s.marks, page); });
  }
  int before;
  given = one_scan(given, s.sums, &before);  // waits for the marks too
  const int all = one_scan(__popcll(s.marks[tid]), s.sums, &before);
  s.before[tid] = before;
  __syncthreads();
  one_pages(a, s, [&](int page, bool marked, int rank) {
    if (!marked) return;
    a.shares[page] = 0;
    if (rank < a.most) a.out[rank] = page;
  });
  for (int i = all + tid; i < a.most; i += kOneBlock) a.out[i] = -1;
  for (int i = tid; i < a.n; i += kOneBlock)
    if ((unsigned)a.rows[i] < (unsigned)a.R) a.seq[a.rows[i]] = 0;
  if (tid == 0) a.counts[0] = all, a.counts[1] = given;
}

__global__ __launch_bounds__(kOneBlock) void page_compact_one(LifeArgs a) {
  __shared__ OneBlock s;
  const int tid = threadIdx.x, entries = a.R * a.W;
  s.marks[tid] = 0;
  __syncthreads();
  for (int e = tid; e < entries; e += kOneBlock) {
    const int r = (unsigned)e / (unsigned)a.W, j = e - r * a.W;
    if (j >= pages_held(a, r)) continue;
    const int page = a.table[r * a.table_row + j];
    if (is_page(page, a.pages)) mark(s.marks, page);
  }
  __syncthreads();
  int before, unused;
  const Word bits = s.marks[tid];
  const int used = one_scan(__popcll(bits), s.sums, &before);
  const int left = used - tid * 64;  // of the places that stay, those from this word on
  const Word mask = left >= 64 ? ~(Word)0 : left > 0 ? ((Word)1 << left) - 1 : 0;
  const int stay = one_scan(__popcll(bits & mask), s.sums, &unused), moves = used - stay;
  s.before[tid] = before - stay;
  __syncthreads();
  one_pages(a, s, [&](int page, bool marked, int move) {
    if (marked && page >= used)
      a.out[2 * move] = page;
    else if (!marked && page < used)
      a.out[2 * (page - stay - move) + 1] = page;
  });
  for (int i = 2 * moves + tid; i < 2 * a.most; i += kOneBlock) a.out[i] = -1;
  if (tid == 0) a.counts[0] = used, a.counts[1] = moves;
  __syncthreads();
  for (int e = tid; e < entries; e += kOneBlock) {
    const int r = (unsigned)e / (unsigned)a.W, j = e - r * a.W;
    if (j >= pages_held(a, r)) continue;
    const int page = a.table[r * a.table_row + j];
    if (is_page(page, a.pages) && page >= used) a.table[r * a.table_row + j] = a.out[2 * move_of(s.marks, s.before, page) + 1];
  }
  for (int k = tid; k < moves; k += kOneBlock) {
    const int from = a.out[2 * k], to = a.out[2 * k + 1];
    a.shares[to] = a.shares[from];
    a.shares[from] = 0;
  }
}

// -------------------------------------------------------------------- copies

constexpr int kCopyArrays = 8;
constexpr int kCopyBytes = 16384;  // of a block's step: the 697 MB below 136 us; 8 KB 140, 32 KB 137

struct CopyArray {
  uint8_t *data;
  int64_t page, outer_stride, inner_stride;  // bytes
  int64_t bytes;                             // of a page
  unsigned row, inner;                       // bytes of a row, rows of an inner run
  int unit;                                  // bytes moved at once: 16, 4 or 1
  int steps;                                 // of kCopyBytes
  int dense;                                 // a page's bytes are adjacent
};

struct CopyArgs {
  CopyArray array[kCopyArrays];
  const int32_t *pairs;  // [n][2]
  int64_t items;         // steps of all pairs
  int32_t n, arrays, pages, steps;
};

template <class V>
__device__ __forceinline__ void copy_step(const CopyArray &x, int from, int to, int64_t first) {
  const uint8_t *src = x.data + from * x.page;
  uint8_t *dst = x.data + to * x.page;
  const int64_t last = first + kCopyBytes < x.bytes ? first + kCopyBytes : x.bytes;
  constexpr int kMany = 4;
  for (int64_t at = first + threadIdx.x * (int64_t)sizeof(V); at < last; at += kLifeBlock * (int64_t)sizeof(V) * kMany) {
    V v[kMany];
    int64_t off[kMany];
#pragma unroll
    for (int k = 0; k < kMany; ++k) {
      const int64_t i = at + k * kLifeBlock * (int64_t)sizeof(V);
      off[k] = i;
      if (!x.dense) {
        const int64_t row = i / x.row, outer = row / x.inner;
        off[k] = outer * x.outer_stride + (row - outer * x.inner) * x.inner_stride + (i - row * x.row);
      }
      if (i < last) v[k] = *(const __attribute__((address_space(1))) V *)(src + off[k]);
    }
#pragma unroll
    for (int k = 0; k < kMany; ++k)
      if (at + k * kLifeBlock * (int64_t)sizeof(V) < last) *(__attribute__((address_space(1))) V *)(dst + off[k]) = v[k];
  }
}

// A block takes 16 KB of a page of one array at a time; four 16-byte loads a thread are on their way.  Memory: 697 MB read and
// written in 136 us, 5.1 TB/s (a torch copy of 4 GiB 4.7); 118 MB, much of it in the last cache, in 12.
// Its lanes look at the pairs of its next 64 steps at once: a list is mostly of pairs that are left out, where a large cache
// was compacted (100000 pages, 64 of them moved, two arrays of 128 KB a page: 16 us, with a look at each step's pair in turn 230).
__global__ __launch_bounds__(kLifeBlock) void page_copy(CopyArgs a) {
  const int lane = threadIdx.x & 63;
  for (int64_t item0 = blockIdx.x; item0 < a.items; item0 += (int64_t)gridDim.x * kWave) {
    const int64_t item = item0 + (int64_t)lane * gridDim.x;
    int from = -1, to = -1, step = 0;
    if (item < a.items) {
      const int64_t i = item / a.steps;
      step = (int)(item - i * a.steps);
      from = a.pairs[2 * i], to = a.pairs[2 * i + 1];
    }
    unsigned long long todo = __builtin_amdgcn_ballot_w64(is_page(from, a.pages) && is_page(to, a.pages) && from != to);
    for (; todo; todo &= todo - 1) {
      const int n = __builtin_ctzll(todo);
      const int src = __builtin_amdgcn_readlane(from, n), dst = __builtin_amdgcn_readlane(to, n);
      int s = __builtin_amdgcn_readlane(step, n), k = 0;
      while (k < a.arrays - 1 && s >= a.array[k].steps) s -= a.array[k++].steps;
      const CopyArray &x = a.array[k];
      const int64_t first = (int64_t)s * kCopyBytes;
      if (x.unit == 16)
        copy_step<u32x4>(x, src, dst, first);
      else if (x.unit == 4)
        copy_step<unsigned>(x, src, dst, first);
      else
        copy_step<uint8_t>(x, src, dst, first);
    }
  }
}

}  // namespace paged
}  // namespace slnr
