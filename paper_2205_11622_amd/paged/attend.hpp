// Attention over a paged cache: the SDDMM q.k, the softmax and the SpMM p v of
// one (request, KV head) in one pass, with the running maximum and sum of the
// softmax.  The query heads of a KV head are rows of one matrix product.
#pragma once

#include "common.hpp"

namespace slnr {
namespace paged {

struct AttendArgs {
  const void *q;         // [T][Hq][D], strides q_token, q_head
  int64_t q_token, q_head;
  const void *k, *v;     // [pages][P][Hkv][D]
  int64_t k_page, k_slot, k_head, v_page, v_slot, v_head;
  const int32_t *table;  // [R][W], row stride table_row
  int64_t table_row;
  const int32_t *seq;    // [R]
  const int32_t *qptr;   // [R + 1]
  const int32_t *sel;    // [T][Hkv][top], sparse form only
  void *out;             // [T][Hq][D], densely packed
  float *lse;            // [T][Hq] or null
  float *part;           // per piece of a split tile: rows x DP values, then rows maxima and sums
  int32_t *meta;         // per piece, what the join has to know (see kMeta)
  int32_t R, T, W, pages, shift, Hq, Hkv, G, D, top, window;
  int32_t few;           // requests with at most this many rows belong to attend_few, the others to attend_many
  int32_t target;        // pieces that the work is cut into, about
  float scale2;          // scale * log2(e)
};

// meta[0]: slots that this call uses.  From kMeta * (1 + slot) on: pieces of this tile
// if the slot is its first, else 0; the tile's first row (token * G + head of the
// group), its rows, and the KV head.
constexpr int kMeta = 4;

__device__ __forceinline__ int imin(int a, int b) { return a < b ? a : b; }
__device__ __forceinline__ int imax(int a, int b) { return a > b ? a : b; }

// Scores are kept as they come out of q.k and scaled inside the exponent, exp2(s c - m c),
// except in fp32: there s c comes first, so that the largest weight is exactly one.
// Maxima are in the same unit; this is what takes it to the exponent of two.
template <class T>
__device__ __forceinline__ float score_unit(const AttendArgs &a) {
  return sizeof(T) == 4 ? 1.0f : a.scale2;
}

template <class T>
struct Pack4 {
  typedef i16x4 V;
};
template <>
struct Pack4<float> {
  typedef f32x4 V;
};

// Adds weight * v to four columns of a query that sees the key, for those of the
// values v[d .. d + 3] that are infinite or NaN.
template <class T, class F>
__device__ __forceinline__ void add_odd(const T *v, int d, int D, float weight, bool seen, F add) {
  if (d < D) {
    union {
      typename Pack4<T>::V v;
      T t[4];
    } w;
    w.v = *(const __attribute__((address_space(1))) typename Pack4<T>::V *)(v + d);
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const float x = (float)w.t[c];
      add(c, seen && !(fabsf(x) < __builtin_inff()) ? weight * x : 0.0f);
    }
  }
  asm volatile("" ::: "memory");  // one load at a time: this is rare, registers are not
}

// Whether a row of V has infinities or NaN; the same in all lanes.
template <class T>
__device__ __forceinline__ bool has_odd(const T *v, int D, int lane) {
  bool bad = false;
  if (lane * 8 < D) {
    typename Type<T>::Vec x = load8_global<T>(v + lane * 8);
    bad = clean8<T>(x);
  }
  return __builtin_amdgcn_ballot_w64(bad) != 0;
}

// Eight terms of q.k.
template <class T>
__device__ __forceinline__ float dot8(typename Type<T>::Vec q, const T *k, int d, int D) {
  float s = 0.0f;
  if (d < D) {
    const typename Type<T>::Vec x = load8_global<T>(k + d);
#pragma unroll
    for (int i = 0; i < 8; ++i) s = __builtin_fmaf((float)q[i], (float)x[i], s);
  }
  asm volatile("" ::: "memory");
  return s;
}

struct Request {
  int first, n, S;  // first token, tokens, visible length
};

// Whatever the arrays hold, tokens stay in [0, T) and keys in the table's row.
__device__ __forceinline__ Request request_of(const AttendArgs &a, int r) {
  Request q;
  const int b = imin(imax(a.qptr[r], 0), a.T);
  const int e = imin(imax(a.qptr[r + 1], 0), a.T);
  q.first = b;
  q.n = imax(e - b, 0);
  const int64_t room = (int64_t)a.W << a.shift;
  const int s = imax(a.seq[r], 0);
  q.S = s < room ? s : (int)room;
  return q;
}

// ------------------------------------------------------------- split of the work
//
// A tile is up to ROWS rows (token, head of the group) of one request and KV head.
// Tiles whose keys take more than `cap` steps are cut into np equal pieces of the
// key axis, whose results the join adds up; cap is such that all the work makes
// about `target` pieces, so long contexts are cut where there are few tiles and
// left whole where there are many.  With a tail, the tiles behind the first 70% of the
// work are cut kTailCuts times finer: the blocks that are done early find something
// to fill the time with until the longest one is done (see has_tail).
// Every block derives the split from the lengths by one scan: nothing has to be
// planned, copied or known on the host.

constexpr int kTailCuts = 3;
constexpr int kTailSteps = 40;

template <int NT>
struct Split {
  int begin[NT];         // pieces (of one KV head) before this thread's requests
  int slot[NT];          // the same of split tiles only
  long long before[NT];  // steps before them
  long long work[NT / kWave], least[NT / kWave];
  int wave_a[NT / kWave], wave_b[NT / kWave];
  long long whole;       // steps up to which tiles are cut by cap, behind them by cap_tail
  int total, total_split, cap, cap_tail, per;
};

struct Piece {
  int r, tile, part, np, slot;  // slot < 0: the tile is whole
};

// A request's tiles before the tail, and the pieces of a tile before and in it.
struct Cut {
  int front, np, np_tail;
};

template <int NT>
__device__ __forceinline__ Cut cut_of(const Split<NT> &sh, long long before, int tiles, int steps) {
  Cut c;
  const int s = imax(steps, 1);
  const long long left = sh.whole - before;
  c.front = left <= 0 ? 0 : left >= (long long)tiles * s ? tiles : (int)((left + s - 1) / s);
  c.np = (s + sh.cap - 1) / sh.cap;
  c.np_tail = (s + sh.cap_tail - 1) / sh.cap_tail;
  return c;
}

// A tail pays where long tiles are a little more than the rounds that the units take them in, so that the last
// round is nearly empty; elsewhere it only makes more pieces to be joined.  Only attend_many has one: a block of it
// fills a compute unit.  attend_few has three pieces a unit, two at a time, anyway.  `least` is the sum of all tiles'
// steps, each request's at its shortest one.  us with / without, 32 / 8 heads of 128 in bf16 on 256 units, one request:
// behind 8000 tokens 2048 of them (256 tiles) 383 / 328, 2112 (264) 387 / 501, 2560 (320) 429 / 528, 2816 (352) 501 /
// 543, 3584 (448) 633 / 592, 4096 (512) 785 / 658, 4160 (520) 792 / 873, 5632 (704) 1039 / 1005; from 768 tiles on
// they are shorter than the cut, alike; two requests behind 3000, 2 x 1056 185 / 221; four behind 1500, 4 x 528 126 / 138, but
// 4 x 1040 227 / 213; none cached, 2112 100 / 87, 4160 219 / 187.
__device__ __forceinline__ bool has_tail(const AttendArgs &a, long long tiles, long long least) {
  const long long all = tiles * a.Hkv, over = all % a.target;
  return all > a.target && over > 0 && over <= a.target * 3 / 8 && least >= tiles * kTailSteps;
}

// count(r, tiles, steps) gives a request's tiles and the steps of its longest one; shortest(r, steps) with a
// tail those of its shortest one.
struct NoTail {
  __device__ int operator()(int, int steps) const { return steps; }
};

template <int NT, class F, class S = NoTail>
__device__ void split_scan(Split<NT> &sh, const AttendArgs &a, int min_steps, F count, S shortest = S()) {
  constexpr bool kTail = !__is_same(S, NoTail);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int per = (a.R + NT - 1) / NT;
  const int r0 = imin(tid * per, a.R), r1 = imin(r0 + per, a.R);
  long long w = 0, least = 0;
  int rows = 0;
  for (int r = r0; r < r1; ++r) {
    int tiles, steps;
    count(r, tiles, steps);
    w += (long long)tiles * imax(steps, 1);
    if (kTail) least += (long long)tiles * shortest(r, steps), rows += tiles;
  }
  if (kTail) {
#pragma unroll
    for (int o = 32; o; o >>= 1) least += __shfl_xor(least, o), rows += __shfl_xor(rows, o);
    if (lane == 0) sh.least[wave] = least, sh.wave_a[wave] = rows;
  }
  long long upto = w;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const long long x = __shfl_up(upto, o);
    if (lane >= o) upto += x;
  }
  if (lane == 63) sh.work[wave] = upto;
  __syncthreads();
  long long all = 0;
#pragma unroll
  for (int i = 0; i < NT / kWave; ++i) {
    if (i < wave) upto += sh.work[i];
    all += sh.work[i];
  }
  if (tid == 0) {
    bool tail = false;
    if (kTail) {
      long long tiles = 0;
      least = 0;
#pragma unroll
      for (int i = 0; i < NT / kWave; ++i) least += sh.least[i], tiles += sh.wave_a[i];
      tail = has_tail(a, tiles, least);
    }
    const long long want = (all * a.Hkv + a.target - 1) / a.target;
    sh.cap = imax(min_steps, (int)(want < (1 << 28) ? want : (1 << 28)));
    sh.cap_tail = tail ? imax(min_steps, (sh.cap + kTailCuts - 1) / kTailCuts) : sh.cap;
    sh.whole = tail ? all - all * 3 / 10 : all;
    sh.per = per;
  }
  __syncthreads();
  int np = 0, ns = 0;
  long long before = upto - w;
  sh.before[tid] = before;
  for (int r = r0; r < r1; ++r) {
    int tiles, steps;
    count(r, tiles, steps);
    const Cut c = cut_of(sh, before, tiles, steps);
    before += (long long)tiles * imax(steps, 1);
    const int x = c.front * c.np, y = (tiles - c.front) * c.np_tail;
    np += x + y;
    ns += (c.np > 1 ? x : 0) + (c.np_tail > 1 ? y : 0);
  }
  int x = np, y = ns;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int px = __shfl_up(x, o), py = __shfl_up(y, o);
    if (lane >= o) x += px, y += py;
  }
  if (lane == 63) sh.wave_a[wave] = x, sh.wave_b[wave] = y;
  __syncthreads();
  int bx = 0, by = 0, total = 0, total_split = 0;
#pragma unroll
  for (int i = 0; i < NT / kWave; ++i) {
    if (i < wave) bx += sh.wave_a[i], by += sh.wave_b[i];
    total += sh.wave_a[i];
    total_split += sh.wave_b[i];
  }
  sh.begin[tid] = bx + x - np;
  sh.slot[tid] = by + y - ns;
  if (tid == 0) sh.total = total, sh.total_split = total_split;
  __syncthreads();
}

// The piece number q of one KV head, 0 <= q < total.
template <int NT, class F>
__device__ Piece split_find(const Split<NT> &sh, const AttendArgs &a, int q, F count) {
  // the last thread that begins at or before q (those without pieces begin where the
  // next one does)
  int lo = 0, hi = NT - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (sh.begin[mid] <= q)
      lo = mid;
    else
      hi = mid - 1;
  }
  int left = q - sh.begin[lo], slot = sh.slot[lo];
  long long before = sh.before[lo];
  Piece p{};
  for (int r = lo * sh.per; r < a.R; ++r) {
    int tiles, steps;
    count(r, tiles, steps);
    const Cut c = cut_of(sh, before, tiles, steps);
    before += (long long)tiles * imax(steps, 1);
    const int x = c.front * c.np, y = (tiles - c.front) * c.np_tail;
    if (left < x + y) {
      const bool in_tail = left >= x;
      if (in_tail) {
        left -= x;
        if (c.np > 1) slot += x;
      }
      p.r = r;
      p.np = in_tail ? c.np_tail : c.np;
      const int t = left / p.np;
      p.tile = tiles - 1 - (in_tail ? c.front + t : t);  // the longest (last) tile of a causal chunk first
      p.part = left - t * p.np;
      p.slot = p.np > 1 ? slot + left : -1;
      return p;
    }
    left -= x + y;
    slot += (c.np > 1 ? x : 0) + (c.np_tail > 1 ? y : 0);
  }
  p.r = -1;
  return p;
}

// ---------------------------------------------------------------- few rows
//
// attend_few: a block of four waves takes one piece of a tile of 16 rows (the
// heads of one token of a decode step, or of a few tokens; the heads of one token
// over its selected pages in the sparse form).  Each wave walks every fourth tile
// of 32 keys.  S^T = K Q^T puts a query into a lane's column, so the softmax
// needs two exchanges between lanes a tile, and P^T stays in the registers in
// which O^T = V^T P^T wants it.  K goes from memory straight to the matrix cores'
// operands; V passes through LDS to be transposed.  The waves' results are joined
// in LDS.
//
// Bound by memory: a key is read once for all heads of its group.  16 KB of K and V
// are in flight per wave while the previous tile is worked on.
//
// 64 requests of 513 to 15096 keys, 32 / 8 heads of 128 in bf16 (1190 MB): 252 us, 4.7 TB/s,
// what a copy of 4 GiB reaches; the join adds 6.  32 tokens over 32 selected
// pages of 64 keys (269 MB): 63 us, 4.2 TB/s, and 5.  4 requests of 635 to 933 keys, 8 / 2
// heads of 64 in fp32 (3 MB): 12 us and 4, the latency of the lengths, the split, the
// table, a tile, the four waves' join and the launches.

constexpr int kFewBlock = 256;
constexpr int kFewWaves = kFewBlock / kWave;
constexpr int kFewRows = 16;
constexpr int kFewKeys = 32;                           // keys of a wave's tile
constexpr int kFewStep = kFewKeys * kFewWaves;         // keys of a block's step

template <class T, int DP>
struct FewShared {
  union {
    T v[kFewWaves][kFewKeys * Tile<T, DP>::kStride];
    float o[kFewWaves][kFewRows * DP];
  };
  float m[kFewWaves][kFewRows], l[kFewWaves][kFewRows];
  Split<kFewBlock> split;
};

template <class T, int DP, bool SPARSE>
__global__ __launch_bounds__(kFewBlock) void attend_few(AttendArgs a) {
  typedef typename Type<T>::Vec Vec;
  constexpr int KS = DP / 32;   // steps of the summed axis of q.k
  constexpr int DT = DP / 16;   // tiles of output columns
  extern __shared__ __align__(16) char raw[];
  FewShared<T, DP> &sh = *reinterpret_cast<FewShared<T, DP> *>(raw);
  const float sc = score_unit<T>(a);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int col = lane & 15, grp = lane >> 4;
  const int row_tiles = (a.G + kFewRows - 1) / kFewRows;  // sparse form: of one token
  const int P = 1 << a.shift;
  auto count = [&](int r, int &tiles, int &steps) {
    const Request q = request_of(a, r);
    const long long rows = (long long)q.n * a.G;
    tiles = rows > a.few ? 0 : (int)((rows + kFewRows - 1) / kFewRows);
    const int lo = a.window ? imax(q.S - q.n - a.window + 1, 0) : 0;
    steps = (q.S - lo + kFewStep - 1) / kFewStep;
  };
  int total, used, np_sparse = 1;
  int steps_sparse = 0;
  if constexpr (SPARSE) {
    const long long keys = (long long)a.top << a.shift;
    steps_sparse = (int)((keys + kFewStep - 1) / kFewStep);
    const long long tiles = (long long)a.T * row_tiles * a.Hkv;
    // all tiles are alike: cut until there are `target` pieces
    const long long k = a.target / (tiles > 0 ? tiles : 1);
    np_sparse = imax(1, (int)(k < steps_sparse ? k : steps_sparse));
    total = a.T * row_tiles * np_sparse;
    used = np_sparse > 1 ? total : 0;
  } else {
    split_scan<kFewBlock>(sh.split, a, 1, count);
    total = sh.split.total;
    used = sh.split.total_split;
  }
  if (blockIdx.x == 0 && tid == 0) a.meta[0] = used * a.Hkv;

  for (unsigned p = blockIdx.x; p < (unsigned)total * (unsigned)a.Hkv; p += gridDim.x) {
    const int h = (int)(p % (unsigned)a.Hkv), qn = (int)(p / (unsigned)a.Hkv);
    // ------------------------------------------------ which rows and keys
    int r, row0, rows, pos_first, pos_last, lo, hi, part, np, slot;
    const int32_t *sel = nullptr;
    Request rq;
    if constexpr (SPARSE) {
      part = qn % np_sparse;
      const int t2 = qn / np_sparse;
      const int t = t2 / row_tiles, rt = t2 % row_tiles;
      // the request of token t: the last r with qptr[r] <= t
      int x = 0, y = a.R - 1;
      while (x < y) {
        const int mid = (x + y + 1) >> 1;
        if (a.qptr[mid] <= t)
          x = mid;
        else
          y = mid - 1;
      }
      r = x;
      rq = request_of(a, r);
      np = np_sparse;
      slot = np > 1 ? qn : -1;
      if (t < rq.first || t >= rq.first + rq.n) {  // no request's token
        if (slot >= 0 && tid == 0) a.meta[(1 + (int64_t)slot * a.Hkv + h) * kMeta] = 0;
        continue;
      }
      row0 = t * a.G + rt * kFewRows;
      rows = imin(a.G - rt * kFewRows, kFewRows);
      pos_first = pos_last = rq.S - rq.n + (t - rq.first);
      sel = a.sel + ((int64_t)t * a.Hkv + h) * a.top;
      lo = 0;
      hi = a.top << a.shift;
    } else {
      const Piece pc = split_find<kFewBlock>(sh.split, a, qn, count);
      if (pc.r < 0) continue;
      r = pc.r;
      part = pc.part;
      np = pc.np;
      slot = pc.slot;
      rq = request_of(a, r);
      const int first = pc.tile * kFewRows;  // of the request's rows
      rows = imin(rq.n * a.G - first, kFewRows);
      row0 = rq.first * a.G + first;
      pos_first = rq.S - rq.n + first / a.G;
      pos_last = rq.S - rq.n + (first + rows - 1) / a.G;
      lo = a.window ? imax(pos_first - a.window + 1, 0) : 0;
      hi = imin(pos_last + 1, rq.S);
    }
    const int tiles = hi > lo ? (hi - lo + kFewKeys - 1) / kFewKeys : 0;
    const int steps = (tiles + kFewWaves - 1) / kFewWaves;
    const int s0 = (int)((long long)steps * part / np), s1 = (int)((long long)steps * (part + 1) / np);
    const int32_t *table = a.table + (int64_t)r * a.table_row;

    // ------------------------------------------------ the queries, as columns
    const bool have_row = col < rows;
    const int rho = row0 + (have_row ? col : 0);
    const int tok = rho / a.G, head = h * a.G + rho % a.G;
    const int pos = rq.S - rq.n + (tok - rq.first);
    Vec q[KS];
    {
      const T *src = (const T *)a.q + (int64_t)tok * a.q_token + (int64_t)head * a.q_head;
#pragma unroll
      for (int i = 0; i < KS; ++i) {
        const int d = i * 32 + grp * 8;
        q[i] = load8_global<T>(have_row && d < a.D ? src + d : (const T *)kZeroRow);
      }
    }

    // ------------------------------------------------ walk of the keys
    f32x4 o[DT];
#pragma unroll
    for (int i = 0; i < DT; ++i) o[i] = f32x4{0, 0, 0, 0};
    float m = kNegInf, l = 0.0f;

    // The page of key u of the piece's axis; -1 where no row of the tile sees it.
    auto find = [&](int u) {
      int page = -1;
      if (u < hi) {
        int b = u >> a.shift, at = u;
        if constexpr (SPARSE) {
          b = sel[b];
          at = (b << a.shift) | (u & (P - 1));
        }
        if (b >= 0 && b < a.W) page = table[b];
        if ((unsigned)page >= (unsigned)a.pages || at > pos_last) page = -1;
      }
      return page;
    };
    int page[2], page2[2];  // of the tile to load, and of the one after it
    Vec kr[2][KS], vr[2][KS];
    unsigned live;  // bit: this key of the tile is there
    auto load = [&](int base) {
      live = 0;
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const bool ok = page[s] >= 0;
        live |= ((unsigned)__builtin_amdgcn_ballot_w64(ok) & 0xffffu) << (16 * s);
        const int64_t in = ((base + s * 16 + col) & (P - 1));
        const T *ks = (const T *)a.k + (int64_t)page[s] * a.k_page + in * a.k_slot + (int64_t)h * a.k_head;
        const T *vs = (const T *)a.v + (int64_t)page[s] * a.v_page + in * a.v_slot + (int64_t)h * a.v_head;
#pragma unroll
        for (int i = 0; i < KS; ++i) {
          const int d = i * 32 + grp * 8;
          const bool in_row = ok && d < a.D;
          kr[s][i] = load8_global<T>(in_row ? ks + d : (const T *)kZeroRow);
          vr[s][i] = load8_global<T>(in_row ? vs + d : (const T *)kZeroRow);
        }
      }
    };
    // Rows of several tokens see different keys.
    auto is_mixed = [&](int tile) {
      return !SPARSE && pos_first != pos_last &&
             (tile + kFewKeys - 1 > pos_first || (a.window && tile <= pos_last - a.window));
    };
    bool odd = false;
    T *vt = sh.v[wave];
    int base = lo + (s0 * kFewWaves + wave) * kFewKeys;
    const int end = imin(lo + s1 * kFewStep, hi);
    auto look = [&](int base, int out[2]) {
#pragma unroll
      for (int s = 0; s < 2; ++s) out[s] = base < end ? find(base + s * 16 + col) : -1;
    };
    look(base, page);
    look(base + kFewStep, page2);
    if (base < end) load(base);
    while (base < end) {
      const unsigned now = live;
      const int tile = base;
      base += kFewStep;
      page[0] = page2[0], page[1] = page2[1];
      look(base + kFewStep, page2);
      // S^T = K Q^T
      f32x4 x[2];
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        x[s] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < KS; ++i) x[s] = Type<T>::dot16(kr[s][i], q[i], x[s]);
        if constexpr (sizeof(T) == 4) x[s] *= a.scale2;
      }
      // A key that some rows see and others do not must not reach the latter through 0 *
      // inf: infinities and NaN of V are taken out of the product and added at the end.
      const bool mixed = is_mixed(tile);
      if (mixed) {
        bool bad = false;
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
          for (int i = 0; i < KS; ++i) bad |= clean8<T>(vr[s][i]);
        if (__builtin_amdgcn_ballot_w64(bad)) odd = true;
      }
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int i = 0; i < KS; ++i)
          store8<T>(vt + Tile<T, DP>::at(s * 16 + col, i * 32 + grp * 8), vr[s][i]);
      load(base);  // the next tile's rows are on their way from here on

      if (now != 0xffffffffu || mixed) {
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int key = s * 16 + grp * 4 + i;
            bool seen = (now >> key) & 1;
            if (mixed) seen = seen && tile + key <= pos && (!a.window || tile + key > pos - a.window);
            x[s][i] = seen ? x[s][i] : kNegInf;
          }
      }
      float top = x[0][0];
#pragma unroll
      for (int i = 1; i < 8; ++i) top = fmaxf(top, x[i >> 2][i & 3]);
      top = max_across_16(top);
      const float mn = fmaxf(m, top);
      const float ms = mn == kNegInf ? 0.0f : mn * sc;  // nothing seen yet: exp2(-inf - 0) = 0
      const float fade = exp2_of(m * sc - ms);          // 0 at the first key seen
      m = mn;
      l *= fade;
      Vec pv;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float e = exp2_of(__builtin_fmaf(x[i >> 2][i & 3], sc, -ms));
        l += e;
        x[i >> 2][i & 3] = e;
        // the weights go to the matrix cores in the type of V, their sum stays in fp32
        pv[i] = (T)e;
      }
#pragma unroll
      for (int i = 0; i < DT; ++i) o[i] *= fade;
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int i = 0; i < DT; ++i) {
        union {
          Vec v;
          T t[8];
        } w;
        Tile<T, DP>::read4(vt, grp * 4, i * 16, lane, w.t);
        Tile<T, DP>::read4(vt, 16 + grp * 4, i * 16, lane, w.t + 4);
        o[i] = Type<T>::dot16(w.v, pv, o[i]);
      }
      __builtin_amdgcn_wave_barrier();
    }
    if (odd) {  // rare
      for (int tile = lo + (s0 * kFewWaves + wave) * kFewKeys; tile < end; tile += kFewStep)
        if (is_mixed(tile))
          for (int u = tile; u < tile + kFewKeys; ++u) {
            const int pg = find(u);
            if (pg < 0) continue;
            const T *vs = (const T *)a.v + pg * a.v_page + (u & (P - 1)) * a.v_slot + (int64_t)h * a.v_head;
            if (!has_odd<T>(vs, a.D, lane)) continue;
            const T *ks = (const T *)a.k + pg * a.k_page + (u & (P - 1)) * a.k_slot + (int64_t)h * a.k_head;
            float s = 0.0f;
#pragma unroll
            for (int i = 0; i < KS; ++i) s += dot8<T>(q[i], ks, i * 32 + grp * 8, a.D);
            s = sum_across_16(s);
            if constexpr (sizeof(T) == 4) s *= a.scale2;
            const float e = exp2_of((s - m) * sc);
            const bool seen = u <= pos && (!a.window || u > pos - a.window);
#pragma unroll
            for (int i = 0; i < DT; ++i)
              add_odd<T>(vs, i * 16 + grp * 4, a.D, e, seen, [&](int c, float y) { o[i][c] += y; });
          }
    }

    // ------------------------------------------------ the four waves' results
    l = sum_across_16(l);
    if (l != l) m = __builtin_inff();  // NaN among the scores: the whole row is NaN
    __syncthreads();  // every wave is done with its tile of V
    if (grp == 0) sh.m[wave][col] = m, sh.l[wave][col] = l;
    __syncthreads();
    float mall = kNegInf;
#pragma unroll
    for (int w = 0; w < kFewWaves; ++w) mall = fmaxf(mall, sh.m[w][col]);
    {
      const float f = m == kNegInf ? 0.0f : exp2_of((m - mall) * sc);
#pragma unroll
      for (int i = 0; i < DT; ++i)
        *reinterpret_cast<f32x4 *>(&sh.o[wave][col * DP + i * 16 + grp * 4]) = m == kNegInf ? f32x4{0, 0, 0, 0} : o[i] * f;
    }
    __syncthreads();
    const int threads_row = DP / 8;
    for (int e = tid; e < rows * threads_row; e += kFewBlock) {
      const int i = e / threads_row, d = (e % threads_row) * 8;
      float mx = kNegInf, sum = 0.0f;
#pragma unroll
      for (int w = 0; w < kFewWaves; ++w) mx = fmaxf(mx, sh.m[w][i]);
#pragma unroll
      for (int w = 0; w < kFewWaves; ++w)
        sum += sh.m[w][i] == kNegInf ? 0.0f : sh.l[w][i] * exp2_of((sh.m[w][i] - mx) * sc);
      f32x4 lo4{0, 0, 0, 0}, hi4{0, 0, 0, 0};
#pragma unroll
      for (int w = 0; w < kFewWaves; ++w) {
        lo4 += *reinterpret_cast<const f32x4 *>(&sh.o[w][i * DP + d]);
        hi4 += *reinterpret_cast<const f32x4 *>(&sh.o[w][i * DP + d + 4]);
      }
      if (slot >= 0) {
        const int64_t s = (int64_t)slot * a.Hkv + h;
        float *dst = a.part + s * (kFewRows * (DP + 2)) + i * DP + d;
        *reinterpret_cast<f32x4 *>(dst) = lo4;
        *reinterpret_cast<f32x4 *>(dst + 4) = hi4;
        if (d == 0) {
          float *ml = a.part + s * (kFewRows * (DP + 2)) + kFewRows * DP + i * 2;
          ml[0] = mx;
          ml[1] = sum;
        }
      } else {
        const int rr = row0 + i, t = rr / a.G, hd = h * a.G + rr % a.G;
        const float inv = mx == kNegInf ? 0.0f : 1.0f / sum;
        if (d < a.D) {
          Vec w;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            w[j] = (T)(mx == kNegInf ? 0.0f : lo4[j] * inv);
            w[4 + j] = (T)(mx == kNegInf ? 0.0f : hi4[j] * inv);
          }
          store8<T>((T *)a.out + ((int64_t)t * a.Hq + hd) * a.D + d, w);
        }
        if (d == 0 && a.lse)
          a.lse[(int64_t)t * a.Hq + hd] = mx == kNegInf ? kNegInf : mx * (sc * kLn2) + __logf(sum);
      }
    }
    if (slot >= 0 && tid == 0) {
      int32_t *mt = a.meta + (1 + (int64_t)slot * a.Hkv + h) * kMeta;
      mt[0] = part == 0 ? np : 0;
      mt[1] = row0;
      mt[2] = rows;
      mt[3] = h;
    }
    __syncthreads();
  }
}

// --------------------------------------------------------------- many rows
//
// attend_many: a block takes one piece of a tile of 32 * NW rows, 32 to a wave, and
// walks it in tiles of 64 keys that all its waves share through LDS (two buffers of K and
// of V, the next stage's rows on their way in registers).  As above S^T = K Q^T and
// O^T = V^T P^T, here on the 32 x 32 x 16 products: a lane holds one query and half
// the keys of a tile, so a row's maximum takes one exchange and P^T is used where it
// lies; V^T comes out of LDS through transposing reads.
//
// Bound by the matrix products and by what feeds them: a product of 32 cycles takes 1 KB of
// K or V from LDS, so four SIMDs at once use all of its 128 bytes a cycle, and
// two waves of a SIMD take turns, one in its products, one in its softmax.  4073 tokens
// behind 6818 and 7894, 32 / 8 heads of 128 in bf16 (559 GFLOP): 632 and 654 us on
// two cards, 0.85 to 0.88 PFLOP/s, after a first 10 ms at up to 730, and 34 us for the join (a product of 8192^3: 1.2).  Of that time, the
// same with work left out: 0.97 without exponentials, 0.96 without loads, 0.65 without P V.
// 24 requests under a window of 1024, 16 / 4 heads of 64 in fp16 (2.3 GFLOP): 26 us, two
// tiles deep and bound by latency.
// Measured and not taken: V transposed on its way into LDS, 1.07 times as long; all waves
// in the same phase 1.08; the late half in odd waves, two of them on each of two SIMDs, 1.17;
// 64 rows to a wave, one wave to a SIMD, 1.35 (half the bytes from LDS, but one wave issues its
// softmax and its products one after the other).
//
// NW: eight waves, two to a SIMD; four where O of 256 columns or fp32 takes the
// registers or the LDS of two.
template <class T, int DP, int NW>
struct ManyShared {
  T k[2][64 * Tile<T, DP>::kStride];
  T v[2][64 * Tile<T, DP>::kStride];
  int odd;  // infinities or NaN were taken out of V
  Split<NW * kWave> split;
};

constexpr int kManyKeys = 64;
// The maximum that weights are taken at may be so many powers of two low, so that O is seldom rescaled.
// This costs precision: at the exact maximum the largest weight is one and is not rounded to the type of V; an error of
// 2.1e-3 of the chunk's result below becomes 2.3e-3.  It pays above 64 columns (us with / without, 32 / 8 heads in bf16: 128
// columns 4 of 500 tokens behind 3000 144 / 150, 1 of 4000 175 / 183, 64 of 1 to 200 410 / 436; 256 columns, 16 / 4
// heads, 208 / 218, 252 / 279, 597 / 646); at 64 the maximum is exact (132 / 126, 151 / 144, 365 / 358; fp16
// 126 / 121, 144 / 147, 363 / 367).
template <class T, int DP>
constexpr float kLag = sizeof(T) == 2 && DP > 64 ? 8.0f : 0.0f;
// Instruction classes of sched_group_barrier.
constexpr int kMfma = 0x008, kDsRead = 0x100;
// A piece is at least so many tiles of keys long.  It decides little: at 4, 12 and 16 ten of eleven batches take
// within 2% of the time at 8 (16 of 64 tokens behind 4000 133, 133 and 132 us against 134); 8 of 40 behind 2000 72, 57 and 67
// against 73.
constexpr int kManyMinSteps = 8;

// ONE_PAGE: every tile of 64 keys lies in one page (64 positions and more, which begin
// at multiples of 64), so its address is a scalar to which a lane adds 32 bits.
template <class T, int DP, int NW, bool ONE_PAGE>
__global__ __launch_bounds__(NW *kWave) void attend_many(AttendArgs a) {
  typedef typename Type<T>::Vec Vec;
  typedef Tile<T, DP> L;
  constexpr int NT = NW * kWave, ROWS = 32 * NW;
  constexpr int KS = DP / 16;               // steps of the summed axis of q.k
  constexpr int DT = DP / 32;               // tiles of output columns
  constexpr int NC = DP / 8;                // chunks of eight values of a row
  constexpr int CH = kManyKeys * NC / NT;   // chunks of K and of V that a thread carries
  constexpr int RS = NT / NC;               // rows between two of them
  extern __shared__ __align__(16) char raw[];
  ManyShared<T, DP, NW> &sh = *reinterpret_cast<ManyShared<T, DP, NW> *>(raw);
  const float sc = score_unit<T>(a);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int col = lane & 31, half = lane >> 5;
  const int P = 1 << a.shift;
  auto count = [&](int r, int &tiles, int &steps) {
    const Request q = request_of(a, r);
    const long long rows = (long long)q.n * a.G;
    tiles = rows > a.few ? (int)((rows + ROWS - 1) / ROWS) : 0;
    const int lo = (a.window ? imax(q.S - q.n - a.window + 1, 0) : 0) & -kManyKeys;
    steps = (q.S - lo + kManyKeys - 1) / kManyKeys;
  };
  split_scan<NT>(sh.split, a, kManyMinSteps, count, [&](int r, int steps) {
    const Request q = request_of(a, r);
    return a.window ? steps : imax(steps - q.n / kManyKeys, 0);  // causal: the first tile sees the context only
  });
  const int total = sh.split.total;
  if (blockIdx.x == 0 && tid == 0) a.meta[0] = sh.split.total_split * a.Hkv;

  for (unsigned p = blockIdx.x; p < (unsigned)total * (unsigned)a.Hkv; p += gridDim.x) {
    const int h = (int)(p % (unsigned)a.Hkv);
    const Piece pc = split_find<NT>(sh.split, a, (int)(p / (unsigned)a.Hkv), count);
    if (pc.r < 0) continue;
    const Request rq = request_of(a, pc.r);
    const int before = rq.S - rq.n;  // position of the request's first token
    const int first = pc.tile * ROWS, rows = imin(rq.n * a.G - first, ROWS);
    const int pos_first = before + first / a.G, pos_last = before + (first + rows - 1) / a.G;
    const int lo = (a.window ? imax(pos_first - a.window + 1, 0) : 0) & -kManyKeys;
    const int hi = imin(pos_last + 1, rq.S);
    const int tiles = hi > lo ? (hi - lo + kManyKeys - 1) / kManyKeys : 0;
    const int t0 = (int)((long long)tiles * pc.part / pc.np), t1 = (int)((long long)tiles * (pc.part + 1) / pc.np);
    const int32_t *table = a.table + (int64_t)pc.r * a.table_row;

    // ------------------------------------------------ the queries, as columns
    const int mine = first + wave * 32 + col;  // this lane's row of the request
    const bool have_row = mine < first + rows;
    const int rho = have_row ? mine : first;
    const int tok = rq.first + rho / a.G, head = h * a.G + rho % a.G;
    const int pos = before + rho / a.G;
    const int wave_rows = imin(rows - wave * 32, 32);
    const int wave_first = wave_rows > 0 ? before + (first + wave * 32) / a.G : 0;
    const int wave_last = wave_rows > 0 ? before + (first + wave * 32 + wave_rows - 1) / a.G : -1;
    Vec q[KS];
    {
      const T *src = (const T *)a.q + (int64_t)tok * a.q_token + (int64_t)head * a.q_head;
#pragma unroll
      for (int i = 0; i < KS; ++i) {
        const int d = i * 16 + half * 8;
        q[i] = load8_global<T>(have_row && d < a.D ? src + d : (const T *)kZeroRow);
      }
    }
    f32x16 o[DT];
#pragma unroll
    for (int i = 0; i < DT; ++i)
#pragma unroll
      for (int j = 0; j < 16; ++j) o[i][j] = 0.0f;
    float m = kNegInf, l = 0.0f;

    // ------------------------------------------------ K and V into LDS
    const int n = t1 - t0;          // tiles of this piece
    const int k0 = lo + t0 * kManyKeys;
    // The table's entry for key `lane` of tile i (ONE_PAGE: for all of them), or of the
    // last key there is (there is one wherever this is called), and the page it stands for.
    auto find = [&](int i) {
      return table[imin(k0 + i * kManyKeys + (ONE_PAGE ? 0 : lane), hi - 1) >> a.shift];
    };
    auto valid = [&](int i, int page) {
      if constexpr (ONE_PAGE) page = __builtin_amdgcn_readfirstlane(page);
      const bool in = k0 + i * kManyKeys + (ONE_PAGE ? 0 : lane) < hi;
      return in && (unsigned)page < (unsigned)a.pages ? page : -1;
    };
    auto live_of = [&](int i, int page) -> unsigned long long {  // bit: this key is there
      if constexpr (ONE_PAGE) {
        const int keys = hi - (k0 + i * kManyKeys);
        return page < 0 ? 0 : keys >= kManyKeys ? ~0ull : (1ull << keys) - 1;
      } else {
        return __builtin_amdgcn_ballot_w64(page >= 0);
      }
    };
    // a tile of which some of the block's rows see a part only
    auto mixed = [&](int i) {
      const int b = k0 + i * kManyKeys;
      return b + kManyKeys - 1 > pos_first || (a.window && b <= pos_last - a.window);
    };
    const int c8 = (tid % NC) * 8, row_of = tid / NC;
    const bool in_row = c8 < a.D;
    // Rows that are not there are read from a page that is, and zeroed on their way to
    // LDS: a load then has no condition.
    const T *k_head = (a.pages ? (const T *)a.k : (const T *)kZeroRow) + (a.pages ? (int64_t)h * a.k_head : 0);
    const T *v_head = (a.pages ? (const T *)a.v : (const T *)kZeroRow) + (a.pages ? (int64_t)h * a.v_head : 0);
    const int64_t k_page = a.pages ? a.k_page : 0, k_slot = a.pages ? a.k_slot : 0;
    const int64_t v_page = a.pages ? a.v_page : 0, v_slot = a.pages ? a.v_slot : 0;
    const unsigned k_lane = (unsigned)(row_of * (int)k_slot + (in_row ? c8 : 0)) * (unsigned)sizeof(T);
    const unsigned v_lane = (unsigned)(row_of * (int)v_slot + (in_row ? c8 : 0)) * (unsigned)sizeof(T);
    Vec kr[CH], vr[CH];
    auto load = [&](Vec r[CH], int i, int page, const T *base, int64_t page_stride, int64_t slot_stride,
                    unsigned lane_bytes) {
      if constexpr (ONE_PAGE) {
        const int in = (k0 + i * kManyKeys) & (P - 1);
        const char *src = (const char *)(base + imax(page, 0) * page_stride + in * slot_stride);
#pragma unroll
        for (int c = 0; c < CH; ++c) {
          r[c] = load8_global<T>((const T *)(src + lane_bytes));
          src += RS * slot_stride * (int64_t)sizeof(T);
        }
      } else {
#pragma unroll
        for (int c = 0; c < CH; ++c) {
          const int row = c * RS + row_of;
          const int pg = imax(__shfl(page, row), 0);
          const int in = (k0 + i * kManyKeys + row) & (P - 1);
          r[c] = load8_global<T>(base + pg * page_stride + in * slot_stride + (in_row ? c8 : 0));
        }
      }
    };
    auto load_k = [&](int i, int page) { load(kr, i, page, k_head, k_page, k_slot, k_lane); };
    auto load_v = [&](int i, int page) { load(vr, i, page, v_head, v_page, v_slot, v_lane); };
    // Rows that are not there become zeros, and V of a tile of which some rows see a part
    // only loses its infinities and NaN (kept for those who see them: see `values`).
    auto clean = [&](Vec r[CH], unsigned long long live) {
      if (live != ~0ull || a.D != DP) {
#pragma unroll
        for (int c = 0; c < CH; ++c) {
          const bool keep = in_row && ((live >> (c * RS + row_of)) & 1);
#pragma unroll
          for (int j = 0; j < 8; ++j) r[c][j] = keep ? r[c][j] : (T)0.0f;
        }
      }
    };
    auto clean_v = [&](int i, unsigned long long live) {
      clean(vr, live);
      if (mixed(i)) {
        bool bad = false;
#pragma unroll
        for (int c = 0; c < CH; ++c) bad |= clean8<T>(vr[c]);
        if (__builtin_amdgcn_ballot_w64(bad)) sh.odd = 1;
      }
    };
    auto store = [&](T *dst, Vec r[CH]) {
#pragma unroll
      for (int c = 0; c < CH; ++c)  // 16 rows on, a row's chunks are permuted alike
        store8<T>(dst + L::at((c * RS) % 16 + row_of, c8) + (c * RS) / 16 * 16 * L::kStride, r[c]);
    };
    // A barrier that waits for LDS only: loads on their way stay there.
    auto sync = [&]() {
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
      __builtin_amdgcn_s_barrier();
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
    };

    const unsigned k_at = lds_address(sh.k[0]) + L::k_first(col, half);
    const unsigned v_at = lds_address(sh.v[0]) + L::v_first(lane);
    f32x16 x[2];
    Vec pv[4];

    // S^T = K Q^T of tile i
    auto scores = [&](int i) {
      if constexpr (sizeof(T) == 2) {
        unsigned at = k_at + (i & 1) * (int)sizeof(sh.k[0]);
        asm("" : "+v"(at));  // the addresses made of it here take an instruction each, kept ones a register
        Vec k[KS][2];
#pragma unroll
        for (int c = 0; c < KS; ++c)
#pragma unroll
          for (int s = 0; s < 2; ++s) k[c][s] = lds_read<Vec>((at ^ (c << 5)) + s * 32 * L::kRowBytes);
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
          for (int j = 0; j < 16; ++j) x[s][j] = 0.0f;
#pragma unroll
        for (int c = 0; c < KS; ++c)
#pragma unroll
          for (int s = 0; s < 2; ++s) x[s] = Type<T>::dot32(k[c][s], q[c], x[s]);
        // four operands ahead of the products
        __builtin_amdgcn_sched_group_barrier(kDsRead, 4, 0);
#pragma unroll
        for (int c = 0; c < 2 * KS - 4; ++c) {
          __builtin_amdgcn_sched_group_barrier(kMfma, 1, 0);
          __builtin_amdgcn_sched_group_barrier(kDsRead, 1, 0);
        }
        __builtin_amdgcn_sched_group_barrier(kMfma, 4, 0);
        __builtin_amdgcn_sched_barrier(0);
      } else {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
#pragma unroll
          for (int j = 0; j < 16; ++j) x[s][j] = 0.0f;
#pragma unroll
          for (int c = 0; c < KS; ++c)
            x[s] = Type<T>::dot32(load8<T>(sh.k[i & 1] + L::at(s * 32 + col, c * 16 + half * 8)), q[c], x[s]);
          x[s] *= a.scale2;
        }
      }
    };

    // P^T of tile i out of S^T, and what was summed so far brought to its maximum
    auto weights = [&](int i, unsigned long long live) {
      const int b = k0 + i * kManyKeys;
      if (live != ~0ull || b + kManyKeys - 1 > wave_first || (a.window && b <= wave_last - a.window)) {
        // bit: this lane's query sees the key; the lane's keys begin at 4 half
        const int most = pos - b, least = a.window ? most - a.window : -1;
        unsigned long long seen = live;
        seen &= most < 0 ? 0 : most >= 63 ? ~0ull : (2ull << most) - 1;
        seen &= least < 0 ? ~0ull : least >= 63 ? 0 : ~0ull << (least + 1);
        seen >>= 4 * half;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          const unsigned bits = (unsigned)(seen >> (32 * s));
#pragma unroll
          for (int j = 0; j < 16; ++j) x[s][j] = bits & (1u << (8 * (j >> 2) + (j & 3))) ? x[s][j] : kNegInf;
        }
      }
      float top = x[0][0];
#pragma unroll
      for (int j = 1; j < 32; ++j) top = fmaxf(top, x[j >> 4][j & 15]);
      top = max_across_32(top);
      if (__builtin_amdgcn_ballot_w64((top - m) * sc > kLag<T, DP>)) {
        const float mn = fmaxf(m, top);
        const float fade = mn == kNegInf ? 1.0f : exp2_of((m - mn) * sc);
        l *= fade;
#pragma unroll
        for (int c = 0; c < DT; ++c) o[c] *= fade;
        m = mn;
      }
      const float ms = m == kNegInf ? 0.0f : m * sc;
#pragma unroll
      for (int j = 0; j < 32; ++j) {
        const float e = exp2_of(__builtin_fmaf(x[j >> 4][j & 15], sc, -ms));
        l += e;
        // the weights go to the matrix cores in the type of V, their sum stays in fp32
        pv[j >> 3][j & 7] = (T)e;
      }
    };

    // O^T += V^T P^T of tile i
    auto values = [&](int i) {
      if constexpr (sizeof(T) == 2) {
        unsigned at = v_at + (i & 1) * (int)sizeof(sh.v[0]);
        asm("" : "+v"(at));
        union Operand {
          i16x4 h[2];
          Vec v;
        } v[4][DT];
#pragma unroll
        for (int s = 0; s < 4; ++s)
#pragma unroll
          for (int c = 0; c < DT; ++c) {
            const unsigned to = (at ^ (c << 6)) + s * 16 * L::kRowBytes;
            v[s][c].h[0] = lds_read_transposed(to);
            v[s][c].h[1] = lds_read_transposed((to ^ L::kEight) + 8 * L::kRowBytes);
          }
#pragma unroll
        for (int s = 0; s < 4; ++s)
#pragma unroll
          for (int c = 0; c < DT; ++c) o[c] = Type<T>::dot32(v[s][c].v, pv[s], o[c]);
        __builtin_amdgcn_sched_group_barrier(kDsRead, 8, 1);
#pragma unroll
        for (int c = 0; c < 4 * DT - 4; ++c) {
          __builtin_amdgcn_sched_group_barrier(kMfma, 1, 1);
          __builtin_amdgcn_sched_group_barrier(kDsRead, 2, 1);
        }
        __builtin_amdgcn_sched_group_barrier(kMfma, 4, 1);
        __builtin_amdgcn_sched_barrier(0);
      } else {
#pragma unroll
        for (int s = 0; s < 4; ++s)
#pragma unroll
          for (int c = 0; c < DT; ++c) {
            union {
              Vec v;
              T t[8];
            } w;
            const int row = s * 16 + half * 4, d0 = c * 32 + (lane & 16);
            L::read4(sh.v[i & 1], row, d0, lane, w.t);
            L::read4(sh.v[i & 1], row + 8, d0, lane, w.t + 4);
            o[c] = Type<T>::dot32(w.v, pv[s], o[c]);
          }
      }
    };

    // ------------------------------------------------ the walk, in two phases a tile
    // Products (O += P V of the tile before, S = K Q of this one) and the softmax after
    // them alternate behind barriers.  Half of the waves, one of the two on each
    // SIMD, run a phase behind, so that one wave's products go beside the other's
    // softmax.  Stage i is K of tile i + 1 and V of tile i, which must be in LDS before
    // the products of tile i + 1; a wave stores its share of it among the products of
    // tile i, when both buffers are free, and sets off the next stage's loads.  Where a
    // wave has no more to see, its weights are zeros.
    const int late = NW == 8 && wave >= NW / 2 ? 1 : 0;
    sync();  // the last piece's tiles are done with
    if (tid == 0) sh.odd = 0;
    sync();
    if (n > 0) {
      const int page0 = valid(0, find(0));
      int v_pg = valid(1, find(1)), k_pg = valid(2, find(2));  // pages of stage i + 1 (V, K), while stage i is at hand
      int next_pg = find(3);  // not looked at before its time: that would wait for the loads before it
      unsigned long long live = live_of(0, page0), live1 = live_of(1, v_pg), live2 = live_of(2, k_pg);
      load_k(0, page0);
      clean(kr, live);
      store(sh.k[0], kr);
      load_k(1, v_pg);
      load_v(0, page0);
      clean(kr, live1);
      clean_v(0, live);
      sync();
      if (late) sync();
      for (int i = 0; i < n; ++i) {
        scores(i);
        // stage i: K of tile i + 1, V of tile i
        store(sh.k[(i + 1) & 1], kr);
        store(sh.v[i & 1], vr);
        load_k(i + 2, k_pg);
        load_v(i + 1, v_pg);
        __builtin_amdgcn_sched_barrier(0);
        if (i > 0) values(i - 1);
        sync();
        // among the softmax: what the stage on its way needs before it goes to LDS, and the next one's pages
        weights(i, live);
        if (live2 != ~0ull || a.D != DP) clean(kr, live2);
        if (live1 != ~0ull || a.D != DP || mixed(i + 1)) clean_v(i + 1, live1);
        v_pg = k_pg;
        k_pg = valid(i + 3, next_pg);
        live = live1, live1 = live2, live2 = live_of(i + 3, k_pg);
        next_pg = find(i + 4);
        sync();
      }
      values(n - 1);
      if (!late) sync();
      sync();
      if (sh.odd) {  // rare
        for (int i = 0; i < n; ++i)
          if (mixed(i))
            for (int key = 0; key < kManyKeys; ++key) {
              const int u = k0 + i * kManyKeys + key;
              const int page = u < hi ? table[u >> a.shift] : -1;
              if ((unsigned)page >= (unsigned)a.pages) continue;
              const T *vs = (const T *)a.v + page * a.v_page + (u & (P - 1)) * a.v_slot + (int64_t)h * a.v_head;
              if (!has_odd<T>(vs, a.D, lane)) continue;
              const T *ks = (const T *)a.k + page * a.k_page + (u & (P - 1)) * a.k_slot + (int64_t)h * a.k_head;
              float s = 0.0f;
#pragma unroll
              for (int c = 0; c < KS; ++c) s += dot8<T>(q[c], ks, c * 16 + half * 8, a.D);
              s = sum_across_32(s);
              if constexpr (sizeof(T) == 4) s *= a.scale2;
              const float e = exp2_of((s - m) * sc);
              const bool seen = u <= pos && (!a.window || u > pos - a.window);
#pragma unroll
              for (int c = 0; c < DT; ++c)
#pragma unroll
                for (int j = 0; j < 16; j += 4)
                  add_odd<T>(vs, c * 32 + 2 * j + 4 * half, a.D, e, seen, [&](int k, float y) { o[c][j + k] += y; });
            }
      }
    }

    // ------------------------------------------------ out, or to the join
    l = sum_across_32(l);
    if (l != l) m = __builtin_inff();  // NaN among the scores: the whole row is NaN
    if (pc.slot >= 0) {
      const int64_t s = (int64_t)pc.slot * a.Hkv + h;
      float *dst = a.part + s * (ROWS * (DP + 2));
      const int i = wave * 32 + col;
      if (have_row) {
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
          for (int j = 0; j < 4; ++j)
            *reinterpret_cast<f32x4 *>(dst + (int64_t)i * DP + t * 32 + j * 8 + half * 4) =
                f32x4{o[t][4 * j], o[t][4 * j + 1], o[t][4 * j + 2], o[t][4 * j + 3]};
        if (half == 0) {
          dst[ROWS * DP + i * 2] = m;
          dst[ROWS * DP + i * 2 + 1] = l;
        }
      }
      if (tid == 0) {
        int32_t *mt = a.meta + (1 + s) * kMeta;
        mt[0] = pc.part == 0 ? pc.np : 0;
        mt[1] = rq.first * a.G + first;
        mt[2] = rows;
        mt[3] = h;
      }
    } else if (have_row) {
      const float inv = m == kNegInf ? 0.0f : 1.0f / l;
      T *dst = (T *)a.out + ((int64_t)tok * a.Hq + head) * a.D;
#pragma unroll
      for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int d = t * 32 + j * 8 + half * 4;
          if (d < a.D) {
            union {
              T t[4];
              typename Pack4<T>::V v;
            } w;
#pragma unroll
            for (int k = 0; k < 4; ++k) w.t[k] = (T)(m == kNegInf ? 0.0f : o[t][4 * j + k] * inv);
            *reinterpret_cast<typename Pack4<T>::V *>(dst + d) = w.v;
          }
        }
      if (half == 0 && a.lse)
        a.lse[(int64_t)tok * a.Hq + head] = m == kNegInf ? kNegInf : m * (sc * kLn2) + __logf(l);
    }
  }
}

// ------------------------------------------------------------------ the join
//
// Adds the pieces of one row of a split tile: the largest of their maxima, their
// sums and values rescaled to it, in the order of the pieces.  A block goes through
// every gridDim.x-th slot that is a tile's first piece and every gridDim.y-th row of
// it.  The pieces of a tile are Hkv slots apart.

constexpr int kJoinBlock = 256;

template <class T, int DP>
__global__ __launch_bounds__(kJoinBlock) void join_few(AttendArgs a) {
  constexpr int ROWS = kFewRows;
  constexpr int kLanes = DP / 4;                    // threads of a row
  constexpr int kSide = kJoinBlock / kLanes;        // pieces side by side
  __shared__ float acc[kSide][DP];
  __shared__ float weight[kJoinBlock];
  __shared__ float red[2][kJoinBlock / kWave];
  const float sc = score_unit<T>(a);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int used = a.meta[0];
  for (int64_t s = blockIdx.x; s < used; s += gridDim.x) {
    const int32_t *mt = a.meta + (1 + s) * kMeta;
    const int np = mt[0];
    if (np <= 1) continue;
    constexpr int64_t kSize = (int64_t)ROWS * (DP + 2);
    const float *part = a.part + s * kSize;
    const int64_t next = (int64_t)a.Hkv * kSize;
    for (int i = blockIdx.y; i < mt[2]; i += gridDim.y) {
      const float *ml = part + ROWS * DP + i * 2;
      float mx = kNegInf;
      for (int j = tid; j < np; j += kJoinBlock) mx = fmaxf(mx, ml[j * next]);
#pragma unroll
      for (int o = 32; o; o >>= 1) mx = fmaxf(mx, __shfl_xor(mx, o));
      if (lane == 0) red[0][wave] = mx;
      __syncthreads();
#pragma unroll
      for (int w = 0; w < kJoinBlock / kWave; ++w) mx = fmaxf(mx, red[0][w]);
      const int c = (tid % kLanes) * 4, g = tid / kLanes;
      f32x4 o{0, 0, 0, 0};
      float sum = 0.0f;
      for (int j0 = 0; j0 < np; j0 += kJoinBlock) {
        const int j = j0 + tid;
        float w = 0.0f;
        if (j < np) {
          const float mj = ml[j * next];
          w = mj == kNegInf ? 0.0f : exp2_of((mj - mx) * sc);
          sum += w == 0.0f ? 0.0f : w * ml[j * next + 1];
        }
        __syncthreads();
        weight[tid] = w;
        __syncthreads();
        const int n = imin(np - j0, kJoinBlock);
#pragma unroll 8
        for (int k = g; k < n; k += kSide) {
          const f32x4 x = *reinterpret_cast<const f32x4 *>(part + (j0 + k) * next + i * DP + c);
          const float f = weight[k];
          if (f != 0.0f) o += x * f;
        }
      }
#pragma unroll
      for (int k = 32; k; k >>= 1) sum += __shfl_xor(sum, k);
      if (lane == 0) red[1][wave] = sum;
      *reinterpret_cast<f32x4 *>(&acc[g][c]) = o;
      __syncthreads();
      sum = 0.0f;
#pragma unroll
      for (int w = 0; w < kJoinBlock / kWave; ++w) sum += red[1][w];
      const int row = mt[1] + i, t = row / a.G, hd = mt[3] * a.G + row % a.G;
      const int64_t at = (int64_t)t * a.Hq + hd;
      if (tid < a.D) {
        float v = 0.0f;
#pragma unroll
        for (int k = 0; k < kSide; ++k) v += acc[k][tid];
        ((T *)a.out)[at * a.D + tid] = (T)(mx == kNegInf ? 0.0f : v / sum);
      }
      if (tid == 0 && a.lse) a.lse[at] = mx == kNegInf ? kNegInf : mx * (sc * kLn2) + __logf(sum);
      __syncthreads();
    }
  }
}

// The same for the tiles of attend_many: many rows of few pieces, a wave per row.
// Bound by memory and by the chain of its loads, so a wave has two rows on their way: 27 us behind the 559 GFLOP above, 7
// behind the window's batch, 10 behind the one in 4 bits (one row after the other 34, 9 and 13; one row a wave 44, 18
// and 13; four rows 11 for the last).
constexpr int kJoinRows = 8;  // rows of a block, two of them side by side in each wave

template <class T, int DP, int ROWS>
__global__ __launch_bounds__(kJoinBlock) void join_many(AttendArgs a) {
  constexpr int C = DP / 64;  // columns of a lane
  const float sc = score_unit<T>(a);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  constexpr int64_t kSize = (int64_t)ROWS * (DP + 2);
  const int64_t next = (int64_t)a.Hkv * kSize;
  const int used = a.meta[0];
  for (int64_t s = blockIdx.x; s < used; s += gridDim.x) {
    const int32_t *mt = a.meta + (1 + s) * kMeta;
    const int np = mt[0], rows = mt[2];
    if (np <= 1) continue;
    constexpr int kSide = kJoinRows / (kJoinBlock / kWave);  // rows of a wave
    const int i0 = blockIdx.y * kJoinRows + wave;
    if (i0 >= rows) continue;
    const float *part[kSide], *ml[kSide];
    float mx[kSide], sum[kSide], o[kSide][C];
#pragma unroll
    for (int k = 0; k < kSide; ++k) {
      const int i = i0 + k * (kJoinBlock / kWave) < rows ? i0 + k * (kJoinBlock / kWave) : i0;
      part[k] = a.part + s * kSize + i * DP + lane * C;
      ml[k] = a.part + s * kSize + ROWS * DP + i * 2;
      mx[k] = kNegInf, sum[k] = 0.0f;
#pragma unroll
      for (int c = 0; c < C; ++c) o[k][c] = 0.0f;
    }
    for (int j = lane; j < np; j += kWave)
#pragma unroll
      for (int k = 0; k < kSide; ++k) mx[k] = fmaxf(mx[k], ml[k][j * next]);
#pragma unroll
    for (int n = 32; n; n >>= 1)
#pragma unroll
      for (int k = 0; k < kSide; ++k) mx[k] = fmaxf(mx[k], __shfl_xor(mx[k], n));
#pragma unroll 2
    for (int j = 0; j < np; ++j) {
      float x[kSide][C], mj[kSide], lj[kSide];
#pragma unroll
      for (int k = 0; k < kSide; ++k) {
        mj[k] = ml[k][j * next], lj[k] = ml[k][j * next + 1];
#pragma unroll
        for (int c = 0; c < C; ++c) x[k][c] = part[k][j * next + c];
      }
#pragma unroll
      for (int k = 0; k < kSide; ++k) {
        const float w = mj[k] == kNegInf ? 0.0f : exp2_of((mj[k] - mx[k]) * sc);
        if (w != 0.0f) {
          sum[k] += w * lj[k];
#pragma unroll
          for (int c = 0; c < C; ++c) o[k][c] += w * x[k][c];
        }
      }
    }
#pragma unroll
    for (int k = 0; k < kSide; ++k) {
      const int i = i0 + k * (kJoinBlock / kWave);
      if (i >= rows) break;
      const int row = mt[1] + i, t = row / a.G, hd = mt[3] * a.G + row % a.G;
      const int64_t at = (int64_t)t * a.Hq + hd;
#pragma unroll
      for (int c = 0; c < C; ++c)
        if (lane * C + c < a.D) ((T *)a.out)[at * a.D + lane * C + c] = (T)(mx[k] == kNegInf ? 0.0f : o[k][c] / sum[k]);
      if (lane == 0 && a.lse) a.lse[at] = mx[k] == kNegInf ? kNegInf : mx[k] * (sc * kLn2) + __logf(sum[k]);
    }
  }
}

}  // namespace paged
}  // namespace slnr
