// Attention of many queries over selected pages, by pages: where a page is
// selected by several queries it is read once for all of them instead of once for each.
//
// The selection (a row per token and KV head, its columns the pages) is transposed by
// counting: how many queries select a page, where its list of them begins, the lists.
// attend_pages then takes a page and up to 128 rows (queries of its list, heads of the
// group) as two dense products with a softmax over the page's keys between them, and
// join_pages adds a query's pages up in the order of its selection, so results do
// not depend on the order within the lists, which the counting leaves open.
//
// What it moves: every selected page once, and D + 2 values in 32 bits per row and page,
// written and read; against 2 P D values per query and page that the walk by queries
// (attend_few) gathers.  2020 tokens over 16 pages of 64 keys, 32 / 8 heads of 128 in
// bf16: 545 MB there and back and 360 MB of pages, in 46 us for the lists, 4 times 60 for the
// pages and 4 times 29 for the join; by queries 8.5 GB are gathered.
#pragma once

#include "attend.hpp"

namespace slnr {
namespace paged {

struct PagesArgs {
  int32_t *count, *begin, *tile_begin;  // per bucket (h, r, b): queries, where their list and their tiles begin
  int32_t *total;                       // tiles in all
  int32_t *rank;                        // per (token, h, j): place in its page's list, -1: no page
  int32_t *list;                        // (token - t0) * top + j
  int32_t *tile;                        // bucket of a tile
  float *part, *ml;                     // per (token, h - h0, j, g): DP values; maximum and sum
  int32_t t0, tokens, buckets, per_tile;  // per_tile: queries of a tile
  int32_t h0, heads;                    // the KV heads of this launch
};

constexpr int kPagesBlock = 256;
constexpr int kPagesRows = 128;
constexpr int kPagesKeys = 64;

static __global__ __launch_bounds__(kPagesBlock) void pages_clear(PagesArgs p) {
  const int i = blockIdx.x * kPagesBlock + threadIdx.x;
  if (i < p.buckets) p.count[i] = 0;
}

// The page of entry i = (token, h, j) of the selection: its bucket, or -1 if there is none to see.
__device__ __forceinline__ int bucket_of(const AttendArgs &a, const PagesArgs &p, int i) {
  const int j = i % a.top, h = (i / a.top) % a.Hkv, t = p.t0 + i / (a.top * a.Hkv);
  const int b = a.sel[((int64_t)t * a.Hkv + h) * a.top + j];
  if (b < 0 || b >= a.W) return -1;
  int x = 0, y = a.R - 1;  // the last request that begins at or before t
  while (x < y) {
    const int mid = (x + y + 1) >> 1;
    if (a.qptr[mid] <= t)
      x = mid;
    else
      y = mid - 1;
  }
  const Request rq = request_of(a, x);
  if (t < rq.first || t >= rq.first + rq.n) return -1;
  const int pos = rq.S - rq.n + (t - rq.first);
  if ((int64_t)b << a.shift > pos) return -1;
  const int page = a.table[(int64_t)x * a.table_row + b];
  if ((unsigned)page >= (unsigned)a.pages) return -1;
  return (h * a.R + x) * a.W + b;
}

// Neighbouring lanes are neighbouring tokens: pages that all tokens select (the first, the
// last) are then counted once a wave: 21 us for the 2020 tokens above, most of it atomics
// on their way; one by one 28.
static __global__ __launch_bounds__(kPagesBlock) void pages_count(AttendArgs a, PagesArgs p) {
  const int e = blockIdx.x * kPagesBlock + threadIdx.x;
  const bool in = e < p.tokens * a.Hkv * a.top;
  const int i = in ? (e % p.tokens) * a.Hkv * a.top + e / p.tokens : 0;  // (h, j) slowest
  const int bucket = in ? bucket_of(a, p, i) : -1;
  int rank = -1;
  const unsigned long long some = __builtin_amdgcn_ballot_w64(bucket >= 0);
  if (some) {
    const int lane = threadIdx.x & 63, lead = __builtin_ctzll(some);
    const int common = __shfl(bucket, lead);
    const unsigned long long same = __builtin_amdgcn_ballot_w64(bucket == common);
    // one atomic a lane, on their way together
    const bool shared = bucket == common;
    int got = 0;
    if (bucket >= 0 && (!shared || lane == lead)) got = atomicAdd(&p.count[bucket], shared ? __popcll(same) : 1);
    const int base = __shfl(got, lead);
    if (bucket >= 0) rank = shared ? base + __popcll(same & ((1ull << lane) - 1)) : got;
  }
  if (in) p.rank[i] = rank;
}

// Running sums over the buckets, by one block: a share of them per thread, then a scan.
constexpr int kScanBlock = 1024;

static __global__ __launch_bounds__(kScanBlock) void pages_scan(PagesArgs p) {
  __shared__ int wave_a[kScanBlock / kWave], wave_b[kScanBlock / kWave];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int per = (p.buckets + kScanBlock - 1) / kScanBlock;
  const int i0 = imin(tid * per, p.buckets), i1 = imin(i0 + per, p.buckets);
  int n = 0, m = 0;
#pragma unroll 8
  for (int i = i0; i < i1; ++i) {
    const int c = p.count[i];
    n += c;
    m += (c + p.per_tile - 1) / p.per_tile;
  }
  int x = n, y = m;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int px = __shfl_up(x, o), py = __shfl_up(y, o);
    if (lane >= o) x += px, y += py;
  }
  if (lane == 63) wave_a[wave] = x, wave_b[wave] = y;
  __syncthreads();
  int all = 0;
#pragma unroll
  for (int i = 0; i < kScanBlock / kWave; ++i) {
    if (i < wave) x += wave_a[i], y += wave_b[i];
    all += wave_b[i];
  }
  x -= n, y -= m;
#pragma unroll 8
  for (int i = i0; i < i1; ++i) {
    const int c = p.count[i];
    p.begin[i] = x;
    p.tile_begin[i] = y;
    x += c;
    y += (c + p.per_tile - 1) / p.per_tile;
  }
  if (tid == 0) *p.total = all;
}

static __global__ __launch_bounds__(kPagesBlock) void pages_fill(AttendArgs a, PagesArgs p) {
  const int i = blockIdx.x * kPagesBlock + threadIdx.x;
  if (i >= p.tokens * a.Hkv * a.top) return;
  const int rank = p.rank[i];
  if (rank < 0) return;
  const int bucket = bucket_of(a, p, i);
  const int j = i % a.top, t = i / (a.top * a.Hkv);
  p.list[p.begin[bucket] + rank] = t * a.top + j;
  if (rank % p.per_tile == 0) p.tile[p.tile_begin[bucket] + rank / p.per_tile] = bucket;
}

template <class T, int DP>
struct PagesShared {
  T k[kPagesKeys * Tile<T, DP>::kStride];
  T v[kPagesKeys * Tile<T, DP>::kStride];
  int odd;  // infinities or NaN were taken out of V
};

// A block of four waves, 32 rows each, as attend_many; a page is short, so nothing is
// pipelined here: other blocks on the compute unit fill the waits.  Bound by memory, by the
// partial results above all: 134 MB of them written, 130 MB read in 60 us, 4.4 TB/s.
template <class T, int DP>
__global__ __launch_bounds__(kPagesBlock, DP <= 128 ? 2 : 1) void attend_pages(AttendArgs a, PagesArgs pa) {
  typedef typename Type<T>::Vec Vec;
  typedef Tile<T, DP> L;
  constexpr int NT = kPagesBlock;
  constexpr int KS = DP / 16, DT = DP / 32, NC = DP / 8;
  constexpr int CH = kPagesKeys * NC / NT;  // chunks of K and of V that a thread carries
  constexpr int RS = NT / NC;               // rows between two of them
  extern __shared__ __align__(16) char raw[];
  PagesShared<T, DP> &sh = *reinterpret_cast<PagesShared<T, DP> *>(raw);
  const float sc = score_unit<T>(a);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int col = lane & 31, half = lane >> 5;
  const int per_head = a.R * a.W, last = pa.h0 + pa.heads;  // tiles lie by heads
  const int tile = pa.tile_begin[pa.h0 * per_head] + (int)blockIdx.x;
  if (tile >= (last < a.Hkv ? pa.tile_begin[last * per_head] : *pa.total)) return;
  const int bucket = pa.tile[tile];
  const int b = bucket % a.W, r = (bucket / a.W) % a.R, h = bucket / (a.W * a.R);
  const int e0 = (tile - pa.tile_begin[bucket]) * pa.per_tile;
  const int entries = imin(pa.count[bucket] - e0, pa.per_tile);
  const int32_t *list = pa.list + pa.begin[bucket] + e0;
  const int page = a.table[(int64_t)r * a.table_row + b];
  const Request rq = request_of(a, r);
  const int before = rq.S - rq.n;
  const int P = 1 << a.shift, start = b << a.shift;
  const int keys = imin(P, rq.S - start);                // of the page that are written
  const bool mixed = start + P - 1 > before;             // some new tokens may see a part only

  // ------------------------------------------------ the queries, as columns
  const int row = wave * 32 + col;
  const bool have_row = row < entries * a.G;
  const int entry = have_row ? row / a.G : 0, g = have_row ? row % a.G : 0;
  const int which = list[entry];  // (token - t0) * top + j
  const int t = which / a.top, j_of = which % a.top;
  const int pos = before + (pa.t0 + t - rq.first);
  Vec q[KS];
  {
    const T *src = (const T *)a.q + (int64_t)(pa.t0 + t) * a.q_token + (int64_t)(h * a.G + g) * a.q_head;
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
  const int c8 = (tid % NC) * 8, row_of = tid / NC;
  const bool in_row = c8 < a.D;
  const T *k_page = (const T *)a.k + page * a.k_page + (int64_t)h * a.k_head;
  const T *v_page = (const T *)a.v + page * a.v_page + (int64_t)h * a.v_head;
  const unsigned k_at = lds_address(sh.k) + L::k_first(col, half), v_at = lds_address(sh.v) + L::v_first(lane);
  if (tid == 0) sh.odd = 0;

  for (int k0 = 0; k0 < keys; k0 += kPagesKeys) {
    __syncthreads();
    Vec kr[CH], vr[CH];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int key = k0 + c * RS + row_of;
      const bool ok = in_row && key < keys;
      kr[c] = load8_global<T>(ok ? k_page + key * a.k_slot + c8 : (const T *)kZeroRow);
      vr[c] = load8_global<T>(ok ? v_page + key * a.v_slot + c8 : (const T *)kZeroRow);
    }
    if (mixed) {
      bool bad = false;
#pragma unroll
      for (int c = 0; c < CH; ++c) bad |= clean8<T>(vr[c]);
      if (__builtin_amdgcn_ballot_w64(bad)) sh.odd = 1;
    }
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int at = L::at(c * RS + row_of, c8);
      store8<T>(sh.k + at, kr[c]);
      store8<T>(sh.v + at, vr[c]);
    }
    __syncthreads();
    if (wave * 32 >= entries * a.G) continue;  // no rows for this wave
    // S^T = K Q^T
    f32x16 x[2];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
#pragma unroll
      for (int j = 0; j < 16; ++j) x[s][j] = 0.0f;
#pragma unroll
      for (int c = 0; c < KS; ++c) {
        Vec k;
        if constexpr (sizeof(T) == 2)
          k = lds_read<Vec>((k_at ^ (c << 5)) + s * 32 * L::kRowBytes);
        else
          k = load8<T>(sh.k + L::at(s * 32 + col, c * 16 + half * 8));
        x[s] = Type<T>::dot32(k, q[c], x[s]);
      }
      if constexpr (sizeof(T) == 4) x[s] *= a.scale2;
    }
    if (mixed || k0 + kPagesKeys > keys) {
      const int most = imin(pos - start, keys - 1) - k0 - 4 * half;  // the last key of the tile that the query sees
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int j = 0; j < 16; ++j)
          x[s][j] = s * 32 + 8 * (j >> 2) + (j & 3) <= most ? x[s][j] : kNegInf;
    }
    float top = x[0][0];
#pragma unroll
    for (int j = 1; j < 32; ++j) top = fmaxf(top, x[j >> 4][j & 15]);
    top = max_across_32(top);
    const float mn = fmaxf(m, top);
    const float ms = mn == kNegInf ? 0.0f : mn * sc;
    const float fade = exp2_of(m * sc - ms);
    m = mn;
    l *= fade;
    Vec pv[4];
#pragma unroll
    for (int j = 0; j < 32; ++j) {
      const float e = exp2_of(__builtin_fmaf(x[j >> 4][j & 15], sc, -ms));
      l += e;
      pv[j >> 3][j & 7] = (T)e;
    }
    if (k0)
#pragma unroll
      for (int c = 0; c < DT; ++c) o[c] *= fade;
#pragma unroll
    for (int s = 0; s < 4; ++s)
#pragma unroll
      for (int c = 0; c < DT; ++c) {
        union {
          Vec v;
          i16x4 h[sizeof(T)];
          T t[8];
        } w;
        if constexpr (sizeof(T) == 2) {
          const unsigned at = (v_at ^ (c << 6)) + s * 16 * L::kRowBytes;
          w.h[0] = lds_read_transposed(at);
          w.h[1] = lds_read_transposed((at ^ L::kEight) + 8 * L::kRowBytes);
        } else {
          const int from = s * 16 + half * 4, d0 = c * 32 + (lane & 16);
          L::read4(sh.v, from, d0, lane, w.t);
          L::read4(sh.v, from + 8, d0, lane, w.t + 4);
        }
        o[c] = Type<T>::dot32(w.v, pv[s], o[c]);
      }
  }
  __syncthreads();
  if (sh.odd) {  // rare: infinities and NaN of V to the rows that see them
    for (int key = 0; key < keys; ++key) {
      const T *vs = v_page + key * a.v_slot;
      if (!has_odd<T>(vs, a.D, lane)) continue;
      const T *ks = k_page + key * a.k_slot;
      float s = 0.0f;
#pragma unroll
      for (int c = 0; c < KS; ++c) s += dot8<T>(q[c], ks, c * 16 + half * 8, a.D);
      s = sum_across_32(s);
      if constexpr (sizeof(T) == 4) s *= a.scale2;
      const float e = exp2_of((s - m) * sc);
#pragma unroll
      for (int c = 0; c < DT; ++c)
#pragma unroll
        for (int j = 0; j < 16; j += 4)
          add_odd<T>(vs, c * 32 + 2 * j + 4 * half, a.D, e, start + key <= pos, [&](int k, float z) { o[c][j + k] += z; });
    }
  }
  l = sum_across_32(l);
  if (l != l) m = __builtin_inff();  // NaN among the scores: the whole row is NaN
  if (have_row) {
    const int64_t at = (((int64_t)t * pa.heads + (h - pa.h0)) * a.top + j_of) * a.G + g;
    float *dst = pa.part + at * DP;
#pragma unroll
    for (int c = 0; c < DT; ++c)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        *reinterpret_cast<f32x4 *>(dst + c * 32 + j * 8 + half * 4) =
            f32x4{o[c][4 * j], o[c][4 * j + 1], o[c][4 * j + 2], o[c][4 * j + 3]};
    if (half == 0) {
      pa.ml[at * 2] = m;
      pa.ml[at * 2 + 1] = l;
    }
  }
}

// The pages of one row (token, head) added up, a wave per row; eight pages' values on
// their way at a time.  Bound by memory: 136 MB in 29 us, 4.7 TB/s.
template <class T, int DP>
__global__ __launch_bounds__(kPagesBlock) void join_pages(AttendArgs a, PagesArgs pa) {
  constexpr int C = DP / 64;  // columns of a lane
  typedef float Cols __attribute__((ext_vector_type(C)));
  const float sc = score_unit<T>(a);
  const int lane = threadIdx.x & 63;
  const int64_t row = (int64_t)blockIdx.x * (kPagesBlock / kWave) + (threadIdx.x >> 6);  // of the launch's (token, head)
  const int share = pa.heads * a.G;
  if (row >= (int64_t)pa.tokens * share) return;
  const int t = (int)(row / share), hs = (int)(row % share) / a.G, g = (int)(row % share) % a.G;
  const int h = pa.h0 + hs, hd = h * a.G + g;
  const int tok = pa.t0 + t;
  if (tok < a.qptr[0] || tok >= a.qptr[a.R]) return;  // of no request
  const int64_t first = ((int64_t)t * pa.heads + hs) * a.top;
  const int32_t *rank = pa.rank + ((int64_t)t * a.Hkv + h) * a.top;
  float mx = kNegInf;
  for (int j = lane; j < a.top; j += kWave)
    if (rank[j] >= 0) mx = fmaxf(mx, pa.ml[((first + j) * a.G + g) * 2]);
#pragma unroll
  for (int o = 32; o; o >>= 1) mx = fmaxf(mx, __shfl_xor(mx, o));
  float sum = 0.0f;
  Cols o;
#pragma unroll
  for (int c = 0; c < C; ++c) o[c] = 0.0f;
#pragma unroll 8
  for (int j = 0; j < a.top; ++j) {
    const int64_t at = (first + j) * a.G + g;
    const bool there = rank[j] >= 0;
    const Cols x = *reinterpret_cast<const Cols *>(pa.part + at * DP + lane * C);
    const float mj = there ? pa.ml[at * 2] : kNegInf, lj = pa.ml[at * 2 + 1];
    const float w = mj == kNegInf ? 0.0f : exp2_of((mj - mx) * sc);
    if (w != 0.0f) {
      sum += w * lj;
      o += x * w;
    }
  }
  const int64_t at = (int64_t)tok * a.Hq + hd;
  T *dst = (T *)a.out + at * a.D + lane * C;
#pragma unroll
  for (int c = 0; c < C; ++c)
    if (lane * C + c < a.D) dst[c] = (T)(mx == kNegInf ? 0.0f : o[c] / sum);
  if (lane == 0 && a.lse) a.lse[at] = mx == kNegInf ? kNegInf : mx * (sc * kLn2) + __logf(sum);
}

}  // namespace paged
}  // namespace slnr
