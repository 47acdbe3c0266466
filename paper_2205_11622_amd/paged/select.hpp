// Which pages a query attends: a cheap score of every page and an exact top-k.
#pragma once

#include "common.hpp"

namespace slnr {
namespace paged {

struct SelectArgs {
  const void *q;  // [T][Hq][D]
  int64_t q_token, q_head;
  const int8_t *kq;     // [pages][Hkv][D]
  const float *kscale;  // [pages][Hkv]
  const int32_t *table;
  int64_t table_row;
  const int32_t *seq, *qptr;
  int32_t *sel;  // [T][Hkv][top]
  int32_t R, T, W, pages, shift, Hkv, G, D, top, first, local;
  int32_t tile0;     // number of the launch's first tile
  int32_t capacity;  // entries of a row in LDS: top carried ones, then a segment of pages
};

constexpr int kSelectWaves = 16;
constexpr int kSelectBlock = kSelectWaves * kWave;
constexpr int kSelectMaxTop = 256;

// Keys that order as the scores do, as unsigned numbers: 0 is no page, ~0 one that
// is always taken.  NaN ranks above every number (the minimum of NaN and a number is the
// number), and -0 and 0 are one score.
__device__ __forceinline__ unsigned rank_of(float s) {
  const float big = 3.402823466e38f;
  const unsigned b = __float_as_uint(fmaxf(fminf(s, big), -big) + 0.0f);
  return b ^ (unsigned)((int)b >> 31 | (int)0x80000000);
}

// The largest `cut` that at least `top` of the wave's values reach (there are more than
// `top` values above 0), found bit by bit; `reach` is how many do.
__device__ __forceinline__ unsigned kth_largest(unsigned v, int top, int &reach) {
  unsigned cut = 0;
  for (int bit = 31; bit >= 0; --bit) {
    const unsigned next = cut | (1u << bit);
    const int c = __popcll(__builtin_amdgcn_ballot_w64(v >= next));
    if (c >= top) {
      cut = next;
      reach = c;
      if (c == top) break;
    }
  }
  return cut;
}

constexpr int kSelectFew = 64;  // as many pages as a wave has lanes

// The `top` <= 64 largest of a wave's values above 0, v[i] in lane l being number 64 i + l,
// equal ones by the lowest number: lane e < kept gets the e-th of them in the order of
// the numbers.  The top-th largest of the lanes' maxima bounds the answer from
// below, and few values are above it; they are put one to a lane through `room` (128
// words), where the search goes on.  False, if there are more than 64 of them.
template <int NR>
__device__ __forceinline__ bool choose_few(const unsigned (&v)[NR], int top, unsigned *room, int lane, int &kept,
                                           unsigned &key, int &number) {
  unsigned most = v[0];
#pragma unroll
  for (int i = 1; i < NR; ++i) most = most > v[i] ? most : v[i];
  unsigned low = 1;
  int reach = 0;
  if (__popcll(__builtin_amdgcn_ballot_w64(most > 0)) > top) low = kth_largest(most, top, reach);
  int n = 0;
  const unsigned long long below = (1ull << lane) - 1;
#pragma unroll
  for (int i = 0; i < NR; ++i) {
    const unsigned long long b = __builtin_amdgcn_ballot_w64(v[i] >= low);
    if (b) {
      const int at = n + __popcll(b & below);
      if (v[i] >= low && at < kWave) {
        room[at] = v[i];
        room[kWave + at] = i * kWave + lane;
      }
      n += __popcll(b);
    }
  }
  if (n > kWave) return false;
  key = lane < n ? room[lane] : 0;
  number = lane < n ? (int)room[kWave + lane] : 0;
  kept = n;
  if (n > top) {
    reach = n;
    const unsigned c = kth_largest(key, top, reach);
    const unsigned long long over = __builtin_amdgcn_ballot_w64(key > c), tied = __builtin_amdgcn_ballot_w64(key == c);
    const int ties = top - __popcll(over);
    const bool take = key > c || (key == c && __popcll(tied & below) < ties);
    const unsigned long long b = __builtin_amdgcn_ballot_w64(take);
    if (take) {
      room[__popcll(b & below)] = key;
      room[kWave + __popcll(b & below)] = number;
    }
    kept = top;
    key = lane < kept ? room[lane] : 0;
    number = lane < kept ? (int)room[kWave + lane] : 0;
  }
  return true;
}

// Scores: the group's query heads are added up in 64 bits, rounded once and cut to
// 8 bits; its product with a page's 8-bit mean key is a whole number below 2^24,
// exact on the integer matrix cores, and the page's step makes it the score.  So a
// score has one rounding, in no order, and equal scores are equal numbers.
//
// A block takes TM tokens of one request and one KV head: 16 (rows of the 16 x 16
// x 64 products, one wave per token in the choice) or one (a decode step: all 16 waves
// share the choice).  Scores stay in LDS as keys; a longer context is taken in
// segments, the best so far carried in front of the next one, which keeps the
// order of the indices.  Up to 64 pages are chosen as choose_few says (one token: by every
// wave among its pages, then by the first wave among those).  More of them, or
// too many equal scores: the k-th largest key is found bit by bit, with a count over
// the row per bit, up to the first prefix that exactly k keys reach; equal keys
// at the end go by the lowest index.
//
// Bound by latency: the table, the summaries behind it, the choice's steps one after
// the other.  32 tokens, 8 heads of 128, contexts of 8302 to 55936 in pages of 64 (13 MB):
// 16 us; 2020 tokens behind 34227 and 40918 (19 MB, 2.5 Gop): 53 us, of which vector instructions
// fill a third.  There two blocks share a compute unit (64 registers to a wave): us with / with one block of 128, 128
// columns 2 requests of 1000 behind 30000 47 / 55, 8 of 250 behind 4000 28 / 38, 1 of 4000 behind 30000 70 / 88; 64 columns 43 / 46, 25 /
// 25, 63 / 65.
//
// NR: keys of a row that a lane holds in the choice.
template <class T, int DP, int TM, int NR>
__global__ __launch_bounds__(kSelectBlock, TM > 1 && NR <= 16 && DP <= 128 ? 8 : 4) void block_select(SelectArgs a) {
  constexpr int KS = DP / 64;
  constexpr int WPR = kSelectWaves / TM;  // waves of a row in the choice
  static_assert(TM == 1 || TM == kSelectWaves, "one wave per token, or all for one");
  extern __shared__ __align__(16) char raw[];
  const int stride = a.capacity + 4;
  unsigned *keys = reinterpret_cast<unsigned *>(raw);               // [TM][stride]
  int *carried = reinterpret_cast<int *>(keys + TM * stride);       // [TM][top], indices
  int8_t *q8 = reinterpret_cast<int8_t *>(carried + TM * a.top + ((-TM * a.top) & 3));  // [16][DP + 16]
  constexpr int QS = DP + 16;
  int *count = reinterpret_cast<int *>(q8 + 16 * QS);               // [2][16] of the waves
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int col = lane & 15, grp = lane >> 4;
  const int h = blockIdx.y;

  // ------------------------------------------------------ which tokens
  // TM = 16: request r's tiles begin at number floor(qptr[r] / 16) + r, which leaves
  // room for all of them and never runs back.  TM = 1: token by token.
  const int id = a.tile0 + (int)blockIdx.x;
  auto start = [&](int r) {
    int b = a.qptr[r];
    b = b < 0 ? 0 : b > a.T ? a.T : b;
    return TM == 1 ? b : b / TM + r;
  };
  int x = 0, y = a.R - 1;
  while (x < y) {
    const int mid = (x + y + 1) >> 1;
    if (start(mid) <= id)
      x = mid;
    else
      y = mid - 1;
  }
  const int r = x;
  int qb = a.qptr[r], qe = a.qptr[r + 1];
  qb = qb < 0 ? 0 : qb > a.T ? a.T : qb;
  qe = qe < 0 ? 0 : qe > a.T ? a.T : qe;
  const int t0 = qb + (id - start(r)) * TM;
  if (id < start(r) || t0 >= qe) return;
  const int tokens = qe - t0 < TM ? qe - t0 : TM;
  const int64_t row_ends = (int64_t)a.W << a.shift;  // a longer request ends with its table's row, as in attention
  int seq = a.seq[r];
  seq = seq < 0 ? 0 : seq < row_ends ? seq : (int)row_ends;
  const int pos0 = seq - (qe - qb) + (t0 - qb);  // position of the first token
  const int pos1 = pos0 + tokens - 1;
  const int32_t *table = a.table + (int64_t)r * a.table_row;
  const int near1 = pos1 < 0 ? -1 : pos1 >> a.shift;
  const int blocks = near1 + 1 < a.W ? near1 + 1 : a.W;

  auto table_entry = [&](int b) { return b < blocks ? table[b] : -1; };
  constexpr int U = TM == 1 ? 4 : 1;  // groups of 16 pages that a wave has on their way (16 tokens: two 55 us, one 53)
  int ahead[U];  // table entries of the next ones (a segment that is not the last has some for every wave)
#pragma unroll
  for (int u = 0; u < U; ++u) ahead[u] = table_entry((wave + u * kSelectWaves) * 16 + col);

  // ------------------------------------------------------ the queries in 8 bits
  if (wave < TM) {  // a wave per token
    float u[DP / 64];
    float most = 0.0f;
#pragma unroll
    for (int i = 0; i < DP / 64; ++i) {
      const int d = i * 64 + lane;
      double s = 0;
      if (wave < tokens && d < a.D) {
        const T *src = (const T *)a.q + (int64_t)(t0 + wave) * a.q_token + (int64_t)h * a.G * a.q_head + d;
#pragma unroll 4
        for (int g = 0; g < a.G; ++g) s += (double)(float)src[g * a.q_head];
      }
      u[i] = (float)s;
      const float z = fabsf(u[i]);
      most = z <= 3.402823466e38f ? fmaxf(most, z) : __builtin_inff();
    }
#pragma unroll
    for (int o = 32; o; o >>= 1) most = fmaxf(most, __shfl_xor(most, o));
    const bool fine = most < __builtin_inff();
    const float step = most * kStep127;
#pragma unroll
    for (int i = 0; i < DP / 64; ++i)
      q8[wave * QS + i * 64 + lane] = fine && step > 0.0f ? whole8(u[i], step) : (int8_t)0;
  }
  if (TM == 1)  // the other columns of the product are not used
    for (int i = tid; i < 15 * QS; i += kSelectBlock) q8[QS + i] = 0;
  __syncthreads();
  i32x4 qv[KS];
#pragma unroll
  for (int i = 0; i < KS; ++i) qv[i] = *reinterpret_cast<const i32x4 *>(q8 + col * QS + i * 64 + grp * 16);

  const int near0 = pos0 < 0 ? -1 : pos0 >> a.shift;  // page of the first token
  const int my_token = TM == 1 ? 0 : wave;                   // row of the choice
  const int room_of_segment = a.capacity - a.top;
  int held = 0;                                              // carried entries of my row
  for (int seg = 0; seg == 0 || seg < blocks; seg += room_of_segment) {
    const int n = blocks - seg < room_of_segment ? (blocks - seg > 0 ? blocks - seg : 0) : room_of_segment;
    // ---------------------------------------------------- scores of a segment
    // Rows of the product are the tokens, columns 16 pages, so a lane has one page for
    // four tokens.  U groups at once: their entries, then their summaries are on their
    // way together.
    for (int g0 = wave * 16; g0 < n; g0 += U * kSelectWaves * 16) {
      int page[U];
      const int next = g0 + U * kSelectWaves * 16 < n ? seg + g0 + U * kSelectWaves * 16 : seg + room_of_segment + wave * 16;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        page[u] = ahead[u];
        ahead[u] = table_entry(next + u * kSelectWaves * 16 + col);
      }
      i32x4 kv[U][KS];
      float scale[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if ((unsigned)page[u] >= (unsigned)a.pages) page[u] = -1;
        const int64_t row = (int64_t)(page[u] < 0 ? 0 : page[u]) * a.Hkv + h;
        const int8_t *src = page[u] < 0 ? (const int8_t *)kZeroRow : a.kq + row * a.D;
#pragma unroll
        for (int i = 0; i < KS; ++i) {
          const int d = i * 64 + grp * 16;
          typedef const __attribute__((address_space(1))) uint2 *G;
          union {
            i32x4 v;
            uint2 u[2];
          } w;
          const G g = (G)(d < a.D ? src + d : (const int8_t *)kZeroRow);
          const G g8 = (G)(d + 8 < a.D ? src + d + 8 : (const int8_t *)kZeroRow);
          w.u[0].x = g->x, w.u[0].y = g->y;
          w.u[1].x = g8->x, w.u[1].y = g8->y;
          kv[u][i] = w.v;
        }
        scale[u] = page[u] < 0 ? 0.0f : a.kscale[row];
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int b0 = g0 + u * kSelectWaves * 16;
        if (b0 >= n) break;
        i32x4 acc{0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < KS; ++i) acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(qv[i], kv[u][i], acc, 0, 0, 0);
        unsigned key[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) key[i] = rank_of(__fmul_rn((float)acc[i], scale[u]));
        const int bb = seg + b0 + col;
        // all pages there, seen by all tokens and chosen by score alone, as most are
        if (seg + b0 < a.first || seg + b0 + 15 > near0 - a.local || b0 + 15 >= n ||
            __builtin_amdgcn_ballot_w64(page[u] < 0)) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int p = pos0 + grp * 4 + i;
            const int near = p < 0 ? -1 : p >> a.shift;
            if (bb < a.first || bb > near - a.local) key[i] = ~0u;
            if (page[u] < 0 || bb > near) key[i] = 0;
          }
        }
        if (b0 + col < n && (TM > 1 || grp == 0)) {
          unsigned *dst = keys + grp * 4 * stride + a.top + b0 + col;
#pragma unroll
          for (int i = 0; i < (TM == 1 ? 1 : 4); ++i) dst[i * stride] = key[i];
        }
      }
    }
    __syncthreads();

    // ---------------------------------------------------- the best of carried and new
    // Entries: the carried ones at [top - held, top), then the segment's n.
    unsigned *row = keys + my_token * stride;
    int *names = carried + my_token * a.top;
    const int first_entry = a.top - held, entries = held + n;
    const int base = TM == 1 ? wave * (NR * kWave) : 0;  // a wave's entries are one run of them
    unsigned v[NR];
#pragma unroll
    for (int i = 0; i < NR; ++i) {
      const int e = base + i * kWave + lane;
      v[i] = e < entries ? row[first_entry + e] : 0;
    }
    const bool last = seg + room_of_segment >= blocks;
    int32_t *dst = a.sel + ((int64_t)(t0 + my_token) * a.Hkv + h) * a.top;
    const bool mine = my_token < tokens;
    bool done = false;
    // Two numbers a lane of LDS for a wave: the row that is now in registers, or (one
    // token) the words behind the counts.
    unsigned *room = TM == 1 ? reinterpret_cast<unsigned *>(count + 2 * kSelectWaves) + wave * 2 * kWave : row + a.top;
    if (a.top <= kSelectFew) {
      int kept;
      unsigned key;
      int number;
      done = choose_few(v, a.top, room, lane, kept, key, number);
      if constexpr (WPR > 1) {
        // every wave's choice behind the one of the wave before, then once more among them
        if (lane == 0) count[wave] = done ? kept : kWave + 1;
        __syncthreads();
        int before = 0, all = 0;
#pragma unroll
        for (int w = 0; w < kSelectWaves; ++w) {
          const int c = count[w];
          done = done && c <= kWave;
          if (w < wave) before += c;
          all += c;
        }
        if (done) {  // in all waves or in none
          number = base + number;
          const int name = number < held ? names[number] : seg + (number - held);
          unsigned *list = room - wave * 2 * kWave + kSelectWaves * 2 * kWave;
          if (lane < kept) list[before + lane] = key, list[kSelectWaves * kWave + before + lane] = (unsigned)name;
          __syncthreads();
          if (wave == 0) {
            unsigned c[kSelectWaves];
#pragma unroll
            for (int i = 0; i < kSelectWaves; ++i) c[i] = i * kWave + lane < all ? list[i * kWave + lane] : 0;
            done = choose_few(c, a.top, room, lane, kept, key, number);
            if (done && lane < kept) {
              const int chosen = (int)list[kSelectWaves * kWave + number];
              if (last) {
                dst[lane] = chosen;
              } else {
                names[lane] = chosen;
                row[a.top - kept + lane] = key;
              }
            }
            if (done && last && lane >= kept && lane < a.top) dst[lane] = -1;
            if (lane == 0) count[kSelectWaves] = done ? kept : -1;
          }
          __syncthreads();
          held = count[kSelectWaves] < 0 ? held : count[kSelectWaves];
          done = count[kSelectWaves] >= 0;
        }
        __syncthreads();
      } else if (done) {
        int name = 0;
        if (lane < kept) name = number < held ? names[number] : seg + (number - held);
        if (last) {
          if (mine && lane < a.top) dst[lane] = lane < kept ? name : -1;
        } else if (lane < kept) {
          names[lane] = name;
          row[a.top - kept + lane] = key;
        }
        held = kept;
      }
    }
    if (done) {
      __syncthreads();
      continue;
    }
    // Keys of the row that are at least `than`.
    int turn = 0;
    auto at_least = [&](unsigned than) {
      int c = 0;
#pragma unroll
      for (int i = 0; i < NR; ++i) c += __popcll(__builtin_amdgcn_ballot_w64(v[i] >= than));
      if constexpr (WPR > 1) {
        if (lane == 0) count[turn * kSelectWaves + wave] = c;
        __syncthreads();
        c = 0;
#pragma unroll
        for (int w = 0; w < kSelectWaves; ++w) c += count[turn * kSelectWaves + w];
        turn ^= 1;
      }
      return c;
    };
    unsigned cut = 1;  // keys from here on are taken
    int reach = at_least(1);
    if (reach > a.top) {
      cut = 0;
      for (int bit = 31; bit >= 0 && reach != a.top; --bit) {
        const unsigned next = cut | (1u << bit);
        const int c = at_least(next);
        if (c >= a.top) cut = next, reach = c;
      }
    }
    const int over = reach > a.top ? at_least(cut + 1) : reach;  // cut < ~0: fewer than top are forced
    const int ties = reach > a.top ? a.top - over : reach;       // keys equal to cut that are taken, lowest first
    const bool cut_ties = reach > a.top;
    // taken and tied entries before this wave's
    int out = 0, tied = 0;
    if constexpr (WPR > 1) {
      int c = 0, e = 0;
#pragma unroll
      for (int i = 0; i < NR; ++i) {
        c += __popcll(__builtin_amdgcn_ballot_w64(cut_ties ? v[i] > cut : v[i] >= cut));
        e += __popcll(__builtin_amdgcn_ballot_w64(cut_ties && v[i] == cut));
      }
      __syncthreads();
      if (lane == 0) count[wave] = c, count[kSelectWaves + wave] = e;
      __syncthreads();
      for (int w = 0; w < wave; ++w) out += count[w], tied += count[kSelectWaves + w];
      out += tied < ties ? tied : ties;
    }
    // Names of the entries: read before the carried ones are written over, by other
    // waves (one token) or by this one, which writes behind where it reads.
    auto name_of = [&](int i) {
      const int e = base + i * kWave + lane;
      return e < held ? names[e] : seg + (e - held);
    };
    int name[WPR > 1 ? NR : 1];
    if constexpr (WPR > 1) {
#pragma unroll
      for (int i = 0; i < NR; ++i) name[i] = name_of(i);
      __syncthreads();
    }
    int taken = out;
    const int kept = reach > a.top ? a.top : reach;  // entries that the row keeps
#pragma unroll
    for (int i = 0; i < NR; ++i) {
      const bool eq = cut_ties && v[i] == cut;
      const unsigned long long be = __builtin_amdgcn_ballot_w64(eq);
      const unsigned long long below = (1ull << lane) - 1;
      const bool take = (cut_ties ? v[i] > cut : v[i] >= cut) || (eq && tied + __popcll(be & below) < ties);
      const unsigned long long b = __builtin_amdgcn_ballot_w64(take);
      int its = 0;
      if constexpr (WPR > 1)
        its = name[i];
      else
        its = name_of(i);
      __builtin_amdgcn_wave_barrier();
      if (take) {
        const int at = taken + __popcll(b & below);
        if (last) {
          if (mine) dst[at] = its;
        } else {
          names[at] = its;
          row[a.top - kept + at] = v[i];
        }
      }
      taken += __popcll(b);
      tied += __popcll(be);
    }
    if (last && mine)
      for (int e = kept + (TM == 1 ? tid : lane); e < a.top; e += TM == 1 ? kSelectBlock : kWave) dst[e] = -1;
    held = kept;
    __syncthreads();
  }
}

}  // namespace paged
}  // namespace slnr
