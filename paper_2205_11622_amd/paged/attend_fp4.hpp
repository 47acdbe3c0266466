// Attention over a paged cache in 4 bits: as attend.hpp, with the split of the work, the softmax and
// the joins from there.  q.k is taken on the cache's bytes as they are; V becomes 16-bit
// values, exactly, on its way into LDS.
#pragma once

#include "fp4.hpp"

namespace slnr {
namespace paged {

// k, v: the bytes; all strides of the cache in bytes.
struct AttendFp4Args : AttendArgs {
  const uint8_t *ks, *vs;
  int64_t ks_page, ks_slot, ks_head, vs_page, vs_slot, vs_head;
  int32_t groups;  // of a row
};

// A weight as the sum of N values of the type of V: one for 16-bit results, three for 24 bits.
template <class V4, int N>
__device__ __forceinline__ void split_weight(float e, typename Type<V4>::Vec out[N], int at) {
#pragma unroll
  for (int p = 0; p < N; ++p) {
    const V4 w = (V4)e;
    out[p][at] = w;
    if (p + 1 < N) e -= (float)w;
  }
}

// Loads from device memory (see load8_global), and those of what is read once.
template <class V>
__device__ __forceinline__ V load_global(const uint8_t *p) {
  return *(const __attribute__((address_space(1))) V *)p;
}
template <class V>
__device__ __forceinline__ V load_once(const uint8_t *p) {
  return __builtin_nontemporal_load((const __attribute__((address_space(1))) V *)p);
}

// ------------------------------------------------------------- split of the work
//
// The steps of all tiles of a KV head, one request after the other, are one line of `all` steps that
// `n` blocks share evenly, so that all end at the same time: block i takes the steps from all i / n to
// all (i + 1) / n, which are the end of a tile, whole tiles and the beginning of one.  A tile that is
// cut has pieces in the blocks i0 .. i1; the first is the last thing that block i0 does, the others are the first
// thing that theirs do, so two places a block hold all pieces there are.
template <int NT>
struct Line {
  long long before[NT];  // steps before this thread's requests
  long long work[NT / kWave];
};

// The steps of a KV head.  count(r, tiles, steps) gives a request's tiles and the steps of each.
template <int NT, class F>
__device__ __forceinline__ long long line_scan(Line<NT> &sh, const AttendArgs &a, int per, F count) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int r0 = imin(tid * per, a.R), r1 = imin(r0 + per, a.R);
  long long w = 0;
  for (int r = r0; r < r1; ++r) {
    int tiles, steps;
    count(r, tiles, steps);
    w += (long long)tiles * imax(steps, 1);
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
  sh.before[tid] = upto - w;
  __syncthreads();
  return all;
}

// Whole numbers of a line: up to 2^28 rows of up to 2^23 steps, times n < 2^12, fit 64 bits.
__device__ __forceinline__ int block_of(long long step, int n, long long all) {
  return (int)(((step + 1) * n - 1) / all);
}

// --------------------------------------------------------------- few rows
//
// attend_few_fp4: as attend_few, tiles of 16 rows and blocks of four waves, each of which walks every fourth
// tile of 64 keys.  A lane loads 16 bytes of K, which are one group of a key and,
// with its exponent, an operand of a product over 128 dimensions; the query's pieces
// are the other.  V goes through LDS 32 keys at a time.  The next tile's K is on its way while this one's scores become weights,
// its V while the last products run; rows that are read once go past the caches (128 us, through them 137).  Memory: 96 single
// tokens of 32/8 heads of 128 in bf16, 584 MB, 122 us, 4.8 TB/s; the join 5.  Small batches are bound by latency: 3
// requests of up to 900 keys 11 us, their join 4.
constexpr int kFew4Keys = 64;                        // of a wave's tile
constexpr int kFew4Step = kFew4Keys * kFewWaves;     // of a block's step

// A tile of V in LDS (see Tile) whose 16-byte chunks are permuted for reads of 16 columns: LDS moves 128 bytes
// a cycle, which are two chunks of four rows in a read and one of eight rows in a write.  The permutation is an exclusive or and the same
// 16 rows on, so a lane's addresses differ from its first ones in single bits.
template <int DP>
struct Tile16 {
  static constexpr int kRowBytes = 2 * DP;
  static __device__ __forceinline__ unsigned chunk(int row) {
    return ((row & 3) << 1) | ((row >> 2) & 1) | (DP >= 128 ? row & 8 : 0);
  }
  // Columns column .. + 7 (a multiple of 8) of row `row` < 16; those 8 i on: ^ (i << 4).
  static __device__ __forceinline__ unsigned write_first(int row, int column) {
    return row * kRowBytes + (((column >> 3) ^ chunk(row)) << 4);
  }
  // Keys 4 (lane >> 4) .. + 3 of column lane & 15, by a transposing read; columns 16 i on: ^ (i << 5).
  static __device__ __forceinline__ unsigned read_first(int lane) {
    const int row = (lane >> 4) * 4 + ((lane >> 2) & 3), column = (lane & 3) * 4;
    return row * kRowBytes + (((column >> 3) ^ chunk(row)) << 4) + (column & 7) * 2;
  }
};

template <class T, int DP>
struct Few4Shared {
  typedef typename Four<T>::V4 V4;
  union {
    alignas(512) V4 v[kFewWaves][32 * DP];
    float o[kFewWaves][kFewRows * DP];
  };
  float m[kFewWaves][kFewRows], l[kFewWaves][kFewRows];
  Line<kFewBlock> line;
};

// Blocks of a compute unit that the registers leave room for.  Those 96 tokens: one block a unit 176 us, two 122, three
// (fewer registers, some of them in memory) 143.
template <class T, int DP>
constexpr int kFew4PerCu = DP == 256 ? 1 : 2;

template <class T, int DP, bool ONE_PAGE>
__global__ __launch_bounds__(kFewBlock, (kFew4PerCu<T, DP>)) void attend_few_fp4(AttendFp4Args a) {
  typedef typename Four<T>::V4 V4;
  typedef typename Type<V4>::Vec Vec;
  typedef Tile16<DP> L;
  constexpr int NQ = Four<T>::kQ, NP = Four<T>::kP;
  constexpr int DT = DP / 16;               // tiles of output columns
  constexpr int KR = DP == 256 ? 2 : 1;     // operands of a key
  constexpr int NM = DP == 64 ? (NQ + 1) / 2 : NQ * KR;  // products of 128 of the summed axis
  constexpr int VW = DP / 32;               // words of V of a lane and key
  constexpr int VS = DP == 256 ? 2 : 1;     // their groups
  extern __shared__ __align__(16) char raw[];
  Few4Shared<T, DP> &sh = *reinterpret_cast<Few4Shared<T, DP> *>(raw);
  const float sc = score_unit<T>(a);
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);  // a scalar: so are its tiles, their addresses and conditions
  const int col = lane & 15, grp = lane >> 4;
  const int P = 1 << a.shift;
  auto count = [&](int r, int &tiles, int &steps) {
    const Request q = request_of(a, r);
    const long long rows = (long long)q.n * a.G;
    tiles = rows > a.few ? 0 : (int)((rows + kFewRows - 1) / kFewRows);
    const int lo = (a.window ? imax(q.S - q.n - a.window + 1, 0) : 0) & -kFew4Keys;
    steps = (q.S - lo + kFew4Step - 1) / kFew4Step;
  };
  const int per = (a.R + kFewBlock - 1) / kFewBlock;
  const long long all = line_scan<kFewBlock>(sh.line, a, per, count);
  const int h = (int)(blockIdx.x % (unsigned)a.Hkv), me = (int)(blockIdx.x / (unsigned)a.Hkv);
  const int blocks = (int)(gridDim.x / (unsigned)a.Hkv), n = all < blocks ? (int)all : blocks;
  int32_t *record = a.meta + (int64_t)blockIdx.x * kMeta;  // of the tile that begins here and goes on in other blocks
  if (tid == 0) record[0] = 0;
  if (me >= n) return;
  long long u = all * me / n;
  const long long u_end = all * (me + 1) / n;
  // the request of step u: of the last thread that begins at or before it
  int r = 0, r_tiles, r_steps;
  long long r_begin;
  {
    int x = 0, y = kFewBlock - 1;
    while (x < y) {
      const int mid = (x + y + 1) >> 1;
      if (sh.line.before[mid] <= u)
        x = mid;
      else
        y = mid - 1;
    }
    r = x * per;
    r_begin = sh.line.before[x];
  }

  for (; u < u_end && r < a.R;) {
    count(r, r_tiles, r_steps);
    const int units = imax(r_steps, 1);  // of a tile
    if (u >= r_begin + (long long)r_tiles * units) {
      r_begin += (long long)r_tiles * units;
      ++r;
      continue;
    }
    const int tile_of = (int)((u - r_begin) / units);
    const long long begin = r_begin + (long long)tile_of * units;
    const int from = (int)(u - begin), to = (int)(u_end - begin < units ? u_end - begin : units);
    u = begin + to;
    const bool split = from > 0 || to < units;
    const int i0 = split ? block_of(begin, n, all) : me;
    const int np = split ? block_of(begin + units - 1, n, all) - i0 + 1 : 1;
    const int slot = !split ? -1 : 2 * me + (me == i0);
    const Request rq = request_of(a, r);
    const int first = tile_of * kFewRows;  // of the request's rows
    const int rows = imin(rq.n * a.G - first, kFewRows);
    const int row0 = rq.first * a.G + first;
    const int pos_first = rq.S - rq.n + first / a.G;
    const int pos_last = rq.S - rq.n + (first + rows - 1) / a.G;
    const int lo = (a.window ? imax(pos_first - a.window + 1, 0) : 0) & -kFew4Keys;
    const int hi = imin(pos_last + 1, rq.S);
    const int tiles = hi > lo ? (hi - lo + kFew4Keys - 1) / kFew4Keys : 0;
    const int steps = (tiles + kFewWaves - 1) / kFewWaves;
    const int s0 = (int)((long long)steps * from / units), s1 = (int)((long long)steps * to / units);
    const int32_t *table = a.table + (int64_t)r * a.table_row;

    // ------------------------------------------------ the queries, as columns
    // Product m of a key's operand c has piece m / KR for 128 columns and more; for 64 the
    // lanes' two upper groups take the piece after that of the two lower ones.
    const bool have_row = col < rows;
    const int rho = row0 + (have_row ? col : 0);
    const int tok = rho / a.G, head = h * a.G + rho % a.G;
    const int pos = rq.S - rq.n + (tok - rq.first);
    u32x6 q[NM];
    int q_scale[NM];
    {
      const T *src = (const T *)a.q + (int64_t)tok * a.q_token + (int64_t)head * a.q_head;
#pragma unroll
      for (int c = 0; c < KR; ++c) {
        const int d0 = (DP == 64 ? grp & 1 : c * 4 + grp) * kGroup;
        f32x32 x;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int d = d0 + i * 8;
          const typename Type<T>::Vec in = load8_global<T>(have_row && d < a.D ? src + d : (const T *)kZeroRow);
#pragma unroll
          for (int j = 0; j < 8; ++j) x[i * 8 + j] = (float)in[j];
        }
        const Query<NQ> s = split_query<NQ>(x);
        if constexpr (DP == 64) {
#pragma unroll
          for (int m = 0; m < NM; ++m) {
            const u32x6 zero{0, 0, 0, 0, 0, 0};
            q[m] = grp < 2 ? s.piece[2 * m] : 2 * m + 1 < NQ ? s.piece[imin(2 * m + 1, NQ - 1)] : zero;
            q_scale[m] = grp < 2 ? s.scale[2 * m] : 2 * m + 1 < NQ ? s.scale[imin(2 * m + 1, NQ - 1)] : 127;
          }
        } else {
#pragma unroll
          for (int m = 0; m < NQ; ++m) q[m * KR + c] = s.piece[m], q_scale[m * KR + c] = s.scale[m];
        }
      }
    }

    // ------------------------------------------------ walk of the keys
    __builtin_amdgcn_sched_barrier(0);  // the first keys' registers are not wanted before: the pieces take many
    f32x4 o[DT];
#pragma unroll
    for (int i = 0; i < DT; ++i) o[i] = f32x4{0, 0, 0, 0};
    float m = kNegInf, l = 0.0f;

    // Of 64 keys: 16 of each of four parts, four lanes a key.
    struct Keys {
      u32x4 k[4][KR];
      uint8_t k_scale[4][KR];  // bytes: made words where they are loaded, they would be waited for there
      unsigned v[4][VW];
      uint8_t v_scale[4][VS];
      unsigned long long live;  // bit: this key is there
    };
    // The page of key `lane` of a tile (ONE_PAGE: of all of them); -1 where there is none.
    const int end = imin(lo + s1 * kFew4Step, hi);
    auto find = [&](int base) {
      const int u = base + (ONE_PAGE ? 0 : lane);
      int page = -1;
      if (u < end) {
        page = table[u >> a.shift];
        if ((unsigned)page >= (unsigned)a.pages) page = -1;
      }
      return page;
    };
    const int kg = DP == 64 ? grp & 1 : grp;  // this lane's group of the key's first operand
    const int v0 = grp * (DP / 4);            // this lane's first column of V
    const uint8_t *zero = (const uint8_t *)kZeroRow;
    // ONE_PAGE: a tile's address is a scalar, to which a lane adds 32 bits.  Rows that are not there are read
    // from a page that is, and zeroed or not looked at: a load then has no condition.
    const bool any = a.pages > 0;
    const uint8_t *k_head = any ? (const uint8_t *)a.k + h * a.k_head : zero;
    const uint8_t *v_head = any ? (const uint8_t *)a.v + h * a.v_head : zero;
    const uint8_t *ks_head = any ? a.ks + h * a.ks_head : zero;
    const uint8_t *vs_head = any ? a.vs + h * a.vs_head : zero;
    const int k_row = any ? (int)a.k_slot : 0, v_row = any ? (int)a.v_slot : 0;
    const int ks_row = any ? (int)a.ks_slot : 0, vs_row = any ? (int)a.vs_slot : 0;
    unsigned k_at[KR], ks_at[KR], v_at[(VW + 3) / 4], vs_at[VS];
    if constexpr (ONE_PAGE) {
#pragma unroll
      for (int c = 0; c < KR; ++c) {
        const int g = kg + c * 4 < a.groups ? kg + c * 4 : 0;
        k_at[c] = col * k_row + g * kGroupBytes, ks_at[c] = col * ks_row + g;
      }
#pragma unroll
      for (int i = 0; i < (VW + 3) / 4; ++i) v_at[i] = col * v_row + (v0 + i * 32 < a.groups * kGroup ? v0 / 2 + i * 16 : 0);
#pragma unroll
      for (int i = 0; i < VS; ++i) vs_at[i] = col * vs_row + (v0 / kGroup + i < a.groups ? v0 / kGroup + i : 0);
    }
    auto load_k = [&](Keys &x, int base, int found) {
      if constexpr (ONE_PAGE) {
        const int page = __builtin_amdgcn_readfirstlane(found);
        const int keys = end - base;
        x.live = page < 0 ? 0 : keys >= kFew4Keys ? ~0ull : (1ull << keys) - 1;
        const int in = base & (P - 1);
        const int64_t pg = any ? imax(page, 0) : 0;
        const uint8_t *kp = k_head + pg * a.k_page + (int64_t)in * k_row;
        const uint8_t *ksp = ks_head + pg * a.ks_page + (int64_t)in * ks_row;
#pragma unroll
        for (int s = 0; s < 4; ++s) {
#pragma unroll
          for (int c = 0; c < KR; ++c) {
            x.k[s][c] = load_once<u32x4>(kp + k_at[c]);
            x.k_scale[s][c] = load_once<uint8_t>(ksp + ks_at[c]);
          }
          kp += 16 * k_row, ksp += 16 * ks_row;
        }
      } else {
        x.live = __builtin_amdgcn_ballot_w64(found >= 0);
#pragma unroll
        for (int s = 0; s < 4; ++s) {
          const int page = __shfl(found, s * 16 + col);
          const bool ok = page >= 0;
          const int64_t in = (base + s * 16 + col) & (P - 1);
          const uint8_t *kp = (const uint8_t *)a.k + page * a.k_page + in * a.k_slot + h * a.k_head;
          const uint8_t *ksp = a.ks + page * a.ks_page + in * a.ks_slot + h * a.ks_head;
#pragma unroll
          for (int c = 0; c < KR; ++c) {
            const int g = kg + c * 4;
            const bool in_row = ok && g < a.groups;
            x.k[s][c] = load_once<u32x4>(in_row ? kp + g * kGroupBytes : zero);
            x.k_scale[s][c] = load_once<uint8_t>(in_row ? ksp + g : zero);
          }
        }
      }
    };
    auto load_v = [&](Keys &x, int base, int found) {
      if constexpr (ONE_PAGE) {
        const int in = base & (P - 1);
        const int64_t pg = any ? imax(__builtin_amdgcn_readfirstlane(found), 0) : 0;
        const uint8_t *vp = v_head + pg * a.v_page + (int64_t)in * v_row;
        const uint8_t *vsp = vs_head + pg * a.vs_page + (int64_t)in * vs_row;
#pragma unroll
        for (int s = 0; s < 4; ++s) {
          if constexpr (VW == 2) {
            const u32x2 w = load_once<u32x2>(vp + v_at[0]);
            x.v[s][0] = w[0], x.v[s][1] = w[1];
          } else {
#pragma unroll
            for (int i = 0; i < VW; i += 4) {
              const u32x4 w = load_once<u32x4>(vp + v_at[i / 4]);
#pragma unroll
              for (int j = 0; j < 4; ++j) x.v[s][i + j] = w[j];
            }
          }
#pragma unroll
          for (int i = 0; i < VS; ++i) x.v_scale[s][i] = load_once<uint8_t>(vsp + vs_at[i]);
          vp += 16 * v_row, vsp += 16 * vs_row;
        }
      } else {
#pragma unroll
        for (int s = 0; s < 4; ++s) {
          const int page = __shfl(found, s * 16 + col);
          const bool ok = page >= 0;
          const int64_t in = (base + s * 16 + col) & (P - 1);
          const uint8_t *vp = (const uint8_t *)a.v + page * a.v_page + in * a.v_slot + h * a.v_head;
          const uint8_t *vsp = a.vs + page * a.vs_page + in * a.vs_slot + h * a.vs_head;
          if constexpr (VW == 2) {
            const u32x2 w = load_once<u32x2>(ok && v0 < a.groups * kGroup ? vp + v0 / 2 : zero);
            x.v[s][0] = w[0], x.v[s][1] = w[1];
          } else {
#pragma unroll
            for (int i = 0; i < VW; i += 4) {
              const u32x4 w = load_once<u32x4>(ok && v0 + i * 8 < a.groups * kGroup ? vp + v0 / 2 + i * 4 : zero);
#pragma unroll
              for (int j = 0; j < 4; ++j) x.v[s][i + j] = w[j];
            }
          }
#pragma unroll
          for (int i = 0; i < VS; ++i) {
            const int g = v0 / kGroup + i;
            x.v_scale[s][i] = load_once<uint8_t>(ok && g < a.groups ? vsp + g : zero);
          }
        }
      }
    };
    // Rows of several tokens see different keys.
    auto is_mixed = [&](int tile) {
      return (pos_first != pos_last && tile + kFew4Keys - 1 > pos_first) || (a.window && tile <= pos_last - a.window);
    };
    bool odd = false;
    const unsigned to_first = lds_address(sh.v[wave]) + L::write_first(col, v0);
    const unsigned from_first = lds_address(sh.v[wave]) + L::read_first(lane);
    Keys k;
    int base = lo + (s0 * kFewWaves + wave) * kFew4Keys;
    int next = find(base + kFew4Step);
    if (base < end) {
      const int found = find(base);
      load_k(k, base, found);
      load_v(k, base, found);
    }
    while (base < end) {
      const int tile = base;
      base += kFew4Step;
      const int found = next;
      next = find(base + kFew4Step);
      // S^T = K Q^T
      f32x4 x[4];
#pragma unroll
      for (int s = 0; s < 4; ++s) x[s] = f32x4{0, 0, 0, 0};
#pragma unroll
      for (int i = 0; i < NM; ++i)
#pragma unroll
        for (int s = 0; s < 4; ++s)
          x[s] = fp4_dot16(k.k[s][i % KR], k.k_scale[s][i % KR], q[i], q_scale[i], x[s]);
      if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int s = 0; s < 4; ++s) x[s] *= a.scale2;
      }
      // V that is not there, or not in the row, is zero; a NaN that some rows see and others do not must not
      // reach the latter through 0 * NaN, so it is taken out of the product and added at the end.
      const bool mixed = is_mixed(tile);
      const unsigned long long live = k.live;
      if (live != ~0ull || mixed || a.groups * kGroup != DP) {
        bool bad = false;
        const unsigned long long mine = live >> col;
#pragma unroll
        for (int s = 0; s < 4; ++s) {
          const bool there = (unsigned)(mine >> (32 * (s >> 1))) & (1u << (16 * (s & 1)));
#pragma unroll
          for (int i = 0; i < VS; ++i) {
            const bool keep = there && v0 + i * kGroup < a.groups * kGroup;
            const bool nan = keep && mixed && k.v_scale[s][i] == kNanScale;
            bad |= nan;
            if (!keep || nan) {
              k.v_scale[s][i] = 127;
#pragma unroll
              for (int j = i * VW / VS; j < (i + 1) * VW / VS; ++j) k.v[s][j] = 0;
            }
          }
        }
        if (__builtin_amdgcn_ballot_w64(bad)) odd = true;
      }
      load_k(k, base, found);  // the next tile's keys are on their way from here on, its V from below

      if (live != ~0ull || mixed) {
        // bit: this lane's query sees the key; the lane's keys begin at 4 grp
        unsigned long long seen = live;
        if (mixed) {
          const int most = pos - tile, least = a.window ? most - a.window : -1;
          seen &= most < 0 ? 0 : most >= 63 ? ~0ull : (2ull << most) - 1;
          seen &= least < 0 ? ~0ull : least >= 63 ? 0 : ~0ull << (least + 1);
        }
        seen >>= 4 * grp;
#pragma unroll
        for (int s = 0; s < 4; ++s) {
          const unsigned bits = (unsigned)(seen >> (32 * (s >> 1)));
#pragma unroll
          for (int i = 0; i < 4; ++i) x[s][i] = bits & (1u << (16 * (s & 1) + i)) ? x[s][i] : kNegInf;
        }
      }
      float top = x[0][0];
#pragma unroll
      for (int i = 1; i < 16; ++i) top = fmaxf(top, x[i >> 2][i & 3]);
      top = max_across_16(top);
      if (__builtin_amdgcn_ballot_w64(top > m)) {  // seldom behind the first tiles
        const float mn = fmaxf(m, top);
        const float fade = mn == kNegInf ? 1.0f : exp2_of((m - mn) * sc);  // 0 at the first key seen
        m = mn;
        l *= fade;
#pragma unroll
        for (int i = 0; i < DT; ++i) o[i] *= fade;
      }
      const float ms = m == kNegInf ? 0.0f : m * sc;  // nothing seen yet: exp2(-inf - 0) = 0
      Vec pv[2][NP];
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float e = exp2_of(__builtin_fmaf(x[i >> 2][i & 3], sc, -ms));
        l += e;
        // the weights go to the matrix cores in the type of V, their sum stays in fp32
        split_weight<V4, NP>(e, pv[i >> 3], i & 7);
      }
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        // the addresses made of these here take an instruction each, kept ones a register
        unsigned to = to_first, from = from_first;
        asm("" : "+v"(to), "+v"(from));
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
          for (int i = 0; i < VW; ++i)
            *(__attribute__((address_space(3))) Vec *)(uintptr_t)((to ^ (i << 4)) + s * 16 * L::kRowBytes) =
                eight_of<V4>(k.v[half * 2 + s][i], scale_of(k.v_scale[half * 2 + s][i * VS / VW]));
        if (half == 1) load_v(k, base, found);
        __builtin_amdgcn_wave_barrier();
        union {
          Vec v;
          i16x4 h[2];
        } w[DT];
#pragma unroll
        for (int i = 0; i < DT; ++i) {
          w[i].h[0] = lds_read_transposed(from ^ (i << 5));
          w[i].h[1] = lds_read_transposed((from ^ (i << 5)) + 16 * L::kRowBytes);
        }
#pragma unroll
        for (int i = 0; i < DT; ++i)
#pragma unroll
          for (int p = 0; p < NP; ++p) o[i] = Type<V4>::dot16(w[i].v, pv[half][p], o[i]);
        // operands ahead of the products
        constexpr int kAhead = DT < 4 ? DT : 4;
        __builtin_amdgcn_sched_group_barrier(kDsRead, 2 * kAhead, 2);
#pragma unroll
        for (int i = 0; i < DT - kAhead; ++i) {
          __builtin_amdgcn_sched_group_barrier(kMfma, NP, 2);
          __builtin_amdgcn_sched_group_barrier(kDsRead, 2, 2);
        }
        __builtin_amdgcn_sched_group_barrier(kMfma, NP * kAhead, 2);
      }
    }
    if (odd) {  // rare
      for (int tile = lo + (s0 * kFewWaves + wave) * kFew4Keys; tile < end; tile += kFew4Step)
        if (is_mixed(tile))
          for (int u = tile; u < tile + kFew4Keys && u < end; ++u) {
            const int page = table[u >> a.shift];
            if ((unsigned)page >= (unsigned)a.pages) continue;
            const uint8_t *vsp = a.vs + page * a.vs_page + (u & (P - 1)) * a.vs_slot + h * a.vs_head;
            const bool seen = u <= pos && (!a.window || u > pos - a.window);
#pragma unroll
            for (int i = 0; i < DT; ++i) {
              const int g = i * 16 / kGroup;
              if (g < a.groups && vsp[g] == kNanScale && seen) o[i] += __builtin_nanf("");
            }
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
          typename Type<T>::Vec w;
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
    if (slot >= 0 && me == i0 && tid == 0) {
      record[0] = np;
      record[1] = row0;
      record[2] = rows;
    }
    __syncthreads();
  }
}

// Adds the pieces of one row of a tile that is cut up (see join_few): of the tile that begins in block i0 of
// a KV head, at places 2 i0 + 1, 2 (i0 + 1), 2 (i0 + 2), ...  A block takes one of the n * Hkv records and every
// gridDim.y-th row.
template <class T, int DP>
__global__ __launch_bounds__(kJoinBlock) void join_few_fp4(AttendArgs a) {
  constexpr int kLanes = DP / 4;              // threads of a row
  constexpr int kSide = kJoinBlock / kLanes;  // pieces side by side
  __shared__ float acc[kSide][DP];
  __shared__ float weight[kJoinBlock];
  __shared__ float red[2][kJoinBlock / kWave];
  const float sc = score_unit<T>(a);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int32_t *record = a.meta + (int64_t)blockIdx.x * kMeta;
  const int np = record[0], row0 = record[1], rows = record[2];
  if (np <= 1) return;
  const int h = (int)(blockIdx.x % (unsigned)a.Hkv);
  const int64_t i0 = blockIdx.x / (unsigned)a.Hkv;
  constexpr int64_t kSize = (int64_t)kFewRows * (DP + 2);
  auto piece = [&](int j) { return a.part + ((2 * (i0 + j) + (j == 0)) * a.Hkv + h) * kSize; };
  for (int i = blockIdx.y; i < rows; i += gridDim.y) {
    const int ml = kFewRows * DP + i * 2;
    float mx = kNegInf;
    for (int j = tid; j < np; j += kJoinBlock) mx = fmaxf(mx, piece(j)[ml]);
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
        const float mj = piece(j)[ml];
        w = mj == kNegInf ? 0.0f : exp2_of((mj - mx) * sc);
        sum += w == 0.0f ? 0.0f : w * piece(j)[ml + 1];
      }
      __syncthreads();
      weight[tid] = w;
      __syncthreads();
      const int n = imin(np - j0, kJoinBlock);
#pragma unroll 8
      for (int k = g; k < n; k += kSide) {
        const f32x4 x = *reinterpret_cast<const f32x4 *>(piece(j0 + k) + i * DP + c);
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
    const int row = row0 + i, t = row / a.G, hd = h * a.G + row % a.G;
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

// -------------------------------------------------------------- many rows
//
// attend_many_fp4: as attend_many, 32 rows to a wave over tiles of 64 keys in LDS, two
// phases a tile.  K lies in LDS as its bytes and exponents: a product over 64 dimensions takes
// 32 cycles, as one over 16 in 16 bits, so that three pieces of a bf16 query take three quarters
// of the 16-bit products' time (four all of it), and 1 KB of LDS serves all of them.  In one phase the waves of a SIMD multiply, one of them
// the weights of the last tile with V, then the next scores; in the other they make weights of scores: two
// waves a SIMD take turns.  The query is scaled before it is split and a product begins at the negative maximum, so that a
// weight is one exponential of what comes out.  Above 64 columns the maximum of 16-bit types may lag by 2^8, and the weights are
// rounded to the type, both as in attend_many (see kLag): the chunk's result is off by 2.3e-3 in all, by 1.7e-3 with exact weights.  4010 tokens of 2 requests behind 5000 to 13000 keys, 32/8 heads of 128 in
// bf16, 694 GFLOP: 573 to 623 us by card, 1.11 to 1.21 PFLOP/s, the rate of a bf16 library product.  The matrix cores are
// busy 49% of the time at 2.0 GHz; without the exponentials it takes 8% less, without most of V's products 18%.
template <class V4, int DP>
struct Many4Shared {
  uint8_t k[2][64 * DP / 2];
  uint8_t k_scale[2][64 * (DP == 256 ? 8 : 4)];
  alignas(512) V4 v[2][64 * Tile<V4, DP>::kStride];  // the addresses of a row's chunks differ in single bits
  int odd;  // NaN was taken out of V
};
template <class T, int DP, int NW>
struct Many4SharedOf : Many4Shared<typename Four<T>::V4, DP> {
  Split<NW * kWave> split;
};

template <int BYTES>
struct Words;  // as many as a thread carries of a row
template <>
struct Words<4> {
  typedef unsigned V;
};
template <>
struct Words<8> {
  typedef u32x2 V;
};
template <>
struct Words<16> {
  typedef u32x4 V;
};

template <class T, int DP, int NW, bool ONE_PAGE, int NQ>
__global__ __launch_bounds__(NW *kWave) void attend_many_fp4(AttendFp4Args a) {
  typedef typename Four<T>::V4 V4;
  typedef typename Type<V4>::Vec Vec;
  typedef Tile<V4, DP> L;
  constexpr int NP = Four<T>::kP;
  constexpr int NT = NW * kWave, ROWS = 32 * NW;
  constexpr int KS = DP / 64;               // products of the summed axis of q.k, of each piece
  constexpr int DT = DP / 32;               // tiles of output columns
  constexpr int RB = DP / 2;                // bytes of a row
  constexpr int CB = 64 * RB / NT > 16 ? 16 : 64 * RB / NT;  // bytes of a chunk
  constexpr int NC = RB / CB;               // chunks of a row
  constexpr int CH = 64 * NC / NT;          // chunks of K and of V that a thread carries
  constexpr int RS = NT / NC;               // rows between two of them
  constexpr int CW = CB / 4;                // words of a chunk
  constexpr int G16 = DP / kGroup;          // groups of a row, 16 bytes each
  constexpr int SB = DP == 256 ? 8 : 4;     // bytes of a key's exponents in LDS
  typedef typename Words<CB>::V Chunk;
  extern __shared__ __align__(16) char raw[];
  Many4SharedOf<T, DP, NW> &sh = *reinterpret_cast<Many4SharedOf<T, DP, NW> *>(raw);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
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
    u32x6 q[KS][NQ];
    int q_scale[KS][NQ];
    {
      const T *src = (const T *)a.q + (int64_t)tok * a.q_token + (int64_t)head * a.q_head;
#pragma unroll
      for (int c = 0; c < KS; ++c) {
        f32x32 x;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int d = c * 64 + half * 32 + i * 8;
          const typename Type<T>::Vec in = load8_global<T>(have_row && d < a.D ? src + d : (const T *)kZeroRow);
#pragma unroll
          for (int j = 0; j < 8; ++j) x[i * 8 + j] = (float)in[j] * a.scale2;  // scores come out as exponents of two
        }
        const Query<NQ> s = split_query<NQ>(x);
#pragma unroll
        for (int i = 0; i < NQ; ++i) q[c][i] = s.piece[i], q_scale[c][i] = s.scale[i];
      }
    }
    f32x16 o[DT];
#pragma unroll
    for (int i = 0; i < DT; ++i)
#pragma unroll
      for (int j = 0; j < 16; ++j) o[i][j] = 0.0f;
    float m = kNegInf, l = 0.0f;
    f32x16 low;  // -m in all of them, 0 before the first key: the products of a tile begin from it
#pragma unroll
    for (int j = 0; j < 16; ++j) low[j] = 0.0f;

    // ------------------------------------------------ K and V into LDS
    const int n = t1 - t0;          // tiles of this piece
    const int k0 = lo + t0 * kManyKeys;
    // Tiles from `tail` on some of the block's rows see a part of only, and with a window those before `head`.
    const int tail = imin(imax((pos_first + 1 - k0) >> 6, 0), n);
    const int head_end = a.window ? imin(imax(((pos_last - a.window - k0) >> 6) + 1, 0), n) : 0;
    auto mixed = [&](int i) { return i >= tail || i < head_end; };
    // The table's entry for key `lane` of tile i (ONE_PAGE: for all of them), or of the
    // last key there is (there is one wherever this is called), and the page it stands for.
    auto find = [&](int i) {
      return table[imin(k0 + i * kManyKeys + (ONE_PAGE ? 0 : lane), hi - 1) >> a.shift];
    };
    auto valid = [&](int i, int page) {
      if constexpr (ONE_PAGE) {
        page = __builtin_amdgcn_readfirstlane(page);
        return i < n && (unsigned)page < (unsigned)a.pages ? page : -1;
      } else {
        return k0 + i * kManyKeys + lane < hi && (unsigned)page < (unsigned)a.pages ? page : -1;
      }
    };
    auto live_of = [&](int i, int page) -> unsigned long long {  // bit: this key is there
      if constexpr (ONE_PAGE) {
        const int keys = hi - (k0 + i * kManyKeys);
        return page < 0 ? 0 : keys >= kManyKeys ? ~0ull : (1ull << keys) - 1;
      } else {
        return __builtin_amdgcn_ballot_w64(page >= 0);
      }
    };
    // Few tiles are anything but 64 keys that are there and that all rows see: what the others need has its
    // scalars worked out where it is needed only.
    auto plain = [&](int i, int page) {
      if constexpr (ONE_PAGE)
        return page >= 0 && !mixed(i);
      else
        return __builtin_amdgcn_ballot_w64(page >= 0) == ~0ull && !mixed(i);
    };
    const int c_of = tid % NC, row_of = tid / NC;
    const int g_of = c_of * CB / kGroupBytes;  // group of this thread's chunks
    const bool in_row = g_of < a.groups;
    // Rows that are not there are read from a page that is, and zeroed on their way to
    // LDS: a load then has no condition.
    const bool any = a.pages > 0;
    const uint8_t *zero = (const uint8_t *)kZeroRow;
    const uint8_t *k_head = any ? (const uint8_t *)a.k + h * a.k_head : zero;
    const uint8_t *v_head = any ? (const uint8_t *)a.v + h * a.v_head : zero;
    const uint8_t *ks_head = any ? a.ks + h * a.ks_head : zero;
    const uint8_t *vs_head = any ? a.vs + h * a.vs_head : zero;
    const int64_t k_page = any ? a.k_page : 0, k_slot = any ? a.k_slot : 0;
    const int64_t v_page = any ? a.v_page : 0, v_slot = any ? a.v_slot : 0;
    const int64_t ks_page = any ? a.ks_page : 0, ks_slot = any ? a.ks_slot : 0;
    const int64_t vs_page = any ? a.vs_page : 0, vs_slot = any ? a.vs_slot : 0;
    const unsigned c_at = in_row ? c_of * CB : 0, s_at = in_row ? g_of : 0;
    // ONE_PAGE: this lane's first row of page 0, to which a tile adds a scalar (see one_page: strides are 32 bits)
    const uint8_t *k_lane = k_head + row_of * k_slot + c_at, *v_lane = v_head + row_of * v_slot + c_at;
    const uint8_t *ks_lane = ks_head + row_of * ks_slot + s_at, *vs_lane = vs_head + row_of * vs_slot + s_at;
    Chunk kr[CH], vr[CH];
    uint8_t kb[CH], vb[CH];  // bytes: made words where they are loaded, they would be waited for there
    auto load = [&](Chunk r[CH], uint8_t b[CH], int i, int page, const uint8_t *base, int64_t page_stride,
                    int64_t slot_stride, const uint8_t *s_base, int64_t s_page, int64_t s_slot) {
      if constexpr (ONE_PAGE) {
        const unsigned in = (k0 + i * kManyKeys) & (P - 1), pg = imax(page, 0);
        const uint8_t *src = base + ((uint64_t)pg * (unsigned)page_stride + in * (unsigned)slot_stride);
        const uint8_t *s_src = s_base + ((uint64_t)pg * (unsigned)s_page + in * (unsigned)s_slot);
#pragma unroll
        for (int c = 0; c < CH; ++c) {
          r[c] = load_global<Chunk>(src + c * RS * (int)slot_stride);
          b[c] = load_global<uint8_t>(s_src + c * RS * (int)s_slot);
        }
      } else {
#pragma unroll
        for (int c = 0; c < CH; ++c) {
          const int row = c * RS + row_of;
          const int64_t pg = imax(__shfl(page, row), 0);
          const int in = (k0 + i * kManyKeys + row) & (P - 1);
          r[c] = load_global<Chunk>(base + pg * page_stride + in * slot_stride + c_at);
          b[c] = load_global<uint8_t>(s_base + pg * s_page + in * s_slot + s_at);
        }
      }
    };
    auto load_k = [&](int i, int page) {
      load(kr, kb, i, page, ONE_PAGE ? k_lane : k_head, k_page, k_slot, ONE_PAGE ? ks_lane : ks_head, ks_page, ks_slot);
    };
    auto load_v = [&](int i, int page) {
      load(vr, vb, i, page, ONE_PAGE ? v_lane : v_head, v_page, v_slot, ONE_PAGE ? vs_lane : vs_head, vs_page, vs_slot);
    };
    // Rows that are not there become zeros, and V of a tile of which some rows see a part
    // only loses its NaN (kept for those who see them: see the end of the walk).
    const bool whole_rows = a.groups == G16;
    auto clean = [&](Chunk r[CH], uint8_t b[CH], unsigned long long live) {
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        const bool keep = in_row && ((live >> (c * RS + row_of)) & 1);
        r[c] = keep ? r[c] : Chunk(0);
        b[c] = keep ? b[c] : (uint8_t)127;
      }
    };
    auto clean_k = [&](int i, int page) {
      if (!whole_rows || !plain(i, page)) clean(kr, kb, live_of(i, page));
    };
    auto clean_v = [&](int i, int page) {
      if (whole_rows && plain(i, page)) return;
      clean(vr, vb, live_of(i, page));
      if (mixed(i)) {
        bool bad = false;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
          const bool nan = vb[c] == kNanScale;
          bad |= nan;
          vr[c] = nan ? Chunk(0) : vr[c];
          vb[c] = nan ? (uint8_t)127 : vb[c];
        }
        if (__builtin_amdgcn_ballot_w64(bad)) sh.odd = 1;
      }
    };
    // 16 bytes of 16 rows, read at once, lie in different banks: a row's are permuted by the row.
    constexpr int kPer = 16 / G16;  // rows of 256 bytes
    auto swizzle = [](int row) { return (row / kPer) & (G16 - 1); };
    auto store_k = [&](int buffer) {
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        const int row = c * RS + row_of;
        const int at = c_of * CB;
        *reinterpret_cast<Chunk *>(&sh.k[buffer][row * RB + ((g_of ^ swizzle(row)) << 4) + (at & 15)]) = kr[c];
        sh.k_scale[buffer][row * SB + g_of] = kb[c];  // all threads of a group the same: no condition, no other block
      }
    };
    auto store_v = [&](int buffer) {
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        const float scale = scale_of(vb[c]);
#pragma unroll
        for (int w = 0; w < CW; ++w) {
          unsigned word;
          if constexpr (CW == 1)
            word = vr[c];
          else
            word = vr[c][w];
          store8<V4>(sh.v[buffer] + L::at(c * RS + row_of, (c_of * CW + w) * 8), eight_of<V4>(word, scale));
        }
      }
    };
    // A barrier that waits for LDS only: loads on their way stay there.
    auto sync = [&]() {
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
      __builtin_amdgcn_s_barrier();
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
    };

    const unsigned v_at = lds_address(sh.v[0]) + L::v_first(lane);
    f32x16 x[2];
    Vec pv[4][NP];

    // S^T = K Q^T of tile i, less the maximum so far
    auto scores = [&](int i) {
      const int buffer = i & 1;
      u32x4 k[2][KS];
      u32x2 e[2];
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const int row = s * 32 + col;
        if constexpr (DP == 256)
          e[s] = *reinterpret_cast<const u32x2 *>(&sh.k_scale[buffer][row * SB]);
        else
          e[s][0] = *reinterpret_cast<const unsigned *>(&sh.k_scale[buffer][row * SB]), e[s][1] = 0;
        // this lane's groups are c * 2 + half: they come to lie at the bytes 0 and 2 of a word
        e[s][0] >>= half * 8, e[s][1] >>= half * 8;
#pragma unroll
        for (int c = 0; c < KS; ++c)
          k[s][c] = *reinterpret_cast<const u32x4 *>(&sh.k[buffer][row * RB + (((c * 2 + half) ^ swizzle(row)) << 4)]);
      }
      x[0] = low, x[1] = low;
#pragma unroll
      for (int c = 0; c < KS; ++c)
#pragma unroll
        for (int w = 0; w < NQ; ++w)
#pragma unroll
          for (int s = 0; s < 2; ++s)
            x[s] = c & 1 ? fp4_dot32<2>(k[s][c], (int)e[s][c >> 1], q[c][w], q_scale[c][w], x[s])
                         : fp4_dot32<0>(k[s][c], (int)e[s][c >> 1], q[c][w], q_scale[c][w], x[s]);
    };

    // P^T of tile i out of S^T, and what was summed so far brought to its maximum
    auto weights = [&](int i, int page) {
      if (!plain(i, page)) {
        // bit: this lane's query sees the key; the lane's keys begin at 4 half
        const int b = k0 + i * kManyKeys, most = pos - b, least = a.window ? most - a.window : -1;
        unsigned long long seen = live_of(i, page);
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
      const bool none = m == kNegInf;
      if (__builtin_amdgcn_ballot_w64(top > (none ? kNegInf : kLag<T, DP>))) {
        const float up = none ? top : fmaxf(top, 0.0f);  // by how much the maximum rises
        const float mn = none ? top : m + up;
        const float fade = mn == kNegInf ? 1.0f : exp2_of(m - mn);
        l *= fade;
#pragma unroll
        for (int c = 0; c < DT; ++c) o[c] *= fade;
        m = mn;
        const float less = mn == kNegInf ? 0.0f : up;
#pragma unroll
        for (int j = 0; j < 32; ++j) x[j >> 4][j & 15] -= less;
#pragma unroll
        for (int j = 0; j < 16; ++j) low[j] = mn == kNegInf ? 0.0f : -mn;
      }
#pragma unroll
      for (int j = 0; j < 32; ++j) {
        const float e = exp2_of(x[j >> 4][j & 15]);
        l += e;
        // the weights go to the matrix cores in the type of V, their sum stays in fp32
        split_weight<V4, NP>(e, pv[j >> 3], j & 7);
      }
    };

    // O^T += V^T P^T of tile i
    auto values = [&](int i) {
      unsigned at = v_at + (i & 1) * (int)sizeof(sh.v[0]);
      asm("" : "+v"(at));  // the addresses made of it here take an instruction each, kept ones a register
      union Operand {
        i16x4 h[2];
        Vec v;
      } v[4][DT];
#pragma unroll
      for (int s = 0; s < 4; ++s)
#pragma unroll
        for (int c = 0; c < DT; ++c) {
          v[s][c].h[0] = lds_read_transposed((at ^ (c << 6)) + s * 16 * L::kRowBytes);
          v[s][c].h[1] = lds_read_transposed((at ^ (c << 6) ^ L::kEight) + (s * 16 + 8) * L::kRowBytes);
        }
#pragma unroll
      for (int s = 0; s < 4; ++s)
#pragma unroll
        for (int w = 0; w < NP; ++w)
#pragma unroll
          for (int c = 0; c < DT; ++c) o[c] = Type<V4>::dot32(v[s][c].v, pv[s][w], o[c]);
    };

    // ------------------------------------------------ the walk, in two phases a tile
    // As in attend_many: products (O += P V of the tile before, S = K Q of this one) and the
    // softmax after them alternate behind barriers, half of the waves a phase behind the others.
    // Stage i is K of tile i + 1 and V of tile i.
    const int late = NW == 8 && wave >= NW / 2 ? 1 : 0;
    sync();  // the last piece's tiles are done with
    if (tid == 0) sh.odd = 0;
    sync();
    if (n > 0) {
      int pg = valid(0, find(0));  // page of tile i
      int v_pg = valid(1, find(1)), k_pg = valid(2, find(2));  // of stage i + 1 (V, K), while stage i is at hand
      int next_pg = find(3);  // not looked at before its time: that would wait for the loads before it
      load_k(0, pg);
      clean_k(0, pg);
      store_k(0);
      load_k(1, v_pg);
      load_v(0, pg);
      clean_k(1, v_pg);
      clean_v(0, pg);
      sync();
      if (late) sync();
      // Stage i, K of tile i + 1 and V of tile i, goes to LDS among the products of tile i, and the next stage's loads set off.
      auto stage = [&](int i) {
        store_k((i + 1) & 1);
        store_v(i & 1);
        load_k(i + 2, k_pg);
        load_v(i + 1, v_pg);
      };
      // The softmax, and among it what the stage on its way needs before it goes to LDS, and the next one's pages.
      auto softmax = [&](int i) {
        weights(i, pg);
        clean_k(i + 2, k_pg);
        clean_v(i + 1, v_pg);
        pg = v_pg, v_pg = k_pg, k_pg = valid(i + 3, next_pg);
        next_pg = find(i + 4);
      };
      scores(0);
      stage(0);
      sync();
      softmax(0);
      sync();
      for (int i = 1; i < n; ++i) {
        values(i - 1);
        stage(i);
        scores(i);
        // four operands of V ahead of its products, K's behind them
        constexpr int kValues = 4 * DT;
        __builtin_amdgcn_sched_group_barrier(kDsRead, 8, 1);
#pragma unroll
        for (int c = 0; c < kValues - 4; ++c) {
          __builtin_amdgcn_sched_group_barrier(kMfma, NP, 1);
          __builtin_amdgcn_sched_group_barrier(kDsRead, 2, 1);
        }
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          __builtin_amdgcn_sched_group_barrier(kMfma, NP, 1);
          __builtin_amdgcn_sched_group_barrier(kDsRead, (KS + 1) / 2, 1);
        }
        __builtin_amdgcn_sched_group_barrier(kDsRead, 2 + 2 * KS, 1);
        __builtin_amdgcn_sched_group_barrier(kMfma, 2 * KS * NQ, 1);
        __builtin_amdgcn_sched_barrier(0);
        sync();
        softmax(i);
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
              const uint8_t *vsp = a.vs + page * a.vs_page + (u & (P - 1)) * a.vs_slot + h * a.vs_head;
              const bool seen = u <= pos && (!a.window || u > pos - a.window);
#pragma unroll
              for (int c = 0; c < DT; ++c)
                if (c < a.groups && vsp[c] == kNanScale && seen) o[c] += __builtin_nanf("");
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
        for (int t = 0; t < DT; ++t) {
          if (t >= a.groups) break;
#pragma unroll
          for (int j = 0; j < 4; ++j)
            *reinterpret_cast<f32x4 *>(dst + (int64_t)i * DP + t * 32 + j * 8 + half * 4) =
                f32x4{o[t][4 * j], o[t][4 * j + 1], o[t][4 * j + 2], o[t][4 * j + 3]};
        }
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
        a.lse[(int64_t)tok * a.Hq + head] = m == kNegInf ? kNegInf : m * kLn2 + __logf(l);
    }
  }
}

}  // namespace paged
}  // namespace slnr
