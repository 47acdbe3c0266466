// A cache in 4 bits: what its bytes stand for, new rows into it, and rows out of it.
//
// A row of dim values is ceil(dim / 32) groups of 32, the last one filled up with zeros.  A
// value is a sign and one of {0, 0.5, 1, 1.5, 2, 3, 4, 6} (E2M1), two to a byte, the
// first in the low half; a group has one byte e + 127 (E8M0) and its values are
// multiplied by 2^e.  The matrix cores take both as they are.
#pragma once

#include "attend.hpp"

namespace slnr {
namespace paged {

typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x6 __attribute__((ext_vector_type(6)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x32 __attribute__((ext_vector_type(32)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

constexpr int kGroup = 32;          // values that share an exponent
constexpr int kGroupBytes = 16;
constexpr unsigned kNanScale = 255;  // a group with infinities or NaN: all of it is NaN

// V4: the type that 4-bit values are taken into for products with the weights, all of them
// exactly.  kLeast, kMost: exponents of a group.  0.5 * 2^kLeast and 6 * 2^kMost are normal values of bf16 and values of fp16, so
// that no code is lost or becomes infinite on its way back.  What it costs: values above 7 * 2^13 in fp16 and above
// 7 * 2^125 in bf16 and fp32, the last quarter of their last binade, become 6 times the power, and in bf16 and fp32 groups of up to
// 2^-127 become zeros.
// kQ: pieces that a query is split into (see split_query), kQOut: as many as out needs, which is rounded to bf16
// while lse is not; kP: pieces of a weight.
template <class T>
struct Four;
template <>
struct Four<__bf16> {
  typedef __bf16 V4;
  static constexpr int kLeast = -125, kMost = 125, kQ = 4, kQOut = 3, kP = 1;
};
template <>
struct Four<_Float16> {
  typedef _Float16 V4;
  static constexpr int kLeast = -23, kMost = 13, kQ = 4, kQOut = 4, kP = 1;
};
template <>
struct Four<float> {
  typedef __bf16 V4;
  static constexpr int kLeast = -125, kMost = 125, kQ = 5, kQOut = 5, kP = 3;
};

__device__ __forceinline__ float scale_of(unsigned byte) { return __uint_as_float(byte << 23); }

// Eight values of a word.  The scale of a NaN group, an infinity as a number, makes all of them NaN.
template <class V4>
__device__ __forceinline__ typename Type<V4>::Vec eight_of(unsigned word, float scale) {
  typename Type<V4>::Vec v;
  if constexpr (__is_same(V4, __bf16)) {
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, 0);
    const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, 1);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, 2);
    const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, 3);
    v = bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
  } else {
    const f16x2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(word, scale, 0);
    const f16x2 b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(word, scale, 1);
    const f16x2 c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(word, scale, 2);
    const f16x2 d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(word, scale, 3);
    v = f16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
  }
  return v;
}

// ------------------------------------------------------------------ new rows

struct Fp4Args {
  const void *k, *v;  // append: [T][Hkv][D], strides in values; read: written densely
  int64_t k_token, k_head_in, v_token, v_head_in;
  const int64_t *slots;  // [T]
  uint8_t *kc, *vc, *ks, *vs;
  // strides in bytes
  int64_t k_page, k_slot, k_head, v_page, v_slot, v_head;
  int64_t ks_page, ks_slot, ks_head, vs_page, vs_slot, vs_head;
  int32_t T, pages, shift, Hkv, D;
};

constexpr int kFp4Block = 256;

// Four lanes take the 32 values of a group: the largest of them gives the exponent, the least e
// with max|x| <= 7 * 2^e, so that no value is further off than half a step of the 4-bit grid (6 is
// followed by 8); x / 2^e is rounded to the nearest, ties to an even code.
// The values are read while the slot is on its way.  Latency: 64 tokens of 8 heads of 128 3.2 us; 6258 tokens of 4 heads of
// 80 6.7 us, 10 MB at 1.5 TB/s.
template <class T>
__global__ __launch_bounds__(kFp4Block) void fp4_append(Fp4Args a) {
  const int groups = (a.D + kGroup - 1) / kGroup;
  const unsigned lanes = groups * 4, row = 2 * (unsigned)a.Hkv * lanes;  // of a row, of a token
  const int64_t all = (int64_t)a.T * row;
  for (int64_t i = (int64_t)blockIdx.x * kFp4Block + threadIdx.x; i < all; i += (int64_t)gridDim.x * kFp4Block) {
    const int64_t t = i / row;
    unsigned e = (unsigned)(i - t * row);
    const bool is_v = e >= row / 2;
    if (is_v) e -= row / 2;
    const unsigned h = e / lanes, c = e - h * lanes;
    const int64_t slot = a.slots[t];
    const T *src = is_v ? (const T *)a.v + t * a.v_token + h * a.v_head_in
                        : (const T *)a.k + t * a.k_token + h * a.k_head_in;
    float x[8];
    {
      const typename Type<T>::Vec in = load8_global<T>((int)c * 8 < a.D ? src + c * 8 : (const T *)kZeroRow);
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = (float)in[j];
    }
    // as whole numbers: the bits of numbers without sign are in their order, infinities and NaN last
    unsigned top = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const unsigned b = __float_as_uint(x[j]) & 0x7fffffffu;
      top = b > top ? b : top;
    }
#pragma unroll
    for (int o = 1; o < 4; o <<= 1) {
      const unsigned b = __shfl_xor(top, o);
      top = b > top ? b : top;
    }
    int power = (int)(top >> 23) - 2 + ((top & 0x7fffffu) > 0x600000u);  // e + 127; 7 = 1.75 * 4
    power = imin(imax(power, Four<T>::kLeast + 127), Four<T>::kMost + 127);
    const float scale = scale_of(power);
    unsigned word = 0;
    word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, x[0], x[1], scale, 0);
    word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, x[2], x[3], scale, 1);
    word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, x[4], x[5], scale, 2);
    word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, x[6], x[7], scale, 3);
    const bool odd = top >= 0x7f800000u;
    const int64_t page = slot >> a.shift, in = slot & ((1 << a.shift) - 1);
    if (slot < 0 || page >= a.pages) continue;
    uint8_t *codes = is_v ? a.vc + page * a.v_page + in * a.v_slot + h * a.v_head
                          : a.kc + page * a.k_page + in * a.k_slot + h * a.k_head;
    *reinterpret_cast<unsigned *>(codes + c * 4) = odd ? 0 : word;
    if ((c & 3) == 0) {
      uint8_t *scales = is_v ? a.vs + page * a.vs_page + in * a.vs_slot + h * a.vs_head
                             : a.ks + page * a.ks_page + in * a.ks_slot + h * a.ks_head;
      scales[c >> 2] = odd ? (uint8_t)kNanScale : (uint8_t)power;
    }
  }
}

// The rows of some slots as values; zeros for slots outside the cache.  A lane takes eight values: 3.1 and 5.8 us for
// as many rows.
template <class T>
__global__ __launch_bounds__(kFp4Block) void fp4_read(Fp4Args a) {
  const unsigned lanes = a.D / 8, row = 2 * (unsigned)a.Hkv * lanes;
  const int64_t all = (int64_t)a.T * row;
  for (int64_t i = (int64_t)blockIdx.x * kFp4Block + threadIdx.x; i < all; i += (int64_t)gridDim.x * kFp4Block) {
    const int64_t t = i / row;
    unsigned e = (unsigned)(i - t * row);
    const bool is_v = e >= row / 2;
    if (is_v) e -= row / 2;
    const unsigned h = e / lanes, c = e - h * lanes;
    const int64_t slot = a.slots[t], page = slot >> a.shift, in = slot & ((1 << a.shift) - 1);
    unsigned word = 0, scale = 127;
    if (slot >= 0 && page < a.pages) {
      word = *reinterpret_cast<const unsigned *>((is_v ? a.vc + page * a.v_page + in * a.v_slot + h * a.v_head
                                                       : a.kc + page * a.k_page + in * a.k_slot + h * a.k_head) + c * 4);
      scale = (is_v ? a.vs + page * a.vs_page + in * a.vs_slot + h * a.vs_head
                    : a.ks + page * a.ks_page + in * a.ks_slot + h * a.ks_head)[c >> 2];
    }
    const auto x = eight_of<typename Four<T>::V4>(word, scale_of(scale));
    typename Type<T>::Vec out;
#pragma unroll
    for (int j = 0; j < 8; ++j) out[j] = (T)x[j];
    store8<T>((T *)(is_v ? a.v : a.k) + ((t * a.Hkv + h) * a.D + c * 8), out);
  }
}

// ------------------------------------------------- a query for the matrix cores
//
// The products q.k take the cache's bytes as they are, in the matrix cores' form for operands with an
// exponent per 32 values.  The other operand may have 6 bits (E2M3: a sign and steps of 1/8 up
// to 2, of 1/4 up to 4, of 1/2 up to 7.5) at four times the rate of a 16-bit
// product, so a query is written as a sum of such pieces, each the rest of those before it,
// with an exponent of its own per group.  A first piece leaves at most 1/4 of its unit, 4 units of a second
// one 16 times finer; each further piece is 32 times finer.  The first unit is at most the group's largest value divided by
// 3.75, so three pieces leave 2^-13 of that value, four 2^-18, five 2^-23.  All of this goes by the group's
// largest value: where a channel is A times the others (A times less in K), what is left of the others counts A times as much.
// Relative error of out over 1000 keys at dim 128 by three | four pieces, A = 1: 3.5e-5 | 1.1e-6, 30: 4.0e-4 | 1.3e-5, 100:
// 1.4e-3 | 4.3e-5, 300: 4.2e-3 | 1.3e-4; the rounding of the result is 1.6e-3 in bf16 and 2e-4 in fp16.  So bf16's out takes three, up to
// A = 100 no more than its rounding, and fp16's takes four.  lse is fp32: over 1000 keys at dim 96 three
// pieces put it off by up to 1.9e-4, four by 4e-6.
constexpr int query_step(int piece) { return piece == 0 ? 0 : 5 * piece - 1; }

template <int N>
struct Query {
  u32x6 piece[N];
  int scale[N];  // e + 127
};

// 32 values in steps of `unit`: even and odd ones, and back.  These instructions take several passes and
// write while they still read: where the result begins inside an operand, or on the unit's register, it
// is wrong, and the compiler does not know.  The empty statements keep the operands until after it, in registers
// of their own.
__device__ __forceinline__ u32x6 to_fp6(f32x16 even, f32x16 odd, float unit) {
  u32x6 r = __builtin_amdgcn_cvt_scalef32_2xpk16_fp6_f32(even, odd, unit);
  asm volatile("" : "+v"(r) : "v"(even), "v"(odd), "v"(unit));
  return r;
}
__device__ __forceinline__ f32x32 from_fp6(u32x6 x, float unit) {
  f32x32 r = __builtin_amdgcn_cvt_scalef32_pk32_f32_fp6(x, unit);
  asm volatile("" : "+v"(r) : "v"(x), "v"(unit));
  return r;
}

// x: the 32 values of a group.
template <int N>
__device__ __forceinline__ Query<N> split_query(f32x32 x) {
  Query<N> q;
  unsigned top = 0;
#pragma unroll
  for (int j = 0; j < 32; ++j) {
    const unsigned b = __float_as_uint(x[j]) & 0x7fffffffu;
    top = b > top ? b : top;
  }
  // 7.5 = 1.875 * 4; the last piece's exponent stays in the numbers' range
  const int first = imax((int)(top >> 23) - 2 + ((top & 0x7fffffu) > 0x700000u), query_step(N - 1) + 2);
#pragma unroll
  for (int p = 0; p < N; ++p) {
    q.scale[p] = first - query_step(p);
    const float unit = scale_of(q.scale[p]);
    f32x16 even, odd;
#pragma unroll
    for (int j = 0; j < 16; ++j) even[j] = x[2 * j], odd[j] = x[2 * j + 1];
    q.piece[p] = to_fp6(even, odd, unit);
    if (p + 1 < N) x -= from_fp6(q.piece[p], unit);
  }
  if (top >= 0x7f800000u) q.scale[0] = kNanScale;
  return q;
}

// The operand of 32 values a lane: groups of four words (4 bits) or six (6 bits).
__device__ __forceinline__ i32x8 operand(u32x4 k) { return i32x8{(int)k[0], (int)k[1], (int)k[2], (int)k[3], 0, 0, 0, 0}; }
__device__ __forceinline__ i32x8 operand(u32x6 q) {
  return i32x8{(int)q[0], (int)q[1], (int)q[2], (int)q[3], (int)q[4], (int)q[5], 0, 0};
}
constexpr int kE2M1 = 4, kE2M3 = 2;

// D(16x16) += A(16x128) B(128x16): lane l holds row l & 15 of A and column l & 15 of B, group l >> 4, and gets
// D as dot16 does.
__device__ __forceinline__ f32x4 fp4_dot16(u32x4 k, int k_scale, u32x6 q, int q_scale, f32x4 c) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(operand(k), operand(q), c, kE2M1, kE2M3, 0, k_scale, 0,
                                                          q_scale);
}
// D(32x32) += A(32x64) B(64x32): row and column l & 31, group l >> 5, D as dot32 does.  BYTE: of the scales' word.
template <int BYTE>
__device__ __forceinline__ f32x16 fp4_dot32(u32x4 k, int k_scale, u32x6 q, int q_scale, f32x16 c) {
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(operand(k), operand(q), c, kE2M1, kE2M3, BYTE, k_scale, 0,
                                                         q_scale);
}

}  // namespace paged
}  // namespace slnr
