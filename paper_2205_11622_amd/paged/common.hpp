// Types, matrix-core products and address arithmetic shared by the kernels of
// the paged cache.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace slnr {
namespace paged {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef short i16x8 __attribute__((ext_vector_type(8)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

constexpr int kWave = 64;
constexpr float kNegInf = -__builtin_inff();
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// Rows that are not there (past the end, page given back) are read from here:
// as many zeros as the widest row has bytes.
constexpr int kMaxDim = 256;
static __device__ __align__(16) const float kZeroRow[kMaxDim] = {};

// ------------------------------------------------------------- the three types

// `Vec` is what a lane holds of a matrix-core operand: eight values along the
// summed axis.  dot16: D(16x16) += A(16x32) B(32x16), lane l holds A[l & 15][8 (l >> 4) + 0..7]
// and B[8 (l >> 4) + 0..7][l & 15] and gets D[4 (l >> 4) + 0..3][l & 15].
// dot32: D(32x32) += A(32x16) B(16x32), lane l holds A[l & 31][8 (l >> 5) + 0..7], B likewise, and gets
// D[8 (i / 4) + 4 (l >> 5) + i % 4][l & 31] in element i.  In fp32 the eight
// values go to eight products of the fp32 matrix cores, which take one value a
// lane: the same sum, its axis in another order.
template <class T>
struct Type;

template <>
struct Type<__bf16> {
  typedef bf16x8 Vec;
  static constexpr int kBytes = 2;
  static constexpr unsigned kExpMask = 0x7f807f80u, kExpOne = 0x00800080u;
  static __device__ f32x4 dot16(Vec a, Vec b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
  }
  static __device__ f32x16 dot32(Vec a, Vec b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
  }
};

template <>
struct Type<_Float16> {
  typedef f16x8 Vec;
  static constexpr int kBytes = 2;
  static constexpr unsigned kExpMask = 0x7c007c00u, kExpOne = 0x04000400u;
  static __device__ f32x4 dot16(Vec a, Vec b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
  }
  static __device__ f32x16 dot32(Vec a, Vec b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
  }
};

template <>
struct Type<float> {
  typedef f32x8 Vec;
  static constexpr int kBytes = 4;
  static __device__ f32x4 dot16(Vec a, Vec b, f32x4 c) {
#pragma unroll
    for (int i = 0; i < 8; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], b[i], c, 0, 0, 0);
    return c;
  }
  static __device__ f32x16 dot32(Vec a, Vec b, f32x16 c) {
#pragma unroll
    for (int i = 0; i < 8; ++i) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[i], b[i], c, 0, 0, 0);
    return c;
  }
};

// Eight values from 16-byte aligned memory.
template <class T>
__device__ __forceinline__ typename Type<T>::Vec load8(const T *p) {
  typename Type<T>::Vec v;
  if constexpr (sizeof(T) == 2) {
    v = *reinterpret_cast<const typename Type<T>::Vec *>(p);
  } else {
    const f32x4 lo = *reinterpret_cast<const f32x4 *>(p);
    const f32x4 hi = *reinterpret_cast<const f32x4 *>(p + 4);
    v = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  }
  return v;
}

// The same from device memory: the pointer may be one of two objects, which would
// otherwise make the load a flat one, and that waits for LDS too.
template <class T>
__device__ __forceinline__ typename Type<T>::Vec load8_global(const T *p) {
  typedef const __attribute__((address_space(1))) u32x4 *G;
  union {
    u32x4 u[sizeof(T) / 2];
    typename Type<T>::Vec v;
  } w;
  const G g = (G)p;
  w.u[0] = g[0];
  if constexpr (sizeof(T) == 4) w.u[1] = g[1];
  return w.v;
}

template <class T>
__device__ __forceinline__ void store8(T *p, typename Type<T>::Vec v) {
  if constexpr (sizeof(T) == 2) {
    *reinterpret_cast<typename Type<T>::Vec *>(p) = v;
  } else {
    *reinterpret_cast<f32x4 *>(p) = __builtin_shufflevector(v, v, 0, 1, 2, 3);
    *reinterpret_cast<f32x4 *>(p + 4) = __builtin_shufflevector(v, v, 4, 5, 6, 7);
  }
}

// ------------------------------------------------------- a tile of V in LDS
//
// Rows are keys, columns head dimensions.  O^T = V^T P^T needs eight keys of one
// column per lane: the transposing LDS read gives a lane four keys of its column
// where the 16 lanes of a group point at four rows of 16 values.  16-byte chunks
// of a row are permuted by the row, so that both the rows' writes (one chunk of 16
// rows) and these reads (four rows, two chunks) spread over all banks.  fp32 rows
// are read value by value and padded by four instead.
template <class T, int DP>
struct Tile {
  static constexpr int kStride = sizeof(T) == 2 ? DP : DP + 4;  // values a row

  static __device__ __forceinline__ int chunk(int row) {
    if constexpr (DP >= 128)
      return ((row & 3) << 2) | ((row >> 2) & 3);
    else
      return (row & 6) | ((row >> 3) & 1);
  }
  // column is a multiple of 8 (4 is fine too: half a chunk)
  static __device__ __forceinline__ int at(int row, int column) {
    if constexpr (sizeof(T) == 2)
      return row * kStride + ((((column >> 3) ^ chunk(row)) << 3) | (column & 7));
    else
      return row * kStride + column;
  }
  // Operands of a 32 x 32 product in 16 bits.  The permutation is an exclusive or, so
  // a lane's address for step i differs from its first one in single bits:
  // K, row `row + 32 s` (row < 32), values 16 i + 8 half ..:  k_first ^ (i << 5), + 32 s rows;
  // V, keys 16 s + 4 half + 8 p .., column 32 i + (lane & 31): v_first ^ (i << 6) ^ p * kEight, + 16 s + 8 p rows.
  static constexpr int kRowBytes = kStride * (int)sizeof(T);
  static constexpr unsigned kEight = DP >= 128 ? 32 : 16;  // chunk(row + 8) ^ chunk(row), in bytes
  static __device__ __forceinline__ unsigned k_first(int row, int half) {
    return row * kRowBytes + ((half ^ chunk(row)) << 4);
  }
  static __device__ __forceinline__ unsigned v_first(int lane) {
    const int row = (lane >> 5) * 4 + ((lane >> 2) & 3);
    return at(row, (lane & 16) + (lane & 3) * 4) * (int)sizeof(T);
  }
  // Keys row .. row + 3 of column `column + (lane & 15)`; row and column are the
  // same in all 16 lanes of a group, multiples of 4 and 16.
  static __device__ __forceinline__ void read4(const T *tile, int row, int column, int lane, T out[4]) {
    if constexpr (sizeof(T) == 2) {
      const T *p = tile + at(row + ((lane >> 2) & 3), column + (lane & 3) * 4);
      union {
        i16x4 i;
        T t[4];
      } u;
      u.i = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          (__attribute__((address_space(3))) i16x4 *)p);
      out[0] = u.t[0], out[1] = u.t[1], out[2] = u.t[2], out[3] = u.t[3];
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) out[i] = tile[at(row + i, column + (lane & 15))];
    }
  }
};

// Reads at a byte address of LDS.
template <class V>
__device__ __forceinline__ V lds_read(unsigned address) {
  return *(const __attribute__((address_space(3))) V *)(uintptr_t)address;
}
__device__ __forceinline__ i16x4 lds_read_transposed(unsigned address) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4 *)(uintptr_t)address);
}
template <class T>
__device__ __forceinline__ unsigned lds_address(const T *p) {
  return (unsigned)(uintptr_t)(const __attribute__((address_space(3))) T *)p;
}

// ------------------------------------------------------------------ lanes

__device__ __forceinline__ float max_across_16(float x) {  // over lanes l, l ^ 16, l ^ 32, l ^ 48
  auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

__device__ __forceinline__ float sum_across_16(float x) {
  auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

__device__ __forceinline__ float max_across_32(float x) {  // over lanes l, l ^ 32
  auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

__device__ __forceinline__ float sum_across_32(float x) {
  auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }

// A vector in 8 bits: steps of max|x| times this.
constexpr float kStep127 = 1.0f / 127.0f;

// x in steps of `step` > 0, at most 127 of them (a subnormal step is rounded enough for more).
__device__ __forceinline__ int8_t whole8(float x, float step) {
  return (int8_t)(int)fminf(fmaxf(rintf(__fdiv_rn(x, step)), -127.0f), 127.0f);
}

// Whether any of eight values is infinite or NaN, and the values with such ones
// set to zero.
template <class T>
__device__ __forceinline__ bool clean8(typename Type<T>::Vec &v) {
  bool bad = false;
  if constexpr (sizeof(T) == 2) {
    union {
      typename Type<T>::Vec v;
      unsigned u[4];
    } x;
    x.v = v;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      // an exponent of ones carries into its sign bit
      const unsigned over = ((x.u[i] & Type<T>::kExpMask) + Type<T>::kExpOne) & 0x80008000u;
      bad |= over != 0;
      const unsigned drop = (over >> 15) * 0xffffu;
      x.u[i] &= ~drop;
    }
    v = x.v;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const bool b = !(fabsf(v[i]) < __builtin_inff());
      bad |= b;
      v[i] = b ? 0.0f : v[i];
    }
  }
  return bad;
}

}  // namespace paged
}  // namespace slnr
