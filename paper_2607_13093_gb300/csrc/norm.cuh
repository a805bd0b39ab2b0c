// What the layer norm's two directions share: pieces of rows, parameters and results of any type.
#pragma once

#include <type_traits>

#include "f2.cuh"
#include "rows.cuh"
#include "sm100_ptx.cuh"
#include "sph_internal.h"

namespace sph {

// A thread holds a row in pieces of eight columns.  MODE:
//   0  any row: the eight are 32 columns apart, a warp's accesses 32 columns side by side
//      wherever the row starts;
//   1  d is a multiple of 8, and all rows and parameters are on 16 bytes (fp32: 32): the eight
//      are neighbours, read and written in one access;
//   2  (the norm alone) the same, and parameters and results have the type of x: no branch on a
//      type;
//   3  the same with fp32 parameters (16384 x 5120 bf16 56 us, with a branch 62; 10000 x 8192 58
//      and 70).
template <int MODE>
__device__ __forceinline__ int piece_col(int i, int t, int threads) {
  return MODE ? (i * threads + t) * 8 : (i * threads + (t & ~31)) * 8 + (t & 31);
}
template <int MODE> constexpr int kStep = MODE ? 1 : 32;
// The first and the last of the eight are before d.
template <int MODE>
__device__ __forceinline__ bool whole(int col, int d) { return MODE || col + 7 * 32 < d; }

// Eight columns as they were read: 16-bit ones stay packed.  MODE 0: those from d on read as zeros.
template <class T, int MODE>
struct Eight {
  uint32_t w[4];
  __device__ __forceinline__ void load(const T* row, int col, int d) {
    if constexpr (MODE) {
      const uint4 q = *reinterpret_cast<const uint4*>(row + col);
      w[0] = q.x; w[1] = q.y; w[2] = q.z; w[3] = q.w;
    } else {
      const uint16_t* bits = reinterpret_cast<const uint16_t*>(row) + col;
      uint32_t e[8];
      if (whole<MODE>(col, d)) {
#pragma unroll
        for (int j = 0; j < 8; ++j) e[j] = bits[j * 32];
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) e[j] = col + j * 32 < d ? bits[j * 32] : 0u;
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) w[j] = e[2 * j] | e[2 * j + 1] << 16;
    }
  }
  __device__ __forceinline__ float get(int j) const {
    if constexpr (std::is_same<T, __half>::value)
      return __half2float(__ushort_as_half((uint16_t)(j & 1 ? w[j >> 1] >> 16 : w[j >> 1] & 0xFFFFu)));
    else
      return __uint_as_float(j & 1 ? w[j >> 1] & 0xFFFF0000u : w[j >> 1] << 16);
  }
  __device__ __forceinline__ F2 two(int k) const { return f2(get(2 * k), get(2 * k + 1)); }
};
template <int MODE>
struct Eight<float, MODE> {
  float v[8];
  __device__ __forceinline__ void load(const float* row, int col, int d) {
    if constexpr (MODE) {
      load_v8(row + col, v);
    } else if (whole<MODE>(col, d)) {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = row[col + j * 32];
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = col + j * 32 < d ? row[col + j * 32] : 0.f;
    }
  }
  __device__ __forceinline__ float get(int j) const { return v[j]; }
  __device__ __forceinline__ F2 two(int k) const { return f2(v[2 * k], v[2 * k + 1]); }
};

template <class T, int MODE>
__device__ __forceinline__ void load_eight(const void* p, int col, int d, F2 (&v)[4]) {
  Eight<T, MODE> e;
  e.load(static_cast<const T*>(p), col, d);
#pragma unroll
  for (int k = 0; k < 4; ++k) v[k] = e.two(k);
}
template <class T, int MODE>
__device__ __forceinline__ void store_eight(void* p, int64_t at, int col, int d, const F2 (&v2)[4]) {
  T* row = static_cast<T*>(p) + at;
  float v[8];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const float2 r = both(v2[k]);
    v[2 * k] = r.x; v[2 * k + 1] = r.y;
  }
  if constexpr (MODE == 0) {
    if (whole<MODE>(col, d)) {
#pragma unroll
      for (int j = 0; j < 8; ++j) row[col + j * 32] = from_f32<T>(v[j]);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (col + j * 32 < d) row[col + j * 32] = from_f32<T>(v[j]);
    }
  } else if constexpr (sizeof(T) == 4) {
    store_v8(row + col, v);
  } else {
    store_cols<T, true>(row, col, col + 8, v);
  }
}
// Eight columns of a parameter row in fp32 (T: x's type).
template <class T, int MODE>
__device__ __forceinline__ void load_param(const void* p, int type, int col, int d, F2 (&v)[4]) {
  if (MODE == 2) load_eight<T, MODE>(p, col, d, v);
  else if (MODE == 3) load_eight<float, MODE>(p, col, d, v);
  else if (type == TAB_FP32) load_eight<float, MODE>(p, col, d, v);
  else if (type == TAB_BF16) load_eight<__nv_bfloat16, MODE>(p, col, d, v);
  else load_eight<__half, MODE>(p, col, d, v);
}
// Eight columns of a result row.
template <class T, int MODE>
__device__ __forceinline__ void store_row(void* p, int type, int64_t at, int col, int d,
                                          const F2 (&v)[4]) {
  if (MODE >= 2) store_eight<T, MODE>(p, at, col, d, v);
  else if (type == TAB_FP32) store_eight<float, MODE>(p, at, col, d, v);
  else if (type == TAB_BF16) store_eight<__nv_bfloat16, MODE>(p, at, col, d, v);
  else store_eight<__half, MODE>(p, at, col, d, v);
}

// Rows of `type` can be read and written eight columns an access.
inline bool wide_rows(const void* p, int64_t ld, int type) {
  const int size = type_size(type);
  return ((uintptr_t)p & (size * 8 - 1)) == 0 && (ld & 7) == 0;
}

}  // namespace sph
