// Rows of bf16, fp32 or fp16 at any address, eight columns a thread: loads by 16-byte
// words wherever the row starts, conversions, stores.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

#include <type_traits>

#include "sph_internal.h"

namespace sph {

// N words of elements of SIZE bytes that start `off` bytes into x (less than 16): moved to
// x's start.
template <int N, int SIZE>
__device__ __forceinline__ void shift_words(uint32_t (&x)[N + 4], int off) {
#pragma unroll
  for (int i = 0; i < N + 3; ++i) x[i] = off & 4 ? x[i + 1] : x[i];
#pragma unroll
  for (int i = 0; i < N + 2; ++i) x[i] = off & 8 ? x[i + 2] : x[i];
  if constexpr (SIZE == 2) {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = __funnelshift_r(x[i], x[i + 1], off & 2 ? 16 : 0);
  }
}

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__half x) { return __half2float(x); }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
template <class T> __device__ __forceinline__ T from_f32(float x);
template <> __device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <> __device__ __forceinline__ __half from_f32<__half>(float x) { return __float2half_rn(x); }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float x) {
  return __float2bfloat16_rn(x);
}
// Two values in a word, the first in the low half.
template <class T>
__device__ __forceinline__ uint32_t two_of(float lo, float hi) {
  if constexpr (std::is_same<T, __half>::value) {
    const __half2 h = __floats2half2_rn(lo, hi);
    return (uint32_t)__half_as_ushort(h.x) | (uint32_t)__half_as_ushort(h.y) << 16;
  } else {
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return (uint32_t)__bfloat16_as_ushort(h.x) | (uint32_t)__bfloat16_as_ushort(h.y) << 16;
  }
}

// Eight fp32 values at an address on 32 bytes, one access (in two, lanes 32 bytes apart
// touch every sector twice).
__device__ __forceinline__ void load_v8(const float* p, float (&v)[8]) {
  asm volatile("ld.global.v8.f32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]),
                 "=f"(v[7])
               : "l"(p)
               : "memory");
}
__device__ __forceinline__ void store_v8(float* p, const float (&v)[8]) {
  asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "f"(v[0]),
               "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7])
               : "memory");
}
__device__ __forceinline__ void load_v8(const void* p, uint32_t (&v)[8]) {
  asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]),
                 "=r"(v[7])
               : "l"(p)
               : "memory");
}
__device__ __forceinline__ void store_v8(void* p, const uint32_t (&v)[8]) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(v[0]),
               "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7])
               : "memory");
}
__device__ __forceinline__ bool on32(const void* p) { return ((uintptr_t)p & 31) == 0; }

// Eight consecutive elements at any address, by the 16-byte words that hold them (each of
// which holds one of the elements at least).
template <class T>
__device__ __forceinline__ void load_8(const T* p, float (&v)[8]) {
  constexpr int N = 2 * (int)sizeof(T);         // words
  const int off = (int)((uintptr_t)p & 15);
  const uint4* w = reinterpret_cast<const uint4*>((uintptr_t)p - off);
  uint32_t x[N + 4];
#pragma unroll
  for (int i = 0; i <= N / 4; ++i) {
    const uint4 q = i < N / 4 || off ? w[i] : make_uint4(0, 0, 0, 0);
    x[4 * i] = q.x; x[4 * i + 1] = q.y; x[4 * i + 2] = q.z; x[4 * i + 3] = q.w;
  }
  shift_words<N, sizeof(T)>(x, off);
  const T* e = reinterpret_cast<const T*>(x);
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = to_f32(e[j]);
}

// A thread's eight columns of a row, col .. col + 7 (those in 0 .. d - 1; zeros for the
// others).  VEC: rows and col are on 16 bytes.
template <class T, bool VEC>
__device__ __forceinline__ void load_cols(const T* row, int col, int d, float (&v)[8]) {
  const bool all = (VEC || col >= 0) && col + 8 <= d;
  if (VEC && all) {
    uint4 w[sizeof(T) / 2];
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i)
      w[i] = reinterpret_cast<const uint4*>(row + col)[i];
    const T* e = reinterpret_cast<const T*>(w);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = to_f32(e[j]);
  } else if (all) {
    load_8(row + col, v);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      v[j] = col + j >= 0 && col + j < d ? to_f32(row[col + j]) : 0.f;
  }
}
// ON16: row + col is on 16 bytes.
template <class T, bool ON16>
__device__ __forceinline__ void store_cols(T* row, int col, int d, const float (&v)[8]) {
  if (ON16 && col >= 0 && col + 8 <= d) {
    uint32_t w[2 * sizeof(T)];
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int j = 0; j < 8; ++j) w[j] = __float_as_uint(v[j]);
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) w[j] = two_of<T>(v[2 * j], v[2 * j + 1]);
    }
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i)
      reinterpret_cast<uint4*>(row + col)[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (col + j >= 0 && col + j < d) row[col + j] = from_f32<T>(v[j]);
  }
}

inline bool on16(const void* p, int64_t ld, int size) {
  return ((uintptr_t)p & 15) == 0 && (ld * size & 15) == 0;
}
inline int type_size(int t) { return t == TAB_FP32 ? 4 : 2; }

}  // namespace sph
