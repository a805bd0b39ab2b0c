// Microscaled 4-bit floating point: e2m1 codes with a scale for each block of
// a row, in the two forms the table operators hold rows in.
//
//   e8m0   32-column blocks; scale 2^(floor(log2(amax)) - 2), at least 2^-126
//   e4m3   16-column blocks; scale RNE_e4m3(amax / 6 / 2^k), where 2^k is the
//          row's own: the least with amax(row) <= 6 * 448 * 2^k
//
// A value stands for code * scale (* 2^k); every product of these factors has
// at most 6 significant bits, so it is exact in fp32 and in bf16.  A block that
// holds a NaN or an infinity gets a NaN scale and stands for NaN throughout.
#pragma once

#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <stdint.h>

namespace sph {

enum Mx4Format : int { MX4_E8M0 = 0, MX4_E4M3 = 1 };

template <int FMT>
struct Mx4 {
  static constexpr int kBlock = FMT == MX4_E4M3 ? 16 : 32;     // columns of a scale
  static constexpr uint32_t kNanScale = FMT == MX4_E4M3 ? 0x7Fu : 0xFFu;
};

constexpr unsigned kInfBits = 0x7F800000u;

// The row exponent k of the e4m3 form from the bits of the row's largest finite
// magnitude; 0 for a row of zeros.  2688 = 6 * 448 = 1.3125 * 2^11.  k stays in
// [-110, 116], where 2^k, its inverse and the steps below are normal numbers.
__device__ __forceinline__ int mx4_row_exp(unsigned amax_bits) {
  if (amax_bits == 0) return 0;
  const int k = (int)(amax_bits >> 23) - 127 - 11 + ((amax_bits & 0x7FFFFFu) > 0x280000u);
  return min(116, max(-110, k));
}
__device__ __forceinline__ float exp2_int(int k) {      // 2^k for k in [-126, 127]
  return __uint_as_float((unsigned)(k + 127) << 23);
}

// The scale byte of a block whose largest magnitude has the bits `amax`
// (finite), and the step (scale times row scale) that its codes count in.
template <int FMT>
__device__ __forceinline__ uint32_t mx4_scale(unsigned amax, int row_exp, float* step) {
  if constexpr (FMT == MX4_E4M3) {
    // amax / 6 as IEEE division rounds it (as in mx4_codes below)
    const float a = __uint_as_float(amax) * exp2_int(-row_exp), r6 = 1.0f / 6.0f;
    float v = a * r6;
    v = __fmaf_rn(__fmaf_rn(-6.0f, v, a), r6, v);
    const __nv_fp8_storage_t b = __nv_cvt_float_to_fp8(v, __NV_SATFINITE, __NV_E4M3);
    const __half_raw h = __nv_cvt_fp8_to_halfraw(b, __NV_E4M3);
    *step = __half2float(__half(h)) * exp2_int(row_exp);
    return b;
  } else {
    const int e = max((int)(amax >> 23) - 127 - 2, -126);
    *step = exp2_int(e);
    return (uint32_t)(e + 127);
  }
}

// The float that a scale byte stands for (e8m0: 0 is 2^-127, 255 NaN).
template <int FMT>
__device__ __forceinline__ float mx4_scale_value(uint32_t b) {
  if constexpr (FMT == MX4_E4M3) {
    const __half_raw h = __nv_cvt_fp8_to_halfraw((__nv_fp8_storage_t)b, __NV_E4M3);
    return __half2float(__half(h));
  } else {
    return __uint_as_float(b == 0 ? 0x00400000u : b == 255 ? 0x7FFFFFFFu : b << 23);
  }
}

// Eight e2m1 codes (column j in bits 4j) as floats.
__device__ __forceinline__ void e2m1x8_to_float(uint32_t codes, float (&v)[8]) {
  uint32_t h[4];
  asm("{\n .reg .b8 b0, b1, b2, b3;\n mov.b32 {b0, b1, b2, b3}, %4;\n"
      " cvt.rn.f16x2.e2m1x2 %0, b0;\n cvt.rn.f16x2.e2m1x2 %1, b1;\n"
      " cvt.rn.f16x2.e2m1x2 %2, b2;\n cvt.rn.f16x2.e2m1x2 %3, b3;\n}\n"
      : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3])
      : "r"(codes));
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h[i]));
    v[2 * i] = f.x;
    v[2 * i + 1] = f.y;
  }
}

// Eight floats to the nearest e2m1 codes (ties to even, saturating at 6).
__device__ __forceinline__ uint32_t float_to_e2m1x8(const float (&t)[8]) {
  uint32_t c;
  asm("{\n .reg .b8 b0, b1, b2, b3;\n"
      " cvt.rn.satfinite.e2m1x2.f32 b0, %2, %1;\n cvt.rn.satfinite.e2m1x2.f32 b1, %4, %3;\n"
      " cvt.rn.satfinite.e2m1x2.f32 b2, %6, %5;\n cvt.rn.satfinite.e2m1x2.f32 b3, %8, %7;\n"
      " mov.b32 %0, {b0, b1, b2, b3};\n}\n"
      : "=r"(c)
      : "f"(t[0]), "f"(t[1]), "f"(t[2]), "f"(t[3]), "f"(t[4]), "f"(t[5]), "f"(t[6]), "f"(t[7]));
  return c;
}

// Codes of N values (8 to a word) in units of `step` (0: a block that underflowed,
// all codes zero).  x / step is rounded as IEEE division rounds it, from the
// correctly rounded reciprocal and two fused steps (Markstein, IBM J. Res.
// Dev. 34, 1990): a division a value would cost as much as the pass's memory
// traffic.  The rounded quotient meets a midpoint of two codes only where the
// exact one does (step has 4 significant bits), so codes are the nearest ones
// exactly.  An e8m0 step is a power of two and needs one product.
template <int FMT, int N>
__device__ __forceinline__ void mx4_codes(const float (&x)[N], float step, uint32_t (&codes)[N / 8]) {
  const float r = step > 0.f ? __frcp_rn(step) : 0.f;
#pragma unroll
  for (int w = 0; w < N / 8; ++w) {
    float t[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float v = x[8 * w + j];
      t[j] = v * r;
      if constexpr (FMT == MX4_E4M3) t[j] = __fmaf_rn(__fmaf_rn(-t[j], step, v), r, t[j]);
    }
    codes[w] = float_to_e2m1x8(t);
  }
}

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

}  // namespace sph
