// e4m3 with an fp32 scale for each block of 128 columns (of one row, or of 128 rows):
//
//   scale = max(amax / 448, 2^-126), rounded to fp32, of the block's largest magnitude
//   code  = the e4m3 value nearest to x / scale, ties to the even code
//
// A value stands for code * scale.  A block that holds a NaN or an infinity gets a NaN
// scale and codes of zero, and stands for NaN throughout.
#pragma once

#include <cuda_fp8.h>
#include <stdint.h>

#include "sph_internal.h"

namespace sph {

constexpr unsigned kFp8Inf = 0x7F800000u;

// A block's scale from the bits of its largest magnitude, and what its codes need: x is
// coded as (x * lift) / step, where lift is 1 or, for small scales, the exact 2^64 that keeps
// the remainders below clear of fp32's least step.
struct Fp8Scale {
  float scale, step, lift, inv;
};
__device__ __forceinline__ Fp8Scale fp8_scale(unsigned amax_bits) {
  Fp8Scale s;
  if (amax_bits >= kFp8Inf) {
    s.scale = __uint_as_float(0x7FFFFFFFu);
    s.step = s.lift = s.inv = 0.f;
    return s;
  }
  s.scale = fmaxf(__uint_as_float(amax_bits) / 448.f, 0x1p-126f);
  s.lift = s.scale < 0x1p-60f ? 0x1p64f : 1.f;
  s.step = s.scale * s.lift;
  s.inv = 1.f / s.step;
  return s;
}

// x / step, such that e4m3's rounding of it is that of the exact quotient.  The quotient by
// the reciprocal is within an ulp or two, one correction leaves it the nearest fp32 value
// or next to it; where that lies on a border of two codes (or on a code: its low 19 bits are
// zeros, a code's 3 bits and the border's one being above them) the remainder tells on which
// side the exact one is, and the quotient moves one step that way.
__device__ __forceinline__ float fp8_quotient(float x, const Fp8Scale& s) {
  const float v = x * s.lift;
  float q = v * s.inv;
  q = copysignf(__fmaf_rn(__fmaf_rn(-q, s.step, v), s.inv, q), v);      // (-0 stays -0)
  if ((__float_as_uint(q) & 0x7FFFFu) == 0 && q != 0.f) {
    const float rest = __fmaf_rn(-q, s.step, v);          // exact
    if (rest != 0.f) q = __int_as_float(__float_as_int(q) + ((rest > 0.f) == (q > 0.f) ? 1 : -1));
  }
  return q;
}

// Four values to four codes, the first in the low byte (saturating at 448).
__device__ __forceinline__ uint32_t fp8_codes4(float a, float b, float c, float d) {
  const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
  const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(c, d), __NV_SATFINITE, __NV_E4M3);
  return lo | hi << 16;
}

}  // namespace sph
