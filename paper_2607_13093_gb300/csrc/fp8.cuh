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

#include "f2.cuh"
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
// or next to it.  Where that lies on a border of two codes (or on a code: its low 19 bits are
// zeros, a code's 3 bits and the border's one being above them) the remainder tells on which
// side the exact one is, and the quotient moves one step that way (fp8_settled).
//
// rest: q step - x lift, exact.  (With the remainder's sign so, -0 stays -0.)
struct Fp8Two {
  F2 q, rest;
};
__device__ __forceinline__ Fp8Two fp8_quotients(F2 x, const Fp8Scale& s) {
  const F2 minus = mul2(x, f2(-s.lift));
  F2 q = mul2(minus, f2(-s.inv));
  q = fma2(fma2(q, f2(s.step), minus), f2(-s.inv), q);
  return {q, fma2(q, f2(s.step), minus)};
}
__device__ __forceinline__ float fp8_settled(float q, float rest) {
  const int bits = __float_as_int(q);
  const int less = (bits ^ __float_as_int(rest)) >> 31 | 1;       // -1: q is too small in magnitude
  const bool moves = ((bits & 0x7FFFF) == 0) & (rest != 0.f) & (q != 0.f);
  return __int_as_float(moves ? bits - less : bits);
}

// The same codes for x and amax of at most 11 significant bits (bf16, fp16), by a product.  The
// ideal quotient x 448 / amax is a border of two codes (an integer of 5 bits or fewer and a power
// of two) or off it by 1 / (31 * 2047) at least, 2^-16.  x / scale differs from it by what
// rounding the scale took, less than 2^-23, on the same side for the whole block: so all that lie
// next to a border go one way, and x times the reciprocal moved by 2^-19 that way has the same
// codes as x / scale.  Where the scale was not rounded (amax is a multiple of 7), quotients on a
// border are exact: rounded to 18 bits they stay there, free of the product's error.  A scale of
// 2^-126 has an exact reciprocal.  (Quotients on a border are not rare here: 1 of 400 of normal
// bf16 values, so that most warps met some; with exact quotients and a branch for them
// 32000 x 4096 bf16 was coded in 82 us, so in 59.)
struct Fp8Product {
  F2 inv, nudge;
  bool on_border;
};
__device__ __forceinline__ Fp8Product fp8_product(unsigned amax_bits, const Fp8Scale& s) {
  const float off = __fmaf_rn(s.scale, 448.f, -__uint_as_float(amax_bits));      // exact
  const bool rounded = s.scale > 0x1p-126f && off != 0.f;
  Fp8Product p;
  p.on_border = s.scale > 0x1p-126f && off == 0.f;
  p.inv = f2(s.inv * s.lift);
  p.nudge = f2(!rounded ? 1.f : off > 0.f ? 1.f - 0x1p-19f : 1.f + 0x1p-19f);
  return p;
}
// ROUND: some lane's block has quotients on a border.
template <bool ROUND>
__device__ __forceinline__ float2 fp8_by_product(float lo, float hi, const Fp8Product& p, F2 inv_nudged) {
  if constexpr (!ROUND) {
    return both(mul2(f2(lo, hi), inv_nudged));
  } else {
    const F2 q = mul2(f2(lo, hi), p.inv), c = mul2(q, f2(65.f));
    const F2 high = fma2(fma2(q, f2(-1.f), c), f2(-1.f), c);             // c - (c - q): 18 bits
    return both(mul2(high, p.nudge));
  }
}

// Four values to four codes, the first in the low byte (saturating at 448).
__device__ __forceinline__ uint32_t fp8_codes4(float a, float b, float c, float d) {
  const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
  const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(c, d), __NV_SATFINITE, __NV_E4M3);
  return lo | hi << 16;
}

}  // namespace sph
