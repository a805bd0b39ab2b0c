// What the layer norm's two directions share: parameters of any type, results of any type.
#pragma once

#include "rows.cuh"
#include "sph_internal.h"

namespace sph {

// Eight columns of a weight or bias row in fp32.
template <bool VEC>
__device__ __forceinline__ void load_param(const void* p, int type, bool on16, int col, int d,
                                           float (&v)[8]) {
  if (type == TAB_FP32) {
    if (VEC && on16) load_cols<float, true>(static_cast<const float*>(p), col, d, v);
    else load_cols<float, false>(static_cast<const float*>(p), col, d, v);
  } else if (type == TAB_BF16) {
    if (VEC && on16) load_cols<__nv_bfloat16, true>(static_cast<const __nv_bfloat16*>(p), col, d, v);
    else load_cols<__nv_bfloat16, false>(static_cast<const __nv_bfloat16*>(p), col, d, v);
  } else {
    if (VEC && on16) load_cols<__half, true>(static_cast<const __half*>(p), col, d, v);
    else load_cols<__half, false>(static_cast<const __half*>(p), col, d, v);
  }
}
// Columns of a result row of any type (ON16: as store_cols).
template <bool ON16>
__device__ __forceinline__ void store_row(void* p, int type, int64_t at, int col, int d,
                                          const float (&v)[8]) {
  if (type == TAB_FP32) store_cols<float, ON16>(static_cast<float*>(p) + at, col, d, v);
  else if (type == TAB_BF16) store_cols<__nv_bfloat16, ON16>(static_cast<__nv_bfloat16*>(p) + at, col, d, v);
  else store_cols<__half, ON16>(static_cast<__half*>(p) + at, col, d, v);
}

}  // namespace sph
