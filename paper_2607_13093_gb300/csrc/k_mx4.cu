// Rows into microscaled 4-bit floating point: the table form (codes and scales
// row by row) and the operand form of the 4-bit product, whose scales lie
// stage by stage as it copies them and which holds a row as the sum of several
// terms, each the 4-bit form of what the terms before it left over.
//
// Bound by memory: an element is read once (2 or 4 bytes) and leaves 4.5 or
// 4.25 bits.  A row belongs to a warp or a block, whose threads hold it in
// registers, 8 consecutive columns a thread and step, while the row's and the
// blocks' maxima are made (a block's by one or two shuffles); rows too long for
// the registers are read twice.
#include <cuda_bf16.h>

#include "mx4.cuh"
#include "sm100_ptx.cuh"
#include "sph_internal.h"

namespace sph {
namespace {

constexpr int kQuantUnits = 4;      // 8-column steps a thread holds in registers

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__half x) { return __half2float(x); }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }

// Columns col .. col + 7 of a row of d columns; zeros beyond it.  vec: the row
// starts on 16 bytes.  Coherent loads: the caller's kernel may have written x
// just before.
template <class T>
__device__ __forceinline__ void load8(const T* row, int col, int d, bool vec, float (&v)[8]) {
  if (vec && col + 8 <= d) {
    uint4 w[sizeof(T) / 2];
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i)
      w[i] = reinterpret_cast<const uint4*>(row + col)[i];
    const T* e = reinterpret_cast<const T*>(w);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = to_f32(e[j]);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = col + j < d ? to_f32(row[col + j]) : 0.f;
  }
}

// Bits of the largest magnitude of a block, from its threads' eights.
template <int FMT>
__device__ __forceinline__ unsigned block_amax(const float (&v)[8]) {
  unsigned m = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) m = max(m, __float_as_uint(v[j]) & 0x7FFFFFFFu);
  m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, 1));
  if constexpr (FMT == MX4_E8M0) m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, 2));
  return m;
}

// TPR threads a row.  OPERAND: the product's form.
template <class T, int FMT, int TPR, bool OPERAND>
__global__ void __launch_bounds__(TPR < 128 ? 128 : TPR)
quant_kernel(const Mx4Quant a) {
  constexpr int kRows = TPR < 128 ? 128 / TPR : 1;     // rows of a block
  constexpr int kSpan = TPR * kQuantUnits;             // 8-column steps a turn
  ptx::griddep_wait();
  ptx::griddep_launch_dependents();
  const int t = threadIdx.x % TPR, lane = threadIdx.x & 31;
  const int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / TPR;
  if (row >= a.rows) return;                           // (whole warps; TPR >= 128: whole blocks)
  const T* x = static_cast<const T*>(a.x) + row * a.ld_x;
  const bool vec = a.aligned != 0;
  const int turns = (a.scale_cols / 8 + kSpan - 1) / kSpan;
  float v[kQuantUnits][8];
  unsigned amax[kQuantUnits];
  auto load = [&](int turn) {
#pragma unroll
    for (int i = 0; i < kQuantUnits; ++i)
      load8(x, (turn * kSpan + i * TPR + t) * 8, a.d, vec, v[i]);
#pragma unroll
    for (int i = 0; i < kQuantUnits; ++i) amax[i] = block_amax<FMT>(v[i]);
  };
  int row_exp = 0;
  if constexpr (FMT == MX4_E4M3) {
    unsigned top = 0;
    for (int turn = 0; turn < turns; ++turn) {
      load(turn);
#pragma unroll
      for (int i = 0; i < kQuantUnits; ++i)
        if (amax[i] < kInfBits) top = max(top, amax[i]);
    }
    top = __reduce_max_sync(0xFFFFFFFFu, top);
    if constexpr (TPR > 32) {
      __shared__ unsigned s_top[TPR / 32];
      if (lane == 0) s_top[threadIdx.x / 32] = top;
      __syncthreads();
#pragma unroll
      for (int w = 0; w < TPR / 32; ++w) top = max(top, s_top[w]);
    }
    row_exp = mx4_row_exp(top);
  }
  if (t == 0 && a.row_scale) a.row_scale[row] = exp2_int(row_exp);
  // the row's scale words: word i at at_scale + i / tile_words * step + i % tile_words
  // words (table form: one after another)
  int64_t at_scale, step;
  int words;
  if constexpr (OPERAND) {
    const int tile = (int)(row / a.tile_rows), r = (int)(row % a.tile_rows);
    words = a.tile_words;
    at_scale = (int64_t)tile * a.tile_bytes + r * words * 4;
    step = a.tile_rows * words * 4;
  } else {
    words = 1;
    at_scale = row * a.ld_scales;
    step = 4;
  }
  uint8_t* codes = a.codes + row * a.ld_codes;
  const int code_cols = (a.d + 31) / 32 * 32;
  for (int turn = 0; turn < turns; ++turn) {
    if (FMT == MX4_E8M0 || turns > 1) load(turn);
    for (int p = 0; p < a.planes; ++p) {
#pragma unroll
      for (int i = 0; i < kQuantUnits; ++i) {
        const int unit = turn * kSpan + i * TPR + t, col = unit * 8;
        if (p > 0) amax[i] = block_amax<FMT>(v[i]);
        const bool bad = amax[i] >= kInfBits;
        float unit_step = 0.f;
        uint32_t s = 0, c = 0;
        if (bad) {
          s = Mx4<FMT>::kNanScale;
        } else if (col / Mx4<FMT>::kBlock * Mx4<FMT>::kBlock < a.d) {
          s = mx4_scale<FMT>(amax[i], row_exp, &unit_step);
          c = mx4_codes<FMT>(v[i], unit_step);
        }
        if (col < code_cols) *reinterpret_cast<uint32_t*>(codes + p * a.plane_codes + unit * 4) = c;
        // four scales to a word, stored by the lane that holds the first
        constexpr int kLanes = Mx4<FMT>::kBlock / 8;
        s |= __shfl_down_sync(0xFFFFFFFFu, s, kLanes) << 8;
        s |= __shfl_down_sync(0xFFFFFFFFu, s, 2 * kLanes) << 16;
        if (lane % (4 * kLanes) == 0 && col < a.scale_cols) {
          const int w = unit / (4 * kLanes);
          *reinterpret_cast<uint32_t*>(a.scales + p * a.plane_scales + at_scale +
                                       w / words * step + w % words * 4) = s;
        }
        if (p + 1 < a.planes && !bad) {
          float q[8];
          e2m1x8_to_float(c, q);
#pragma unroll
          for (int j = 0; j < 8; ++j) v[i][j] = __fmaf_rn(-q[j], unit_step, v[i][j]);   // exact
        }
      }
    }
  }
}

template <class T, int FMT, bool OPERAND>
cudaError_t launch(const Mx4Quant& a, cudaStream_t st) {
  // one warp a row up to 1024 columns, a block of 128 threads up to 4096, of
  // 256 above: each holds its row in registers up to 8192 columns.
  if (a.scale_cols <= 32 * kQuantUnits * 8)
    return launch_pdl(quant_kernel<T, FMT, 32, OPERAND>, dim3((unsigned)((a.rows + 3) / 4)),
                      dim3(128), 0, st, a);
  if (a.scale_cols <= 128 * kQuantUnits * 8)
    return launch_pdl(quant_kernel<T, FMT, 128, OPERAND>, dim3((unsigned)a.rows), dim3(128), 0, st,
                      a);
  return launch_pdl(quant_kernel<T, FMT, 256, OPERAND>, dim3((unsigned)a.rows), dim3(256), 0, st,
                    a);
}
template <class T>
cudaError_t launch_t(const Mx4Quant& a, int fmt, bool operand, cudaStream_t st) {
  if (fmt == MX4_E4M3)
    return operand ? launch<T, MX4_E4M3, true>(a, st) : launch<T, MX4_E4M3, false>(a, st);
  return operand ? launch<T, MX4_E8M0, true>(a, st) : launch<T, MX4_E8M0, false>(a, st);
}

}  // namespace

cudaError_t launch_mx4_quant(Mx4Quant a, int fmt, int x_type, bool operand, cudaStream_t st) {
  const int es = x_type == TAB_FP32 ? 4 : 2;
  a.aligned = ((uintptr_t)a.x & 15) == 0 && (a.ld_x * es & 15) == 0;
  if (x_type == TAB_FP32) return launch_t<float>(a, fmt, operand, st);
  if (x_type == TAB_BF16) return launch_t<__nv_bfloat16>(a, fmt, operand, st);
  return launch_t<__half>(a, fmt, operand, st);
}

}  // namespace sph
