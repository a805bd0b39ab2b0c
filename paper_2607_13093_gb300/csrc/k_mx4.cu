// Rows into microscaled 4-bit floating point: the table form (codes and scales
// row by row) and the operand form of the 4-bit product, whose scales lie
// stage by stage as it copies them and which holds a row as the sum of several
// terms, each the 4-bit form of what the terms before it left over.
//
// Bound by memory: an element is read once (2 or 4 bytes) and leaves 4.5 or
// 4.25 bits.  A row belongs to a warp or a block, whose threads hold it as it was
// read, 16 consecutive columns a thread and step, while the row's and the blocks'
// maxima are made; rows too long for the registers are read twice.  What a
// block's scale costs is shared by its 16 columns (with 8 columns a thread,
// 32000 x 4096 bf16 rows took 125 us, the readback included; so 113).
#include <cuda_bf16.h>

#include <type_traits>

#include "mx4.cuh"
#include "rows.cuh"
#include "sm100_ptx.cuh"
#include "sph_internal.h"

namespace sph {
namespace {

constexpr int kCols = 16;           // columns of a thread and step

// 16 columns as they lie in memory.
template <class T>
struct Raw {
  uint4 w[sizeof(T)];
};
template <class T> __device__ __forceinline__ float element(const Raw<T>& r, int j);
template <> __device__ __forceinline__ float element<float>(const Raw<float>& r, int j) {
  return reinterpret_cast<const float*>(r.w)[j];
}
template <> __device__ __forceinline__ float element<__half>(const Raw<__half>& r, int j) {
  return __half2float(reinterpret_cast<const __half*>(r.w)[j]);
}
template <> __device__ __forceinline__ float element<__nv_bfloat16>(const Raw<__nv_bfloat16>& r,
                                                                     int j) {
  const uint32_t w = reinterpret_cast<const uint32_t*>(r.w)[j / 2];
  return __uint_as_float(j % 2 ? w & 0xFFFF0000u : w << 16);
}

// Columns col .. col + 15 of a row, zeros past column d.  aligned: the row starts on 16
// bytes.  Other rows are read by the 16-byte words that hold the columns (each of which
// holds one at least) and shifted (32000 x 4095 bf16 75 us; column by column through
// shared memory 93).  Coherent loads: the caller's kernel may have
// written x just before.
template <class T>
__device__ __forceinline__ void load_raw(const T* row, int col, int d, bool aligned, Raw<T>& r) {
  constexpr int N = (int)sizeof(T);             // 16-byte words of the columns
  if (col + kCols > d) {
#pragma unroll
    for (int i = 0; i < N; ++i) r.w[i] = make_uint4(0, 0, 0, 0);
    T* e = reinterpret_cast<T*>(r.w);
#pragma unroll
    for (int j = 0; j < kCols; ++j)
      if (col + j < d) e[j] = row[col + j];
  } else if (aligned) {
#pragma unroll
    for (int i = 0; i < N; ++i) r.w[i] = reinterpret_cast<const uint4*>(row + col)[i];
  } else {
    const int off = (int)((uintptr_t)(row + col) & 15);
    const uint4* w = reinterpret_cast<const uint4*>((uintptr_t)(row + col) - off);
    uint32_t x[4 * N + 4];
#pragma unroll
    for (int i = 0; i <= N; ++i) {
      const uint4 q = i < N || off ? w[i] : make_uint4(0, 0, 0, 0);
      x[4 * i] = q.x; x[4 * i + 1] = q.y; x[4 * i + 2] = q.z; x[4 * i + 3] = q.w;
    }
    shift_words<4 * N, N>(x, off);
#pragma unroll
    for (int i = 0; i < N; ++i)
      r.w[i] = make_uint4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]);
  }
}

// Bits of the largest magnitude of a block as fp32 (kInfBits or more: it holds a
// NaN or an infinity).  16-bit types compare two columns an instruction, as bits.
template <int FMT, class T>
__device__ __forceinline__ unsigned block_amax(const Raw<T>& r) {
  unsigned m = 0;
  const uint32_t* w = reinterpret_cast<const uint32_t*>(r.w);
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int j = 0; j < kCols; ++j) m = max(m, w[j] & 0x7FFFFFFFu);
  } else {
#pragma unroll
    for (int j = 0; j < kCols / 2; ++j) m = __vmaxu2(m, w[j] & 0x7FFF7FFFu);
    m = max(m >> 16, m & 0xFFFFu);
  }
  if constexpr (FMT == MX4_E8M0) m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, 1));
  if constexpr (std::is_same<T, __nv_bfloat16>::value) m <<= 16;
  if constexpr (std::is_same<T, __half>::value)
    m = m >= 0x7C00u ? kInfBits : __float_as_uint(__half2float(__ushort_as_half((unsigned short)m)));
  return m;
}
template <int FMT>
__device__ __forceinline__ unsigned block_amax(const float (&v)[kCols]) {
  unsigned m = 0;
#pragma unroll
  for (int j = 0; j < kCols; ++j) m = max(m, __float_as_uint(v[j]) & 0x7FFFFFFFu);
  if constexpr (FMT == MX4_E8M0) m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, 1));
  return m;
}

// TPR threads a row, U steps of 16 columns a thread and turn.  OPERAND: the
// product's form.
template <class T, int FMT, int TPR, int U, bool OPERAND>
__global__ void __launch_bounds__(TPR < 128 ? 128 : TPR) quant_kernel(const Mx4Quant a) {
  constexpr int kThreads = TPR < 128 ? 128 : TPR;
  constexpr int kRows = kThreads / TPR;                // rows of a block
  constexpr int kSpan = TPR * U;                       // steps a turn
  ptx::griddep_wait();
  ptx::griddep_launch_dependents();
  if constexpr (OPERAND) {
    for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < a.zeros;
         i += (int64_t)gridDim.x * kThreads)
      a.zero[i] = 0;
  }
  const int t = threadIdx.x % TPR, lane = threadIdx.x & 31;
  const int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / TPR;
  if (row >= a.rows) return;                           // (whole warps; TPR >= 128: whole blocks)
  const T* x = static_cast<const T*>(a.x) + row * a.ld_x;
  const bool aligned = a.aligned != 0;
  const int turns = (a.scale_cols / kCols + kSpan - 1) / kSpan;
  Raw<T> raw[U];
  unsigned amax[U];
  auto load = [&](int turn) {
#pragma unroll
    for (int i = 0; i < U; ++i)
      load_raw<T>(x, (turn * kSpan + i * TPR + t) * kCols, a.d, aligned, raw[i]);
#pragma unroll
    for (int i = 0; i < U; ++i) amax[i] = block_amax<FMT>(raw[i]);
  };
  int row_exp = 0;
  if constexpr (FMT == MX4_E4M3) {
    unsigned top = 0;
    for (int turn = 0; turn < turns; ++turn) {
      load(turn);
#pragma unroll
      for (int i = 0; i < U; ++i)
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
  // the row's scale words: word i at at_scale + i / words * step + i % words * 4
  // (table form: one after another)
  int64_t at_scale, step;
  int words;
  if constexpr (OPERAND) {
    const int tile = (int)(row / a.tile_rows), r = (int)(row % a.tile_rows);
    words = a.tile_words;
    at_scale = (int64_t)tile * a.tile_bytes + r * words * 4;
    step = a.stage_bytes;
  } else {
    words = 1;
    at_scale = row * a.ld_scales;
    step = 4;
  }
  uint8_t* codes = a.codes + row * a.ld_codes;
  const int code_cols = (a.d + 31) / 32 * 32;
  for (int turn = 0; turn < turns; ++turn) {
    if (FMT == MX4_E8M0 || turns > 1) load(turn);
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int unit = turn * kSpan + i * TPR + t, col = unit * kCols;
      float v[kCols];
#pragma unroll
      for (int j = 0; j < kCols; ++j) v[j] = element<T>(raw[i], j);
      for (int p = 0; p < (OPERAND ? a.planes : 1); ++p) {
        if (p > 0) amax[i] = block_amax<FMT>(v);
        const bool bad = amax[i] >= kInfBits;
        float unit_step = 0.f;
        uint32_t s = 0, c[kCols / 8] = {0, 0};
        if (bad) {
          s = Mx4<FMT>::kNanScale;
        } else if (col / Mx4<FMT>::kBlock * Mx4<FMT>::kBlock < a.d) {
          s = mx4_scale<FMT>(amax[i], row_exp, &unit_step);
          mx4_codes<FMT>(v, unit_step, c);
        }
        if (col < code_cols)
          *reinterpret_cast<uint2*>(codes + (OPERAND ? p * a.plane_codes : 0) + unit * (kCols / 2)) =
              make_uint2(c[0], c[1]);
        // four scales to a word, stored by the lane that holds the first
        constexpr int kLanes = Mx4<FMT>::kBlock / kCols;
        s |= __shfl_down_sync(0xFFFFFFFFu, s, kLanes) << 8;
        s |= __shfl_down_sync(0xFFFFFFFFu, s, 2 * kLanes) << 16;
        if (lane % (4 * kLanes) == 0 && col < a.scale_cols) {
          const int w = unit / (4 * kLanes);
          *reinterpret_cast<uint32_t*>(a.scales + (OPERAND ? p * a.plane_scales : 0) + at_scale +
                                       w / words * step + w % words * 4) = s;
        }
        if (OPERAND && p + 1 < a.planes && !bad) {
#pragma unroll
          for (int h = 0; h < kCols / 8; ++h) {
            float q[8];
            e2m1x8_to_float(c[h], q);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[8 * h + j] = __fmaf_rn(-q[j], unit_step, v[8 * h + j]);  // exact
          }
        }
      }
    }
  }
}

template <class T, int FMT, int TPR, int U, bool OPERAND>
cudaError_t launch(const Mx4Quant& a, cudaStream_t st) {
  constexpr int kThreads = TPR < 128 ? 128 : TPR, kRows = kThreads / TPR;
  return launch_pdl(quant_kernel<T, FMT, TPR, U, OPERAND>,
                    dim3((unsigned)(((int64_t)a.rows + kRows - 1) / kRows)), dim3(kThreads), 0, st, a);
}
// Hidden states are few, and the product waits for them: one step a thread and as
// many threads as a row has, up to 512 (128 / 512 threads, the product and all, us: 32 x
// 12000 ids x 3840 11.3 / 10.2, 320 x 12000 x 3584 28.6 / 25.7, 1 x 2048 x 448 6.5 / 6.8).
// A table's rows are many, and a block's threads, waiting for each other's maxima, hide
// less of the memory's time than as many warps with rows of their own: a warp a row up to
// 2048 columns (32000 x 2048 bf16 28.9 us, by 128 threads 46.7), 128 threads above, with
// as many steps as hold the row in registers, up to 8192 columns (32000 x 5120 bf16
// three steps 73, four 81, 256 threads of two 101; 16000 x 4096 fp32 44.7, by a warp of eight
// steps 50.0).  32000 x 4096 bf16 take 59.5 us, 5.6 TB/s.
template <class T, int FMT>
cudaError_t launch_f(const Mx4Quant& a, bool operand, cudaStream_t st) {
  if (operand) {
    if (a.scale_cols <= 128 * kCols) return launch<T, FMT, 128, 1, true>(a, st);
    return launch<T, FMT, 512, 1, true>(a, st);
  }
  if (a.scale_cols <= 32 * 1 * kCols) return launch<T, FMT, 32, 1, false>(a, st);
  if (a.scale_cols <= 32 * 2 * kCols) return launch<T, FMT, 32, 2, false>(a, st);
  if (a.scale_cols <= 32 * 4 * kCols) return launch<T, FMT, 32, 4, false>(a, st);
  if (a.scale_cols <= 128 * 2 * kCols) return launch<T, FMT, 128, 2, false>(a, st);
  if (a.scale_cols <= 128 * 3 * kCols) return launch<T, FMT, 128, 3, false>(a, st);
  return launch<T, FMT, 128, 4, false>(a, st);
}
template <class T>
cudaError_t launch_t(const Mx4Quant& a, int fmt, bool operand, cudaStream_t st) {
  return fmt == MX4_E4M3 ? launch_f<T, MX4_E4M3>(a, operand, st)
                         : launch_f<T, MX4_E8M0>(a, operand, st);
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
