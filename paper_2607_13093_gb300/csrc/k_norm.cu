// Layer norm of rows.
//
//   mean = sum_c x / d (0 without centring)     rstd = (sum_c (x - mean)^2 / d + eps)^-1/2
//   y    = (x - mean) * rstd * w + b
//
// All of it is fp32, the result rounded once.  The variance is taken about the mean, from
// the row in registers (E[x^2] - mean^2 would lose what a large mean leaves).
//
// Bound by memory: x is read once and y written.  A row belongs to a warp (up to 1024 columns)
// or a block, whose threads hold eight columns a piece as they were read.  Of many rows a block
// is small and its threads hold several pieces, so that many rows are on their way to an SM at
// once and few threads wait for each other: 16384 x 5120 bf16 56 us (6.0 TB/s), fp32 97 us (6.9
// TB/s).  320 threads a row took 98 us, a ring of rows in shared memory that two groups of these
// took in turn 171, and pieces with the code for rows at any address beside the aligned one's 74
// (a quarter of the stalls were waits for code).  Rows at any address: 16384 x 5119 bf16 101 us.
// Of few rows a block has as many threads as there are pieces: 500 x 4096 bf16 4.0 us.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "norm.cuh"
#include "sm100_ptx.cuh"

namespace sph {
namespace {

constexpr int kMaxThreads = 512;         // of a block that holds a row
constexpr int kLongThreads = 1024;

__device__ __forceinline__ float sum_warp(float v) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
  return v;
}
// Sum over the threads of a row: a warp, or the block (`red`: a word a warp, not used again
// before the block's next barrier).
template <bool WARP>
__device__ __forceinline__ float sum_row(float v, float* red) {
  v = sum_warp(v);
  if constexpr (!WARP) {
    const int lane = threadIdx.x & 31, warps = (int)blockDim.x >> 5;
    if (lane == 0) red[threadIdx.x >> 5] = v;
    __syncthreads();
    v = sum_warp(lane < warps ? red[lane] : 0.f);
  }
  return v;
}

// ---------------------------------------------------------------------------
// forward
// ---------------------------------------------------------------------------
// The weighted columns of a piece.
template <class T, int MODE>
__device__ __forceinline__ void finish_piece(const Norm& a, int64_t row, int col, float mean,
                                             float rstd, const Eight<T, MODE>& x) {
  F2 v[4], p[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) v[k] = mul2(add2(x.two(k), f2(-mean)), f2(rstd));
  if (a.weight) {
    load_param<T, MODE>(a.weight, a.param_type, col, a.d, p);
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = mul2(v[k], p[k]);
  }
  if (a.bias) {
    load_param<T, MODE>(a.bias, a.param_type, col, a.d, p);
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = add2(v[k], p[k]);
  }
  store_row<T, MODE>(a.out, a.out_type, row * a.ld_out, col, a.d, v);
}
template <class T, int MODE>
__device__ __forceinline__ float sum_piece(const Eight<T, MODE>& x) {
  return sum_of(add2(add2(x.two(0), x.two(1)), add2(x.two(2), x.two(3))));
}
// Squares about the mean of the piece's columns before d.
template <class T, int MODE>
__device__ __forceinline__ float square_piece(const Eight<T, MODE>& x, float mean, int col, int d) {
  if (whole<MODE>(col, d)) {
    F2 q = f2(0.f);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const F2 v = add2(x.two(k), f2(-mean));
      q = fma2(v, v, q);
    }
    return sum_of(q);
  }
  float q = 0.f;
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if (col + j * kStep<MODE> < d) q = __fmaf_rn(x.get(j) - mean, x.get(j) - mean, q);
  return q;
}

// U pieces a thread.
template <class T, int U, int MODE, bool WARP>
__global__ void __launch_bounds__(WARP ? 128 : U == 1 ? 1024 : 512) norm_kernel(const Norm a) {
  __shared__ float red[2][32];
  ptx::griddep_wait();
  ptx::griddep_launch_dependents();
  const int threads = WARP ? 32 : (int)blockDim.x;
  const int t = WARP ? threadIdx.x & 31 : threadIdx.x;
  const int64_t row = WARP ? (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5) : blockIdx.x;
  if (WARP && row >= a.rows) return;
  const T* x = static_cast<const T*>(a.x) + row * a.ld_x;
  Eight<T, MODE> v[U];
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const int col = piece_col<MODE>(i, t, threads);
    if (col < a.d) v[i].load(x, col, a.d);
  }
  float mean = 0.f;
  if (a.centre) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < U; ++i)
      if (piece_col<MODE>(i, t, threads) < a.d) s += sum_piece(v[i]);
    mean = sum_row<WARP>(s, red[0]) / (float)a.d;
  }
  float q = 0.f;
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const int col = piece_col<MODE>(i, t, threads);
    if (col < a.d) q += square_piece(v[i], mean, col, a.d);
  }
  const float rstd = 1.f / sqrtf(sum_row<WARP>(q, red[1]) / (float)a.d + a.eps);
  if (t == 0) {
    if (a.mean) a.mean[row] = mean;
    if (a.rstd) a.rstd[row] = rstd;
  }
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const int col = piece_col<MODE>(i, t, threads);
    if (col < a.d) finish_piece(a, row, col, mean, rstd, v[i]);
  }
}

// Rows too long for the registers: read three times, the second and third from the L2.
template <class T>
__global__ void __launch_bounds__(kLongThreads) norm_long_kernel(const Norm a) {
  __shared__ float red[2][32];
  ptx::griddep_wait();
  ptx::griddep_launch_dependents();
  const int64_t row = blockIdx.x;
  const T* x = static_cast<const T*>(a.x) + row * a.ld_x;
  const int first = piece_col<0>(0, threadIdx.x, kLongThreads);
  Eight<T, 0> v;
  float mean = 0.f;
  if (a.centre) {
    float s = 0.f;
    for (int col = first; col < a.d; col += kLongThreads * 8) {
      v.load(x, col, a.d);
      s += sum_piece(v);
    }
    mean = sum_row<false>(s, red[0]) / (float)a.d;
  }
  float q = 0.f;
  for (int col = first; col < a.d; col += kLongThreads * 8) {
    v.load(x, col, a.d);
    q += square_piece(v, mean, col, a.d);
  }
  const float rstd = 1.f / sqrtf(sum_row<false>(q, red[1]) / (float)a.d + a.eps);
  if (threadIdx.x == 0) {
    if (a.mean) a.mean[row] = mean;
    if (a.rstd) a.rstd[row] = rstd;
  }
  for (int col = first; col < a.d; col += kLongThreads * 8) {
    v.load(x, col, a.d);
    finish_piece(a, row, col, mean, rstd, v);
  }
}

template <class T, int MODE>
cudaError_t launch_norm_v(const Norm& a, int sm_count, cudaStream_t st) {
  auto warps = [&](auto kernel) {
    return launch_pdl(kernel, dim3((unsigned)((a.rows + 3) / 4)), dim3(128), 0, st, a);
  };
  auto block = [&](auto kernel, int u) {
    const int threads = ((a.d + 8 * u - 1) / (8 * u) + 31) / 32 * 32;
    return launch_pdl(kernel, dim3((unsigned)a.rows), dim3(threads), 0, st, a);
  };
  if (a.d <= 32 * 8) return warps(norm_kernel<T, 1, MODE, true>);
  // (few rows: as many threads as a row has)
  const bool few = a.rows <= 2 * (int64_t)sm_count;
  if (!few && a.d <= 32 * 16) return warps(norm_kernel<T, 2, MODE, true>);
  if (!few && a.d <= 32 * 32) return warps(norm_kernel<T, 4, MODE, true>);
  if (few && a.d <= 1024 * 8) return block(norm_kernel<T, 1, MODE, false>, 1);
  if (a.d <= 128 * 16) return block(norm_kernel<T, 2, MODE, false>, 2);
  if (a.d <= 128 * 32) return block(norm_kernel<T, 4, MODE, false>, 4);
  // (five where a block of 128 threads or fewer then holds the row: 16384 x 4104, 4608, 5120 bf16
  // 51, 53, 56 us; eight pieces 57, 59, 63)
  if (a.d <= 128 * 40) return block(norm_kernel<T, 5, MODE, false>, 5);
  if (a.d <= kMaxThreads * 64) return block(norm_kernel<T, 8, MODE, false>, 8);
  return launch_pdl(norm_long_kernel<T>, dim3((unsigned)a.rows), dim3(kLongThreads), 0, st, a);
}
template <class T>
cudaError_t launch_norm_t(const Norm& a, int mode, int sm_count, cudaStream_t st) {
  if constexpr (sizeof(T) == 2)
    if (mode == 3) return launch_norm_v<T, 3>(a, sm_count, st);
  return mode == 2   ? launch_norm_v<T, 2>(a, sm_count, st)
         : mode == 1 ? launch_norm_v<T, 1>(a, sm_count, st)
                     : launch_norm_v<T, 0>(a, sm_count, st);
}

}  // namespace

cudaError_t launch_norm(const Norm& a, int x_type, int sm_count, cudaStream_t st) {
  const bool wide = a.d % 8 == 0 && wide_rows(a.x, a.ld_x, x_type) &&
                    wide_rows(a.out, a.ld_out, a.out_type) && wide_rows(a.weight, 0, a.param_type) &&
                    wide_rows(a.bias, 0, a.param_type);
  const bool none = !a.weight && !a.bias, same = none || a.param_type == x_type;
  const int mode = !wide                                    ? 0
                   : a.out_type != x_type                   ? 1
                   : same                                   ? 2
                   : a.param_type == TAB_FP32               ? 3
                                                            : 1;
  if (x_type == TAB_FP32) return launch_norm_t<float>(a, mode, sm_count, st);
  if (x_type == TAB_BF16) return launch_norm_t<__nv_bfloat16>(a, mode, sm_count, st);
  return launch_norm_t<__half>(a, mode, sm_count, st);
}

}  // namespace sph
