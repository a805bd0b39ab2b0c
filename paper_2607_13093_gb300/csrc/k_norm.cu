// Layer norm of rows.
//
//   mean = sum_c x / d (0 without centring)     rstd = (sum_c (x - mean)^2 / d + eps)^-1/2
//   y    = (x - mean) * rstd * w + b
//
// All of it is fp32, the result rounded once.  The variance is taken about the mean, from
// the row in registers (E[x^2] - mean^2 would lose what a large mean leaves).
//
// Bound by memory: x is read once and y written.  A row belongs to a warp (up to 1024
// columns) or a block, whose threads hold eight columns a piece.
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
// The weighted columns of a piece.  (A row's first piece may start before it, see below.)
template <bool VEC>
__device__ __forceinline__ void finish_piece(const Norm& a, int64_t row, int col, float mean,
                                             float rstd, float (&v)[8]) {
  float p[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = (v[j] - mean) * rstd;
  if (a.weight) {
    load_param<VEC>(a.weight, a.param_type, a.param16 != 0, col, a.d, p);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] *= p[j];
  }
  if (a.bias) {
    load_param<VEC>(a.bias, a.param_type, a.param16 != 0, col, a.d, p);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] += p[j];
  }
  store_row<true>(a.out, a.out_type, row * a.ld_out, col, a.d, v);
}

// U pieces a thread.  VEC: rows of x and out are on 16 bytes.  Other rows: the first piece
// ends at the output row's first 16-byte boundary, so that the others are stored in 16-byte
// words.
template <class T, int U, bool VEC, bool WARP>
__global__ void __launch_bounds__(WARP ? 128 : U == 1 ? 1024 : kMaxThreads) norm_kernel(const Norm a) {
  __shared__ float red[2][32];
  ptx::griddep_wait();
  ptx::griddep_launch_dependents();
  const int threads = WARP ? 32 : (int)blockDim.x;
  const int t = WARP ? threadIdx.x & 31 : threadIdx.x;
  const int64_t row = WARP ? (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5) : blockIdx.x;
  if (WARP && row >= a.rows) return;
  const T* x = static_cast<const T*>(a.x) + row * a.ld_x;
  int first = t * 8;
  if constexpr (!VEC) {
    const int size = a.out_type == TAB_FP32 ? 4 : 2;
    const int head = (int)(-(intptr_t)((uintptr_t)a.out + row * a.ld_out * size) & 15) / size;
    first += head ? head - 8 : 0;
  }
  float v[U][8];
#pragma unroll
  for (int i = 0; i < U; ++i) load_cols<T, VEC>(x, first + i * threads * 8, a.d, v[i]);
  float mean = 0.f;
  if (a.centre) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < U; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) s += v[i][j];
    mean = sum_row<WARP>(s, red[0]) / (float)a.d;
  }
  float q = 0.f;
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const int col = first + i * threads * 8;
    if (col >= 0 && col + 8 <= a.d) {
#pragma unroll
      for (int j = 0; j < 8; ++j) q = __fmaf_rn(v[i][j] - mean, v[i][j] - mean, q);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (col + j >= 0 && col + j < a.d) q = __fmaf_rn(v[i][j] - mean, v[i][j] - mean, q);
    }
  }
  const float rstd = 1.f / sqrtf(sum_row<WARP>(q, red[1]) / (float)a.d + a.eps);
  if (t == 0) {
    if (a.mean) a.mean[row] = mean;
    if (a.rstd) a.rstd[row] = rstd;
  }
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const int col = first + i * threads * 8;
    if (col < a.d) finish_piece<VEC>(a, row, col, mean, rstd, v[i]);
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
  const int size = a.out_type == TAB_FP32 ? 4 : 2;
  const int head = (int)(-(intptr_t)((uintptr_t)a.out + row * a.ld_out * size) & 15) / size;
  const int first = (int)threadIdx.x * 8 + (head ? head - 8 : 0);
  float mean = 0.f, v[8];
  if (a.centre) {
    float s = 0.f;
    for (int col = first; col < a.d; col += kLongThreads * 8) {
      load_cols<T, false>(x, col, a.d, v);
      float part = 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) part += v[j];
      s += part;
    }
    mean = sum_row<false>(s, red[0]) / (float)a.d;
  }
  float q = 0.f;
  for (int col = first; col < a.d; col += kLongThreads * 8) {
    load_cols<T, false>(x, col, a.d, v);
    float part = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (col + j >= 0 && col + j < a.d) part = __fmaf_rn(v[j] - mean, v[j] - mean, part);
    q += part;
  }
  const float rstd = 1.f / sqrtf(sum_row<false>(q, red[1]) / (float)a.d + a.eps);
  if (threadIdx.x == 0) {
    if (a.mean) a.mean[row] = mean;
    if (a.rstd) a.rstd[row] = rstd;
  }
  for (int col = first; col < a.d; col += kLongThreads * 8) {
    load_cols<T, false>(x, col, a.d, v);
    finish_piece<false>(a, row, col, mean, rstd, v);
  }
}

template <class T, bool VEC>
cudaError_t launch_norm_v(const Norm& a, int sm_count, cudaStream_t st) {
  // columns that the pieces of a row have to cover
  const int cover = a.d + (VEC ? 0 : 7);
  auto warps = [&](auto kernel) {
    return launch_pdl(kernel, dim3((unsigned)((a.rows + 3) / 4)), dim3(128), 0, st, a);
  };
  auto block = [&](auto kernel, int u) {
    const int threads = ((cover + 8 * u - 1) / (8 * u) + 31) / 32 * 32;
    return launch_pdl(kernel, dim3((unsigned)a.rows), dim3(threads), 0, st, a);
  };
  if (cover <= 32 * 8) return warps(norm_kernel<T, 1, VEC, true>);
  const bool few = a.rows <= 2 * (int64_t)sm_count;
  if (!few && cover <= 32 * 16) return warps(norm_kernel<T, 2, VEC, true>);
  if (!few && cover <= 32 * 32) return warps(norm_kernel<T, 4, VEC, true>);
  if (few && cover <= 1024 * 8) return block(norm_kernel<T, 1, VEC, false>, 1);
  if (cover <= kMaxThreads * 16) return block(norm_kernel<T, 2, VEC, false>, 2);
  if (cover <= kMaxThreads * 32) return block(norm_kernel<T, 4, VEC, false>, 4);
  return launch_pdl(norm_long_kernel<T>, dim3((unsigned)a.rows), dim3(kLongThreads), 0, st, a);
}
template <class T>
cudaError_t launch_norm_t(const Norm& a, bool vec, int sm_count, cudaStream_t st) {
  return vec ? launch_norm_v<T, true>(a, sm_count, st) : launch_norm_v<T, false>(a, sm_count, st);
}

}  // namespace

cudaError_t launch_norm(Norm a, int x_type, int sm_count, cudaStream_t st) {
  const bool vec = on16(a.x, a.ld_x, type_size(x_type)) && on16(a.out, a.ld_out, type_size(a.out_type));
  a.param16 = (((uintptr_t)a.weight | (uintptr_t)a.bias) & 15) == 0;
  if (x_type == TAB_FP32) return launch_norm_t<float>(a, vec, sm_count, st);
  if (x_type == TAB_BF16) return launch_norm_t<__nv_bfloat16>(a, vec, sm_count, st);
  return launch_norm_t<__half>(a, vec, sm_count, st);
}

}  // namespace sph
