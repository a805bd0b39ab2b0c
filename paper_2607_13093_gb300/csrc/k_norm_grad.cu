// Layer norm's gradients.  With n = (x - mean) * rstd and g = dy * w,
//
//   dx = rstd * (g - sum_c g / d - n * sum_c (g * n) / d)   (centring gives the second term)
//   dw = sum_r dy * n          db = sum_r dy
//
// All of it is fp32, each result rounded once.
//
// Bound by memory: x and dy are read once and dx written.  A row belongs to a warp (up to
// 512 columns) or a block.  The gradients of w and b are sums over rows: each block takes
// rows in turn and keeps the sums of its columns in registers; a second kernel adds the
// blocks' sums in order, so equal inputs give equal bits.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "norm.cuh"
#include "sm100_ptx.cuh"

namespace sph {
namespace {

constexpr int kMaxThreads = 512;         // of a block that holds a row
constexpr int kLongThreads = 1024;

// Sums of a row's g and g n over its threads, in one exchange.
template <bool WARP>
__device__ __forceinline__ float2 sum_row2(float a, float b, float2* red) {
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    a += __shfl_xor_sync(0xFFFFFFFFu, a, o);
    b += __shfl_xor_sync(0xFFFFFFFFu, b, o);
  }
  if constexpr (!WARP) {
    const int lane = threadIdx.x & 31, warps = (int)blockDim.x >> 5;
    if (lane == 0) red[threadIdx.x >> 5] = make_float2(a, b);
    __syncthreads();
    const float2 r = lane < warps ? red[lane] : make_float2(0.f, 0.f);
    a = r.x;
    b = r.y;
#pragma unroll
    for (int o = 16; o; o >>= 1) {
      a += __shfl_xor_sync(0xFFFFFFFFu, a, o);
      b += __shfl_xor_sync(0xFFFFFFFFu, b, o);
    }
  }
  return make_float2(a, b);
}

// Rows first, first + step, ... of a block (or warp), which keeps the sums of its columns
// for the weight's and the bias's gradient.  VEC: rows of x, dy and dx are on 16 bytes.
template <class TX, class TY, int U, bool VEC, bool WARP>
__global__ void __launch_bounds__(WARP ? 128 : kMaxThreads) norm_grad_kernel(const NormGrad a) {
  __shared__ float2 red[2][32];
  ptx::griddep_wait();
  ptx::griddep_launch_dependents();
  const int threads = WARP ? 32 : (int)blockDim.x;
  const int t = WARP ? threadIdx.x & 31 : threadIdx.x;
  const int owner = WARP ? (int)blockIdx.x * 4 + (threadIdx.x >> 5) : (int)blockIdx.x;
  const float inv_d = 1.f / (float)a.d;
  float sw[U][8], sb[U][8];
#pragma unroll
  for (int i = 0; i < U; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) sw[i][j] = sb[i][j] = 0.f;
  int turn = 0;
  for (int64_t row = owner; row < a.rows; row += a.parts, turn ^= 1) {
    const TX* x = static_cast<const TX*>(a.x) + row * a.ld_x;
    const TY* y = static_cast<const TY*>(a.dy) + row * a.ld_dy;
    float n[U][8], g[U][8];
#pragma unroll
    for (int i = 0; i < U; ++i) {
      load_cols<TX, VEC>(x, (i * threads + t) * 8, a.d, n[i]);
      load_cols<TY, VEC>(y, (i * threads + t) * 8, a.d, g[i]);
    }
    const float mean = a.mean ? a.mean[row] : 0.f, rstd = a.rstd[row];
    float s1 = 0.f, s2 = 0.f;
#pragma unroll
    for (int i = 0; i < U; ++i) {
      float p[8];
      const int col = (i * threads + t) * 8;
      if (a.weight && col < a.d) load_param<VEC>(a.weight, a.weight_type, a.param16 != 0, col, a.d, p);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        n[i][j] = (n[i][j] - mean) * rstd;
        sw[i][j] = __fmaf_rn(g[i][j], n[i][j], sw[i][j]);
        sb[i][j] += g[i][j];
        if (a.weight) g[i][j] *= p[j];
        if (col + j >= a.d) g[i][j] = 0.f;      // (there p and n are not the row's)
        s1 += g[i][j];
        s2 = __fmaf_rn(g[i][j], n[i][j], s2);
      }
    }
    const float2 s = sum_row2<WARP>(s1, s2, red[turn]);
    const float c1 = a.mean ? s.x * inv_d : 0.f, c2 = s.y * inv_d;
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int col = (i * threads + t) * 8;
      if (col >= a.d) break;
#pragma unroll
      for (int j = 0; j < 8; ++j) g[i][j] = rstd * (g[i][j] - c1 - n[i][j] * c2);
      store_row<VEC>(a.dx, a.dx_type, row * a.ld_dx, col, a.d, g[i]);
    }
  }
  if (a.partial) {
    float* pw = a.partial + (int64_t)owner * 2 * a.ld_partial;
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int col = (i * threads + t) * 8;
      if (col >= a.d) break;
      store_cols<float, true>(pw, col, (int)a.ld_partial, sw[i]);
      store_cols<float, true>(pw + a.ld_partial, col, (int)a.ld_partial, sb[i]);
    }
  }
}

// Rows too long for the registers: the sums of the columns first (dx may be x or dy), a
// block for 256 columns and some of the rows, then dx, each row read twice.
template <class TX, class TY>
__global__ void __launch_bounds__(256) norm_columns_kernel(const NormGrad a) {
  __shared__ float part[8][32][17];
  ptx::griddep_wait();
  ptx::griddep_launch_dependents();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int col = (int)blockIdx.x * 256 + lane * 8;
  float sw[8], sb[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) sw[j] = sb[j] = 0.f;
  for (int64_t row = (int64_t)blockIdx.y * 8 + warp; row < a.rows; row += (int64_t)a.parts * 8) {
    float n[8], g[8];
    load_cols<TX, false>(static_cast<const TX*>(a.x) + row * a.ld_x, col, a.d, n);
    load_cols<TY, false>(static_cast<const TY*>(a.dy) + row * a.ld_dy, col, a.d, g);
    const float mean = a.mean ? a.mean[row] : 0.f, rstd = a.rstd[row];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      sw[j] = __fmaf_rn(g[j], (n[j] - mean) * rstd, sw[j]);
      sb[j] += g[j];
    }
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    part[warp][lane][j] = sw[j];
    part[warp][lane][8 + j] = sb[j];
  }
  __syncthreads();
  const int c = (int)blockIdx.x * 256 + (int)threadIdx.x;
  if (c >= a.d) return;
  float w = 0.f, b = 0.f;
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    w += part[k][threadIdx.x / 8][threadIdx.x % 8];
    b += part[k][threadIdx.x / 8][8 + threadIdx.x % 8];
  }
  float* p = a.partial + (int64_t)blockIdx.y * 2 * a.ld_partial;
  p[c] = w;
  p[a.ld_partial + c] = b;
}
template <class TX, class TY>
__global__ void __launch_bounds__(kLongThreads) norm_grad_long_kernel(const NormGrad a) {
  __shared__ float2 red[32];
  ptx::griddep_wait();
  ptx::griddep_launch_dependents();
  const int64_t row = blockIdx.x;
  const TX* x = static_cast<const TX*>(a.x) + row * a.ld_x;
  const TY* y = static_cast<const TY*>(a.dy) + row * a.ld_dy;
  const float mean = a.mean ? a.mean[row] : 0.f, rstd = a.rstd[row], inv_d = 1.f / (float)a.d;
  float n[8], g[8], p[8], s1 = 0.f, s2 = 0.f;
  auto load = [&](int col) {
    load_cols<TX, false>(x, col, a.d, n);
    load_cols<TY, false>(y, col, a.d, g);
    if (a.weight) load_param<false>(a.weight, a.weight_type, false, col, a.d, p);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      n[j] = (n[j] - mean) * rstd;
      if (a.weight) g[j] *= p[j];
      if (col + j >= a.d) g[j] = 0.f;
    }
  };
  for (int col = (int)threadIdx.x * 8; col < a.d; col += kLongThreads * 8) {
    load(col);
    float t1 = 0.f, t2 = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      t1 += g[j];
      t2 = __fmaf_rn(g[j], n[j], t2);
    }
    s1 += t1;
    s2 += t2;
  }
  const float2 s = sum_row2<false>(s1, s2, red);
  const float c1 = a.mean ? s.x * inv_d : 0.f, c2 = s.y * inv_d;
  for (int col = (int)threadIdx.x * 8; col < a.d; col += kLongThreads * 8) {
    load(col);
#pragma unroll
    for (int j = 0; j < 8; ++j) g[j] = rstd * (g[j] - c1 - n[j] * c2);
    store_row<false>(a.dx, a.dx_type, row * a.ld_dx, col, a.d, g);
  }
}

// The parts' sums of 32 columns, added in order, to the weight's and the bias's gradient.
// A warp adds every eighth part.
constexpr int kJoinWarps = 16;
template <class T>
__global__ void __launch_bounds__(kJoinWarps * 32) norm_join_kernel(const NormGrad a) {
  __shared__ float part[2][kJoinWarps][32];
  ptx::griddep_wait();
  ptx::griddep_launch_dependents();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int col = (int)blockIdx.x * 32 + lane;
  float s[2] = {0.f, 0.f};
  if (col < a.d) {
    for (int p = warp; p < a.parts; p += kJoinWarps) {
      const float* q = a.partial + (int64_t)p * 2 * a.ld_partial + col;
      s[0] += q[0];
      s[1] += q[a.ld_partial];
    }
  }
  part[0][warp][lane] = s[0];
  part[1][warp][lane] = s[1];
  __syncthreads();
  void* const to = warp == 0 ? a.dw : warp == 1 ? a.db : nullptr;
  if (!to || col >= a.d) return;
  float v = 0.f;
#pragma unroll
  for (int k = 0; k < kJoinWarps; ++k) v += part[warp][k][lane];
  T* out = static_cast<T*>(to) + col;
  *out = from_f32<T>(a.accumulate ? to_f32(*out) + v : v);
}

// How a call's rows are divided.
struct GradPlan {
  bool warps, is_long;
  int u, threads, parts, blocks;
};
GradPlan grad_plan(int64_t rows, int d, int sm_count) {
  GradPlan p{};
  const int64_t most = (int64_t)sm_count * 4;
  if (d <= 32 * 16) {
    p.warps = true;
    p.u = d <= 32 * 8 ? 1 : 2;
    p.threads = 128;
    const int64_t blocks = (rows + 3) / 4 < 2 * most ? (rows + 3) / 4 : 2 * most;
    p.blocks = (int)(blocks > 0 ? blocks : 1);
    p.parts = p.blocks * 4;
  } else if (d <= kMaxThreads * 16) {
    p.u = d <= kMaxThreads * 8 ? 1 : 2;
    p.threads = ((d + 8 * p.u - 1) / (8 * p.u) + 31) / 32 * 32;
    const int per_sm = 1024 / p.threads;
    const int64_t units = (int64_t)sm_count * (per_sm < 1 ? 1 : per_sm > 4 ? 4 : per_sm);
    p.blocks = p.parts = (int)(rows < units ? (rows > 0 ? rows : 1) : units);
  } else {
    p.is_long = true;
    const int64_t cols = (d + 255) / 256, want = (most + cols - 1) / cols;
    const int64_t by_rows = (rows + 7) / 8;
    p.parts = (int)(by_rows < want ? (by_rows > 0 ? by_rows : 1) : want);
  }
  return p;
}

template <class TX, class TY, bool VEC>
cudaError_t launch_grad_v(const NormGrad& a, const GradPlan& p, cudaStream_t st) {
  const dim3 grid((unsigned)p.blocks), block((unsigned)p.threads);
  if (p.warps)
    return p.u == 1 ? launch_pdl(norm_grad_kernel<TX, TY, 1, VEC, true>, grid, block, 0, st, a)
                    : launch_pdl(norm_grad_kernel<TX, TY, 2, VEC, true>, grid, block, 0, st, a);
  return p.u == 1 ? launch_pdl(norm_grad_kernel<TX, TY, 1, VEC, false>, grid, block, 0, st, a)
                  : launch_pdl(norm_grad_kernel<TX, TY, 2, VEC, false>, grid, block, 0, st, a);
}
template <class TX, class TY>
cudaError_t launch_grad_y(const NormGrad& a, const GradPlan& p, bool vec, cudaStream_t st) {
  if (!p.is_long)
    return vec ? launch_grad_v<TX, TY, true>(a, p, st) : launch_grad_v<TX, TY, false>(a, p, st);
  if (a.partial) {
    const cudaError_t e =
        launch_pdl(norm_columns_kernel<TX, TY>, dim3((unsigned)((a.d + 255) / 256), (unsigned)p.parts),
                   dim3(256), 0, st, a);
    if (e != cudaSuccess) return e;
  }
  if (a.rows == 0) return cudaSuccess;
  return launch_pdl(norm_grad_long_kernel<TX, TY>, dim3((unsigned)a.rows), dim3(kLongThreads), 0, st, a);
}
template <class TX>
cudaError_t launch_grad_x(const NormGrad& a, int dy_type, const GradPlan& p, bool vec, cudaStream_t st) {
  if (dy_type == TAB_FP32) return launch_grad_y<TX, float>(a, p, vec, st);
  if (dy_type == TAB_BF16) return launch_grad_y<TX, __nv_bfloat16>(a, p, vec, st);
  return launch_grad_y<TX, __half>(a, p, vec, st);
}

int64_t partial_ld(int d) { return (d + 31) / 32 * 32; }

}  // namespace

size_t norm_grad_scratch_bytes(int64_t rows, int d, int sm_count) {
  return (size_t)grad_plan(rows, d, sm_count).parts * 2 * (size_t)partial_ld(d) * 4;
}
// At least what any call of up to `rows` rows and d columns takes: a part holds two rows of
// sums, and there are at most 32 parts an SM of rows of 512 columns, four of longer ones.
size_t norm_grad_reserve_bytes(int64_t rows, int64_t d, int sm_count) {
  const int64_t narrow = d < 512 ? d : 512, up = (rows + 3) / 4 * 4;
  const size_t short_parts = (size_t)(up < (int64_t)sm_count * 32 ? up : (int64_t)sm_count * 32);
  const size_t parts = (size_t)(rows < (int64_t)sm_count * 4 ? rows : (int64_t)sm_count * 4);
  const size_t a = short_parts * 2 * (size_t)partial_ld((int)narrow) * 4;
  const size_t b = (parts < 1 ? 1 : parts) * 2 * (size_t)partial_ld((int)d) * 4;
  return a > b ? a : b;
}

cudaError_t launch_norm_grad(NormGrad a, int x_type, int dy_type, int grad_type, void* scratch,
                             int sm_count, cudaStream_t st) {
  const GradPlan p = grad_plan(a.rows, a.d, sm_count);
  const bool vec = on16(a.x, a.ld_x, type_size(x_type)) && on16(a.dy, a.ld_dy, type_size(dy_type)) &&
                   on16(a.dx, a.ld_dx, type_size(a.dx_type));
  a.param16 = ((uintptr_t)a.weight & 15) == 0;
  a.parts = p.parts;
  a.ld_partial = partial_ld(a.d);
  a.partial = a.dw || a.db ? static_cast<float*>(scratch) : nullptr;
  const cudaError_t e = x_type == TAB_FP32   ? launch_grad_x<float>(a, dy_type, p, vec, st)
                        : x_type == TAB_BF16 ? launch_grad_x<__nv_bfloat16>(a, dy_type, p, vec, st)
                                             : launch_grad_x<__half>(a, dy_type, p, vec, st);
  if (e != cudaSuccess || !a.partial) return e;
  const dim3 grid((unsigned)((a.d + 31) / 32)), block(kJoinWarps * 32);
  if (grad_type == TAB_FP32) return launch_pdl(norm_join_kernel<float>, grid, block, 0, st, a);
  if (grad_type == TAB_BF16) return launch_pdl(norm_join_kernel<__nv_bfloat16>, grid, block, 0, st, a);
  return launch_pdl(norm_join_kernel<__half>, grid, block, 0, st, a);
}

}  // namespace sph
