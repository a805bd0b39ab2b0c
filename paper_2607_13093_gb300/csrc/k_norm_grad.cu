// Layer norm's gradients.  With n = (x - mean) * rstd and g = dy * w,
//
//   dx = rstd * (g - sum_c g / d - n * sum_c (g * n) / d)   (centring gives the second term)
//   dw = sum_r dy * n          db = sum_r dy
//
// All of it is fp32, each result rounded once.
//
// Bound by memory: x and dy are read once and dx written.  A row belongs to a warp or a block.
// The gradients of w and b are sums over rows: each block takes rows in turn and keeps the sums
// of its columns in registers, and a second kernel adds the blocks' sums in order, so equal
// inputs give equal bits.  With the sums in registers few warps find room, so the next rows
// are on their way while one is worked on: 16-bit rows three ahead in shared memory, which each
// thread fills and reads by itself (no barrier), fp32 rows one ahead in registers (in shared
// memory 201 us, the two halves of a thread's 32 bytes being two requests of every sector).  The
// weight lies in shared memory in fp32, each thread's own columns (read and converted for each
// row 175 us, kept in registers 194).
// 32768 x 4096 bf16 143 us (5.6 TB/s), fp32 16384 x 4096 136 us (5.9 TB/s).  Rows at any address
// are read 32 columns an access, two or four bytes a lane: 32768 x 4095 bf16 282 us.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "norm.cuh"
#include "sm100_ptx.cuh"

namespace sph {
namespace {

constexpr int kMaxThreads = 512;         // of a block that holds a row
constexpr int kLongThreads = 1024;

// Two sums over the threads of a row (a warp, or a block of at most 16 warps, or 32), in one
// exchange: the half warps take one of them each.
template <bool WARP, int WARPS = 16>
__device__ __forceinline__ float2 sum_row2(float a, float b, float* red) {
  const int lane = threadIdx.x & 31;
  const bool upper = lane & 16;
  float s = (upper ? b : a) + __shfl_xor_sync(0xFFFFFFFFu, upper ? a : b, 16);
#pragma unroll
  for (int o = 8; o; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
  if constexpr (!WARP) {
    const int warps = (int)blockDim.x >> 5;
    if ((lane & 15) == 0) red[(upper ? WARPS : 0) + (threadIdx.x >> 5)] = s;
    __syncthreads();
    const float* mine = red + (upper ? WARPS : 0);
    s = (lane & 15) < warps ? mine[lane & 15] : 0.f;
    if (WARPS > 16 && (lane & 15) + 16 < warps) s += mine[(lane & 15) + 16];
#pragma unroll
    for (int o = 8; o; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
  }
  const float other = __shfl_xor_sync(0xFFFFFFFFu, s, 16);
  return upper ? make_float2(other, s) : make_float2(s, other);
}

__device__ __forceinline__ void cp_async16(uint32_t to, const void* from) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// A thread's pieces of a 16-bit row on their way through its own places in shared memory, kDepth
// rows deep, without a barrier (each thread reads what it asked for).
constexpr int kDepth = 4;
template <class T, int U>
__device__ __forceinline__ void ask_row(uint32_t at, int threads, const T* row, int t, int d) {
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const int col = piece_col<1>(i, t, threads);
    if (col >= d) break;
    cp_async16(at + (i * threads + t) * 16, row + col);
  }
}
template <class T>
__device__ __forceinline__ void take_piece(const unsigned char* at, int threads, int t, int i,
                                           Eight<T, 1>& to) {
  const uint4 v = reinterpret_cast<const uint4*>(at)[i * threads + t];
  to.w[0] = v.x; to.w[1] = v.y; to.w[2] = v.z; to.w[3] = v.w;
}

// Rows first, first + step, ... of a block (or warp), which keeps the sums of its columns
// for the weight's and the bias's gradient.
template <class TX, class TY, int U, int MODE, bool WARP, int THREADS, int BLOCKS>
__global__ void __launch_bounds__(THREADS, BLOCKS) norm_grad_kernel(const NormGrad a) {
  extern __shared__ __align__(128) unsigned char smem[];
  __shared__ float red[2][32];
  // 16-bit rows through shared memory; others a row ahead in registers
  constexpr bool RING = MODE != 0 && sizeof(TX) + sizeof(TY) == 4, AHEAD = MODE != 0 && !RING;
  // n and g of a row stay in registers over the exchange; else, where they do not fit without
  // spills, both are made twice (fp32 16384 x 4096 141 us so, 151 held)
  constexpr bool HOLD = RING;
  ptx::griddep_wait();
  ptx::griddep_launch_dependents();
  const int threads = WARP ? 32 : (int)blockDim.x;
  const int t = WARP ? threadIdx.x & 31 : threadIdx.x;
  const int owner = WARP ? (int)blockIdx.x * 4 + (threadIdx.x >> 5) : (int)blockIdx.x;
  const int owners = WARP ? a.parts * 4 : a.parts;
  const float inv_d = 1.f / (float)a.d;
  F2 sw[U][4], sb[U][4];
#pragma unroll
  for (int i = 0; i < U; ++i)
#pragma unroll
    for (int k = 0; k < 4; ++k) sw[i][k] = sb[i][k] = f2(0.f);

  // the weight in fp32, in shared memory: each thread its own columns
  float4* const w_places = reinterpret_cast<float4*>(smem) + threadIdx.x;
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const int col = piece_col<MODE>(i, t, threads);
    if (col >= a.d) break;
    F2 p[4] = {f2(1.f), f2(1.f), f2(1.f), f2(1.f)};
    if (a.weight) load_param<TX, MODE>(a.weight, a.weight_type, col, a.d, p);
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const float2 lo = both(p[2 * k]), hi = both(p[2 * k + 1]);
      w_places[(2 * i + k) * (int)blockDim.x] = make_float4(lo.x, lo.y, hi.x, hi.y);
    }
  }
  auto weight = [&](int i, F2 (&p)[4]) {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const float4 q = w_places[(2 * i + k) * (int)blockDim.x];
      p[2 * k] = f2(q.x, q.y);
      p[2 * k + 1] = f2(q.z, q.w);
    }
  };

  constexpr int kPlaces = U * 16;             // of a thread, for a row of x or dy
  unsigned char* const way = smem + U * 32 * blockDim.x +
                             (WARP ? (threadIdx.x >> 5) * kDepth * 2 * kPlaces * 32 : 0);
  auto ask = [&](int64_t row, int slot) {
    if constexpr (RING) {
      if (row < a.rows) {
        const uint32_t at = ptx::smem_u32(way) + slot * 2 * kPlaces * threads;
        ask_row<TX, U>(at, threads, static_cast<const TX*>(a.x) + row * a.ld_x, t, a.d);
        ask_row<TY, U>(at + kPlaces * threads, threads, static_cast<const TY*>(a.dy) + row * a.ld_dy, t,
                       a.d);
      }
      cp_async_commit();
    }
  };
  struct Row {
    Eight<TX, MODE> x[U];
    Eight<TY, MODE> y[U];
  };
  auto read = [&](int64_t row, Row& to) {
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int col = piece_col<MODE>(i, t, threads);
      if (col >= a.d) break;
      to.x[i].load(static_cast<const TX*>(a.x) + row * a.ld_x, col, a.d);
      to.y[i].load(static_cast<const TY*>(a.dy) + row * a.ld_dy, col, a.d);
    }
  };
  // (the row's mean and rstd come one row ahead, in registers)
  float next_mean = 0.f, next_rstd = 0.f;
  auto stats = [&](int64_t row) {
    if (row < a.rows) {
      if (a.mean) next_mean = a.mean[row];
      next_rstd = a.rstd[row];
    }
  };
  stats(owner);
  Row next;
  if constexpr (RING) {
#pragma unroll
    for (int k = 0; k < kDepth - 1; ++k) ask(owner + (int64_t)k * owners, k);
  } else if constexpr (AHEAD) {
    if (owner < a.rows) read(owner, next);
  }

  int turn = 0, slot = 0;
  for (int64_t row = owner; row < a.rows; row += owners, turn ^= 1) {
    Row now;
    const float mean = next_mean, rstd = next_rstd;
    if constexpr (RING) {
      cp_async_wait<kDepth - 2>();
      const unsigned char* at = way + slot * 2 * kPlaces * threads;
#pragma unroll
      for (int i = 0; i < U; ++i) {
        if (piece_col<MODE>(i, t, threads) >= a.d) break;
        take_piece(at, threads, t, i, now.x[i]);
        take_piece(at + kPlaces * threads, threads, t, i, now.y[i]);
      }
      ask(row + (int64_t)(kDepth - 1) * owners, slot == 0 ? kDepth - 1 : slot - 1);
      slot = slot == kDepth - 1 ? 0 : slot + 1;
    } else if constexpr (AHEAD) {
      now = next;
      if (row + owners < a.rows) read(row + owners, next);
    } else {
      read(row, now);
    }
    stats(row + owners);
    F2 n[HOLD ? U : 1][4], g[HOLD ? U : 1][4], g1 = f2(0.f), g2 = f2(0.f);
    const auto n_of = [&](int i, int k) { return mul2(add2(now.x[i].two(k), f2(-mean)), f2(rstd)); };
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int col = piece_col<MODE>(i, t, threads);
      if (col >= a.d) break;
      F2 p[4];
      weight(i, p);
      // (behind the row's end dy reads as zero, and n is -mean rstd: finite if the row's is)
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const F2 dy = now.y[i].two(k), n1 = n_of(i, k), g1k = mul2(dy, p[k]);
        sw[i][k] = fma2(dy, n1, sw[i][k]);
        sb[i][k] = add2(sb[i][k], dy);
        g1 = add2(g1, g1k);
        g2 = fma2(g1k, n1, g2);
        if constexpr (HOLD) {
          n[i][k] = n1;
          g[i][k] = g1k;
        }
      }
    }
    const float2 s = sum_row2<WARP>(sum_of(g1), sum_of(g2), red[turn]);
    const F2 k1 = f2(a.mean ? -s.x * inv_d * rstd : 0.f), k2 = f2(-s.y * inv_d * rstd);
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int col = piece_col<MODE>(i, t, threads);
      if (col >= a.d) break;
      const int at = HOLD ? i : 0;
      if constexpr (!HOLD) {
        F2 p[4];
        weight(i, p);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          n[0][k] = n_of(i, k);
          g[0][k] = mul2(now.y[i].two(k), p[k]);
        }
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) g[at][k] = fma2(n[at][k], k2, fma2(g[at][k], f2(rstd), k1));
      store_row<TX, MODE>(a.dx, a.dx_type, row * a.ld_dx, col, a.d, g[at]);
    }
  }
  if (!a.partial) return;
  if constexpr (WARP) {
    // the warps' sums of a column, added in order
    float2* const sums = reinterpret_cast<float2*>(smem);
    const int warp = threadIdx.x >> 5;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < U; ++i)
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        sums[((warp * 2) * U * 4 + i * 4 + k) * 32 + t] = both(sw[i][k]);
        sums[((warp * 2 + 1) * U * 4 + i * 4 + k) * 32 + t] = both(sb[i][k]);
      }
    __syncthreads();
    if (warp >= 2) return;
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int col = piece_col<MODE>(i, t, threads);
      if (col >= a.d) break;
      F2 v[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        v[k] = f2(0.f);
#pragma unroll
        for (int from = 0; from < 4; ++from) {
          const float2 q = sums[((from * 2 + warp) * U * 4 + i * 4 + k) * 32 + t];
          v[k] = add2(v[k], f2(q.x, q.y));
        }
      }
      store_eight<float, MODE>(a.partial, ((int64_t)blockIdx.x * 2 + warp) * a.ld_partial, col, a.d, v);
    }
  } else {
    float* pw = a.partial + (int64_t)owner * 2 * a.ld_partial;
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int col = piece_col<MODE>(i, t, threads);
      if (col >= a.d) break;
      store_eight<float, MODE>(pw, 0, col, a.d, sw[i]);
      store_eight<float, MODE>(pw, a.ld_partial, col, a.d, sb[i]);
    }
  }
}

// Rows too long for the registers: the sums of the columns first (dx may be x or dy), a
// block for 256 columns and some of the rows, then dx, each row read twice.  Three readings where
// one is needed, 32 columns an access wherever rows start: 4096 x 16384 bf16 286 us (59 for what
// has to move), 8000 x 12288 465 (87).
template <class TX, class TY>
__global__ void __launch_bounds__(256) norm_columns_kernel(const NormGrad a) {
  __shared__ float part[8][32][17];
  ptx::griddep_wait();
  ptx::griddep_launch_dependents();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int col = (int)blockIdx.x * 256 + lane;
  F2 sw[4], sb[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) sw[k] = sb[k] = f2(0.f);
  for (int64_t row = (int64_t)blockIdx.y * 8 + warp; row < a.rows; row += (int64_t)a.parts * 8) {
    F2 n[4], g[4];
    load_eight<TX, 0>(static_cast<const TX*>(a.x) + row * a.ld_x, col, a.d, n);
    load_eight<TY, 0>(static_cast<const TY*>(a.dy) + row * a.ld_dy, col, a.d, g);
    const float mean = a.mean ? a.mean[row] : 0.f, rstd = a.rstd[row];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      sw[k] = fma2(g[k], mul2(add2(n[k], f2(-mean)), f2(rstd)), sw[k]);
      sb[k] = add2(sb[k], g[k]);
    }
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const float2 w = both(sw[k]), b = both(sb[k]);
    part[warp][lane][2 * k] = w.x; part[warp][lane][2 * k + 1] = w.y;
    part[warp][lane][8 + 2 * k] = b.x; part[warp][lane][8 + 2 * k + 1] = b.y;
  }
  __syncthreads();
  const int c = (int)blockIdx.x * 256 + (int)threadIdx.x;
  if (c >= a.d) return;
  float w = 0.f, b = 0.f;
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    w += part[k][threadIdx.x % 32][threadIdx.x / 32];
    b += part[k][threadIdx.x % 32][8 + threadIdx.x / 32];
  }
  float* p = a.partial + (int64_t)blockIdx.y * 2 * a.ld_partial;
  p[c] = w;
  p[a.ld_partial + c] = b;
}
template <class TX, class TY>
__global__ void __launch_bounds__(kLongThreads) norm_grad_long_kernel(const NormGrad a) {
  __shared__ float red[64];
  ptx::griddep_wait();
  ptx::griddep_launch_dependents();
  const int64_t row = blockIdx.x;
  const TX* x = static_cast<const TX*>(a.x) + row * a.ld_x;
  const TY* y = static_cast<const TY*>(a.dy) + row * a.ld_dy;
  const float mean = a.mean ? a.mean[row] : 0.f, rstd = a.rstd[row], inv_d = 1.f / (float)a.d;
  const int first = piece_col<0>(0, threadIdx.x, kLongThreads);
  F2 n[4], g[4], p[4];
  auto load = [&](int col) {
    load_eight<TX, 0>(x, col, a.d, n);
    load_eight<TY, 0>(y, col, a.d, g);
    if (a.weight) load_param<TX, 0>(a.weight, a.weight_type, col, a.d, p);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      n[k] = mul2(add2(n[k], f2(-mean)), f2(rstd));
      if (a.weight) g[k] = mul2(g[k], p[k]);
    }
  };
  float s1 = 0.f, s2 = 0.f;
  for (int col = first; col < a.d; col += kLongThreads * 8) {
    load(col);
    F2 t1 = f2(0.f), t2 = f2(0.f);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      t1 = add2(t1, g[k]);
      t2 = fma2(g[k], n[k], t2);
    }
    s1 += sum_of(t1);
    s2 += sum_of(t2);
  }
  const float2 s = sum_row2<false, 32>(s1, s2, red);
  const float c1 = a.mean ? s.x * inv_d : 0.f, c2 = s.y * inv_d;
  for (int col = first; col < a.d; col += kLongThreads * 8) {
    load(col);
#pragma unroll
    for (int k = 0; k < 4; ++k) g[k] = mul2(f2(rstd), fma2(n[k], f2(-c2), add2(g[k], f2(-c1))));
    store_row<TX, 0>(a.dx, a.dx_type, row * a.ld_dx, col, a.d, g);
  }
}

// The parts' sums of 32 columns of the weight's or the bias's gradient, added in order: a warp
// adds every 16th part.
constexpr int kJoinWarps = 16;
template <class T>
__global__ void __launch_bounds__(kJoinWarps * 32) norm_join_kernel(const NormGrad a) {
  __shared__ float part[kJoinWarps][32];
  ptx::griddep_wait();
  ptx::griddep_launch_dependents();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int col = (int)blockIdx.x * 32 + lane;
  void* const to = blockIdx.y ? a.db : a.dw;
  if (!to) return;
  float s = 0.f;
  if (col < a.d) {
    const float* q = a.partial + blockIdx.y * a.ld_partial + col;
#pragma unroll 8
    for (int p = warp; p < a.parts; p += kJoinWarps) s += q[(int64_t)p * 2 * a.ld_partial];
  }
  part[warp][lane] = s;
  __syncthreads();
  if (warp || col >= a.d) return;
  float v = 0.f;
#pragma unroll
  for (int k = 0; k < kJoinWarps; ++k) v += part[k][lane];
  T* out = static_cast<T*>(to) + col;
  *out = from_f32<T>(a.accumulate ? to_f32(*out) + v : v);
}

// How a call's rows are divided.  packed: x and dy have 16 bits; ring: they come through shared
// memory.  Blocks of 256 threads: two an SM, whose threads hold n and g (of the form that read the
// weight for each row, three that make both twice took 196 us where two took 174, threads of four
// pieces 220); rows at any address three (32768 x 4095 bf16 284 us, two 371).  Rows of 512 to 1024
// columns by blocks too (60000 x 1000 75 us, by warps of four pieces 92).
struct GradPlan {
  bool warps, is_long;
  int u, threads, parts;
};
GradPlan grad_plan(int64_t rows, int d, bool packed, bool ring, int sm_count) {
  GradPlan p{};
  const int64_t sms = sm_count;
  int64_t most;
  if (d <= 32 * 16) {
    p.warps = true;
    p.u = d <= 32 * 8 ? 1 : 2;
    p.threads = 128;
    most = sms * (packed && p.u == 1 ? 6 : 4);
    rows = (rows + 3) / 4;
  } else if (d <= kMaxThreads * 16) {
    // (few rows: as many threads as a row has)
    p.u = rows <= 2 * sms && d <= kMaxThreads * 8 ? 1 : 2;
    p.threads = ((d + 8 * p.u - 1) / (8 * p.u) + 31) / 32 * 32;
    const int per_sm = (packed && !ring && p.u == 2 && p.threads <= 256 ? 768 : 512) / p.threads;
    most = sms * (per_sm < 1 ? 1 : per_sm);
  } else {
    p.is_long = true;
    const int64_t cols = (d + 255) / 256;
    most = (sms * 4 + cols - 1) / cols;
    rows = (rows + 7) / 8;
  }
  p.parts = (int)(rows < most ? (rows > 0 ? rows : 1) : most);
  return p;
}

template <class TX, class TY, int MODE>
cudaError_t launch_grad_v(const NormGrad& a, const GradPlan& p, cudaStream_t st) {
  constexpr bool packed = sizeof(TX) + sizeof(TY) == 4;
  auto go = [&](auto kernel) {
    const int on_way = MODE && packed ? kDepth * p.u * 32 * p.threads : 0;
    const int sums = p.warps ? p.u * 64 * 128 : 0;
    const int weights = p.u * 32 * p.threads;
    const int smem = weights + on_way > sums ? weights + on_way : sums;
    if (smem > 40 * 1024) {         // (48 KB hold the static part too)
      const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
      if (e != cudaSuccess) return e;
    }
    return launch_pdl(kernel, dim3((unsigned)p.parts), dim3((unsigned)p.threads), smem, st, a);
  };
  if constexpr (packed) {
    if (p.u == 2 && !p.warps && p.threads <= 256)
      return go(norm_grad_kernel<TX, TY, 2, MODE, false, 256, MODE ? 2 : 3>);
  }
  if (p.warps)
    return p.u == 1 ? go(norm_grad_kernel<TX, TY, 1, MODE, true, 128, packed ? 6 : 4>)
                    : go(norm_grad_kernel<TX, TY, 2, MODE, true, 128, 4>);
  return p.u == 1 ? go(norm_grad_kernel<TX, TY, 1, MODE, false, kMaxThreads, 1>)
                  : go(norm_grad_kernel<TX, TY, 2, MODE, false, kMaxThreads, 1>);
}
template <class TX, class TY>
cudaError_t launch_grad_y(const NormGrad& a, const GradPlan& p, int mode, cudaStream_t st) {
  if (!p.is_long) {
    return mode ? launch_grad_v<TX, TY, 1>(a, p, st) : launch_grad_v<TX, TY, 0>(a, p, st);
  }
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
cudaError_t launch_grad_x(const NormGrad& a, int dy_type, const GradPlan& p, int mode, cudaStream_t st) {
  if (dy_type == TAB_FP32) return launch_grad_y<TX, float>(a, p, mode, st);
  if (dy_type == TAB_BF16) return launch_grad_y<TX, __nv_bfloat16>(a, p, mode, st);
  return launch_grad_y<TX, __half>(a, p, mode, st);
}

int64_t partial_ld(int d) { return (d + 31) / 32 * 32; }

}  // namespace

size_t norm_grad_scratch_bytes(int64_t rows, int d, int x_type, int dy_type, int sm_count) {
  const bool packed = x_type != TAB_FP32 && dy_type != TAB_FP32;
  return (size_t)grad_plan(rows, d, packed, false, sm_count).parts   // (a ring's are fewer)
         * 2 * (size_t)partial_ld(d) * 4;
}
// At least what any call of up to `rows` rows and d columns takes: two rows of sums a part, at
// most one part a row and twelve an SM (768 / 64 threads).
size_t norm_grad_reserve_bytes(int64_t rows, int64_t d, int sm_count) {
  const int64_t most = (int64_t)sm_count * 12, parts = rows < 1 ? 1 : rows < most ? rows : most;
  return (size_t)parts * 2 * (size_t)partial_ld((int)d) * 4;
}

cudaError_t launch_norm_grad(NormGrad a, int x_type, int dy_type, int grad_type, void* scratch,
                             int sm_count, cudaStream_t st) {
  const bool wide = a.d % 8 == 0 && wide_rows(a.x, a.ld_x, x_type) &&
                    wide_rows(a.dy, a.ld_dy, dy_type) && wide_rows(a.dx, a.ld_dx, a.dx_type) &&
                    wide_rows(a.weight, 0, a.weight_type);
  const int mode = wide ? 1 : 0;
  const bool packed = x_type != TAB_FP32 && dy_type != TAB_FP32;
  const GradPlan p = grad_plan(a.rows, a.d, packed, packed && mode, sm_count);
  a.parts = p.parts;
  a.ld_partial = partial_ld(a.d);
  a.partial = a.dw || a.db ? static_cast<float*>(scratch) : nullptr;
  const cudaError_t e = x_type == TAB_FP32   ? launch_grad_x<float>(a, dy_type, p, mode, st)
                        : x_type == TAB_BF16 ? launch_grad_x<__nv_bfloat16>(a, dy_type, p, mode, st)
                                             : launch_grad_x<__half>(a, dy_type, p, mode, st);
  if (e != cudaSuccess || !a.partial) return e;
  const dim3 grid((unsigned)((a.d + 31) / 32), 2), block(kJoinWarps * 32);
  if (grad_type == TAB_FP32) return launch_pdl(norm_join_kernel<float>, grid, block, 0, st, a);
  if (grad_type == TAB_BF16) return launch_pdl(norm_join_kernel<__nv_bfloat16>, grid, block, 0, st, a);
  return launch_pdl(norm_join_kernel<__half>, grid, block, 0, st, a);
}

}  // namespace sph
