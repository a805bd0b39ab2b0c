// Logits with penalties for repeated tokens, biases and masks, and a token from them.
//
//   z -> z / rep (z > 0) or z * rep        for ids among the row's tokens so far
//     -> z - freq * count, then z - pres   for ids among those of its output
//     -> z + the sum of the row's biases for the id
//     -> -inf                              where the row's mask has the id's bit clear
//
// each step rounded to fp32 (no fused multiply-add), the result to the output's type.
//
// Bound by memory: logits are read once and written once, with a bit of mask each.  A block
// takes a run of a row's columns.  What is sparse comes first: it counts the row's tokens
// that fall into its columns in shared memory (integer atomics: no order to depend on), and
// adds the biases that do, in the list's order.  Then its threads take eight columns a piece.
// With a draw the block leaves its largest value, its sum of exp((z - largest) / tau) and the
// first place of the largest; a second kernel, a block a row, joins these and finds the token.
#include <cuda_bf16.h>

#include "rows.cuh"
#include "sm100_ptx.cuh"
#include "sph_common.cuh"
#include "sph_internal.h"

namespace sph {
namespace {

constexpr int kThreads = 256;
constexpr float kLog2e = 1.4426950408889634f;

// exp((z - M) / tau) with M >= z: 1 at M itself (an infinite one too), 0 at -inf, NaN for a NaN.
__device__ __forceinline__ float weight(float z, float M, float l2t) {
  return z == -INFINITY ? 0.f : z == M ? 1.f : ex2_approx((z - M) * l2t);
}

// The column in [lo, hi) whose id is `id`, or -1.
__device__ __forceinline__ int find(const int32_t* ids, int lo, int hi, int id) {
  if (!ids) return id;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (ids[mid] < id) lo = mid + 1;
    else hi = mid;
  }
  return ids[lo] == id ? lo : -1;
}

// Mask bits of columns col .. col + 7 (bit j: column col + j), only those in [0, n) meant.
__device__ __forceinline__ uint32_t mask_bits(const Shape& a, const uint32_t* mask, int col) {
  if (!a.ids) {
    const int from = max(col, 0), w = from >> 5;
    const uint32_t lo = mask[w];
    const uint32_t hi = (from & 31) > 24 && 32 * (w + 1) < a.n ? mask[w + 1] : 0u;
    return __funnelshift_r(lo, hi, from & 31) << (from - col);
  }
  uint32_t bits = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if (col + j >= 0 && col + j < a.n) {
      const uint32_t id = (uint32_t)a.ids[col + j];
      if (id < (uint32_t)a.V) bits |= (mask[id >> 5] >> (id & 31) & 1u) << j;
    }
  return bits;
}

// VEC: rows of z and out are on 16 bytes.  Other rows: pieces are laid so that they begin on
// the output's 16-byte boundaries.
template <class T, class OT, bool VEC>
__global__ void __launch_bounds__(kThreads) shape_kernel(const Shape a) {
  extern __shared__ uint32_t smem[];
  __shared__ float s_max[kThreads / 32], s_sum[kThreads / 32];
  __shared__ int s_at[kThreads / 32];
  ptx::griddep_wait();
  ptx::griddep_launch_dependents();
  const int64_t row = blockIdx.x / a.chunks;
  const int chunk = (int)(blockIdx.x - row * a.chunks);
  OT* out = static_cast<OT*>(a.out) + row * a.ld_out;
  int base = chunk * a.cols;               // column of shared word 0
  if constexpr (!VEC) {
    const int head = (int)(-(intptr_t)out & 15) / (int)sizeof(OT);
    base += head ? head - 8 : 0;
  }
  const int c0 = max(base, 0), c1 = min(base + a.cols, a.n);

  // ---- tokens so far, biases ----
  uint32_t* count = smem;                  // of output tokens; bit 31: a prompt token too
  float* bias = reinterpret_cast<float*>(smem + (a.history ? a.cols : 0));
  int length = 0;
  if (a.history) length = a.lengths ? max(0, min(a.lengths[row], a.max_tokens)) : a.max_tokens;
  const bool counts = length > 0 && c0 < c1, biases = a.n_bias > 0 && c0 < c1;
  if (counts || biases) {
    const int32_t first = a.ids ? a.ids[c0] : c0, last = a.ids ? a.ids[c1 - 1] : c1 - 1;
    for (int i = threadIdx.x; i < a.cols; i += kThreads) {
      if (counts) count[i] = 0;
      if (biases) bias[i] = 0.f;
    }
    __syncthreads();
    if (counts) {
      const int prompt = a.prompts ? a.prompts[row] : 0;
      const int32_t* h = a.history + row * a.ld_history;
      for (int i = threadIdx.x; i < length; i += kThreads) {
        const int32_t id = h[i];
        if (id < first || id > last) continue;
        const int c = find(a.ids, c0, c1 - 1, id);
        if (c < 0) continue;
        if (i < prompt) atomicOr(&count[c - base], 0x80000000u);
        else atomicAdd(&count[c - base], 1u);
      }
    }
    if (biases && threadIdx.x < 32) {
      // (one warp, so that entries for the same id are added in the list's order)
      const int lane = threadIdx.x;
      for (int i0 = 0; i0 < a.n_bias; i0 += 32) {
        int c = -1;
        float b = 0.f;
        if (i0 + lane < a.n_bias) {
          const int32_t id = a.bias_ids[row * a.ld_bias_ids + i0 + lane];
          if (id >= first && id <= last) c = find(a.ids, c0, c1 - 1, id);
          if (c >= 0) b = a.bias_values[row * a.ld_bias_values + i0 + lane];
        }
        const unsigned same = __match_any_sync(0xFFFFFFFFu, c);
        const bool lead = c >= 0 && __ffs(same) - 1 == lane;
        float sum = lead ? bias[c - base] : 0.f;
        for (int l = 0; l < 32; ++l) {
          const float v = __shfl_sync(0xFFFFFFFFu, b, l);
          if (lead && same >> l & 1) sum = __fadd_rn(sum, v);
        }
        if (lead) bias[c - base] = sum;
        __syncwarp();
      }
    }
    __syncthreads();
  }
  const float rep = counts && a.repetition ? a.repetition[row] : 1.f;
  const float freq = counts && a.frequency ? a.frequency[row] : 0.f;
  const float pres = counts && a.presence ? a.presence[row] : 0.f;

  const uint32_t* mask = nullptr;
  if (a.mask) {
    const int64_t m = a.mask_rows ? a.mask_rows[row] : row;
    if (m >= 0 && m < a.n_masks) mask = a.mask + m * a.ld_mask;
    else if (m != -1 && threadIdx.x == 0 && chunk == 0) atomicOr(a.status, ERR_BAD_INDEX);
  }

  // ---- the columns ----
  const T* z = static_cast<const T*>(a.z) + row * a.ld_z;
  float top = -INFINITY, sum = 0.f;
  int at = 0x7FFFFFFF;
  for (int k = (int)threadIdx.x * 8; k < a.cols; k += kThreads * 8) {
    const int col = base + k;
    if (col >= a.n) break;
    float v[8];
    load_cols<T, VEC>(z, col, a.n, v);
    if (counts) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const uint32_t c = count[k + j];
        if (c) {
          float x = v[j];
          if (a.repetition) x = x > 0.f ? __fdiv_rn(x, rep) : __fmul_rn(x, rep);
          if (c & 0x7FFFFFFFu) {
            if (a.frequency) x = __fsub_rn(x, __fmul_rn(freq, (float)(c & 0x7FFFFFFFu)));
            if (a.presence) x = __fsub_rn(x, pres);
          }
          v[j] = x;
        }
      }
    }
    if (biases) {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = __fadd_rn(v[j], bias[k + j]);
    }
    if (mask) {
      const uint32_t bits = mask_bits(a, mask, col);
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (!(bits >> j & 1)) v[j] = -INFINITY;
    }
    store_cols<OT, true>(out, col, a.n, v);
    if (a.draw) {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (col + j < 0 || col + j >= a.n) v[j] = -INFINITY;
      float m = top;
#pragma unroll
      for (int j = 0; j < 8; ++j) m = fmaxf(m, v[j]);
      if (a.greedy) {
        bool bad = false;
#pragma unroll
        for (int j = 7; j >= 0; --j) {
          if (v[j] == m && m > top) at = col + j;
          bad |= v[j] != v[j];
        }
        if (bad) sum = NAN;
      } else {
        if (m > top) sum *= weight(top, m, a.l2t);
#pragma unroll
        for (int j = 0; j < 8; ++j) sum += weight(v[j], m, a.l2t);
      }
      top = m;
    }
  }
  if (!a.draw) return;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  auto join = [&](float m2, float s2, int at2) {
    const float M = fmaxf(top, m2);
    if (m2 > top || (m2 == top && at2 < at)) at = at2;
    if (a.greedy) sum += s2;
    else sum = sum * weight(top, M, a.l2t) + s2 * weight(m2, M, a.l2t);
    top = M;
  };
#pragma unroll
  for (int o = 16; o; o >>= 1)
    join(__shfl_xor_sync(0xFFFFFFFFu, top, o), __shfl_xor_sync(0xFFFFFFFFu, sum, o),
         __shfl_xor_sync(0xFFFFFFFFu, at, o));
  if (lane == 0) {
    s_max[warp] = top;
    s_sum[warp] = sum;
    s_at[warp] = at;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
#pragma unroll
    for (int w = 1; w < kThreads / 32; ++w) join(s_max[w], s_sum[w], s_at[w]);
    a.stats[row * a.chunks + chunk] = make_float4(top, sum, __int_as_float(at), 0.f);
  }
}

// Sum of `v` over the threads before this one, and over all (order: the threads').
__device__ __forceinline__ float scan_block(float v, float* red, float* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  float incl = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const float t = __shfl_up_sync(0xFFFFFFFFu, incl, o);
    if (lane >= o) incl += t;
  }
  __syncthreads();
  if (lane == 31) red[warp] = incl;
  __syncthreads();
  float before = 0.f, all = 0.f;
#pragma unroll
  for (int w = 0; w < kThreads / 32; ++w) {
    if (w < warp) before += red[w];
    all += red[w];
  }
  *total = all;
  return before + incl - v;
}

// Of consecutive runs of [0, n), one a thread, with weights w(i): the first place, in order,
// where the sum from `before` on exceeds the target; the last place with weight where
// rounding leaves none.  Every thread gets the place and the sum before it.
template <class W>
__device__ __forceinline__ int pick(int n, const W& w, float target, float* before, float* red,
                                    int* s_place, float* s_before) {
  const int per = (n + kThreads - 1) / kThreads;
  const int lo = min(n, (int)threadIdx.x * per), hi = min(n, lo + per);
  float local = 0.f, total;
  int last = -1;
  for (int i = lo; i < hi; ++i) {
    const float x = w(i);
    if (x > 0.f) last = i;
    local += x;
  }
  const float from = *before + scan_block(local, red, &total);
  // (threads vote for the first run that passes the target, and the last with weight)
  if (threadIdx.x == 0) { s_place[0] = 0x7FFFFFFF; s_place[1] = -1; }
  __syncthreads();
  if (last >= 0) {
    if (target < from + local) atomicMin(&s_place[0], (int)threadIdx.x);
    atomicMax(&s_place[1], (int)threadIdx.x);
  }
  __syncthreads();
  const int owner = s_place[0] != 0x7FFFFFFF ? s_place[0] : s_place[1];
  __syncthreads();
  if ((int)threadIdx.x == owner) {
    float sum = from, before_last = from;
    int place = last;
    for (int i = lo; i < hi; ++i) {
      const float x = w(i);
      if (x > 0.f) {
        if (target < sum + x) { place = i; before_last = sum; break; }
        if (i == last) before_last = sum;
      }
      sum += x;
    }
    s_place[0] = place;
    *s_before = before_last;
  }
  __syncthreads();
  const int place = s_place[0];
  *before = *s_before;
  __syncthreads();
  return owner < 0 ? -1 : place;
}

__global__ void __launch_bounds__(kThreads) shape_draw_kernel(const Shape a) {
  __shared__ float red[kThreads / 32];
  __shared__ int s_place[2];
  __shared__ float s_before;
  ptx::griddep_wait();
  ptx::griddep_launch_dependents();
  const int64_t row = blockIdx.x;
  const float4* st = a.stats + row * a.chunks;
  float M = -INFINITY, bad = 0.f;
  for (int c = threadIdx.x; c < a.chunks; c += kThreads) {
    const float4 q = st[c];
    M = fmaxf(M, q.x);
    bad += q.y - q.y;                   // (NaN where the sum is one; sums are finite else)
  }
  M = block_max(M, red);
  bad = block_sum(bad, red);
  // no id is allowed, or a NaN is among those that are
  if (M == -INFINITY || bad != 0.f) {
    if (threadIdx.x == 0) a.tokens[row] = -1;
    return;
  }
  if (a.greedy) {
    // the chunks are in order, and so is the first place within each
    int at = 0x7FFFFFFF;
    for (int c = threadIdx.x; c < a.chunks; c += kThreads) {
      const float4 q = st[c];
      if (q.x == M) at = min(at, __float_as_int(q.z));
    }
    at = (int)__reduce_min_sync(0xFFFFFFFFu, (unsigned)at);
    if (threadIdx.x == 0) s_place[0] = 0x7FFFFFFF;
    __syncthreads();
    if ((threadIdx.x & 31) == 0) atomicMin(&s_place[0], at);
    __syncthreads();
    if (threadIdx.x == 0) a.tokens[row] = a.ids ? a.ids[s_place[0]] : s_place[0];
    return;
  }
  auto of_chunk = [&](int c) {
    const float4 q = st[c];
    return q.y * weight(q.x, M, a.l2t);
  };
  float total, before = 0.f;
  {
    const int per = (a.chunks + kThreads - 1) / kThreads;
    const int lo = min(a.chunks, (int)threadIdx.x * per), hi = min(a.chunks, lo + per);
    float local = 0.f;
    for (int c = lo; c < hi; ++c) local += of_chunk(c);
    scan_block(local, red, &total);
  }
  const float target = philox_uniform(a.seed, (uint32_t)row, 0u, a.offset) * total;
  const int chunk = pick(a.chunks, of_chunk, target, &before, red, s_place, &s_before);
  const float* z = static_cast<const float*>(a.out) + row * a.ld_out;
  int base = chunk * a.cols;
  if (!a.vec) {
    const int head = (int)(-(intptr_t)z & 15) / 4;
    base += head ? head - 8 : 0;
  }
  const int c0 = max(base, 0), c1 = min(base + a.cols, a.n);
  const int j = pick(c1 - c0, [&](int i) { return weight(z[c0 + i], M, a.l2t); }, target, &before,
                     red, s_place, &s_before);
  if (threadIdx.x == 0) a.tokens[row] = j < 0 ? -1 : a.ids ? a.ids[c0 + j] : c0 + j;
}

// Columns of a block.
int chunk_cols(int64_t rows, int n, int sm_count) {
  int cols = kThreads * 8;
  while (cols < 4096 && rows * ((n + 2 * cols - 1) / (2 * cols)) >= 4 * (int64_t)sm_count) cols *= 2;
  return cols;
}
int chunk_count(int n, int cols) { return (n + 7 + cols - 1) / cols; }

template <class T, class OT>
cudaError_t launch_shape_t(const Shape& a, size_t smem, cudaStream_t st) {
  const dim3 grid((unsigned)(a.rows * a.chunks));
  return a.vec ? launch_pdl(shape_kernel<T, OT, true>, grid, dim3(kThreads), smem, st, a)
               : launch_pdl(shape_kernel<T, OT, false>, grid, dim3(kThreads), smem, st, a);
}
template <class T>
cudaError_t launch_shape_o(const Shape& a, int out_type, size_t smem, cudaStream_t st) {
  if (out_type == TAB_FP32) return launch_shape_t<T, float>(a, smem, st);
  if (out_type == TAB_BF16) return launch_shape_t<T, __nv_bfloat16>(a, smem, st);
  return launch_shape_t<T, __half>(a, smem, st);
}

}  // namespace

size_t shape_scratch_bytes(int64_t rows, int n, int sm_count) {
  return (size_t)rows * chunk_count(n, chunk_cols(rows, n, sm_count)) * sizeof(float4);
}
// At least what any call of up to so many rows and ids takes.
size_t shape_reserve_bytes(int64_t rows, int64_t n) {
  return (size_t)rows * chunk_count((int)n, kThreads * 8) * sizeof(float4);
}
int64_t shape_blocks(int64_t rows, int n, int sm_count) {
  return rows * chunk_count(n, chunk_cols(rows, n, sm_count));
}

cudaError_t launch_shape(Shape a, int z_type, int out_type, void* scratch, int sm_count,
                         cudaStream_t st) {
  a.cols = chunk_cols(a.rows, a.n, sm_count);
  a.chunks = chunk_count(a.n, a.cols);
  a.stats = static_cast<float4*>(scratch);
  a.vec = on16(a.z, a.ld_z, type_size(z_type)) && on16(a.out, a.ld_out, type_size(out_type));
  a.l2t = a.greedy ? 0.f : kLog2e * a.inv_tau;
  const size_t smem = (size_t)a.cols * 4 * ((a.history ? 1 : 0) + (a.n_bias > 0 ? 1 : 0));
  const cudaError_t e = z_type == TAB_FP32   ? launch_shape_o<float>(a, out_type, smem, st)
                        : z_type == TAB_BF16 ? launch_shape_o<__nv_bfloat16>(a, out_type, smem, st)
                                             : launch_shape_o<__half>(a, out_type, smem, st);
  if (e != cudaSuccess || !a.draw) return e;
  return launch_pdl(shape_draw_kernel, dim3((unsigned)a.rows), dim3(kThreads), 0, st, a);
}

}  // namespace sph
