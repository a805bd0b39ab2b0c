// Rows of a vocabulary table by token, and the table's gradient from them.
//
//   lookup    out[t, :] = scale * W[token_t, :]
//   gradient  dW[v, :] (+)= scale * sum over {t : token_t = v} of dOut[t, :]
//
// Both are bound by memory.  The gradient sorts the token positions by id
// (stable, so equal inputs give equal bits), sums runs of equal ids over ranges
// of sorted positions of one length, whatever the runs' lengths, and joins the
// parts of a run that crosses ranges, in order.  Rows of ids that no token has
// are zeroed while the sort runs.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "mx4.cuh"
#include "sm100_ptx.cuh"
#include "sph_internal.h"

namespace sph {
namespace {

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__half x) { return __half2float(x); }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
template <class T> __device__ __forceinline__ T from_f32(float x);
template <> __device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <> __device__ __forceinline__ __half from_f32<__half>(float x) { return __float2half_rn(x); }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float x) {
  return __float2bfloat16_rn(x);
}

// A thread's eight columns of a row.  VEC: eight consecutive ones, moved in
// 16-byte pieces (rows on 16 bytes); else `stride` apart, so that the threads of a
// warp touch neighbouring columns whatever the row's start.
template <class T, bool VEC>
__device__ __forceinline__ void load_cols(const T* row, int col, int stride, int d, float (&v)[8]) {
  if (VEC && col + 8 <= d) {
    uint4 w[sizeof(T) / 2];
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i)
      w[i] = reinterpret_cast<const uint4*>(row + col)[i];
    const T* e = reinterpret_cast<const T*>(w);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = to_f32(e[j]);
  } else {
    const int s = VEC ? 1 : stride;
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = col + j * s < d ? to_f32(row[col + j * s]) : 0.f;
  }
}
template <class T, bool VEC>
__device__ __forceinline__ void store_cols(T* row, int col, int stride, int d, const float (&v)[8]) {
  if (VEC && col + 8 <= d) {
    uint4 w[sizeof(T) / 2];
    T* e = reinterpret_cast<T*>(w);
#pragma unroll
    for (int j = 0; j < 8; ++j) e[j] = from_f32<T>(v[j]);
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) reinterpret_cast<uint4*>(row + col)[i] = w[i];
  } else {
    const int s = VEC ? 1 : stride;
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (col + j * s < d) row[col + j * s] = from_f32<T>(v[j]);
  }
}

// ---------------------------------------------------------------------------
// lookup
// ---------------------------------------------------------------------------
constexpr int kLookThreads = 128;
constexpr int kLookSpan = kLookThreads * 8;    // columns of a block

struct Mx4Row;     // tag of a table held in 4 bits (FMT says which)

template <class TT, int FMT, bool VEC>
__device__ __forceinline__ void table_cols(const Lookup& a, int64_t id, int col, float (&v)[8]) {
  if constexpr (FMT < 0) {
    load_cols<TT, VEC>(static_cast<const TT*>(a.table) + id * a.ld_table, col, kLookThreads, a.d, v);
  } else {
    // (rows of codes and scales start on 16 bytes and end on a whole 32 columns)
    const uint8_t* codes = static_cast<const uint8_t*>(a.table) + id * a.ld_table;
    const uint8_t* scales = a.scales + id * a.ld_scales;
    const float row = FMT == MX4_E4M3 ? a.row_scale[id] : 1.f;
    if constexpr (VEC) {
      if (col < a.d) {
        e2m1x8_to_float(*reinterpret_cast<const uint32_t*>(codes + col / 2), v);
        const float s = mx4_scale_value<FMT>(scales[col / Mx4<FMT>::kBlock]) * row;
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] *= s;
      }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int c = col + j * kLookThreads;
        if (c < a.d) {
          float q[8];
          e2m1x8_to_float((uint32_t)codes[c / 2] >> (c & 1) * 4 & 15u, q);
          v[j] = q[0] * (mx4_scale_value<FMT>(scales[c / Mx4<FMT>::kBlock]) * row);
        }
      }
    }
  }
}

// TB tokens and kLookSpan columns a block; the tokens' rows are requested together.
template <class TT, int FMT, class OT, bool VEC, int TB>
__global__ void __launch_bounds__(kLookThreads) lookup_kernel(const Lookup a) {
  ptx::griddep_wait();
  ptx::griddep_launch_dependents();
  const int span = (int)(blockIdx.x % a.spans);
  const int64_t t0 = (int64_t)(blockIdx.x / a.spans) * TB;
  const int col = span * kLookSpan + (VEC ? (int)threadIdx.x * 8 : (int)threadIdx.x);
  float v[TB][8];
#pragma unroll
  for (int i = 0; i < TB; ++i) {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[i][j] = 0.f;
    if (t0 + i >= a.n) continue;
    const int64_t id = a.tokens ? a.tokens[t0 + i] : t0 + i;
    if (id >= 0 && id < a.V) table_cols<TT, FMT, VEC>(a, id, col, v[i]);
    else if (id != a.padding && col == 0) atomicOr(a.status, ERR_BAD_INDEX);
  }
#pragma unroll
  for (int i = 0; i < TB; ++i) {
    if (t0 + i >= a.n) break;
#pragma unroll
    for (int j = 0; j < 8; ++j) v[i][j] *= a.scale;
    store_cols<OT, VEC>(static_cast<OT*>(a.out) + (t0 + i) * a.ld_out, col, kLookThreads, a.d, v[i]);
  }
}

template <class TT, int FMT, class OT, bool VEC>
cudaError_t launch_lookup_v(const Lookup& a, int sm_count, cudaStream_t st) {
  // four tokens a block once that still leaves every SM eight blocks
  const int64_t blocks = a.n * a.spans;
  if (blocks >= (int64_t)sm_count * 32)
    return launch_pdl(lookup_kernel<TT, FMT, OT, VEC, 4>,
                      dim3((unsigned)((a.n + 3) / 4 * a.spans)), dim3(kLookThreads), 0, st, a);
  return launch_pdl(lookup_kernel<TT, FMT, OT, VEC, 1>, dim3((unsigned)blocks), dim3(kLookThreads),
                    0, st, a);
}
template <class TT, int FMT, class OT>
cudaError_t launch_lookup_o(const Lookup& a, bool vec, int sm_count, cudaStream_t st) {
  return vec ? launch_lookup_v<TT, FMT, OT, true>(a, sm_count, st)
             : launch_lookup_v<TT, FMT, OT, false>(a, sm_count, st);
}
template <class TT, int FMT>
cudaError_t launch_lookup_t(const Lookup& a, int out_type, bool vec, int sm_count, cudaStream_t st) {
  if (out_type == TAB_FP32) return launch_lookup_o<TT, FMT, float>(a, vec, sm_count, st);
  if (out_type == TAB_BF16) return launch_lookup_o<TT, FMT, __nv_bfloat16>(a, vec, sm_count, st);
  return launch_lookup_o<TT, FMT, __half>(a, vec, sm_count, st);
}

bool on16(const void* p, int64_t ld, int size) {
  return ((uintptr_t)p & 15) == 0 && (ld * size & 15) == 0;
}
int type_size(int t) { return t == TAB_FP32 ? 4 : 2; }

// ---------------------------------------------------------------------------
// gradient: the sort
// ---------------------------------------------------------------------------
constexpr int kSortThreads = 1024, kSortItems = 4, kSortTile = kSortThreads * kSortItems;
constexpr int kSortBits = 9, kSortBins = 1 << kSortBits, kSortWarps = kSortThreads / 32;

struct SortSmem {
  uint32_t hist[kSortBins];       // this CTA's count of each digit (read by the cluster)
  uint32_t base[kSortBins];       // where its next element of a digit goes
  uint32_t tile[kSortBins];       // the same at the start of the current tile
  uint32_t part[kSortBins / 32];
  uint16_t warp[kSortWarps][kSortBins];
};

// One cluster sorts: stable radix passes of 9 bits over (id, position), each CTA a
// contiguous part.  A pass counts digits per CTA, reads the counts of the
// cluster's CTAs through distributed shared memory, and moves its part tile by
// tile; within a tile, equal digits of a warp are ranked by match.any, warps by a
// prefix over their counts.  Ids out of range become V, which sorts last.
__global__ void __launch_bounds__(kSortThreads) sort_kernel(const TableGrad a, int parts, int passes) {
  extern __shared__ __align__(16) uint8_t sort_raw[];
  SortSmem& s = *reinterpret_cast<SortSmem*>(sort_raw);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int rank = (int)blockIdx.x;
  ptx::griddep_wait();
  ptx::griddep_launch_dependents();
  const int part = (a.n + parts - 1) / parts;
  const int p0 = min(a.n, rank * part), p1 = min(a.n, p0 + part);
  for (int pass = 0; pass < passes; ++pass) {
    const int shift = pass * kSortBits;
    // passes end in buffer 0: the last one writes it
    const int to = (passes - 1 - pass) & 1;
    const int32_t* src_k = a.keys[to ^ 1];
    const int32_t* src_p = a.pos[to ^ 1];
    int32_t* dst_k = a.keys[to];
    int32_t* dst_p = a.pos[to];
    auto key_of = [&](int i) {
      if (pass > 0) return __ldcg(src_k + i);
      const int32_t id = a.tokens[i];
      return id >= 0 && id < a.V ? id : a.V;
    };
    auto digit = [&](int32_t k) { return (int)((uint32_t)k >> shift) & (kSortBins - 1); };
    for (int b = tid; b < kSortBins; b += kSortThreads) s.hist[b] = 0;
    __syncthreads();
    for (int i = p0 + tid; i < p1; i += kSortThreads) {
      if (pass == 0) {
        const int32_t id = a.tokens[i];
        if ((id < 0 || id >= a.V) && id != a.padding) atomicOr(a.status, ERR_BAD_INDEX);
      }
      atomicAdd(&s.hist[digit(key_of(i))], 1u);
    }
    ptx::cluster_sync();
    uint32_t total = 0, below = 0;
    if (tid < kSortBins) {
      for (int c = 0; c < parts; ++c) {
        uint32_t h;
        asm volatile("ld.shared::cluster.u32 %0, [%1];"
                     : "=r"(h)
                     : "r"(ptx::mapa(ptx::smem_u32(&s.hist[tid]), (uint32_t)c))
                     : "memory");
        if (c < rank) below += h;
        total += h;
      }
    }
    uint32_t incl = total;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t up = __shfl_up_sync(0xFFFFFFFFu, incl, o);
      if (lane >= o) incl += up;
    }
    if (tid < kSortBins && lane == 31) s.part[warp] = incl;
    __syncthreads();
    if (tid < kSortBins) {
      uint32_t before = 0;
      for (int w = 0; w < warp; ++w) before += s.part[w];
      s.base[tid] = before + incl - total + below;
    }
    for (int t0 = p0; t0 < p1; t0 += kSortTile) {
      int32_t k[kSortItems], p[kSortItems];
      uint32_t r[kSortItems];
#pragma unroll
      for (int i = 0; i < kSortItems; ++i) {
        const int at = t0 + warp * (32 * kSortItems) + i * 32 + lane;
        k[i] = at < p1 ? key_of(at) : 0;
        p[i] = at < p1 ? (pass == 0 ? at : __ldcg(src_p + at)) : -1;
      }
      for (int b = lane; b < kSortBins / 2; b += 32)
        reinterpret_cast<uint32_t*>(s.warp[warp])[b] = 0;
      __syncwarp();
#pragma unroll
      for (int i = 0; i < kSortItems; ++i) {
        const unsigned live = __ballot_sync(0xFFFFFFFFu, p[i] >= 0);
        if (p[i] >= 0) {
          const int dg = digit(k[i]);
          const unsigned same = __match_any_sync(live, dg);
          const uint32_t had = s.warp[warp][dg];
          r[i] = had + __popc(same & ((1u << lane) - 1));
          __syncwarp(live);
          if ((same & ((1u << lane) - 1)) == 0) s.warp[warp][dg] = (uint16_t)(had + __popc(same));
        }
        __syncwarp();
      }
      __syncthreads();
      if (tid < kSortBins) {
        uint32_t run = 0;
#pragma unroll 8
        for (int w = 0; w < kSortWarps; ++w) {
          const uint32_t c = s.warp[w][tid];
          s.warp[w][tid] = (uint16_t)run;
          run += c;
        }
        s.tile[tid] = s.base[tid];
        s.base[tid] += run;
      }
      __syncthreads();
#pragma unroll
      for (int i = 0; i < kSortItems; ++i) {
        if (p[i] >= 0) {
          const int dg = digit(k[i]);
          const uint32_t to_at = s.tile[dg] + s.warp[warp][dg] + r[i];
          dst_k[to_at] = k[i];
          dst_p[to_at] = p[i];
        }
      }
      __syncthreads();
    }
    // the pass's writes reach the cluster's other CTAs, and none still reads
    // this one's counts when the next pass clears them
    ptx::cluster_sync();
  }
}

// ---------------------------------------------------------------------------
// gradient: zero rows
// ---------------------------------------------------------------------------
constexpr int kFillThreads = 512, kFillIds = 8192;

// Zeros, by one warp, over bytes of any alignment.
__device__ __forceinline__ void zero_bytes(uint8_t* p, int64_t bytes, int lane) {
  const int64_t head = min(bytes, (int64_t)(-(intptr_t)p & 15));
  // (elements have 2 bytes or more, and so has the row's start)
  if (2 * lane < head) *reinterpret_cast<uint16_t*>(p + 2 * lane) = 0;
  uint4* body = reinterpret_cast<uint4*>(p + head);
  const int64_t n16 = (bytes - head) / 16;
  for (int64_t i = lane; i < n16; i += 32) body[i] = make_uint4(0, 0, 0, 0);
  const int64_t done = head + n16 * 16;
  if (done + 2 * lane < bytes) *reinterpret_cast<uint16_t*>(p + done + 2 * lane) = 0;
}

// Block b zeroes the rows of its share of the ids that no token has: it marks
// the ones that occur from the whole token list (a read of the L2, once per
// kFillIds ids), so nothing is written twice.  Runs beside the sort, and waits
// for it only at its end, so that the kernel after it may take both as done.
// FIRST: it is the call's first kernel, and waits for the caller's work instead.
template <bool FIRST>
__global__ void __launch_bounds__(kFillThreads) fill_kernel(const TableGrad a, int elem) {
  __shared__ uint32_t s_seen[kFillIds / 32];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t v0 = (int64_t)a.V * blockIdx.x / gridDim.x;
  const int64_t v1 = (int64_t)a.V * (blockIdx.x + 1) / gridDim.x;
  if constexpr (FIRST) ptx::griddep_wait();
  ptx::griddep_launch_dependents();
  for (int64_t base = v0; base < v1; base += kFillIds) {
    const int ids = (int)min((int64_t)kFillIds, v1 - base);
    for (int i = threadIdx.x; i < kFillIds / 32; i += kFillThreads) s_seen[i] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < a.n; i += kFillThreads) {
      const int64_t r = (int64_t)a.tokens[i] - base;
      if (r >= 0 && r < ids) atomicOr(&s_seen[r >> 5], 1u << (r & 31));
    }
    __syncthreads();
    for (int r = warp; r < ids; r += kFillThreads / 32)
      if (!(s_seen[r >> 5] >> (r & 31) & 1))
        zero_bytes(static_cast<uint8_t*>(a.out) + (base + r) * a.ld_out * elem,
                   (int64_t)a.d * elem, lane);
    __syncthreads();
  }
  if constexpr (!FIRST) ptx::griddep_wait();
}

// ---------------------------------------------------------------------------
// gradient: sums over ranges of sorted positions, and the join
// ---------------------------------------------------------------------------
constexpr int kSumThreads = 128;
constexpr int kSumBatch = 8;        // rows requested together (4 where columns are scattered)

// Columns of thread `u` of `ct` in column group g.
template <bool VEC>
__device__ __forceinline__ int sum_col(int g, int u, int ct) {
  return g * ct * 8 + (VEC ? u * 8 : u);
}

template <class OT, bool VEC>
__device__ __forceinline__ void write_row(const TableGrad& a, int32_t id, int col, int ct,
                                          const float (&sum)[8]) {
  OT* row = static_cast<OT*>(a.out) + (int64_t)id * a.ld_out;
  float v[8];
  if (a.add) {
    load_cols<OT, VEC>(row, col, ct, a.d, v);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] += a.scale * sum[j];
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = a.scale * sum[j];
  }
  store_cols<OT, VEC>(row, col, ct, a.d, v);
}

// ct threads a range of a.range sorted positions and 8 ct columns (128 / ct
// ranges a block).  A run of equal ids inside the range is written out; the part of
// one that began before the range goes to slot 2 r of the partial sums, that of
// one that begins in it and goes on to slot 2 r + 1.
template <class T, class OT, bool VEC>
__global__ void __launch_bounds__(kSumThreads) sum_kernel(const TableGrad a, int ct) {
  ptx::griddep_wait();
  ptx::griddep_launch_dependents();
  const int u = threadIdx.x % ct;
  const int group = (int)(blockIdx.x % a.groups);
  const int64_t r = (int64_t)(blockIdx.x / a.groups) * (kSumThreads / ct) + threadIdx.x / ct;
  const int64_t i0 = r * a.range;
  const int col = sum_col<VEC>(group, u, ct);
  if (i0 >= a.n || col >= a.d) return;
  const int i1 = (int)min((int64_t)a.n, i0 + a.range);
  const int32_t* keys = a.keys[0];
  const int32_t* pos = a.pos[0];
  float acc[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) acc[j] = 0.f;
  int32_t cur = keys[i0];
  bool open_left = i0 > 0 && keys[i0 - 1] == cur;
  auto flush = [&](bool open_right) {
    if (cur == a.V) return;
    if (!open_left && !open_right) {
      write_row<OT, VEC>(a, cur, col, ct, acc);
    } else {
      float* p = a.partial + (2 * r + (open_left ? 0 : 1)) * a.ld_partial + group * ct * 8 + u * 8;
      reinterpret_cast<float4*>(p)[0] = make_float4(acc[0], acc[1], acc[2], acc[3]);
      reinterpret_cast<float4*>(p)[1] = make_float4(acc[4], acc[5], acc[6], acc[7]);
    }
  };
  constexpr int kBatch = VEC ? kSumBatch : kSumBatch / 2;
  for (int b = (int)i0; b < i1; b += kBatch) {
    int32_t k[kBatch];
    float x[kBatch][8];
#pragma unroll
    for (int q = 0; q < kBatch; ++q) {
      k[q] = b + q < i1 ? keys[b + q] : a.V;
      if (k[q] < a.V)
        load_cols<T, VEC>(static_cast<const T*>(a.d_out) + (int64_t)pos[b + q] * a.ld_d_out, col, ct,
                          a.d, x[q]);
    }
#pragma unroll
    for (int q = 0; q < kBatch; ++q) {
      if (b + q >= i1) break;
      if (k[q] != cur) {
        flush(false);
        cur = k[q];
        open_left = false;
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[j] = 0.f;
      }
      if (k[q] < a.V) {
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[j] += x[q][j];
      }
    }
  }
  flush(i1 < a.n && keys[i1] == cur);
}

constexpr int kJoinThreads = 256;

// A block for each range and column group; it goes on only where a run begins in
// the range and crosses its end.  The run's parts (slot 2 r + 1, then slot 2 j of
// the ranges j it reaches) are shared by the block's thread groups in contiguous
// shares, which are added in order.
template <class OT, bool VEC>
__global__ void __launch_bounds__(kJoinThreads) join_kernel(const TableGrad a, int ct) {
  __shared__ float s_sum[kJoinThreads * 8];
  ptx::griddep_wait();
  ptx::griddep_launch_dependents();
  const int group = (int)(blockIdx.x % a.groups);
  const int64_t r = blockIdx.x / a.groups;
  const int64_t i0 = r * a.range, i1 = i0 + a.range;
  const int32_t* keys = a.keys[0];
  if (i1 >= a.n) return;
  const int32_t id = keys[i1 - 1];
  if (id == a.V || keys[i1] != id) return;
  if (keys[i0] == id && i0 > 0 && keys[i0 - 1] == id) return;     // began earlier
  int64_t parts = 1;
  for (int64_t j = r + 1;; j += kJoinThreads) {
    const int64_t at = (j + threadIdx.x) * a.range;
    const int c = __syncthreads_count(at < a.n && keys[at] == id);
    parts += c;
    if (c < kJoinThreads) break;
  }
  const int u = threadIdx.x % ct, share = threadIdx.x / ct, shares = kJoinThreads / ct;
  const int col = sum_col<VEC>(group, u, ct);
  float sum[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) sum[j] = 0.f;
  if (col < a.d) {
    const int64_t q1 = parts * (share + 1) / shares;
#pragma unroll 4
    for (int64_t q = parts * share / shares; q < q1; ++q) {
      const float4* p = reinterpret_cast<const float4*>(
          a.partial + (q == 0 ? 2 * r + 1 : 2 * (r + q)) * a.ld_partial + group * ct * 8 + u * 8);
      const float4 x = p[0], y = p[1];
      sum[0] += x.x; sum[1] += x.y; sum[2] += x.z; sum[3] += x.w;
      sum[4] += y.x; sum[5] += y.y; sum[6] += y.z; sum[7] += y.w;
    }
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) s_sum[j * kJoinThreads + threadIdx.x] = sum[j];
  __syncthreads();
  if (share > 0 || col >= a.d) return;
  for (int h = 1; h < shares; ++h)
#pragma unroll
    for (int j = 0; j < 8; ++j) sum[j] += s_sum[j * kJoinThreads + h * ct + u];
  write_row<OT, VEC>(a, id, col, ct, sum);
}

template <class T, class OT, bool VEC>
cudaError_t launch_sums(const TableGrad& a, int ct, cudaStream_t st) {
  const int64_t ranges = (a.n + (int64_t)a.range - 1) / a.range;
  const int per = kSumThreads / ct;
  cudaError_t e = launch_pdl(sum_kernel<T, OT, VEC>,
                             dim3((unsigned)((ranges + per - 1) / per * a.groups)),
                             dim3(kSumThreads), 0, st, a, ct);
  if (e != cudaSuccess || ranges < 2) return e;
  return launch_pdl(join_kernel<OT, VEC>, dim3((unsigned)((ranges - 1) * a.groups)),
                    dim3(kJoinThreads), 0, st, a, ct);
}
template <class T, class OT>
cudaError_t launch_sums_v(const TableGrad& a, int ct, bool vec, cudaStream_t st) {
  return vec ? launch_sums<T, OT, true>(a, ct, st) : launch_sums<T, OT, false>(a, ct, st);
}
template <class T>
cudaError_t launch_sums_o(const TableGrad& a, int ct, int out_type, bool vec, cudaStream_t st) {
  if (out_type == TAB_FP32) return launch_sums_v<T, float>(a, ct, vec, st);
  if (out_type == TAB_BF16) return launch_sums_v<T, __nv_bfloat16>(a, ct, vec, st);
  return launch_sums_v<T, __half>(a, ct, vec, st);
}

// Threads that share a range's columns: enough for the row, at most 128.
int sum_threads(int d) {
  int ct = 4;
  while (ct < kSumThreads && ct * 8 < d) ct *= 2;
  return ct;
}

}  // namespace

cudaError_t launch_lookup(Lookup a, int table_type, int out_type, int sm_count, cudaStream_t st) {
  a.spans = (a.d + kLookSpan - 1) / kLookSpan;
  bool vec = on16(a.out, a.ld_out, type_size(out_type));
  if (table_type == TAB_E8M0)
    return launch_lookup_t<Mx4Row, MX4_E8M0>(a, out_type, vec, sm_count, st);
  if (table_type == TAB_E4M3)
    return launch_lookup_t<Mx4Row, MX4_E4M3>(a, out_type, vec, sm_count, st);
  vec = vec && on16(a.table, a.ld_table, type_size(table_type));
  if (table_type == TAB_FP32) return launch_lookup_t<float, -1>(a, out_type, vec, sm_count, st);
  if (table_type == TAB_BF16)
    return launch_lookup_t<__nv_bfloat16, -1>(a, out_type, vec, sm_count, st);
  return launch_lookup_t<__half, -1>(a, out_type, vec, sm_count, st);
}

// Sorted positions a range holds: 32, fewer where that would leave the SMs without
// two blocks each, more where a run through all ranges would make too many parts.
static int grad_range(int64_t n, int d, int sm_count) {
  const int ct = sum_threads(d);
  const int64_t groups = (d + ct * 8 - 1) / (ct * 8), per = kSumThreads / ct;
  if (n > 65536) return (int)(32 * ((n + 65535) / 65536));
  int range = 32;
  while (range > kSumBatch && (n + range - 1) / range * groups < 2 * sm_count * per) range /= 2;
  return range;
}

size_t grad_scratch_bytes(int64_t n, int d, int sm_count) {
  const int ct = sum_threads(d), range = grad_range(n, d, sm_count);
  const int64_t ranges = (n + range - 1) / range;
  const size_t list = ((size_t)n * 4 + 255) / 256 * 256;
  return 4 * list + (size_t)ranges * 2 * ((d + ct * 8 - 1) / (ct * 8) * ct * 8) * 4;
}

// At least what any call of up to n tokens and d columns takes: in ranges of fewer
// than 32 positions a call has at most 4 sm_count * 128 thread columns of partial
// sums, else at most 2048 ranges.
size_t grad_reserve_bytes(int64_t n, int64_t d, int sm_count) {
  const size_t list = ((size_t)n * 4 + 255) / 256 * 256;
  const size_t few = (size_t)sm_count * 4 * kSumThreads * 64;
  const int64_t ranges = n / 32 + 1 < 2048 ? n / 32 + 1 : 2048;
  const size_t many = (size_t)ranges * 2 * ((d + 1023) / 1024 * 1024) * 4;
  return 4 * list + (few > many ? few : many);
}

cudaError_t launch_table_grad(TableGrad a, int src_type, int out_type, void* scratch, int sm_count,
                              cudaStream_t st) {
  const int ct = sum_threads(a.d);
  a.groups = (a.d + ct * 8 - 1) / (ct * 8);
  a.range = grad_range(a.n, a.d, sm_count);
  a.ld_partial = (int64_t)a.groups * ct * 8;
  const size_t list = ((size_t)a.n * 4 + 255) / 256 * 256;
  char* at = static_cast<char*>(scratch);
  for (int i = 0; i < 2; ++i) {
    a.keys[i] = reinterpret_cast<int32_t*>(at);
    a.pos[i] = reinterpret_cast<int32_t*>(at + list);
    at += 2 * list;
  }
  a.partial = reinterpret_cast<float*>(at);
  if (a.n == 0)                 // (not accumulating: the table's gradient is zero)
    return launch_pdl(fill_kernel<true>, dim3((unsigned)(2 * sm_count)), dim3(kFillThreads), 0, st,
                      a, type_size(out_type));
  // a CTA for each tile of tokens, up to a portable cluster
  int parts = 1;
  while (parts < 8 && parts * kSortTile < a.n) parts *= 2;
  int bits = 0;
  while (((int64_t)1 << bits) <= a.V) ++bits;         // keys are 0 .. V
  cudaError_t e = cudaFuncSetAttribute(sort_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                       (int)sizeof(SortSmem));
  if (e != cudaSuccess) return e;
  e = launch_pdl_cluster(sort_kernel, dim3(parts), dim3(kSortThreads), sizeof(SortSmem), st, parts,
                         a, parts, (bits + kSortBits - 1) / kSortBits);
  if (e != cudaSuccess) return e;
  if (!a.add) {
    e = launch_pdl(fill_kernel<false>, dim3((unsigned)(2 * sm_count)), dim3(kFillThreads), 0, st, a,
                   type_size(out_type));
    if (e != cudaSuccess) return e;
  }
  const bool vec = on16(a.out, a.ld_out, type_size(out_type)) &&
                   on16(a.d_out, a.ld_d_out, type_size(src_type));
  if (src_type == TAB_FP32) return launch_sums_o<float>(a, ct, out_type, vec, st);
  if (src_type == TAB_BF16) return launch_sums_o<__nv_bfloat16>(a, ct, out_type, vec, st);
  return launch_sums_o<__half>(a, ct, out_type, vec, st);
}

}  // namespace sph
