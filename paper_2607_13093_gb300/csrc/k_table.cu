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

// A block takes one token and `turns` spans of kLookSpan columns, U of them requested
// together.
template <class TT, int FMT, class OT, bool VEC, int U>
__global__ void __launch_bounds__(kLookThreads) lookup_kernel(const Lookup a) {
  ptx::griddep_wait();
  ptx::griddep_launch_dependents();
  const int64_t t = blockIdx.x / a.blocks;
  const int first = (int)(blockIdx.x % a.blocks) * a.turns * kLookSpan +
                    (VEC ? (int)threadIdx.x * 8 : (int)threadIdx.x);
  const int64_t id = a.tokens ? a.tokens[t] : t;
  const bool there = id >= 0 && id < a.V;
  if (!there && id != a.padding && first == 0) atomicOr(a.status, ERR_BAD_INDEX);
  OT* out = static_cast<OT*>(a.out) + t * a.ld_out;
  for (int n = 0; n < a.turns; n += U) {
    float v[U][8];
#pragma unroll
    for (int i = 0; i < U; ++i) {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] = 0.f;
      const int col = first + (n + i) * kLookSpan;
      if (there && n + i < a.turns && col < a.d) table_cols<TT, FMT, VEC>(a, id, col, v[i]);
    }
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int col = first + (n + i) * kLookSpan;
      if (n + i >= a.turns || col >= a.d) break;
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] *= a.scale;
      store_cols<OT, VEC>(out, col, kLookThreads, a.d, v[i]);
    }
  }
}

template <class TT, int FMT, class OT, bool VEC>
cudaError_t launch_lookup_v(Lookup a, int sm_count, cudaStream_t st) {
  // one block a token once that gives every SM sixteen, else a block for each span
  const int spans = (a.d + kLookSpan - 1) / kLookSpan;
  a.turns = a.n >= (int64_t)sm_count * 16 ? spans : 1;
  a.blocks = (spans + a.turns - 1) / a.turns;
  const dim3 grid((unsigned)(a.n * a.blocks));
  if (a.turns > 1)
    return launch_pdl(lookup_kernel<TT, FMT, OT, VEC, 4>, grid, dim3(kLookThreads), 0, st, a);
  return launch_pdl(lookup_kernel<TT, FMT, OT, VEC, 1>, grid, dim3(kLookThreads), 0, st, a);
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
constexpr int kSortThreads = 512, kSortItems = 16, kSortTile = kSortThreads * kSortItems;
constexpr int kSortBits = 9, kSortBins = 1 << kSortBits, kSortWarps = kSortThreads / 32;

struct SortSmem {
  uint32_t hist[kSortBins];       // this CTA's count of each digit (read by the cluster)
  uint32_t base[kSortBins];       // where its next element of a digit goes
  uint32_t part[kSortWarps];
  uint16_t warp[kSortWarps][kSortBins];
  int32_t key[kSortTile];         // a sort of one tile stays here between passes
  int32_t pos[kSortTile];
};

// One cluster sorts: stable radix passes over (id, position) with digits of at most
// 9 bits, each CTA a contiguous part.  A warp's items are consecutive; equal
// digits within a warp are ranked by match.any, its warps by a prefix over their
// counts, the CTAs by one over theirs, read through distributed shared memory.
// Up to kSortTile tokens (one CTA) the passes stay in shared memory; parts of one
// tile get their counts from the ranking, longer ones from a pass of their own.
// Ids out of range become V, which sorts last.
__global__ void __launch_bounds__(kSortThreads) sort_kernel(const TableGrad a, int parts, int passes,
                                                            int bits) {
  extern __shared__ __align__(16) uint8_t sort_raw[];
  SortSmem& s = *reinterpret_cast<SortSmem*>(sort_raw);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int rank = (int)blockIdx.x;
  ptx::griddep_wait();
  ptx::griddep_launch_dependents();
  const int part = (a.n + parts - 1) / parts;
  const int p0 = min(a.n, rank * part), p1 = min(a.n, p0 + part);
  const bool one = part <= kSortTile, local = parts == 1 && one;
  const int bins = 1 << bits;
  for (int pass = 0; pass < passes; ++pass) {
    const int shift = pass * bits;
    // passes end in buffer 0: the last one writes it
    const int to = (passes - 1 - pass) & 1;
    const bool last = pass == passes - 1;
    auto key_of = [&](int i) {
      if (pass > 0) return local ? s.key[i] : __ldcg(a.keys[to ^ 1] + i);
      const int32_t id = a.tokens[i];
      return id >= 0 && id < a.V ? id : a.V;
    };
    auto digit = [&](int32_t k) { return (int)((uint32_t)k >> shift) & (bins - 1); };
    // Where each digit's elements of this CTA start, from its own counts (thread b:
    // digit b).
    auto place = [&](uint32_t mine) {
      uint32_t total = mine, below = 0;
      if (parts > 1) {
        s.hist[tid] = mine;
        ptx::cluster_sync();
        total = 0;
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
      if (lane == 31) s.part[warp] = incl;
      __syncthreads();
      uint32_t before = 0;
      for (int w = 0; w < warp; ++w) before += s.part[w];
      s.base[tid] = before + incl - total + below;
      __syncthreads();
    };
    if (!one) {
      s.base[tid] = 0;
      __syncthreads();
      for (int i = p0 + tid; i < p1; i += kSortThreads) atomicAdd(&s.base[digit(key_of(i))], 1u);
      __syncthreads();
      const uint32_t mine = s.base[tid];
      __syncthreads();
      place(mine);
    }
    for (int t0 = p0; t0 < p1 || (one && t0 == p0); t0 += kSortTile) {
      // items of a thread: enough for the tile, so that short lists take few rounds
      const int count = min(kSortTile, p1 - t0), rounds = (count + kSortThreads - 1) / kSortThreads;
      int32_t k[kSortItems], p[kSortItems];
      uint32_t r[kSortItems];
      const int first = t0 + warp * 32 * rounds + lane;
#pragma unroll
      for (int i = 0; i < kSortItems; ++i) {
        if (i >= rounds) break;
        const int at = first + i * 32;
        const bool in = at < t0 + count;
        k[i] = in ? key_of(at) : 0;
        p[i] = !in ? -1 : pass == 0 ? at : local ? s.pos[at] : __ldcg(a.pos[to ^ 1] + at);
        if (pass == 0 && in && k[i] == a.V && a.tokens[at] != a.padding)
          atomicOr(a.status, ERR_BAD_INDEX);
      }
      for (int b = lane; b < bins / 2; b += 32) reinterpret_cast<uint32_t*>(s.warp[warp])[b] = 0;
      __syncwarp();
#pragma unroll
      for (int i = 0; i < kSortItems; ++i) {
        if (i >= rounds) break;
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
      uint32_t run = 0;
      if (tid < bins) {
#pragma unroll
        for (int w = 0; w < kSortWarps; ++w) {
          const uint32_t c = s.warp[w][tid];
          s.warp[w][tid] = (uint16_t)run;
          run += c;
        }
      }
      if (one) place(run);
      else __syncthreads();
#pragma unroll
      for (int i = 0; i < kSortItems; ++i) {
        if (i >= rounds) break;
        if (p[i] >= 0) {
          const int dg = digit(k[i]);
          const uint32_t at = s.base[dg] + s.warp[warp][dg] + r[i];
          if (local && !last) {
            s.key[at] = k[i];
            s.pos[at] = p[i];
          } else {
            a.keys[to][at] = k[i];
            a.pos[to][at] = p[i];
          }
        }
      }
      __syncthreads();
      if (!one) {
        s.base[tid] += run;
        __syncthreads();
      }
    }
    // the pass's writes reach the cluster's other CTAs, and none still reads
    // this one's counts when the next pass writes them
    if (parts > 1) ptx::cluster_sync();
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
constexpr int kSumBytes = 256;      // shared memory of a thread: rows requested ahead
constexpr int kShortRun = 32;       // positions of a run that one range takes whole

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

// The part of a run of equal ids around the boundary before position `at` (whose key
// `id` is also that of at - 1): its start and end, exact for runs of at most
// kShortRun positions; longer ones give more than kShortRun.
__device__ __forceinline__ void run_around(const int32_t* keys, int n, int at, int32_t id, int* s,
                                           int* e) {
  int b = at - 1, f = at + 1;
  while (b > 0 && at - b <= kShortRun && keys[b - 1] == id) --b;
  while (f < n && f - b <= kShortRun && keys[f] == id) ++f;
  *s = b;
  *e = f;
}

// ct threads a range of a.range sorted positions and 8 ct columns (128 / ct
// ranges a block).  A run of equal ids of at most kShortRun positions is summed by
// the range that it begins in and written out; of a longer one each range sums its
// own part, into slot 2 r of the partial sums where the run began earlier, into
// slot 2 r + 1 where it begins in the range and goes on (written out where it
// does neither).  A thread's columns of the next rows are on their way to its own
// piece of shared memory while it adds: nothing is shared between threads.  (With
// rows in registers the code for a run's end stood once for each of them:
// 32768 rows x 4096 bf16 159 us.)
template <class T, class OT, bool VEC>
__global__ void __launch_bounds__(kSumThreads) sum_kernel(const TableGrad a, int ct) {
  __shared__ uint4 s_rows[kSumBytes / 16][kSumThreads];
  ptx::griddep_wait();
  ptx::griddep_launch_dependents();
  const int u = threadIdx.x % ct;
  const int group = (int)(blockIdx.x % a.groups);
  const int64_t r = (int64_t)(blockIdx.x / a.groups) * (kSumThreads / ct) + threadIdx.x / ct;
  const int col = sum_col<VEC>(group, u, ct);
  if (r * a.range >= a.n || col >= a.d) return;
  const int i0 = (int)(r * a.range), i1 = min(a.n, i0 + a.range);
  const int32_t* keys = a.keys[0];
  const int32_t* pos = a.pos[0];
  int begin = i0, end = i1;
  bool open_left = false, open_right = false;
  if (i0 > 0 && keys[i0 - 1] == keys[i0]) {
    int s, e;
    run_around(keys, a.n, i0, keys[i0], &s, &e);
    if (e - s > kShortRun) open_left = true;
    else begin = e;
  }
  if (begin >= i1) return;
  if (i1 < a.n && keys[i1 - 1] == keys[i1]) {
    int s, e;
    run_around(keys, a.n, i1, keys[i1], &s, &e);
    if (e - s > kShortRun) open_right = true;
    else end = e;
  }
  float acc[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) acc[j] = 0.f;
  int32_t cur = keys[begin];
  auto flush = [&](bool right) {
    if (!open_left && !right) {
      write_row<OT, VEC>(a, cur, col, ct, acc);
    } else {
      float* p = a.partial + (2 * r + (open_left ? 0 : 1)) * a.ld_partial + group * ct * 8 + u * 8;
      reinterpret_cast<float4*>(p)[0] = make_float4(acc[0], acc[1], acc[2], acc[3]);
      reinterpret_cast<float4*>(p)[1] = make_float4(acc[4], acc[5], acc[6], acc[7]);
    }
  };
  auto add = [&](int32_t k, const float (&x)[8]) {
    if (k != cur) {
      flush(false);
      cur = k;
      open_left = false;
#pragma unroll
      for (int j = 0; j < 8; ++j) acc[j] = 0.f;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[j] += x[j];
  };
  // (ids without a row of their own sort last)
  while (end > begin && keys[end - 1] == a.V) {
    // a whole range of them, or its tail: they end the list, so halve towards the first
    int lo = begin, hi = end - 1;
    while (lo < hi) {
      const int mid = (lo + hi) / 2;
      if (keys[mid] == a.V) hi = mid;
      else lo = mid + 1;
    }
    end = lo;
    open_right = false;
  }
  if (end == begin) return;
  auto row_of = [&](int i) { return static_cast<const T*>(a.d_out) + (int64_t)pos[i] * a.ld_d_out; };
  if constexpr (VEC) {
    constexpr int kPieces = (int)sizeof(T) / 2, kAhead = kSumBytes / 16 / kPieces;
    auto request = [&](int i) {
      if (i < end) {
        const T* row = row_of(i) + col;
        const int slot = (i - begin) % kAhead * kPieces;
#pragma unroll
        for (int q = 0; q < kPieces; ++q) {
          // columns past the row's last are zeros, and not read
          const int bytes = min(16, max(0, (a.d - col) * (int)sizeof(T) - 16 * q));
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(
                           ptx::smem_u32(&s_rows[slot + q][threadIdx.x])),
                       "l"(bytes > 0 ? reinterpret_cast<const uint4*>(row) + q
                                     : reinterpret_cast<const uint4*>(row)),
                       "r"(bytes)
                       : "memory");
        }
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int i = 0; i < kAhead - 1; ++i) request(begin + i);
    for (int i = begin; i < end; ++i) {
      request(i + kAhead - 1);
      asm volatile("cp.async.wait_group %0;" ::"n"(kAhead - 1) : "memory");
      uint4 w[kPieces];
#pragma unroll
      for (int q = 0; q < kPieces; ++q)
        w[q] = s_rows[(i - begin) % kAhead * kPieces + q][threadIdx.x];
      const T* e = reinterpret_cast<const T*>(w);
      float x[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = to_f32(e[j]);
      add(keys[i], x);
    }
  } else {
    constexpr int kAhead = kSumBytes / 32;
    for (int b = begin; b < end; b += kAhead) {
      const int m = min(kAhead, end - b);
#pragma unroll
      for (int h = 0; h < kAhead; h += 4) {
        float x[4][8];
#pragma unroll
        for (int q = 0; q < 4; ++q)
          if (h + q < m) load_cols<T, false>(row_of(b + h + q), col, ct, a.d, x[q]);
#pragma unroll
        for (int q = 0; q < 4; ++q)
          if (h + q < m) {
            s_rows[2 * (h + q)][threadIdx.x] = *reinterpret_cast<const uint4*>(&x[q][0]);
            s_rows[2 * (h + q) + 1][threadIdx.x] = *reinterpret_cast<const uint4*>(&x[q][4]);
          }
      }
      for (int q = 0; q < m; ++q) {
        const uint4 lo = s_rows[2 * q][threadIdx.x], hi = s_rows[2 * q + 1][threadIdx.x];
        const float x[8] = {__uint_as_float(lo.x), __uint_as_float(lo.y), __uint_as_float(lo.z),
                            __uint_as_float(lo.w), __uint_as_float(hi.x), __uint_as_float(hi.y),
                            __uint_as_float(hi.z), __uint_as_float(hi.w)};
        add(keys[b + q], x);
      }
    }
  }
  flush(open_right);
}

constexpr int kJoinThreads = 256;

// A block for each range and column group; it goes on only where a run of more than
// kShortRun positions begins in the range and crosses its end.  The run's parts (slot 2 r + 1, then slot 2 j of
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
  // a run is longer than kShortRun just if more than that many of the kShortRun
  // positions on either side of a boundary in it are its own
  const int64_t near = i1 - kShortRun + threadIdx.x;
  if (__syncthreads_count(threadIdx.x < 2 * kShortRun && near >= 0 && near < a.n &&
                          keys[near] == id) <= kShortRun)
    return;
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
  while (range > 8 && (n + range - 1) / range * groups < 2 * sm_count * per) range /= 2;
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
  // one CTA sorts a tile of tokens; longer lists take a portable cluster
  const int parts = a.n <= kSortTile ? 1 : 8;
  int bits = 1;
  while (((int64_t)1 << bits) <= a.V) ++bits;         // keys are 0 .. V
  const int passes = (bits + kSortBits - 1) / kSortBits;
  cudaError_t e = cudaFuncSetAttribute(sort_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                       (int)sizeof(SortSmem));
  if (e != cudaSuccess) return e;
  e = launch_pdl_cluster(sort_kernel, dim3(parts), dim3(kSortThreads), sizeof(SortSmem), st, parts,
                         a, parts, passes, (bits + passes - 1) / passes);
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
