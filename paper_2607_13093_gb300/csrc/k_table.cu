// Rows of a vocabulary table by token, and the table's gradient from them.
//
//   lookup    out[t, :] = scale * W[token_t, :]
//   gradient  dW[v, :] (+)= scale * sum over {t : token_t = v} of dOut[t, :]
//
// Both are bound by memory.  The gradient sorts the token positions by id
// (stable, so equal inputs give equal bits), sums runs of equal ids over ranges
// of sorted positions of one length, whatever the runs' lengths, and joins the
// parts of a run that crosses ranges, in order.  Rows of ids that no token has
// are zeroed beside the sort.
//
// Measured: lookup of 16384 rows x 5120 of 4 bits into bf16 32.9 us (5.7 TB/s), of 32 x 4096
// bf16 1.9 us; gradient of 32768 rows into 128256 x 4096 bf16 229 us (5.6 TB/s), of 500 into
// 32000 x 4096 fp32 95 us (5.6 TB/s), of 8000 onto 151643 x 3584 fp32 52 us (of which sort 14,
// sums 26 and joins 12).
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "mx4.cuh"
#include "rows.cuh"
#include "sm100_ptx.cuh"
#include "sph_internal.h"

namespace sph {
namespace {

// ---------------------------------------------------------------------------
// lookup
// ---------------------------------------------------------------------------
constexpr int kLookThreads = 128;
constexpr int kLookSpan = kLookThreads * 8;    // columns of a block

struct Mx4Row;     // tag of a table held in 4 bits (FMT says which)

// A thread's eight columns of a table row as they lie in memory, and their values.
// VEC: rows of table and output, and so col, are on 16 bytes.
template <class TT, int FMT, bool VEC>
struct Piece {           // dense rows
  float v[8];
  __device__ __forceinline__ void load(const Lookup& a, int64_t id, int col) {
    load_cols<TT, VEC>(static_cast<const TT*>(a.table) + id * a.ld_table, col, a.d, v);
  }
  __device__ __forceinline__ void values(float, float (&x)[8]) const {
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = v[j];
  }
};
template <int FMT>
struct Piece<Mx4Row, FMT, true> {      // in 4 bits
  uint32_t codes;
  uint8_t scale;
  __device__ __forceinline__ void load(const Lookup& a, int64_t id, int col) {
    codes = *reinterpret_cast<const uint32_t*>(static_cast<const uint8_t*>(a.table) +
                                               id * a.ld_table + col / 2);
    scale = a.scales[id * a.ld_scales + col / Mx4<FMT>::kBlock];
  }
  __device__ __forceinline__ void values(float row, float (&x)[8]) const {
    e2m1x8_to_float(codes, x);
    const float s = mx4_scale_value<FMT>(scale) * row;
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] *= s;
  }
};
template <int FMT>
struct Piece<Mx4Row, FMT, false> {     // columns of two words, and of two blocks
  uint32_t codes;
  uint8_t scale, next;
  int left;                            // columns of the first block
  __device__ __forceinline__ void load(const Lookup& a, int64_t id, int col) {
    constexpr int B = Mx4<FMT>::kBlock;
    const uint32_t* c = reinterpret_cast<const uint32_t*>(static_cast<const uint8_t*>(a.table) +
                                                          id * a.ld_table);
    const uint8_t* s = a.scales + id * a.ld_scales;
    const int from = max(col, 0), i = from / 8;
    const uint32_t hi = from % 8 && 8 * i + 8 < a.d ? c[i + 1] : 0u;
    codes = __funnelshift_r(c[i], hi, from % 8 * 4) << 4 * (from - col);
    scale = s[from / B];
    next = s[min(col + 7, a.d - 1) / B];
    left = B - (col & (B - 1));        // (col < 0: no more than -col, so all are the next's)
  }
  __device__ __forceinline__ void values(float row, float (&x)[8]) const {
    e2m1x8_to_float(codes, x);
    const float s = mx4_scale_value<FMT>(scale) * row, t = mx4_scale_value<FMT>(next) * row;
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] *= j < left ? s : t;
  }
};

// A block takes one token and `turns` spans of kLookSpan columns, U of them requested
// together.
template <class TT, int FMT, class OT, bool VEC, int U>
__global__ void __launch_bounds__(kLookThreads) lookup_kernel(const Lookup a) {
  ptx::griddep_wait();
  ptx::griddep_launch_dependents();
  const int64_t t = blockIdx.x / a.blocks;
  const int span = (int)(blockIdx.x % a.blocks) * a.turns;
  const int64_t id = a.tokens ? a.tokens[t] : t;
  const bool there = id >= 0 && id < a.V && id != a.padding;
  if (!there && id != a.padding && span == 0 && threadIdx.x == 0) atomicOr(a.status, ERR_BAD_INDEX);
  const float row = FMT == MX4_E4M3 && there ? a.row_scale[id] : 1.f;
  OT* out = static_cast<OT*>(a.out) + t * a.ld_out;
  // the first piece ends at the output row's first 16-byte boundary, so that the others
  // are stored in 16-byte words (element by element, us: 16384 x 5119 bf16 171, from e4m3
  // 121; 32000 x 4095 from e4m3 176)
  const int head = VEC ? 0 : (int)(-(intptr_t)out & 15) / (int)sizeof(OT);
  const int first = span * kLookSpan + (int)threadIdx.x * 8 + (head ? head - 8 : 0);
  for (int n = 0; n < a.turns; n += U) {
    Piece<TT, FMT, VEC> piece[U];
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int col = first + (n + i) * kLookSpan;
      if (there && n + i < a.turns && col < a.d) piece[i].load(a, id, col);
    }
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int col = first + (n + i) * kLookSpan;
      if (n + i >= a.turns || col >= a.d) break;
      float v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = 0.f;
      if (there) {
        piece[i].values(row, v);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] *= a.scale;
      }
      store_cols<OT, true>(out, col, a.d, v);
    }
  }
}

template <class TT, int FMT, class OT, bool VEC>
cudaError_t launch_lookup_v(Lookup a, int sm_count, cudaStream_t st) {
  // One block a token once that gives every SM two, else a block for each span
  // (a block a token / a span, us, into bf16: 32 tokens x 5120 from e4m3 2.8 / 2.4, 500
  // 3.5 / 4.1, 1200 4.5 / 7.4; 32 x 4096 from bf16 3.1 / 2.5, 500 3.7 / 3.6, 1200 4.6 / 6.2).
  const int spans = (a.d + (VEC ? 0 : 7) + kLookSpan - 1) / kLookSpan;
  a.turns = a.n >= (int64_t)sm_count * 2 ? spans : 1;
  a.blocks = (spans + a.turns - 1) / a.turns;
  const dim3 grid((unsigned)(a.n * a.blocks));
  if (a.turns > 4 && FMT >= 0)          // (4-bit pieces are two registers each)
    return launch_pdl(lookup_kernel<TT, FMT, OT, VEC, FMT >= 0 && VEC ? 8 : 4>, grid,
                      dim3(kLookThreads), 0, st, a);
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

// ---------------------------------------------------------------------------
// gradient: the sort
// ---------------------------------------------------------------------------
constexpr int kSortThreads = 1024, kSortItems = 8, kSortTile = kSortThreads * kSortItems;
constexpr int kSortShort = 2048;      // tokens that one CTA sorts
constexpr int kSortBits = 9, kSortBins = 1 << kSortBits, kSortWarps = kSortThreads / 32;

struct SortSmem {
  uint32_t hist[kSortBins];       // this CTA's count of each digit, read by the cluster: written
                                  // once a pass, after the barrier that ended the one before
  uint32_t base[kSortBins];       // where its next element of a digit goes
  uint32_t local[kSortBins];      // the same within the current tile
  uint32_t half[kSortBins];       // counts of the first half of the warps, then of the second
  uint32_t part[kSortWarps];
  uint16_t warp[kSortWarps][kSortBins];
  int32_t key[kSortTile];         // the tile in the order of its digits
  int32_t pos[kSortTile];
};

// One cluster sorts: stable radix passes over (id, position) with digits of at most
// 9 bits, each CTA a contiguous part.  A warp's items are consecutive; equal digits
// within a warp are ranked by votes, its warps by a prefix over their counts, the CTAs
// by one over theirs, read through distributed shared memory.
// A tile is put in order in shared memory first and written from there, a digit's
// elements side by side (one by one from the ranking, 8000 tokens took 24 us).  Up
// to kSortTile tokens (one CTA) the passes stay in shared memory; parts of one tile
// get their counts from the ranking, longer ones from a pass of their own.
// The padding id and ids out of range become V, which sorts last.
// FIRST: the call's first kernel.  Else it runs beside the one that zeroes rows, and
// waits for that only at its end, so that the kernel after it may take both as done.
template <bool FIRST>
__global__ void __launch_bounds__(kSortThreads) sort_kernel(const TableGrad a, int parts, int passes,
                                                            int bits) {
  extern __shared__ __align__(16) uint8_t sort_raw[];
  SortSmem& s = *reinterpret_cast<SortSmem*>(sort_raw);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int rank = (int)blockIdx.x;
  if constexpr (FIRST) ptx::griddep_wait();
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
      if (pass > 0) return __ldcg(a.keys[to ^ 1] + i);
      const int32_t id = a.tokens[i];
      return id >= 0 && id < a.V && id != a.padding ? id : a.V;
    };
    auto digit = [&](int32_t k) { return (int)((uint32_t)k >> shift) & (bins - 1); };
    // exclusive sum over the block's threads (thread b: digit b)
    auto sum_before = [&](uint32_t v) {
      uint32_t incl = v;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint32_t up = __shfl_up_sync(0xFFFFFFFFu, incl, o);
        if (lane >= o) incl += up;
      }
      __syncthreads();             // (of s.part, read the last time)
      if (lane == 31) s.part[warp] = incl;
      __syncthreads();
      uint32_t w = lane < warp ? s.part[lane] : 0;
      w = __reduce_add_sync(0xFFFFFFFFu, w);
      return w + incl - v;
    };
    // where each digit's elements of this CTA start, from its own counts
    auto place = [&](uint32_t mine) {
      uint32_t total = mine, below = 0;
      if (parts > 1) {
        if (tid < kSortBins) s.hist[tid] = mine;
        ptx::cluster_sync();
        total = 0;
        if (tid < kSortBins) {
          uint32_t h[8];
#pragma unroll
          for (int c = 0; c < 8; ++c) {
            h[c] = 0;
            if (c < parts)
              asm volatile("ld.shared::cluster.u32 %0, [%1];"
                           : "=r"(h[c])
                           : "r"(ptx::mapa(ptx::smem_u32(&s.hist[tid]), (uint32_t)c))
                           : "memory");
          }
#pragma unroll
          for (int c = 0; c < 8; ++c) {
            if (c < rank) below += h[c];
            total += h[c];
          }
        }
      }
      const uint32_t at = sum_before(total) + below;
      if (tid < kSortBins) s.base[tid] = at;
      __syncthreads();
    };
    if (!one) {
      if (tid < kSortBins) s.base[tid] = 0;
      __syncthreads();
      for (int i = p0 + tid; i < p1; i += kSortThreads) atomicAdd(&s.base[digit(key_of(i))], 1u);
      __syncthreads();
      const uint32_t mine = tid < kSortBins ? s.base[tid] : 0;
      __syncthreads();
      place(mine);
    }
    for (int t0 = p0; t0 < p1 || (one && t0 == p0); t0 += kSortTile) {
      // items of a thread: enough for the tile, so that short lists take few rounds
      const int count = min(kSortTile, p1 - t0), rounds = (count + kSortThreads - 1) / kSortThreads;
      int32_t k[kSortItems], p[kSortItems];
      uint32_t r[kSortItems];
      const int first = t0 + warp * 32 * rounds + lane, stop = t0 + count;
      // (no early end here: the loads of all rounds go out together)
#pragma unroll
      for (int i = 0; i < kSortItems; ++i) {
        const int at = first + i * 32;
        const bool in = i < rounds && at < stop;
        if (pass == 0) {
          k[i] = in ? a.tokens[at] : 0;
          p[i] = in ? at : -1;
        } else if (local) {
          k[i] = in ? s.key[at] : 0;
          p[i] = in ? s.pos[at] : -1;
        } else {
          k[i] = in ? __ldcg(a.keys[to ^ 1] + at) : 0;
          p[i] = in ? __ldcg(a.pos[to ^ 1] + at) : -1;
        }
      }
      if (pass == 0) {
#pragma unroll
        for (int i = 0; i < kSortItems; ++i) {
          const bool out = k[i] < 0 || k[i] >= a.V || k[i] == a.padding;
          if (out && k[i] != a.padding && p[i] >= 0) atomicOr(a.status, ERR_BAD_INDEX);
          if (out) k[i] = a.V;
        }
      }
      for (int b = lane; b < bins / 2; b += 32) reinterpret_cast<uint32_t*>(s.warp[warp])[b] = 0;
      __syncwarp();
#pragma unroll
      for (int i = 0; i < kSortItems; ++i) {
        if (i >= rounds) break;
        const unsigned live = __ballot_sync(0xFFFFFFFFu, p[i] >= 0);
        const int dg = digit(k[i]);
        // lanes with this lane's digit, a vote a bit (match.any is several times slower)
        unsigned same = live;
#pragma unroll
        for (int b = 0; b < kSortBits; ++b) {
          const unsigned ones = __ballot_sync(0xFFFFFFFFu, dg >> b & 1);
          same &= dg >> b & 1 ? ones : ~ones;
        }
        if (p[i] >= 0) {
          const uint32_t had = s.warp[warp][dg];
          r[i] = had + __popc(same & ((1u << lane) - 1));
          __syncwarp(live);
          if ((same & ((1u << lane) - 1)) == 0) s.warp[warp][dg] = (uint16_t)(had + __popc(same));
        }
        __syncwarp();
      }
      __syncthreads();
      // each warp's first place in a digit, and the digit's count (thread b < kSortBins:
      // digit b), two threads a digit
      const int dig = tid % kSortBins, w0 = tid / kSortBins * (kSortWarps / 2);
      uint32_t c[kSortWarps / 2], run = 0;
#pragma unroll
      for (int w = 0; w < kSortWarps / 2; ++w) {
        c[w] = dig < bins ? s.warp[w0 + w][dig] : 0;
        run += c[w];
      }
      if (w0 == 0) s.half[dig] = run;
      __syncthreads();
      uint32_t up = w0 ? s.half[dig] : 0;
      const uint32_t mine = run;
      if (dig < bins) {
#pragma unroll
        for (int w = 0; w < kSortWarps / 2; ++w) {
          s.warp[w0 + w][dig] = (uint16_t)up;
          up += c[w];
        }
      }
      if (w0) s.half[dig] = mine;        // (its only reader so far)
      __syncthreads();
      run = w0 ? 0 : run + s.half[dig];
      if (one && !local) place(run);
      const uint32_t local_at = sum_before(run);
      if (tid < kSortBins) s.local[tid] = local_at;
      __syncthreads();
#pragma unroll
      for (int i = 0; i < kSortItems; ++i) {
        if (i >= rounds) break;
        if (p[i] >= 0) {
          const int dg = digit(k[i]);
          const uint32_t at = s.local[dg] + s.warp[warp][dg] + r[i];
          s.key[at] = k[i];
          s.pos[at] = p[i];
        }
      }
      __syncthreads();
      if (!local || last) {
        for (int i = tid; i < count; i += kSortThreads) {
          const int32_t key = s.key[i];
          const int dg = digit(key);
          const uint32_t at = local ? (uint32_t)i : s.base[dg] + (uint32_t)i - s.local[dg];
          a.keys[to][at] = key;
          a.pos[to][at] = s.pos[i];
        }
        __syncthreads();
      }
      if (!one) {
        if (tid < kSortBins) s.base[tid] += run;
        __syncthreads();
      }
    }
    // the pass's writes reach the cluster's other CTAs, and none still reads
    // this one's counts when the next pass writes them
    if (parts > 1) ptx::cluster_sync();
  }
  if (rank == 0 && tid == 0) a.pos[1][0] = 0;      // (free by now) the count of joins
  if constexpr (!FIRST) ptx::griddep_wait();
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

// Block `b` of `blocks` zeroes the rows of its share of the ids 0 .. V - 1 that
// no token has: it marks the ones that occur from the whole token list (a read of
// the L2, once per kFillIds ids), so nothing is written twice.
__device__ __forceinline__ void zero_rows(const TableGrad& a, int b,
                                          int blocks, int elem, uint32_t* s_seen) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t v0 = (int64_t)a.V * b / blocks;
  const int64_t v1 = (int64_t)a.V * (b + 1) / blocks;
  auto mark = [&](int32_t token, int64_t base, int ids) {
    const int64_t r = (int64_t)token - base;
    if (r >= 0 && r < ids && token != a.padding) atomicOr(&s_seen[r >> 5], 1u << (r & 31));
  };
  // (tokens on 16 bytes: four to a load, and four loads on their way)
  const int quads = ((uintptr_t)a.tokens & 15) == 0 ? a.n / 4 : 0;
  for (int64_t base = v0; base < v1; base += kFillIds) {
    const int ids = (int)min((int64_t)kFillIds, v1 - base);
    for (int i = threadIdx.x; i < kFillIds / 32; i += kFillThreads) s_seen[i] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < quads; i += 4 * kFillThreads) {
      int4 t[4];
#pragma unroll
      for (int q = 0; q < 4; ++q)
        t[q] = i + q * kFillThreads < quads
                   ? reinterpret_cast<const int4*>(a.tokens)[i + q * kFillThreads]
                   : make_int4(-1, -1, -1, -1);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        mark(t[q].x, base, ids);
        mark(t[q].y, base, ids);
        mark(t[q].z, base, ids);
        mark(t[q].w, base, ids);
      }
    }
    for (int i = 4 * quads + threadIdx.x; i < a.n; i += kFillThreads) mark(a.tokens[i], base, ids);
    __syncthreads();
    for (int r = warp; r < ids; r += kFillThreads / 32)
      if (!(s_seen[r >> 5] >> (r & 31) & 1))
        zero_bytes(static_cast<uint8_t*>(a.out) + (base + r) * a.ld_out * elem,
                   (int64_t)a.d * elem, lane);
    __syncthreads();
  }
}

// The call's first kernel where it zeroes rows; the sort runs beside it.  (All rows
// here / 96 MB of them here and the rest beside the joins, us: 32768 tokens into 128256
// x 4096 bf16 228 / 238, 4000 172 / 176; 500 into 32000 x 4096 fp32 91.5 / 90.2.)
__global__ void __launch_bounds__(kFillThreads) head_kernel(const TableGrad a, int elem) {
  __shared__ uint32_t s_seen[kFillIds / 32];
  ptx::griddep_wait();
  ptx::griddep_launch_dependents();
  zero_rows(a, (int)blockIdx.x, (int)gridDim.x, elem, s_seen);
}

// ---------------------------------------------------------------------------
// gradient: sums over ranges of sorted positions, and the join
// ---------------------------------------------------------------------------
constexpr int kSumThreads = 128, kJoinThreads = 512;
constexpr int kSumBytes = 256;      // shared memory of a thread: rows requested ahead
constexpr int kShortRun = 16;       // (at most 32) positions of a run that one range takes whole

// First column of thread `u` of `ct` in column group g.
__device__ __forceinline__ int sum_col(int g, int u, int ct) { return (g * ct + u) * 8; }

// A row of any address, each lane of a warp having eight columns of it, one lane's after
// the other's: lanes store the 16-byte words in which their columns begin, with the
// neighbour's last ones; the first and the last lane what is left, by elements.  For
// whole warps.
template <class OT>
__device__ __forceinline__ void store_shifted(OT* row, int col, int d, const float (&v)[8]) {
  constexpr int N = 2 * (int)sizeof(OT);
  const int lane = threadIdx.x & 31, off = (int)((uintptr_t)(row + col) & 15);
  const int extra = off / (int)sizeof(OT);       // columns of the neighbour
  OT own[8];
  uint32_t x[N + 4];
#pragma unroll
  for (int j = 0; j < 8; ++j) own[j] = from_f32<OT>(v[j]);
  memcpy(x + 4, own, sizeof(own));
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = __shfl_up_sync(0xFFFFFFFFu, x[N + i], 1);
  if (off == 0) {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = x[i + 4];
  } else {
    shift_words<N, sizeof(OT)>(x, 16 - off);
  }
  const int first = col - extra;
  if ((lane > 0 || extra == 0) && first + 8 <= d) {
#pragma unroll
    for (int i = 0; i < N / 4; ++i)
      reinterpret_cast<uint4*>(row + first)[i] =
          make_uint4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]);
  } else {
    const OT* e = reinterpret_cast<const OT*>(x);
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if ((lane > 0 || j >= extra) && first + j < d) row[first + j] = e[j];
  }
  if (lane == 31) {
#pragma unroll
    for (int j = 1; j < 8; ++j)
      if (j >= 8 - extra && col + j < d) row[col + j] = own[j];
  }
}

// (for whole warps)
template <class OT, bool VEC>
__device__ __forceinline__ void write_row(const TableGrad& a, int32_t id, int col,
                                          const float (&sum)[8], const float (&onto)[8]) {
  float v[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = onto[j] + a.scale * sum[j];
  OT* row = static_cast<OT*>(a.out) + (int64_t)id * a.ld_out;
  if constexpr (!VEC) store_shifted<OT>(row, col, a.d, v);
  else if (col < a.d) store_cols<OT, true>(row, col, a.d, v);
}

// ct threads (whole warps) a range of a.range sorted positions and 8 ct columns, 128 /
// ct ranges a block.  A run of equal ids of at most kShortRun positions is summed by
// the range that it begins in and written out; of a longer one each range sums its
// own part, into slot 2 r of the partial sums where the run began earlier, into
// slot 2 r + 1 where it begins in the range and goes on (written out where it does
// neither).  Lanes hold the ids and positions of 32 sorted places each; the words that
// hold a thread's columns of the next rows are on their way to its own piece of shared
// memory while it adds, and nothing is shared between threads.  ADD: so is what the
// table holds for a run, requested with its first row (read at the run's end, it made
// each run wait for memory: 8000 rows x 3584 41 us).  Rows off 16 bytes are shifted into
// place as they are taken, and back as they are stored (element by element: 32768 x 4095
// bf16, the whole call, 541 us; so 289, and 229 for 4096).  (With rows in registers the code for a
// run's end stood once for each of them: 32768 rows x 4096 bf16 159 us.)
template <class T, class OT, bool VEC, bool ADD>
__global__ void __launch_bounds__(kSumThreads) sum_kernel(const TableGrad a, int ct) {
  // 16-byte words a slot: the row's, then the table's (not VEC: those that hold the
  // thread's columns)
  constexpr int kPieces = (int)sizeof(T) / 2 + !VEC;
  constexpr int kOnto = ADD ? (int)sizeof(OT) / 2 + !VEC : 0;
  constexpr int kFit = kSumBytes / 16 / (kPieces + kOnto);
  constexpr int kAhead = kFit >= 16 ? 16 : kFit >= 8 ? 8 : 4;
  __shared__ uint4 s_rows[kAhead * (kPieces + kOnto)][kSumThreads];
  ptx::griddep_wait();
  ptx::griddep_launch_dependents();
  const int u = threadIdx.x % ct, lane = threadIdx.x & 31;
  const int group = (int)(blockIdx.x % a.groups);
  const int64_t r = (int64_t)(blockIdx.x / a.groups) * (kSumThreads / ct) + threadIdx.x / ct;
  if (r * a.range >= a.n) return;
  const int col = sum_col(group, u, ct);
  const bool active = col < a.d;
  const int i0 = (int)(r * a.range), i1 = min(a.n, i0 + a.range);
  const int32_t* keys = a.keys[0];
  const int32_t* pos = a.pos[0];
  auto window = [&](const int32_t* list, int from) {       // 32 places from `from`, -1 outside
    const int at = from + lane;
    return at >= 0 && at < a.n ? list[at] : -1;
  };
  auto matches = [&](int32_t w, int32_t id) { return __popc(__ballot_sync(0xFFFFFFFFu, w == id)); };
  const int32_t before = window(keys, i0 - 32), first = window(keys, i0);
  const int32_t tail = window(keys, i1 - 32), after = window(keys, i1);
  int begin = i0, end = i1;
  bool open_left = false, open_right = false;
  const int32_t id0 = __shfl_sync(0xFFFFFFFFu, first, 0);
  const int32_t id1 = __shfl_sync(0xFFFFFFFFu, tail, 31);
  // (a run's places are neighbours, so its length around a boundary is the count of
  // its id on both sides, exact up to 32)
  if (__shfl_sync(0xFFFFFFFFu, before, 31) == id0) {
    const int f = matches(first, id0);
    if (matches(before, id0) + f > kShortRun) open_left = true;
    else begin = i0 + f;
  }
  if (begin >= i1) return;
  if (__shfl_sync(0xFFFFFFFFu, after, 0) == id1) {
    const int f = matches(after, id1);
    if (matches(tail, id1) + f > kShortRun) open_right = true;
    else end = i1 + f;
  }
  if (id1 == a.V) {        // tokens without a row sort last: none of them, from the first on
    int lo = begin;
    while (lo < end) {
      const int mid = (lo + end) / 2;
      if (keys[mid] == a.V) end = mid;
      else lo = mid + 1;
    }
    open_right = false;
    if (end == begin) return;
  }
  float acc[8], onto[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) acc[j] = onto[j] = 0.f;
  int32_t key = window(keys, begin), at = window(pos, begin);
  int32_t next_key = window(keys, begin + 32), next_at = window(pos, begin + 32);
  int32_t cur = __shfl_sync(0xFFFFFFFFu, key, 0);
  auto flush = [&](bool right) {
    if (!open_left && !right) {
      write_row<OT, VEC>(a, cur, col, acc, onto);
    } else if (active) {
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
  // row of the place `q` after the window's first (less than 64)
  auto row_of = [&](int q) {
    const int32_t t = __shfl_sync(0xFFFFFFFFu, q < 32 ? at : next_at, q & 31);
    return static_cast<const T*>(a.d_out) + (int64_t)t * a.ld_d_out;
  };
  const bool inside = col + 8 <= a.d;
  // word q of those that hold the thread's columns, from p on, of `size` bytes each
  auto copy16 = [&](uint4* dst, const void* p, int q, int size) {
    const int off = VEC ? 0 : (int)((uintptr_t)p & 15);
    // columns past the row's last are zeros, and not read
    const int left = (inside ? 8 : a.d - col) * size + off - 16 * q;
    const int bytes = VEC && inside ? 16 : min(16, max(0, left));
    const void* src = static_cast<const uint8_t*>(p) - off + (bytes > 0 ? 16 * q : 0);
    if (!active) return;
    if (VEC && size == 2)
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(ptx::smem_u32(dst)),
                   "l"(src), "r"(bytes)
                   : "memory");
    else       // (what two lanes, or two words of a lane, share is read from the L2 once)
      asm volatile("cp.async.ca.shared.global [%0], [%1], 16, %2;" ::"r"(ptx::smem_u32(dst)),
                   "l"(src), "r"(bytes)
                   : "memory");
  };
  // the columns out of the words of a slot, which came from p on
  auto take = [&](auto type, const uint4* slot_words, const void* p, float (&v)[8]) {
    using E = decltype(type);
    constexpr int N = (int)sizeof(E) / 2;
    uint32_t x[4 * N + 4];
#pragma unroll
    for (int h = 0; h < N + !VEC; ++h) {
      const uint4 w = slot_words[h * kSumThreads];
      x[4 * h] = w.x; x[4 * h + 1] = w.y; x[4 * h + 2] = w.z; x[4 * h + 3] = w.w;
    }
    if constexpr (!VEC) shift_words<4 * N, sizeof(E)>(x, (int)((uintptr_t)p & 15));
    const E* e = reinterpret_cast<const E*>(x);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = to_f32(e[j]);
  };
  auto table_row = [&](int32_t k) {
    return static_cast<const OT*>(a.out) + (int64_t)k * a.ld_out + col;
  };
  int32_t asked = -1;                       // the id of the last place requested
  auto request = [&](int w0, int i) {       // place i, of the window from w0
    if (i < end) {
      const int slot = (i - begin) % kAhead * (kPieces + kOnto);
      const T* row = row_of(i - w0) + col;
#pragma unroll
      for (int q = 0; q < kPieces; ++q) copy16(&s_rows[slot + q][threadIdx.x], row, q, sizeof(T));
      if constexpr (ADD) {
        const int32_t k = __shfl_sync(0xFFFFFFFFu, i - w0 < 32 ? key : next_key, (i - w0) & 31);
        if (k != asked) {
          const OT* t = table_row(k);
#pragma unroll
          for (int q = 0; q < kOnto; ++q)
            copy16(&s_rows[slot + kPieces + q][threadIdx.x], t, q, sizeof(OT));
          asked = k;
        }
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  for (int i = 0; i < kAhead - 1; ++i) request(begin, begin + i);
  int32_t last = -1;
  for (int w0 = begin; w0 < end; w0 += 32) {
    const int count = min(32, end - w0);
    for (int q = 0; q < count; ++q) {
      request(w0, w0 + q + kAhead - 1);
      asm volatile("cp.async.wait_group %0;" ::"n"(kAhead - 1) : "memory");
      const uint4* slot = &s_rows[(w0 + q - begin) % kAhead * (kPieces + kOnto)][threadIdx.x];
      float x[8];
      take(T(), slot, VEC ? nullptr : row_of(q) + col, x);
      const int32_t k = __shfl_sync(0xFFFFFFFFu, key, q);
      add(k, x);
      if constexpr (ADD) {
        // a run's first row: what it is added to
        if (w0 + q == begin || k != last) take(OT(), slot + kPieces * kSumThreads, table_row(k), onto);
        last = k;
      }
    }
    key = next_key;
    at = next_at;
    next_key = window(keys, w0 + 64);
    next_at = window(pos, w0 + 64);
  }
  flush(open_right);
  if (open_right && !open_left && group == 0 && u == 0)        // a run to join starts here
    a.keys[1][atomicAdd(&a.pos[1][0], 1)] = (int32_t)r;
}

// The last kernel: adds up the runs that cross ranges, from the list that the sums
// left (in any order: each is summed by itself).  A run's parts (slot 2 r + 1 of the
// range r it begins in, then slot 2 j of the ranges j it reaches) are shared by the
// block's thread groups in contiguous shares, which are added in order.
template <class OT, bool VEC>
__global__ void __launch_bounds__(kJoinThreads) join_kernel(const TableGrad a, int ct) {
  __shared__ float s_sum[kJoinThreads * 8];
  ptx::griddep_wait();
  ptx::griddep_launch_dependents();
  const int32_t* keys = a.keys[0];
  const int64_t work = (int64_t)a.pos[1][0] * a.groups;
  for (int64_t item = blockIdx.x; item < work; item += gridDim.x) {
    const int group = (int)(item % a.groups);
    const int64_t r = a.keys[1][item / a.groups];
    const int32_t id = keys[(r + 1) * a.range];
    int64_t parts = 1;
    for (int64_t j = r + 1;; j += kJoinThreads) {
      const int64_t at = (j + threadIdx.x) * a.range;
      const int c = __syncthreads_count(at < a.n && keys[at] == id);
      parts += c;
      if (c < kJoinThreads) break;
    }
    const int u = threadIdx.x % ct, share = threadIdx.x / ct, shares = kJoinThreads / ct;
    const int col = sum_col(group, u, ct);
    float sum[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) sum[j] = 0.f;
    if (col < a.d) {
      const int64_t q1 = parts * (share + 1) / shares;
#pragma unroll 8
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
    if (share == 0) {
      for (int h = 1; h < shares; ++h)
#pragma unroll
        for (int j = 0; j < 8; ++j) sum[j] += s_sum[j * kJoinThreads + h * ct + u];
      float onto[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) onto[j] = 0.f;
      if (a.add && col < a.d)
        load_cols<OT, VEC>(static_cast<const OT*>(a.out) + (int64_t)id * a.ld_out, col, a.d, onto);
      write_row<OT, VEC>(a, id, col, sum, onto);
    }
    __syncthreads();
  }
}

template <class T, class OT, bool VEC>
cudaError_t launch_sums(const TableGrad& a, int ct, int sm_count, cudaStream_t st) {
  const int64_t ranges = (a.n + (int64_t)a.range - 1) / a.range;
  const int per = kSumThreads / ct;
  cudaError_t e = launch_pdl(a.add ? sum_kernel<T, OT, VEC, true> : sum_kernel<T, OT, VEC, false>,
                             dim3((unsigned)((ranges + per - 1) / per * a.groups)),
                             dim3(kSumThreads), 0, st, a, ct);
  if (e != cudaSuccess) return e;
  const int64_t most = (ranges - 1) * a.groups, grid = 2 * (int64_t)sm_count;
  const int joins = a.n <= kShortRun ? 0 : (int)(most < grid ? most : grid);
  if (joins == 0) return e;
  return launch_pdl(join_kernel<OT, VEC>, dim3((unsigned)joins), dim3(kJoinThreads), 0, st, a, ct);
}
template <class T, class OT>
cudaError_t launch_sums_v(const TableGrad& a, int ct, bool vec, int sm_count,
                          cudaStream_t st) {
  return vec ? launch_sums<T, OT, true>(a, ct, sm_count, st)
             : launch_sums<T, OT, false>(a, ct, sm_count, st);
}
template <class T>
cudaError_t launch_sums_o(const TableGrad& a, int ct, int out_type, bool vec, int sm_count,
                          cudaStream_t st) {
  if (out_type == TAB_FP32) return launch_sums_v<T, float>(a, ct, vec, sm_count, st);
  if (out_type == TAB_BF16) return launch_sums_v<T, __nv_bfloat16>(a, ct, vec, sm_count, st);
  return launch_sums_v<T, __half>(a, ct, vec, sm_count, st);
}

// Threads that share a range's columns: enough for the row, a warp at least, at most
// 128.
int sum_threads(int d) {
  int ct = 32;
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
// sixteen blocks each, more where a run through all ranges would make too many parts.
// (8 / 16 / 32, us: 500 tokens x 4096 90 / 94 / 104, 8000 x 3584 56.0 / 56.5 / 70.5; 32768 x
// 4096 263 / 242 / 238.)
static int grad_range(int64_t n, int d, int sm_count) {
  const int ct = sum_threads(d);
  const int64_t groups = (d + ct * 8 - 1) / (ct * 8), per = kSumThreads / ct;
  if (n > 65536) return (int)(32 * ((n + 65535) / 65536));
  int range = 32;
  while (range > 8 && (n + range - 1) / range * groups < 16 * sm_count * per) range /= 2;
  return range;
}

size_t grad_scratch_bytes(int64_t n, int d, int sm_count) {
  const int ct = sum_threads(d), range = grad_range(n, d, sm_count);
  const int64_t ranges = (n + range - 1) / range;
  const size_t list = ((size_t)n * 4 + 255) / 256 * 256;
  return 4 * list + (size_t)ranges * 2 * ((d + ct * 8 - 1) / (ct * 8) * ct * 8) * 4;
}

// At least what any call of up to n tokens and d columns takes: ranges hold 8 positions
// or more; fewer than 32 only while a call has at most 32 sm_count * 128 thread columns
// of partial sums, more where 32 would make over 2048 ranges.
size_t grad_reserve_bytes(int64_t n, int64_t d, int sm_count) {
  const size_t list = ((size_t)n * 4 + 255) / 256 * 256;
  const size_t range = 2 * (size_t)((d + 1023) / 1024 * 1024) * 4;      // bytes of one's parts
  const size_t short_ranges = (size_t)(n / 8 + 1) * range;
  const size_t columns = (size_t)sm_count * 32 * kSumThreads * 64;
  const size_t few = short_ranges < columns ? short_ranges : columns;
  const size_t many = (size_t)(n / 32 + 1 < 2048 ? n / 32 + 1 : 2048) * range;
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
  cudaError_t e = cudaSuccess;
  if (!a.add) {
    e = launch_pdl(head_kernel, dim3((unsigned)(2 * sm_count)), dim3(kFillThreads), 0, st, a,
                   type_size(out_type));
    if (e != cudaSuccess || a.n == 0) return e;
  }
  // one CTA sorts a short list; longer ones take a portable cluster (one CTA / cluster,
  // us of a call with d = 64: 1000 tokens 16.4 / 20.6, 2000 18.7 / 21.0, 3000 20.7 / 21.6,
  // 4000 22.3 / 21.4, 8000 30.5 / 23.5)
  const int parts = a.n <= kSortShort ? 1 : 8;
  int bits = 1;
  while (((int64_t)1 << bits) <= a.V) ++bits;         // keys are 0 .. V
  const int passes = (bits + kSortBits - 1) / kSortBits;
  auto sort = a.add ? sort_kernel<true> : sort_kernel<false>;
  e = cudaFuncSetAttribute(sort, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(SortSmem));
  if (e != cudaSuccess) return e;
  e = launch_pdl_cluster(sort, dim3(parts), dim3(kSortThreads), sizeof(SortSmem), st, parts, a, parts,
                         passes, (bits + passes - 1) / passes);
  if (e != cudaSuccess) return e;
  const bool vec = on16(a.out, a.ld_out, type_size(out_type)) &&
                   on16(a.d_out, a.ld_d_out, type_size(src_type));
  if (src_type == TAB_FP32) return launch_sums_o<float>(a, ct, out_type, vec, sm_count, st);
  if (src_type == TAB_BF16) return launch_sums_o<__nv_bfloat16>(a, ct, out_type, vec, sm_count, st);
  return launch_sums_o<__half>(a, ct, out_type, vec, sm_count, st);
}

}  // namespace sph
