// Logits with penalties for repeated tokens, biases and masks, and a token from them.
//
//   z -> z / rep (z > 0) or z * rep        for ids among the row's tokens so far
//     -> z - freq * count, then z - pres   for ids among those of its output
//     -> z + the sum of the row's biases for the id
//     -> -inf                              where the row's mask has the id's bit clear
//
// each step rounded to fp32 (no fused multiply-add), the result to the output's type.
//
// Bound by memory: logits are read once and written once, with a bit of mask each.  What is
// sparse comes first, in a kernel of its own, a block for a range of a row's columns: tokens
// so far and biases mark their columns in a bitmap in shared memory, whose prefix sums number
// the marked ones; under these numbers tokens are counted (integer atomics: no order to
// depend on) and biases added in the list's order; then each marked column's logit is
// computed and kept with its column, in the columns' order.  The dense kernel, a warp for a
// segment of a row, reads all logits, without waiting for the sparse one, masks and writes
// them, and puts its segment's marked ones over them.  (Counted in shared memory by the
// dense blocks themselves, 4096 columns each, 1024 rows x 128256 ids with 512 tokens and 64
// biases a row took 301 us; with the marked columns written to the result by the sparse
// kernel, single words that the L2 gives back to memory before the dense one comes to them,
// 179 to 255; found by the dense kernel from the bitmap in memory 196.)
// With a draw a warp leaves its largest value, its sum of exp((z - largest) / tau) and the
// first place of the largest; a third kernel, a block a row, joins these and finds the token.
#include <cuda_bf16.h>

#include <type_traits>

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

// Mask bits of columns col .. col + 7 of kept ids (bit j: column col + j; those in [0, n) are
// meant), one by one.
__device__ __forceinline__ uint32_t scattered_bits(const Shape& a, const uint32_t* mask, int col) {
  uint32_t id[8], word[8], bits = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) id[j] = col + j >= 0 && col + j < a.n ? (uint32_t)a.ids[col + j] : ~0u;
#pragma unroll
  for (int j = 0; j < 8; ++j) word[j] = id[j] < (uint32_t)a.V ? mask[id[j] >> 5] : 0u;
#pragma unroll
  for (int j = 0; j < 8; ++j) bits |= (word[j] >> (id[j] & 31) & 1u) << j;
  return bits;
}
// Mask bits of the pieces at columns col, col + 256, ...  Ids ascend, so a piece of eight whose
// last is the first plus 7 is a run, as most are; all pieces' ids are requested together, then
// all their words.
template <int U>
__device__ __forceinline__ void mask_bits(const Shape& a, const uint32_t* mask, int col, uint32_t (&bits)[U]) {
  const uint32_t last = (uint32_t)(a.V - 1) >> 5;
  int first[U], end[U];
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const int c = col + i * 256;
    first[i] = max(c, 0);
    end[i] = first[i] + 7;
    if (a.ids) {
      const bool whole = c >= 0 && c + 8 <= a.n;
      first[i] = whole ? a.ids[c] : 0;
      end[i] = whole ? a.ids[c + 7] : -1;
    }
  }
  uint32_t lo[U], hi[U];
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const bool run = col + i * 256 < a.n && end[i] == first[i] + 7 && first[i] >= 0 && (!a.ids || end[i] < a.V);
    const uint32_t w = (uint32_t)first[i] >> 5;
    lo[i] = run ? mask[w] : 0u;
    hi[i] = run && (first[i] & 31) > 24 && w < last ? mask[w + 1] : 0u;
  }
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const int c = col + i * 256;
    bits[i] = __funnelshift_r(lo[i], hi[i], first[i] & 31);
    if (!a.ids) bits[i] <<= max(c, 0) - c;
    else if (c < a.n && !(end[i] == first[i] + 7 && first[i] >= 0 && end[i] < a.V))
      bits[i] = scattered_bits(a, mask, c);
  }
}

// A row's mask, or nullptr.
__device__ __forceinline__ const uint32_t* mask_of(const Shape& a, int64_t row) {
  if (!a.mask) return nullptr;
  const int64_t m = a.mask_rows ? a.mask_rows[row] : row;
  return m >= 0 && m < a.n_masks ? a.mask + m * a.ld_mask : nullptr;
}

// A piece of the logits; VEC: on the type's eight elements.
template <class T, bool VEC>
__device__ __forceinline__ void load_piece(const T* row, int col, int n, float (&v)[8]) {
  if constexpr (sizeof(T) == 4 && VEC) {
    if (col + 8 <= n && on32(row + col)) {
      load_v8(reinterpret_cast<const float*>(row) + col, v);
      return;
    }
  }
  load_cols<T, VEC>(row, col, n, v);
}
template <class OT>
__device__ __forceinline__ void store_piece(OT* row, int col, int n, const float (&v)[8]) {
  if constexpr (sizeof(OT) == 4) {
    if (col >= 0 && col + 8 <= n && on32(row + col)) {
      store_v8(reinterpret_cast<float*>(row) + col, v);
      return;
    }
  }
  store_cols<OT, true>(row, col, n, v);
}
// Columns that a row's pieces begin before it, so that the others begin on the eight
// elements' boundaries of the output (0 .. 7).
template <class OT>
__device__ __forceinline__ int lead_of(const OT* out) {
  const int head = (int)(-(intptr_t)out & (8 * (int)sizeof(OT) - 1)) / (int)sizeof(OT);
  return head ? 8 - head : 0;
}

// ---------------------------------------------------------------------------
// the sparse part
// ---------------------------------------------------------------------------
// Columns of a block: many, so that few blocks read a row's lists, or, where these blocks
// would be few or the lists could mark more columns than shared memory counts, fewer.
constexpr int kWideRange = 65536, kRange = 16384;
constexpr int kGrid = 256;               // columns whose marks the dense kernel finds together
constexpr int kStep = 64;                // kept ids between those of the first search
constexpr int kShortList = 256;          // biases of a block's columns that are joined at once

// The column in [c0, c1) whose id is `id`, or -1.  steps: every kStep-th kept id from c0 on, in
// shared memory (searched in global memory alone, each step waits for the one before it).
__device__ __forceinline__ int find(const int32_t* ids, const int32_t* steps, int c0, int c1, int id) {
  if (!ids) return id;
  int lo = 0, hi = (c1 - c0 - 1) / kStep;
  while (lo < hi) {                      // the last step whose id is not above
    const int mid = (lo + hi + 1) >> 1;
    if (steps[mid] <= id) lo = mid;
    else hi = mid - 1;
  }
  int a = c0 + lo * kStep, b = min(a + kStep, c1) - 1;
  while (a < b) {
    const int mid = (a + b) >> 1;
    if (ids[mid] < id) a = mid + 1;
    else b = mid;
  }
  return ids[a] == id ? a : -1;
}

template <int RANGE>
struct Marks {                           // in shared memory
  uint32_t bits[RANGE / 32];
  uint32_t before[RANGE / 32];           // marked columns before each word's
  int32_t steps[RANGE / kStep];
  uint32_t warp[32];
  int n_list, place[kShortList], col[kShortList];
  float val[kShortList];
};
template <int RANGE>
__device__ __forceinline__ int number(const Marks<RANGE>& m, int c) {       // of a marked column
  return (int)(m.before[c >> 5] + __popc(m.bits[c >> 5] & ((1u << (c & 31)) - 1u)));
}

// THREADS: 1024 where there are few blocks and long lists.
template <class T, int RANGE, int THREADS>
__global__ void __launch_bounds__(THREADS, THREADS == 256 ? 6 : 1) sparse_kernel(const Shape a) {
  constexpr int kRangeWords = RANGE / 32, kHeld = THREADS == 256 ? 4 : 8, threads = THREADS;
  extern __shared__ __align__(16) uint32_t smem[];
  __shared__ Marks<RANGE> m;
  ptx::griddep_wait();
  ptx::griddep_launch_dependents();
  const int64_t row = blockIdx.x / a.ranges;
  const int range = (int)(blockIdx.x - row * a.ranges);
  const int c0 = range * RANGE, c1 = min(c0 + RANGE, a.n);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  uint32_t* count = smem;                // by number: output tokens; bit 31: a prompt token too
  float* bias = reinterpret_cast<float*>(smem + a.most_marks);
  uint16_t* column = reinterpret_cast<uint16_t*>(smem + a.most_marks * (a.n_bias > 0 ? 2 : 1));

  // (all that depends on nothing is requested at once; a thread's first tokens stay in
  // registers)
  const int32_t* h = a.history + row * a.ld_history;
  const int32_t* bias_ids = a.bias_ids + row * a.ld_bias_ids;
  const float* bias_values = a.bias_values + row * a.ld_bias_values;
  const int max_tokens = a.history ? a.max_tokens : 0;
  int held[kHeld];
#pragma unroll
  for (int k = 0; k < kHeld; ++k) {
    const int i = (int)threadIdx.x + k * threads;
    held[k] = i < max_tokens ? h[i] : -1;
  }
  int32_t bias_id = -1;
  float bias_value = 0.f;
  if ((int)threadIdx.x < a.n_bias) {
    bias_id = bias_ids[threadIdx.x];
    bias_value = bias_values[threadIdx.x];
  }
  const int length = a.history && a.lengths ? max(0, min(a.lengths[row], max_tokens)) : max_tokens;
  const int prompt = a.prompts ? a.prompts[row] : 0;
  const float rep = a.repetition ? a.repetition[row] : 1.f;
  const float freq = a.frequency ? a.frequency[row] : 0.f;
  const float pres = a.presence ? a.presence[row] : 0.f;
  const int32_t first = a.ids ? a.ids[c0] : c0, last = a.ids ? a.ids[c1 - 1] : c1 - 1;
  for (int i = threadIdx.x; i < kRangeWords; i += threads) m.bits[i] = 0;
  if (a.ids)
    for (int i = threadIdx.x; c0 + i * kStep < c1; i += threads) m.steps[i] = a.ids[c0 + i * kStep];
  if (threadIdx.x == 0) m.n_list = 0;
  __syncthreads();
  // the column, from c0, of an id; -1: not one of the block's
  auto col_of = [&](int32_t id) {
    if (id < first || id > last) return -1;
    const int c = find(a.ids, m.steps, c0, c1, id);
    return c < 0 ? -1 : c - c0;
  };

  // ---- marks ----
  // (a frequent id's bit is mostly set; atomics on one word come one after another)
  auto mark = [&](int c) {
    const uint32_t bit = 1u << (c & 31);
    if (!(*const_cast<volatile uint32_t*>(&m.bits[c >> 5]) & bit)) atomicOr(&m.bits[c >> 5], bit);
  };
#pragma unroll
  for (int k = 0; k < kHeld; ++k) {
    const int i = (int)threadIdx.x + k * threads;
    held[k] = i < length ? col_of(held[k]) : -1;
    if (held[k] >= 0) mark(held[k]);
  }
  // (the others in batches, read again below)
  auto others = [&](auto&& use) {
    for (int i0 = (int)threadIdx.x + kHeld * threads; i0 < length; i0 += kHeld * threads) {
      int32_t id[kHeld];
#pragma unroll
      for (int k = 0; k < kHeld; ++k) id[k] = i0 + k * threads < length ? h[i0 + k * threads] : -1;
#pragma unroll
      for (int k = 0; k < kHeld; ++k) {
        const int c = i0 + k * threads < length ? col_of(id[k]) : -1;
        if (c >= 0) use(i0 + k * threads, c);
      }
    }
  };
  others([&](int, int c) { mark(c); });
  for (int i = threadIdx.x; i < a.n_bias; i += threads) {
    const bool own = i == (int)threadIdx.x;
    const int c = col_of(own ? bias_id : bias_ids[i]);
    if (c < 0) continue;
    mark(c);
    const int at = atomicAdd(&m.n_list, 1);
    if (at < kShortList) {
      m.place[at] = i;
      m.col[at] = c;
      m.val[at] = own ? bias_value : bias_values[i];
    }
  }
  __syncthreads();

  // ---- numbers ----
  constexpr int words = kRangeWords >= threads ? kRangeWords / threads : 1;    // of a thread
  const int w0 = min((int)threadIdx.x * words, kRangeWords), w1 = min(w0 + words, kRangeWords);
  uint32_t mine = 0;
  for (int w = w0; w < w1; ++w) mine += __popc(m.bits[w]);
  uint32_t incl = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t up = __shfl_up_sync(0xFFFFFFFFu, incl, o);
    if (lane >= o) incl += up;
  }
  if (lane == 31) m.warp[warp] = incl;
  __syncthreads();
  uint32_t at = incl - mine, marked = 0;
  for (int w = 0; w < threads / 32; ++w) {
    if (w < warp) at += m.warp[w];
    marked += m.warp[w];
  }
  for (int w = w0; w < w1; ++w) {
    m.before[w] = at;
    at += __popc(m.bits[w]);
  }
  for (int i = threadIdx.x; i < (int)marked; i += threads) {
    count[i] = 0;
    if (a.n_bias > 0) bias[i] = 0.f;
  }
  __syncthreads();
  // where the marks of each kGrid columns begin, and how many they are
  for (int g = threadIdx.x; g < RANGE / kGrid && c0 + g * kGrid < a.n; g += threads) {
    const uint32_t from = m.before[g * (kGrid / 32)];
    const uint32_t to = g + 1 < RANGE / kGrid ? m.before[(g + 1) * (kGrid / 32)] : marked;
    a.marks[row * a.ld_marks + range * (RANGE / kGrid) + g] = from | (to - from) << 16;
  }

  // ---- counts and biases under these numbers ----
  // (each names its column: found from the bitmap instead, the frequent ids, which lie side by
  // side, made few threads find most columns)
  auto add = [&](int i, int c) {
    const int k = number(m, c);
    column[k] = (uint16_t)c;
    if (i < prompt) atomicOr(&count[k], 0x80000000u);
    else atomicAdd(&count[k], 1u);
  };
#pragma unroll
  for (int k = 0; k < kHeld; ++k)
    if (held[k] >= 0) add((int)threadIdx.x + k * threads, held[k]);
  others(add);
  const int n = m.n_list;
  if (n <= kShortList) {
    // each column's first entry adds the others, whatever order they were found in
    const int e = threadIdx.x;
    if (e < n) {
      const int c = m.col[e], place = m.place[e];
      bool lead = true, more = false;
      for (int k = 0; k < n; ++k)
        if (m.col[k] == c) {
          lead &= m.place[k] >= place;
          more |= k != e;
        }
      if (lead) {
        float sum = m.val[e];
        for (int done = place; more;) {
          int next = -1;
          for (int k = 0; k < n; ++k)
            if (m.col[k] == c && m.place[k] > done && (next < 0 || m.place[k] < m.place[next])) next = k;
          if (next < 0) break;
          sum = __fadd_rn(sum, m.val[next]);
          done = m.place[next];
        }
        column[number(m, c)] = (uint16_t)c;
        bias[number(m, c)] = sum;
      }
    }
  } else if (warp == 0) {
    // a long list: one warp, 32 entries after another
    for (int i0 = 0; i0 < a.n_bias; i0 += 32) {
      const int c = i0 + lane < a.n_bias ? col_of(bias_ids[i0 + lane]) : -1;
      const float b = c >= 0 ? bias_values[i0 + lane] : 0.f;
      const unsigned same = __match_any_sync(0xFFFFFFFFu, c);
      const bool lead = c >= 0 && __ffs(same) - 1 == lane;
      float sum = lead ? bias[number(m, c)] : 0.f;
      for (int l = 0; l < 32; ++l) {
        const float v = __shfl_sync(0xFFFFFFFFu, b, l);
        if (lead && same >> l & 1) sum = __fadd_rn(sum, v);
      }
      if (lead) {
        column[number(m, c)] = (uint16_t)c;
        bias[number(m, c)] = sum;
      }
      __syncwarp();
    }
  }
  __syncthreads();

  // ---- the marked columns' logits ----
  const uint32_t* mask = mask_of(a, row);
  const T* z = static_cast<const T*>(a.z) + row * a.ld_z + c0;
  float2* pairs = a.pairs + (int64_t)blockIdx.x * a.most_marks;
  for (int i = threadIdx.x; i < (int)marked; i += threads) {
    const uint32_t c = count[i];
    const int col = column[i];
    float x = to_f32(z[col]);
    const uint32_t id = mask ? (uint32_t)(a.ids ? a.ids[c0 + col] : c0 + col) : 0u;
    const bool allowed = !mask || (id < (uint32_t)a.V && (mask[id >> 5] >> (id & 31) & 1u));
    if (c && a.repetition) x = x > 0.f ? __fdiv_rn(x, rep) : __fmul_rn(x, rep);
    if (c & 0x7FFFFFFFu) {
      if (a.frequency) x = __fsub_rn(x, __fmul_rn(freq, (float)(c & 0x7FFFFFFFu)));
      if (a.presence) x = __fsub_rn(x, pres);
    }
    if (a.n_bias > 0) x = __fadd_rn(x, bias[i]);
    pairs[i] = make_float2(__int_as_float(c0 + col), allowed ? x : -INFINITY);
  }
}

// ---------------------------------------------------------------------------
// all columns
// ---------------------------------------------------------------------------
// A piece as it was read: 16-bit logits stay packed.
template <class T, bool VEC>
struct Piece {
  float v[8];
  __device__ __forceinline__ void load(const T* row, int col, int n) { load_piece<T, VEC>(row, col, n, v); }
  __device__ __forceinline__ float value(int j) const { return v[j]; }
};
template <class T>
struct Packed {
  uint4 w;
  __device__ __forceinline__ void load(const T* row, int col, int n) {
    if (col + 8 <= n) {
      w = *reinterpret_cast<const uint4*>(row + col);
    } else {
      w = make_uint4(0, 0, 0, 0);
      T* e = reinterpret_cast<T*>(&w);
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (col + j < n) e[j] = row[col + j];
    }
  }
  __device__ __forceinline__ float value(int j) const { return to_f32(reinterpret_cast<const T*>(&w)[j]); }
};
template <> struct Piece<__nv_bfloat16, true> : Packed<__nv_bfloat16> {};
template <> struct Piece<__half, true> : Packed<__half> {};

// Bits of a float as an integer that orders as the float does (-inf lowest).
__device__ __forceinline__ int ordered(float x) {
  const int b = __float_as_int(x);
  return b ^ (b >> 31 & 0x7FFFFFFF);
}

// A warp takes a segment of 256 U columns, U pieces a lane.  VEC: rows of z and out are on
// 16 bytes.  Other rows: pieces begin on the output's boundaries.
constexpr int kDenseThreads = 128, kDenseWarps = kDenseThreads / 32;
template <class T, class OT, bool VEC, int U>
__global__ void __launch_bounds__(kDenseThreads) shape_kernel(const Shape a) {
  __shared__ uint32_t s_hits[kDenseWarps][32];
  // (after a sparse kernel the logits and masks, which are the caller's, are read before
  // it ends)
  if (!a.marks) {
    ptx::griddep_wait();
    ptx::griddep_launch_dependents();
  }
  const int64_t item = (int64_t)blockIdx.x * kDenseWarps + (threadIdx.x >> 5);
  const int64_t row = item / a.chunks;
  if (row >= a.rows) return;
  const int chunk = (int)(item - row * a.chunks), lane = threadIdx.x & 31;
  OT* out = static_cast<OT*>(a.out) + row * a.ld_out;
  const int base = chunk * (256 * U) - (VEC ? 0 : lead_of(out)) + lane * 8;
  const T* z = static_cast<const T*>(a.z) + row * a.ld_z;
  const uint32_t* mask = mask_of(a, row);
  if (a.mask_rows && !mask && lane == 0 && chunk == 0 && a.mask_rows[row] != -1)
    atomicOr(a.status, ERR_BAD_INDEX);
  Piece<T, VEC> p[U];
  uint32_t bits[U];
#pragma unroll
  for (int i = 0; i < U; ++i)
    if (base + i * 256 < a.n) p[i].load(z, base + i * 256, a.n);
  if (mask) {
    mask_bits<U>(a, mask, base, bits);
  } else {
#pragma unroll
    for (int i = 0; i < U; ++i) bits[i] = 0xFFu;
  }
  // the segment's marks: a lane's own pieces' (bit 8 i + j: column j of piece i), and where
  // the pairs of each of the ranges that it meets (two at most) are
  const int seg0 = max(base - lane * 8, 0), seg1 = min(base - lane * 8 + 256 * U, a.n);
  uint32_t hits = 0;
  const float2* from[2] = {nullptr, nullptr};
  int n_pairs[2] = {0, 0};
  if (a.marks) {
    ptx::griddep_wait();
    ptx::griddep_launch_dependents();
    const int g0 = seg0 / kGrid, g1 = (seg1 - 1) / kGrid;      // at most U + 1 of them
    const uint32_t mark = g0 + lane <= g1 ? a.marks[row * a.ld_marks + g0 + lane] : 0u;
    const int per = (a.wide ? kWideRange : kRange) / kGrid, r0 = g0 / per;
    const int in = g0 + lane <= g1 ? (g0 + lane) / per - r0 : -1;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      if (k == 1 && (VEC || g1 / per == r0)) break;
      n_pairs[k] = (int)__reduce_add_sync(0xFFFFFFFFu, in == k ? mark >> 16 : 0u);
      const int first = k == 0 ? 0 : (r0 + 1) * per - g0;
      from[k] = a.pairs + (row * a.ranges + r0 + k) * a.most_marks +
                (__shfl_sync(0xFFFFFFFFu, mark, first) & 0xFFFFu);
    }
    if (n_pairs[0] + n_pairs[1] > 0) {
      uint32_t* own = s_hits[threadIdx.x >> 5];
      own[lane] = 0;
      __syncwarp();
#pragma unroll
      for (int k = 0; k < 2; ++k)
        for (int e = lane; e < n_pairs[k]; e += 32) {
          const int c = __float_as_int(from[k][e].x);
          if (c < seg0 || c >= seg1) continue;
          const int at = c - (base - lane * 8);
          atomicOr(&own[at >> 3 & 31], 1u << ((at >> 8) * 8 + (at & 7)));
        }
      __syncwarp();
      hits = own[lane];
    }
  }

  float top = -INFINITY, sum = 0.f;
  int at = 0x7FFFFFFF;
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const int col = base + i * 256;
    if (col >= a.n) break;
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = p[i].value(j);
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (!(bits[i] >> j & 1)) v[j] = -INFINITY;
    store_piece<OT>(out, col, a.n, v);
    if (!a.draw) continue;
    if (col < 0 || col + 8 > a.n) {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (col + j < 0 || col + j >= a.n) v[j] = -INFINITY;
    }
    if (hits >> 8 * i & 0xFFu) {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (hits >> (8 * i + j) & 1) v[j] = -INFINITY;
    }
    // (a NaN is the largest here, and goes to the sum)
    float m = v[0];
#pragma unroll
    for (int j = 1; j < 8; ++j) asm("max.NaN.f32 %0, %0, %1;" : "+f"(m) : "f"(v[j]));
    if (m != m) {
      sum = NAN;
      m = -INFINITY;
#pragma unroll
      for (int j = 0; j < 8; ++j) m = fmaxf(m, v[j]);
    }
    if (m > top) {
#pragma unroll
      for (int j = 7; j >= 0; --j)
        if (v[j] == m) at = col + j;
      if (!a.greedy) sum *= weight(top, m, a.l2t);
      top = m;
    }
    if (!a.greedy) {
#pragma unroll
      for (int j = 0; j < 8; ++j) sum += weight(v[j], top, a.l2t);
    }
  }
  // the marked columns over what was stored
  __syncwarp();
#pragma unroll
  for (int k = 0; k < 2; ++k)
    for (int e = lane; e < n_pairs[k]; e += 32) {
      const float2 pair = from[k][e];
      const int c = __float_as_int(pair.x);
      if (c < seg0 || c >= seg1) continue;
      const float x = pair.y;
      out[c] = from_f32<OT>(x);
      if (x != x) sum = NAN;
      if (x > top || (x == top && c < at)) {
        if (!a.greedy) sum *= weight(top, x, a.l2t);
        top = x;
        at = c;
      }
      if (!a.greedy) sum += weight(x, top, a.l2t);
    }
  if (!a.draw) return;
  const int most = __reduce_max_sync(0xFFFFFFFFu, ordered(top));
  const float M = __int_as_float(most ^ (most >> 31 & 0x7FFFFFFF));
  at = (int)__reduce_min_sync(0xFFFFFFFFu, top == M ? (unsigned)at : 0x7FFFFFFFu);
  if (!a.greedy) sum *= weight(top, M, a.l2t);
  sum = warp_sum(sum);
  if (lane == 0) a.stats[row * a.chunks + chunk] = make_float4(M, sum, __int_as_float(at), 0.f);
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
  const int base = chunk * a.cols - (a.vec ? 0 : lead_of(z));
  const int c0 = max(base, 0), c1 = min(base + a.cols, a.n);
  const int j = pick(c1 - c0, [&](int i) { return weight(z[c0 + i], M, a.l2t); }, target, &before,
                     red, s_place, &s_before);
  if (threadIdx.x == 0) a.tokens[row] = j < 0 ? -1 : a.ids ? a.ids[c0 + j] : c0 + j;
}

// Columns of a warp: 1024, fewer where these would leave SMs without work.
int chunk_cols(int64_t rows, int n, int sm_count) {
  const int64_t columns = rows * n;
  return columns >= (int64_t)sm_count * 8 * 1024 ? 1024 : columns >= (int64_t)sm_count * 8 * 512 ? 512 : 256;
}
int chunk_count(int n, int cols) { return (n + 7 + cols - 1) / cols; }
int64_t mark_words(int n) { return ((int64_t)n + 2 * kGrid - 1) / (2 * kGrid) * 2; }      // (even)

template <class T, int RANGE, int THREADS>
cudaError_t launch_sparse(const Shape& a, cudaStream_t st) {
  const size_t smem = (size_t)a.most_marks * (a.n_bias > 0 ? 10 : 6);     // 160 KB at most
  auto kernel = sparse_kernel<T, RANGE, THREADS>;
  const cudaError_t e =
      cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kRange * 10);
  if (e != cudaSuccess) return e;
  return launch_pdl(kernel, dim3((unsigned)(a.rows * a.ranges)), dim3(THREADS), smem, st, a);
}
template <class T, class OT>
cudaError_t launch_shape_t(const Shape& a, cudaStream_t st) {
  const dim3 grid((unsigned)((a.rows * a.chunks + kDenseWarps - 1) / kDenseWarps)), block(kDenseThreads);
  auto dense = [&](auto u) {
    constexpr int U = decltype(u)::value;
    return a.vec ? launch_pdl(shape_kernel<T, OT, true, U>, grid, block, 0, st, a)
                 : launch_pdl(shape_kernel<T, OT, false, U>, grid, block, 0, st, a);
  };
  if (a.cols == 256) return dense(std::integral_constant<int, 1>());
  if (a.cols == 512) return dense(std::integral_constant<int, 2>());
  return dense(std::integral_constant<int, 4>());
}
template <class T>
cudaError_t launch_shape_o(const Shape& a, int out_type, cudaStream_t st) {
  if (a.marks) {
    const cudaError_t e = a.wide             ? launch_sparse<T, kWideRange, 256>(a, st)
                          : a.sparse_threads ? launch_sparse<T, kRange, 1024>(a, st)
                                             : launch_sparse<T, kRange, 256>(a, st);
    if (e != cudaSuccess) return e;
  }
  if (out_type == TAB_FP32) return launch_shape_t<T, float>(a, st);
  if (out_type == TAB_BF16) return launch_shape_t<T, __nv_bfloat16>(a, st);
  return launch_shape_t<T, __half>(a, st);
}

}  // namespace

// How the sparse part is divided.
struct Sparse {
  int wide, ranges, most_marks;
};
Sparse sparse_plan(int64_t rows, int n, int64_t entries, int sm_count) {
  Sparse p;
  p.wide = entries <= kRange && rows * ((n + kWideRange - 1) / kWideRange) >= 2 * (int64_t)sm_count;
  const int range = p.wide ? kWideRange : kRange;
  p.ranges = (n + range - 1) / range;
  const int64_t most = entries < n ? entries : n;
  p.most_marks = (int)((most < kRange ? most : kRange) + 1) & ~1;
  return p;
}

// The statistics of a draw; where each kGrid columns' pairs are, and the pairs.
size_t shape_scratch_bytes(int64_t rows, int n, bool draw, int64_t entries, int sm_count) {
  size_t b = draw ? (size_t)rows * chunk_count(n, chunk_cols(rows, n, sm_count)) * sizeof(float4) : 0;
  if (entries > 0) {
    const Sparse p = sparse_plan(rows, n, entries, sm_count);
    b += (size_t)rows * (mark_words(n) * 4 + (size_t)p.ranges * p.most_marks * 8);
  }
  return b;
}
// At least what any call of up to so many rows and ids takes, whatever its lists: as many
// marks as ids, rounded up to whole ranges (of one, to an even number).
size_t shape_reserve_bytes(int64_t rows, int64_t n) {
  const size_t marks = n <= kRange ? n + 1 : (n + kRange - 1) / kRange * kRange;
  return (size_t)rows * (chunk_count((int)n, 256) * sizeof(float4) + (size_t)mark_words((int)n) * 4 + marks * 8);
}
// Blocks of its largest grid.
int64_t shape_blocks(int64_t rows, int n, int sm_count) {
  return rows * chunk_count(n, chunk_cols(rows, n, sm_count));
}

cudaError_t launch_shape(Shape a, int z_type, int out_type, void* scratch, int sm_count,
                         cudaStream_t st) {
  a.cols = chunk_cols(a.rows, a.n, sm_count);
  a.chunks = chunk_count(a.n, a.cols);
  a.stats = static_cast<float4*>(scratch);
  a.marks = nullptr;
  const int64_t entries = (int64_t)(a.history ? a.max_tokens : 0) + a.n_bias;
  if (entries > 0) {
    const Sparse p = sparse_plan(a.rows, a.n, entries, sm_count);
    a.wide = p.wide; a.ranges = p.ranges; a.most_marks = p.most_marks;
    a.ld_marks = mark_words(a.n);
    a.marks = reinterpret_cast<uint32_t*>(a.stats + (a.draw ? a.rows * a.chunks : 0));
    a.pairs = reinterpret_cast<float2*>(a.marks + a.rows * a.ld_marks);
    a.sparse_threads = entries > 2048 || (entries > 512 && a.rows * a.ranges <= 2 * (int64_t)sm_count);
  }
  a.vec = on16(a.z, a.ld_z, type_size(z_type)) && on16(a.out, a.ld_out, type_size(out_type));
  a.l2t = a.greedy ? 0.f : kLog2e * a.inv_tau;
  const cudaError_t e = z_type == TAB_FP32   ? launch_shape_o<float>(a, out_type, st)
                        : z_type == TAB_BF16 ? launch_shape_o<__nv_bfloat16>(a, out_type, st)
                                             : launch_shape_o<__half>(a, out_type, st);
  if (e != cudaSuccess || !a.draw) return e;
  return launch_pdl(shape_draw_kernel, dim3((unsigned)a.rows), dim3(kThreads), 0, st, a);
}

}  // namespace sph
