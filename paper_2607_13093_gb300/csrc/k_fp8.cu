// Rows into e4m3 with a scale for each block of 128 columns, and rows of such a table back
// (all in order, or by token).
//
// Bound by memory: an element is read once (2 or 4 bytes) and leaves one byte, and the other
// way round.  A thread takes 16 consecutive columns (32 bytes an access: in two of 16 a warp
// asks for every sector twice), eight threads a block's width.  With blocks of one row nothing
// else is shared; with blocks of 128 rows a CTA holds the whole block in registers, four rows a
// thread, until its largest magnitude is known.  32000 x 4096 bf16 in blocks of 128 rows: coded
// in 59 us, coded and decoded in 126 (6.2 TB/s of what has to move), in blocks of a row 135.
#include <cuda_bf16.h>

#include <type_traits>

#include "fp8.cuh"
#include "rows.cuh"
#include "sm100_ptx.cuh"
#include "sph_internal.h"

namespace sph {
namespace {

constexpr int kCols = 16;                // columns of a thread
constexpr int kLanes = kFp8Block / kCols;

// item / spans (a 64-bit division is a hundred instructions)
__device__ __forceinline__ int64_t over(int64_t item, int spans) {
  return item >> 32 ? item / spans : (int64_t)((uint32_t)item / (uint32_t)spans);
}

// A thread's 16 columns as they were read.
template <class T>
struct Cols16 {
  uint32_t w[4 * sizeof(T)];
  __device__ __forceinline__ float get(int j) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[j]);
    else if constexpr (std::is_same<T, __half>::value)
      return __half2float(__ushort_as_half((unsigned short)(j & 1 ? w[j >> 1] >> 16 : w[j >> 1] & 0xFFFFu)));
    else
      return __uint_as_float(j & 1 ? w[j >> 1] & 0xFFFF0000u : w[j >> 1] << 16);
  }
};
// aligned: rows are on 32 bytes.
template <class T>
__device__ __forceinline__ void load16(const T* row, int col, int d, bool aligned, Cols16<T>& r) {
  constexpr int N = (int)sizeof(T);
  if (col + kCols > d) {
#pragma unroll
    for (int j = 0; j < kCols; ++j) {
      if constexpr (N == 4) {
        r.w[j] = col + j < d ? reinterpret_cast<const uint32_t*>(row)[col + j] : 0u;
      } else {
        const uint32_t e = col + j < d ? reinterpret_cast<const uint16_t*>(row)[col + j] : 0u;
        if (j & 1) r.w[j / 2] |= e << 16;
        else r.w[j / 2] = e;
      }
    }
  } else if (aligned) {
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
      uint32_t q[8];
      load_v8(static_cast<const void*>(row + col + i * (32 / N)), q);
#pragma unroll
      for (int k = 0; k < 8; ++k) r.w[8 * i + k] = q[k];
    }
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
    for (int i = 0; i < 4 * N; ++i) r.w[i] = x[i];
  }
}
// Bits of the largest magnitude as fp32 (kFp8Inf or more: a NaN or an infinity).
template <class T>
__device__ __forceinline__ unsigned largest(const Cols16<T>& r) {
  unsigned m = 0;
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int j = 0; j < kCols; ++j) m = max(m, r.w[j] & 0x7FFFFFFFu);
  } else {
#pragma unroll
    for (int j = 0; j < kCols / 2; ++j) m = __vmaxu2(m, r.w[j] & 0x7FFF7FFFu);
    m = max(m >> 16, m & 0xFFFFu);
    if constexpr (std::is_same<T, __nv_bfloat16>::value) m <<= 16;
    else m = m >= 0x7C00u ? kFp8Inf : __float_as_uint(__half2float(__ushort_as_half((unsigned short)m)));
  }
  return m;
}
// The codes of a thread's 16-bit columns; all lanes of the warp call it.
template <class T, bool ROUND>
__device__ __forceinline__ uint4 codes_by_product(const Cols16<T>& r, const Fp8Product& p, unsigned keep) {
  uint32_t c[4];
  const F2 inv = mul2(p.inv, p.nudge);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 a = fp8_by_product<ROUND>(r.get(4 * i), r.get(4 * i + 1), p, inv);
    const float2 b = fp8_by_product<ROUND>(r.get(4 * i + 2), r.get(4 * i + 3), p, inv);
    c[i] = fp8_codes4(a.x, a.y, b.x, b.y) & keep;
  }
  return make_uint4(c[0], c[1], c[2], c[3]);
}
template <class T>
__device__ __forceinline__ uint4 codes16(const Cols16<T>& r, const Fp8Scale& s, unsigned amax) {
  if constexpr (sizeof(T) == 2) {
    const Fp8Product p = fp8_product(amax, s);
    const unsigned keep = s.step > 0.f ? ~0u : 0u;       // (a NaN's block: codes of zero)
    return __any_sync(0xFFFFFFFFu, p.on_border) ? codes_by_product<T, true>(r, p, keep)
                                                : codes_by_product<T, false>(r, p, keep);
  }
  uint32_t c[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const Fp8Two lo = fp8_quotients(f2(r.get(4 * i), r.get(4 * i + 1)), s);
    const Fp8Two hi = fp8_quotients(f2(r.get(4 * i + 2), r.get(4 * i + 3)), s);
    float2 a = both(lo.q), b = both(hi.q);
    const float2 ra = both(lo.rest), rb = both(hi.rest);
    const unsigned border = min(min(__float_as_uint(a.x) << 13, __float_as_uint(a.y) << 13),
                                min(__float_as_uint(b.x) << 13, __float_as_uint(b.y) << 13));
    if (border == 0) {
      a = make_float2(fp8_settled(a.x, ra.x), fp8_settled(a.y, ra.y));
      b = make_float2(fp8_settled(b.x, rb.x), fp8_settled(b.y, rb.y));
    }
    c[i] = s.step > 0.f ? fp8_codes4(a.x, a.y, b.x, b.y) : 0u;
  }
  return make_uint4(c[0], c[1], c[2], c[3]);
}
// Codes of columns col .. col + 15, those past d left as they are.
__device__ __forceinline__ void store16(uint8_t* row, int col, int d, uint4 c) {
  if (col + kCols <= d) {
    *reinterpret_cast<uint4*>(row + col) = c;
  } else {
    const uint32_t w[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
    for (int j = 0; j < kCols; ++j)
      if (col + j < d) row[col + j] = (uint8_t)(w[j / 4] >> 8 * (j % 4));
  }
}

// Blocks of one row: a warp takes four blocks, `spans` of them a row.
constexpr int kRowThreads = 256;
template <class T>
__global__ void __launch_bounds__(kRowThreads) fp8_rows_kernel(const Fp8Quant a) {
  ptx::griddep_wait();
  ptx::griddep_launch_dependents();
  for (int64_t i = (int64_t)blockIdx.x * kRowThreads + threadIdx.x; i < a.zeros;
       i += (int64_t)gridDim.x * kRowThreads)
    a.zero[i] = 0;
  const int lane = threadIdx.x & 31;
  const int64_t item = (int64_t)blockIdx.x * (kRowThreads / 32) + (threadIdx.x >> 5);
  const int64_t row = over(item, a.spans);
  if (row >= a.rows) return;
  const int col = (int)(item - row * a.spans) * 32 * kCols + lane * kCols;
  Cols16<T> r;
  if (col < a.d) load16<T>(static_cast<const T*>(a.x) + row * a.ld_x, col, a.d, a.aligned != 0, r);
  unsigned m = col < a.d ? largest<T>(r) : 0u;
#pragma unroll
  for (int o = 1; o < kLanes; o <<= 1) m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
  const Fp8Scale s = fp8_scale(m);
  const uint4 codes = codes16<T>(r, s, m);
  if (col >= a.d) return;
  store16(a.codes + row * a.ld_codes, col, a.d, codes);
  if (col % kFp8Block == 0) a.scales[row * a.row_step + col / kFp8Block * a.col_step] = s.scale;
}

// Blocks of 128 rows: a CTA a block.
constexpr int kTileThreads = 256;
template <class T>
__global__ void __launch_bounds__(kTileThreads) fp8_tiles_kernel(const Fp8Quant a) {
  constexpr int kTurns = kFp8Block / (kTileThreads / kLanes);      // rows of a thread
  __shared__ unsigned s_max[kTileThreads / 32];
  ptx::griddep_wait();
  ptx::griddep_launch_dependents();
  const int64_t tile = blockIdx.x / a.spans;
  const int cb = (int)(blockIdx.x - tile * a.spans);
  const int col = cb * kFp8Block + (int)(threadIdx.x % kLanes) * kCols;
  const int64_t row0 = tile * kFp8Block + threadIdx.x / kLanes;
  Cols16<T> r[kTurns];
  unsigned m = 0;
#pragma unroll
  for (int i = 0; i < kTurns; ++i) {
    const int64_t row = row0 + i * (kTileThreads / kLanes);
    if (row < a.rows && col < a.d)
      load16<T>(static_cast<const T*>(a.x) + row * a.ld_x, col, a.d, a.aligned != 0, r[i]);
  }
#pragma unroll
  for (int i = 0; i < kTurns; ++i)
    if (row0 + i * (kTileThreads / kLanes) < a.rows && col < a.d) m = max(m, largest<T>(r[i]));
  m = __reduce_max_sync(0xFFFFFFFFu, m);
  if ((threadIdx.x & 31) == 0) s_max[threadIdx.x >> 5] = m;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kTileThreads / 32; ++w) m = max(m, s_max[w]);
  const Fp8Scale s = fp8_scale(m);
#pragma unroll
  for (int i = 0; i < kTurns; ++i) {
    const int64_t row = row0 + i * (kTileThreads / kLanes);
    const uint4 codes = codes16<T>(r[i], s, m);
    if (row < a.rows && col < a.d) store16(a.codes + row * a.ld_codes, col, a.d, codes);
  }
  if (threadIdx.x == 0) a.scales[tile * a.row_step + cb * a.col_step] = s.scale;
}

template <class T>
cudaError_t launch_quant(Fp8Quant a, cudaStream_t st) {
  if (a.block_rows == 1) {
    a.spans = (a.d + 32 * kCols - 1) / (32 * kCols);
    const int64_t items = a.rows * a.spans;
    return launch_pdl(fp8_rows_kernel<T>, dim3((unsigned)((items + kRowThreads / 32 - 1) / (kRowThreads / 32))),
                      dim3(kRowThreads), 0, st, a);
  }
  a.spans = (a.d + kFp8Block - 1) / kFp8Block;
  const int64_t tiles = (a.rows + kFp8Block - 1) / kFp8Block * a.spans;
  return launch_pdl(fp8_tiles_kernel<T>, dim3((unsigned)tiles), dim3(kTileThreads), 0, st, a);
}

// ---------------------------------------------------------------------------
// rows back
// ---------------------------------------------------------------------------
__device__ __forceinline__ float value_of(uint8_t code) {
  const __half_raw h = __nv_cvt_fp8_to_halfraw((__nv_fp8_storage_t)code, __NV_E4M3);
  return __half2float(*reinterpret_cast<const __half*>(&h));
}

// A warp takes 512 columns of a row, 16 a thread: neighbours, or, where the result's rows are not
// on 16 bytes, 32 columns apart, so that a warp's stores are side by side (32000 x 4095 bf16 coded
// and decoded 204 us, by pieces of eight neighbours 812).
constexpr int kLookThreads = 128;
template <class OT, bool ON16>
__global__ void __launch_bounds__(kLookThreads) fp8_lookup_kernel(const Fp8Lookup a) {
  ptx::griddep_wait();
  ptx::griddep_launch_dependents();
  const int64_t item = (int64_t)blockIdx.x * (kLookThreads / 32) + (threadIdx.x >> 5);
  const int64_t t = over(item, a.spans);
  if (t >= a.n) return;
  const int span = (int)(item - t * a.spans), lane = threadIdx.x & 31;
  const int64_t id = a.tokens ? a.tokens[t] : t;
  const bool there = id >= 0 && id < a.V && id != a.padding;
  if (!there && id != a.padding && span == 0 && lane == 0) atomicOr(a.status, ERR_BAD_INDEX);
  OT* out = static_cast<OT*>(a.out) + t * a.ld_out;
  const uint8_t* row = there ? a.codes + id * a.ld_codes : nullptr;
  const float* scales =
      there ? a.scales + (a.block_rows == 1 ? id : id / kFp8Block) * a.ld_scales : nullptr;
  if constexpr (!ON16) {
    const int col = span * 32 * kCols + lane;
    if (col + 31 * kCols >= a.d || !there) {
      for (int c = col; c < min(a.d, (span + 1) * 32 * kCols); c += 32)
        out[c] = from_f32<OT>(there ? value_of(row[c]) * scales[c / kFp8Block] * a.scale : 0.f);
      return;
    }
    uint8_t w[kCols];
#pragma unroll
    for (int j = 0; j < kCols; ++j) w[j] = row[col + 32 * j];
#pragma unroll
    for (int j = 0; j < kCols; j += kFp8Block / 32) {
      const float s = scales[(col + 32 * j) / kFp8Block];
#pragma unroll
      for (int k = j; k < j + kFp8Block / 32; ++k)
        out[col + 32 * k] = from_f32<OT>(value_of(w[k]) * s * a.scale);
    }
    return;
  }
  const int col = span * 32 * kCols + lane * kCols;
  if (col >= a.d) return;
  float v[2][8];
  uint32_t w[4] = {0, 0, 0, 0};
  float s = 0.f;
  if (there) {
    if (col + kCols <= a.d) {
      const uint4 c = *reinterpret_cast<const uint4*>(row + col);
      w[0] = c.x; w[1] = c.y; w[2] = c.z; w[3] = c.w;
    } else {
#pragma unroll
      for (int j = 0; j < kCols; ++j)
        if (col + j < a.d) w[j / 4] |= (uint32_t)row[col + j] << 8 * (j % 4);
    }
    s = scales[col / kFp8Block];
  }
  // (a row that is not there: zeros times 0 times 1)
  const F2 s2 = f2(s), by = f2(there ? a.scale : 1.f);
#pragma unroll
  for (int j = 0; j < kCols; j += 2) {
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(
        (__nv_fp8x2_storage_t)(w[j / 4] >> 8 * (j % 4) & 0xFFFFu), __NV_E4M3);
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
    const float2 r = both(mul2(mul2(f2(f.x, f.y), s2), by));
    v[j / 8][j % 8] = r.x;
    v[j / 8][j % 8 + 1] = r.y;
  }
  if (col + kCols <= a.d && on32(out + col)) {
    if constexpr (sizeof(OT) == 4) {
      store_v8(out + col, v[0]);
      store_v8(out + col + 8, v[1]);
    } else {
      uint32_t w[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) w[k] = two_of<OT>(v[k / 4][2 * k % 8], v[k / 4][2 * k % 8 + 1]);
      store_v8(static_cast<void*>(out + col), w);
    }
    return;
  }
  store_cols<OT, ON16>(out, col, a.d, v[0]);
  store_cols<OT, ON16>(out, col + 8, a.d, v[1]);
}
template <class OT>
cudaError_t launch_look(Fp8Lookup a, cudaStream_t st) {
  a.spans = (a.d + 32 * kCols - 1) / (32 * kCols);
  const int64_t items = a.n * a.spans;
  const dim3 grid((unsigned)((items + kLookThreads / 32 - 1) / (kLookThreads / 32)));
  return on16(a.out, a.ld_out, (int)sizeof(OT))
             ? launch_pdl(fp8_lookup_kernel<OT, true>, grid, dim3(kLookThreads), 0, st, a)
             : launch_pdl(fp8_lookup_kernel<OT, false>, grid, dim3(kLookThreads), 0, st, a);
}

}  // namespace

cudaError_t launch_fp8_quant(Fp8Quant a, int x_type, cudaStream_t st) {
  a.aligned = ((uintptr_t)a.x & 31) == 0 && (a.ld_x * type_size(x_type) & 31) == 0;
  if (x_type == TAB_FP32) return launch_quant<float>(a, st);
  if (x_type == TAB_BF16) return launch_quant<__nv_bfloat16>(a, st);
  return launch_quant<__half>(a, st);
}

cudaError_t launch_fp8_lookup(const Fp8Lookup& a, int out_type, cudaStream_t st) {
  if (out_type == TAB_FP32) return launch_look<float>(a, st);
  if (out_type == TAB_BF16) return launch_look<__nv_bfloat16>(a, st);
  return launch_look<__half>(a, st);
}

}  // namespace sph
