// Product of hidden states and the kept rows of a table held in 4 bits:
//
//   y[r, j] = sum_c X[r, c] * W[ids[j], c] (+ bias[ids[j]])
//
// with X the sum of `planes` terms in the table's own format (k_mx4.cu).  Both
// operands go to the tensor cores in 4 bits with their block scales
// (tcgen05.mma kind::mxf4nvf4): W's rows are the MMA's M = 128, the hidden
// states its N, and the terms of X add into the same accumulator, so a term
// costs its MMAs and no traffic of W.
//
// A CTA keeps a ring of stages of 256 columns, 128 bytes of codes a row, filled
// by three producers: W's codes by TMA, whole boxes where the kept ids are
// consecutive and four gathered rows a copy elsewhere; X's codes and scales by
// TMA; W's scales by four warps, which spread a row's 16 (8) bytes over the
// chunks that tcgen05.cp takes to tensor memory.  One warp issues the MMAs, four
// read the accumulator (double-buffered in tensor memory) and store.
#include <cuda.h>
#include <cuda_bf16.h>

#include <mutex>
#include <type_traits>

#include "mx4.cuh"
#include "sm100_ptx.cuh"
#include "sph_internal.h"

namespace sph {
namespace {

constexpr int kM = 128;                  // table rows of a tile
constexpr int kCols = 256;               // columns of a stage: 128 bytes of codes
constexpr int kABytes = kM * kCols / 2;
constexpr int kThreads = 384;            // 12 warps
constexpr int kWarpW = 0, kWarpMma = 1, kWarpX = 2, kWarpScale = 4, kWarpOut = 8;
constexpr int kMaxStages = 12;
constexpr int kSmemMax = 227 * 1024;
constexpr int kBarBytes = 1024;
constexpr uint32_t kTmemCols = 512;
constexpr long long kDrainCycles = 1ll << 20;

// groups of four scale bytes a stage and row, one chunk of 512 bytes each per 128 rows
__host__ __device__ constexpr int groups_of(int fmt) { return fmt == MX4_E4M3 ? 4 : 2; }

// ---- instructions ------------------------------------------------------------
// Descriptor of a scale chunk: 32 rows of 16 bytes, unswizzled, 8-row groups
// 128 bytes apart.
constexpr uint32_t kChunkDescHi = (128u >> 4) | (1u << 14);
__device__ __forceinline__ uint32_t chunk_desc(uint32_t saddr) { return (saddr >> 4) | (8u << 16); }
// Chunk to four columns of tensor memory, the same in each quarter of the lanes.
__device__ __forceinline__ void copy_scales(uint32_t taddr, uint32_t desc) {
  asm volatile(
      "{\n .reg .pred q;\n .reg .b64 d;\n elect.sync _|q, 0xFFFFFFFF;\n mov.b64 d, {%1, %2};\n"
      " @q tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], d;\n}\n" ::"r"(taddr),
      "r"(desc), "r"(kChunkDescHi)
      : "memory");
}
// e2m1 operands, K-major, fp32 accumulator: N, M / 16, and the scales' format
// (bit 23: e8m0).  With 32-column blocks an MMA's two scales are the low or the
// high half of a scale word (the ids in bits 4 and 29).
template <int FMT>
__host__ __device__ constexpr uint32_t idesc_mx4(int N, int half) {
  return (1u << 7) | (1u << 10) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(kM >> 4) << 24) |
         (FMT == MX4_E8M0 ? 1u << 23 : 0u) | ((uint32_t)(2 * half) << 4) |
         ((uint32_t)(2 * half) << 29);
}
template <int FMT>
__device__ __forceinline__ void mma_mx4(uint32_t d, uint32_t adesc, uint32_t bdesc, uint32_t idesc,
                                        uint32_t sfa, uint32_t sfb, uint32_t accumulate) {
  if constexpr (FMT == MX4_E4M3) {
    asm volatile(
        "{\n .reg .pred p, q;\n .reg .b64 a, b;\n elect.sync _|q, 0xFFFFFFFF;\n"
        " setp.ne.b32 p, %4, 0;\n mov.b64 a, {%1, %5};\n mov.b64 b, {%2, %5};\n"
        " @q tcgen05.mma.cta_group::1.kind::mxf4nvf4.block_scale.scale_vec::4X"
        " [%0], a, b, %3, [%6], [%7], p;\n}\n" ::"r"(d),
        "r"(adesc), "r"(bdesc), "r"(idesc), "r"(accumulate), "r"(ptx::kSdescHi), "r"(sfa), "r"(sfb)
        : "memory");
  } else {
    asm volatile(
        "{\n .reg .pred p, q;\n .reg .b64 a, b;\n elect.sync _|q, 0xFFFFFFFF;\n"
        " setp.ne.b32 p, %4, 0;\n mov.b64 a, {%1, %5};\n mov.b64 b, {%2, %5};\n"
        " @q tcgen05.mma.cta_group::1.kind::mxf4nvf4.block_scale.scale_vec::2X"
        " [%0], a, b, %3, [%6], [%7], p;\n}\n" ::"r"(d),
        "r"(adesc), "r"(bdesc), "r"(idesc), "r"(accumulate), "r"(ptx::kSdescHi), "r"(sfa), "r"(sfb)
        : "memory");
  }
}
__device__ __forceinline__ void tma_gather4(void* dst, const CUtensorMap* map, int x, int4 rows,
                                            uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cluster.global.tile::gather4.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%2, %3, %4, %5, %6}], [%7];" ::"r"(ptx::smem_u32(dst)),
      "l"(map), "r"(x), "r"(rows.x), "r"(rows.y), "r"(rows.z), "r"(rows.w), "r"(ptx::smem_u32(bar))
      : "memory");
}
__device__ __forceinline__ void bulk_load(void* dst, const void* src, uint32_t bytes, uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(
          ptx::smem_u32(dst)),
      "l"(src), "r"(bytes), "r"(ptx::smem_u32(bar))
      : "memory");
}

struct Params {
  Mx4Gemm g;
  const uint8_t* x_scales;      // [plane][row tile][group][chunk][512]
  int64_t x_scale_plane;        // bytes
  const float* x_row;           // [row tiles * bn], e4m3 only
  int bn, row_tiles, tiles, kt; // row tiles are the fast index of a tile
  int stages, stage_bytes, chunks, sf_col;
  long long spin_limit;
};

template <int FMT, bool GATHER, class OT>
__global__ void __launch_bounds__(kThreads, 1)
mx4_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_row,
           const __grid_constant__ CUtensorMap map_x, const Params p) {
  constexpr int kGroups = groups_of(FMT);
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = ptx::smem_u32(smem_raw);
  uint8_t* base = smem_raw + (((raw + 1023) & ~1023u) - raw);
  uint64_t* full = reinterpret_cast<uint64_t*>(base + (size_t)p.stages * p.stage_bytes);
  uint64_t* empty = full + kMaxStages;
  uint64_t* acc_full = empty + kMaxStages;      // [2]
  uint64_t* acc_empty = acc_full + 2;           // [2]
  uint32_t* holder = reinterpret_cast<uint32_t*>(acc_empty + 2);
  volatile int* s_abort = reinterpret_cast<volatile int*>(holder + 1);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const Mx4Gemm& g = p.g;
  // a stage: W codes, X codes (a term after the other), W scales, X scales
  const int x_bytes = p.bn * (kCols / 2);
  const int xs_bytes = kGroups * p.chunks * 512;
  const int off_ws = kABytes + g.planes * x_bytes, off_xs = off_ws + kGroups * 512;

  if (threadIdx.x == 0) {
    for (int s = 0; s < p.stages; ++s) {
      ptx::mbar_init(&full[s], 1 + 1 + 4);      // W codes, X, the four scale warps
      ptx::mbar_init(&empty[s], 1);
    }
    for (int a = 0; a < 2; ++a) {
      ptx::mbar_init(&acc_full[a], 1);
      ptx::mbar_init(&acc_empty[a], 4);
    }
    *s_abort = 0;
    ptx::fence_mbar_init();
  }
  if (warp == kWarpMma) ptx::tmem_alloc(holder, kTmemCols);
  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
  const uint32_t tmem = *holder;
  // (after the allocation, so that no later kernel's CTA takes the tensor memory first)
  ptx::griddep_launch_dependents();

  // A wait that gives up after spin_limit cycles, or once another warp has; the
  // whole warp gets one answer.
  auto wait = [&](uint64_t* bar, uint32_t parity) {
    bool ok = ptx::mbar_try_wait(bar, parity);
    if (!ok) {
      const long long t0 = clock64();
      while (!(ok = ptx::mbar_try_wait(bar, parity))) {
        if (*s_abort) break;
        if (clock64() - t0 > p.spin_limit) {
          atomicOr(g.status, ERR_TIMEOUT);
          *s_abort = 1;
          break;
        }
      }
    }
    return __all_sync(0xFFFFFFFFu, ok) != 0;
  };
  int stage = 0;
  uint32_t phase = 0;
  auto advance = [&] {
    if (++stage == p.stages) { stage = 0; phase ^= 1; }
  };

  if (warp == kWarpW) {
    // ---- W codes -----------------------------------------------------------
    bool ok = true;
    for (int tile = blockIdx.x; ok && tile < p.tiles; tile += gridDim.x) {
      const int j0 = tile / p.row_tiles * kM;
      int4 id;                                   // of rows 4 lane .. 4 lane + 3
      unsigned solid = 0;                        // which 32-row groups are consecutive ids
      if constexpr (GATHER) {
        // rows past the last kept id repeat it
        const int j = j0 + 4 * lane, last = g.n - 1;
        id = make_int4(g.ids[min(j, last)], g.ids[min(j + 1, last)], g.ids[min(j + 2, last)],
                       g.ids[min(j + 3, last)]);
        const bool own = id.y == id.x + 1 && id.z == id.x + 2 && id.w == id.x + 3;
        const int next = __shfl_down_sync(0xFFFFFFFFu, id.x, 1);
        const unsigned four = __ballot_sync(0xFFFFFFFFu, own);
        const unsigned link = __ballot_sync(0xFFFFFFFFu, next == id.w + 1);
#pragma unroll
        for (int q = 0; q < 4; ++q)
          if ((four >> 8 * q & 0xFFu) == 0xFFu && (link >> 8 * q & 0x7Fu) == 0x7Fu) solid |= 1u << q;
      }
      for (int k = 0; k < p.kt; ++k) {
        if (!wait(&empty[stage], phase ^ 1)) { ok = false; break; }
        uint8_t* a = base + (size_t)stage * p.stage_bytes;
        if (lane == 0) ptx::mbar_expect_tx(&full[stage], kABytes);
        __syncwarp();
        if constexpr (GATHER) {
          if (solid >> (lane >> 3) & 1) {
            if ((lane & 7) == 0)
              ptx::tma_load_2d(a + lane * 512, &map_w, k * (kCols / 2), id.x, &full[stage]);
          } else {
            tma_gather4(a + lane * 512, &map_row, k * (kCols / 2), id, &full[stage]);
          }
        } else if (lane == 0) {
          ptx::tma_load_2d(a, &map_w, k * (kCols / 2), j0, &full[stage]);
        }
        advance();
      }
    }
  } else if (warp == kWarpX) {
    // ---- X codes and scales ------------------------------------------------
    ptx::griddep_wait();
    bool ok = true;
    for (int tile = blockIdx.x; ok && tile < p.tiles; tile += gridDim.x) {
      const int rt = tile % p.row_tiles;
      for (int k = 0; k < p.kt; ++k) {
        if (!wait(&empty[stage], phase ^ 1)) { ok = false; break; }
        if (lane == 0) {
          uint8_t* s = base + (size_t)stage * p.stage_bytes;
          ptx::mbar_expect_tx(&full[stage], (uint32_t)(g.planes * (x_bytes + xs_bytes)));
          for (int q = 0; q < g.planes; ++q) {
            ptx::tma_load_3d(s + kABytes + q * x_bytes, &map_x, k * (kCols / 2), rt * p.bn, q,
                             &full[stage]);
            bulk_load(s + off_xs + q * xs_bytes,
                      p.x_scales + q * p.x_scale_plane + ((int64_t)rt * p.kt + k) * xs_bytes,
                      (uint32_t)xs_bytes, &full[stage]);
          }
        }
        __syncwarp();
        advance();
      }
    }
  } else if (warp == kWarpMma) {
    // ---- MMA ---------------------------------------------------------------
    const uint32_t sfa = tmem + p.sf_col, sfb = sfa + 4 * kGroups;
    bool ok = true;
    int acc = 0;
    uint32_t acc_phase = 0;
    for (int tile = blockIdx.x; ok && tile < p.tiles; tile += gridDim.x) {
      if (!wait(&acc_empty[acc], acc_phase ^ 1)) break;
      ptx::tc_fence_after();
      const uint32_t d = tmem + acc * p.bn;
      for (int k = 0; k < p.kt; ++k) {
        if (!wait(&full[stage], phase)) { ok = false; break; }
        ptx::tc_fence_after();
        const uint32_t s = ptx::smem_u32(base) + stage * p.stage_bytes;
        // steps of 64 columns, none past the last column
        const int steps = min(4, (g.d - k * kCols + 63) / 64);
#pragma unroll
        for (int q = 0; q < kGroups; ++q)
          copy_scales(sfa + 4 * q, chunk_desc(s + off_ws + q * 512));
        for (int t = 0; t < g.planes; ++t) {
          const uint32_t sft = sfb + t * kGroups * p.chunks * 4;
          for (int q = 0; q < kGroups * p.chunks; ++q)
            copy_scales(sft + 4 * q, chunk_desc(s + off_xs + t * xs_bytes + q * 512));
          const uint32_t ad = ptx::sdesc_k128(s), bd = ptx::sdesc_k128(s + kABytes + t * x_bytes);
          for (int j = 0; j < steps; ++j) {
            const int q = FMT == MX4_E4M3 ? j : j / 2;
            mma_mx4<FMT>(d, ad + 2 * j, bd + 2 * j,
                         idesc_mx4<FMT>(p.bn, FMT == MX4_E4M3 ? 0 : j % 2), sfa + 4 * q,
                         sft + 4 * q * p.chunks, k > 0 || t > 0 || j > 0);
          }
        }
        ptx::umma_commit(&empty[stage]);
        advance();
      }
      if (!ok) break;
      ptx::umma_commit(&acc_full[acc]);
      acc ^= 1;
      if (acc == 0) acc_phase ^= 1;
    }
  } else if (warp >= kWarpScale && warp < kWarpScale + 4) {
    // ---- W scales ------------------------------------------------------------
    // Thread r holds table row r of the tile; the bytes of four stages are on
    // their way in registers.
    using Word = typename std::conditional<FMT == MX4_E4M3, uint4, uint2>::type;
    constexpr int kBytes = (int)sizeof(Word);
    const int r = threadIdx.x - kWarpScale * 32;
    const int bytes = (g.d + Mx4<FMT>::kBlock - 1) / Mx4<FMT>::kBlock;
    int f_tile = blockIdx.x, f_k = 0;            // what is fetched next
    const uint8_t* f_row = nullptr;
    const uint8_t* n_row = nullptr;              // the row of the tile after it
    auto row_of = [&](int tile) -> const uint8_t* {
      const int j = tile / p.row_tiles * kM + r;
      if (tile >= p.tiles || j >= g.n) return nullptr;
      return g.w_scales + (int64_t)(GATHER ? g.ids[j] : j) * g.ld_scales;
    };
    f_row = row_of(f_tile);
    n_row = row_of(f_tile + gridDim.x);
    auto fetch = [&]() -> Word {
      Word w{};
      const int at = f_k * kBytes;
      if (f_row && at < bytes) {
        w = *reinterpret_cast<const Word*>(f_row + at);
        if (at + kBytes > bytes) {               // bytes past the row's last scale
          uint32_t* e = reinterpret_cast<uint32_t*>(&w);
#pragma unroll
          for (int i = 0; i < kGroups; ++i) {
            const int left = bytes - at - 4 * i;
            if (left < 4) e[i] = left <= 0 ? 0u : e[i] & ((1u << 8 * left) - 1);
          }
        }
      }
      if (++f_k == p.kt) {
        f_k = 0;
        f_tile += gridDim.x;
        f_row = n_row;
        n_row = row_of(f_tile + gridDim.x);
      }
      return w;
    };
    Word w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = fetch();
    const int mine = p.tiles > (int)blockIdx.x ? (p.tiles - 1 - blockIdx.x) / gridDim.x + 1 : 0;
    const int total = mine * p.kt;
    bool ok = true;
    for (int it = 0; ok && it < total; it += 4) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (!ok || it + i >= total) break;
        if (!wait(&empty[stage], phase ^ 1)) { ok = false; break; }
        uint8_t* dst = base + (size_t)stage * p.stage_bytes + off_ws + (r & 31) * 16 + (r >> 5) * 4;
        const uint32_t* e = reinterpret_cast<const uint32_t*>(&w[i]);
#pragma unroll
        for (int q = 0; q < kGroups; ++q) *reinterpret_cast<uint32_t*>(dst + q * 512) = e[q];
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(&full[stage]);
        w[i] = fetch();
        advance();
      }
    }
  } else if (warp >= kWarpOut) {
    // ---- accumulator to y ----------------------------------------------------
    const int quarter = warp - kWarpOut;         // (warp % 4: the lanes it may read)
    ptx::griddep_wait();
    int acc = 0;
    uint32_t acc_phase = 0;
    for (int tile = blockIdx.x; tile < p.tiles; tile += gridDim.x) {
      const int r0 = tile % p.row_tiles * p.bn, rows = min(p.bn, g.rows - r0);
      const int j = tile / p.row_tiles * kM + quarter * 32 + lane;
      const bool live = j < g.n;
      float ws = 1.f, b = 0.f;
      if (live) {
        const int64_t id = GATHER ? g.ids[j] : j;
        if constexpr (FMT == MX4_E4M3) ws = g.w_row[id];
        if (g.bias) b = g.bias[id];
      }
      if (!wait(&acc_full[acc], acc_phase)) break;
      ptx::tc_fence_after();
      const uint32_t t = tmem + acc * p.bn + ((uint32_t)(quarter * 32) << 16);
      OT* y = static_cast<OT*>(g.out) + (int64_t)r0 * g.ld_out + j;
      for (int c = 0; c < rows; c += 16) {
        float v[16];
        ptx::tmem_ld16(t + c, v);
        const int m = min(16, rows - c);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          float x = v[i] * ws;
          if constexpr (FMT == MX4_E4M3) x *= p.x_row[r0 + c + i];
          x += b;
          if (live && i < m) {
            if constexpr (sizeof(OT) == 4) y[(int64_t)(c + i) * g.ld_out] = x;
            else y[(int64_t)(c + i) * g.ld_out] = __float2bfloat16_rn(x);
          }
        }
      }
      ptx::tc_fence_before();
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(&acc_empty[acc]);
      acc ^= 1;
      if (acc == 0) acc_phase ^= 1;
    }
  }

  __syncwarp();
  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
  if (*s_abort) {      // copies and MMAs of the stages given up end within this
    const long long t0 = clock64();
    while (clock64() - t0 < kDrainCycles) {}
    __syncthreads();
  }
  if (warp == kWarpMma) ptx::tmem_dealloc(tmem, kTmemCols);
}

// ---------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------
using EncodeFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*,
                              const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                              const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                              CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeFn encode_fn() {
  static EncodeFn fn = nullptr;
  static std::once_flag once;
  std::call_once(once, [] {
    void* f = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault,
                                         &q) == cudaSuccess &&
        q == cudaDriverEntryPointSuccess)
      fn = reinterpret_cast<EncodeFn>(f);
  });
  return fn;
}
// Byte matrix [planes][rows][bytes a row], boxes of 128 bytes by box_rows.
bool byte_map(CUtensorMap* m, const void* ptr, uint64_t bytes, uint64_t rows, uint64_t ld,
              uint64_t planes, uint64_t plane_ld, uint32_t box_rows) {
  EncodeFn fn = encode_fn();
  if (!fn) return false;
  const cuuint64_t dims[3] = {bytes, rows, planes};
  const cuuint64_t strides[2] = {ld, plane_ld};
  const cuuint32_t box[3] = {128, box_rows, 1};
  const cuuint32_t es[3] = {1, 1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, planes ? 3 : 2, const_cast<void*>(ptr), dims, strides,
            box, es, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

size_t up256(size_t x) { return (x + 255) / 256 * 256; }

struct Plan {
  int bn, row_tiles, tiles, kt, stages, stage_bytes, chunks, sf_col;
};
int stage_bytes_of(int bn, int planes, int fmt) {
  const int chunks = (bn + 127) / 128, g = groups_of(fmt) * 512;
  return (kABytes + planes * bn * (kCols / 2) + g + planes * g * chunks + 1023) / 1024 * 1024;
}
int sf_col_of(int bn) { return (2 * bn + 31) / 32 * 32; }
// The largest tile of hidden-state rows of which three stages fit, and two
// accumulators with a stage's scales; then as many equal tiles as the rows need.
Plan plan_of(int64_t rows, int64_t n, int d, int planes, int fmt) {
  Plan pl{};
  int most = 16;
  for (int bn = 16; bn <= 256; bn += 16) {
    const int cols = sf_col_of(bn) + 4 * groups_of(fmt) * (1 + planes * ((bn + 127) / 128));
    if (3 * stage_bytes_of(bn, planes, fmt) + 1024 + kBarBytes > kSmemMax || cols > (int)kTmemCols)
      break;
    most = bn;
  }
  const int64_t count = (rows + most - 1) / most;
  pl.bn = (int)(((rows + count - 1) / count + 15) / 16 * 16);
  pl.row_tiles = (int)((rows + pl.bn - 1) / pl.bn);
  pl.tiles = (int)((n + kM - 1) / kM) * pl.row_tiles;
  pl.kt = (d + kCols - 1) / kCols;
  pl.stage_bytes = stage_bytes_of(pl.bn, planes, fmt);
  pl.stages = (kSmemMax - 1024 - kBarBytes) / pl.stage_bytes;
  if (pl.stages > kMaxStages) pl.stages = kMaxStages;
  pl.chunks = (pl.bn + 127) / 128;
  pl.sf_col = sf_col_of(pl.bn);
  return pl;
}

struct Operand {        // X in scratch
  int64_t ld, plane, scale_plane;
  size_t scales, row, bytes;
};
Operand operand_of(const Plan& pl, int64_t rows, int d, int planes, int fmt) {
  Operand o{};
  o.ld = (d + 31) / 32 * 16;
  o.plane = (int64_t)up256((size_t)(rows * o.ld));
  o.scale_plane = (int64_t)pl.row_tiles * pl.kt * groups_of(fmt) * pl.chunks * 512;
  o.scales = (size_t)(planes * o.plane);
  o.row = o.scales + (size_t)(planes * o.scale_plane);
  o.bytes = o.row + up256((size_t)pl.row_tiles * pl.bn * 4);
  return o;
}

template <int FMT, bool GATHER, class OT>
cudaError_t launch(const CUtensorMap& w, const CUtensorMap& row, const CUtensorMap& x,
                   const Params& p, int sm_count, cudaStream_t st) {
  const size_t smem = (size_t)p.stages * p.stage_bytes + 1024 + kBarBytes;
  cudaError_t e = cudaFuncSetAttribute(mx4_kernel<FMT, GATHER, OT>,
                                       cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemMax);
  if (e != cudaSuccess) return e;
  const int grid = p.tiles < sm_count ? p.tiles : sm_count;
  return launch_pdl(mx4_kernel<FMT, GATHER, OT>, dim3((unsigned)grid), dim3(kThreads), smem, st, w,
                    row, x, p);
}
template <int FMT, bool GATHER>
cudaError_t launch_o(const CUtensorMap& w, const CUtensorMap& row, const CUtensorMap& x,
                     const Params& p, int sm_count, cudaStream_t st) {
  return p.g.out_type == TAB_FP32 ? launch<FMT, GATHER, float>(w, row, x, p, sm_count, st)
                                  : launch<FMT, GATHER, __nv_bfloat16>(w, row, x, p, sm_count, st);
}

}  // namespace

size_t mx4_gemm_scratch_bytes(int64_t rows, int64_t n, int d, int planes, int fmt) {
  const Plan pl = plan_of(rows, n, d, planes, fmt);
  return operand_of(pl, rows, d, planes, fmt).bytes;
}

// At least what any call of up to `rows` rows and d columns takes: tiles of more
// rows than one has are at least 48 of 128 rows' scale chunks.
size_t mx4_gemm_reserve_bytes(int64_t rows, int64_t d) {
  const size_t r = (size_t)rows, padded = 3 * r + 256, kt = (size_t)((d + kCols - 1) / kCols);
  return 4 * (up256(r * ((size_t)(d + 31) / 32 * 16)) + padded * kt * groups_of(MX4_E4M3) * 4) +
         up256(padded * 4);
}

cudaError_t launch_mx4_gemm(const Mx4Gemm& g, void* scratch, long long spin_limit, int sm_count,
                            cudaStream_t st) {
  const Plan pl = plan_of(g.rows, g.n, g.d, g.planes, g.fmt);
  const Operand o = operand_of(pl, g.rows, g.d, g.planes, g.fmt);
  char* at = static_cast<char*>(scratch);
  Params p{};
  p.g = g;
  p.x_scales = reinterpret_cast<uint8_t*>(at + o.scales);
  p.x_scale_plane = o.scale_plane;
  p.x_row = reinterpret_cast<float*>(at + o.row);
  p.bn = pl.bn; p.row_tiles = pl.row_tiles; p.tiles = pl.tiles; p.kt = pl.kt;
  p.stages = pl.stages; p.stage_bytes = pl.stage_bytes; p.chunks = pl.chunks; p.sf_col = pl.sf_col;
  p.spin_limit = spin_limit;
  CUtensorMap mw, mr, mx;
  const uint64_t bytes = (uint64_t)(g.d + 31) / 32 * 16;
  if (!byte_map(&mx, at, bytes, (uint64_t)g.rows, (uint64_t)o.ld, (uint64_t)g.planes,
                (uint64_t)o.plane, (uint32_t)pl.bn) ||
      !byte_map(&mw, g.w_codes, bytes, (uint64_t)g.V, (uint64_t)g.ld_codes, 0, 0,
                g.ids ? 32 : kM))
    return cudaErrorInvalidValue;
  mr = mw;
  if (g.ids && !byte_map(&mr, g.w_codes, bytes, (uint64_t)g.V, (uint64_t)g.ld_codes, 0, 0, 1))
    return cudaErrorInvalidValue;

  Mx4Quant q{};
  q.x = g.x; q.ld_x = g.ld_x; q.rows = g.rows; q.d = g.d;
  q.codes = reinterpret_cast<uint8_t*>(at); q.ld_codes = o.ld; q.plane_codes = o.plane;
  q.scales = reinterpret_cast<uint8_t*>(at + o.scales); q.plane_scales = o.scale_plane;
  q.row_scale = g.fmt == MX4_E4M3 ? reinterpret_cast<float*>(at + o.row) : nullptr;
  q.planes = g.planes; q.scale_cols = pl.kt * kCols;
  q.tile_rows = pl.bn; q.groups = pl.kt * groups_of(g.fmt);
  cudaError_t e = launch_mx4_quant(q, g.fmt, g.x_type, true, st);
  if (e != cudaSuccess) return e;
  if (g.fmt == MX4_E4M3)
    return g.ids ? launch_o<MX4_E4M3, true>(mw, mr, mx, p, sm_count, st)
                 : launch_o<MX4_E4M3, false>(mw, mr, mx, p, sm_count, st);
  return g.ids ? launch_o<MX4_E8M0, true>(mw, mr, mx, p, sm_count, st)
               : launch_o<MX4_E8M0, false>(mw, mr, mx, p, sm_count, st);
}

}  // namespace sph
