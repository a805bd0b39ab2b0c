// Product of hidden states and the kept rows of a table in e4m3 with a scale for each block
// of 128 columns:
//
//   y[r, j] = sum over blocks b of sx[r, b] * sw[id_j, b] * (qx[r, b] . qw[id_j, b])  (+ bias)
//
// where qx, sx are the hidden states in the same form, a scale for each row and block
// (k_fp8.cu).  W's rows are the MMA's M = 128, the hidden states its N; a stage is one block:
// 128 columns, a 128-byte row of codes.
//
// The scales differ from block to block and are no powers of two, so a block's sums leave
// the tensor core before they are scaled: the MMA warp fills two accumulators in tensor
// memory in turn, one block each, and eight warps (four for few rows) read the one that is
// full and add it, scaled, to sums in their registers: a multiplication and a fused
// multiply-add a value, two values an instruction.
#include <cuda.h>
#include <cuda_bf16.h>

#include <mutex>
#include <type_traits>

#include "fp8.cuh"
#include "sm100_ptx.cuh"
#include "sph_internal.h"

namespace sph {
namespace {

constexpr int kM = 128;                  // table rows of a tile (of a CTA)
constexpr int kABytes = kM * kFp8Block;
constexpr int kThreads = 384;            // 12 warps
constexpr int kWarpW = 0, kWarpMma = 1, kWarpX = 2, kWarpOut = 4;
constexpr int kMaxStages = 12;
constexpr int kMaxBn = 192;              // hidden-state rows of a tile
constexpr int kAccCols = 256;            // columns of an accumulator
constexpr int kSxSlots = 8, kSxRow = 256;
constexpr int kSmemMax = 227 * 1024;
constexpr int kBarBytes = 1024;
constexpr int kExtraBytes = 1024 + kBarBytes + kSxSlots * kSxRow * 4;   // beside the stages
constexpr uint32_t kTmemCols = 512;
constexpr long long kDrainCycles = 1ll << 20;

// ---- instructions ------------------------------------------------------------
__device__ __forceinline__ uint64_t pack2(float a, float b) {
  return (uint64_t)__float_as_uint(b) << 32 | __float_as_uint(a);
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}
// Four rows by one copy, to a pair (bar: a shared::cluster address).
__device__ __forceinline__ void tma_gather4(void* dst, const CUtensorMap* map, int x, int4 rows,
                                            uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile::gather4"
      ".mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5, %6}], [%7];" ::"r"(
          ptx::smem_u32(dst)),
      "l"(map), "r"(x), "r"(rows.x), "r"(rows.y), "r"(rows.z), "r"(rows.w), "r"(bar)
      : "memory");
}
__device__ __forceinline__ void bulk_load(void* dst, const void* src, uint32_t bytes, uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(
          ptx::smem_u32(dst)),
      "l"(src), "r"(bytes), "r"(ptx::smem_u32(bar))
      : "memory");
}
// Arrivals at a barrier of either CTA of a pair (a shared::cluster address); what they
// announce was read from tensor memory or comes by TMA.
__device__ __forceinline__ void arrive_at(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void expect_at(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cluster.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes)
               : "memory");
}
__device__ __forceinline__ void store_value(float* p, float v) { *p = v; }
__device__ __forceinline__ void store_value(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }

struct Params {
  Fp8Gemm g;
  const float* x_scales;        // [block][row tiles * bn]
  int64_t ld_xs;
  int bn, row_tiles, tiles, kt; // row tiles are the fast index of a tile
  int stages, stage_bytes;
  long long spin_limit;
};

// NC columns of an accumulator a thread, in `H` groups of four warps.
template <int NC, int H, bool PAIR>
__global__ void __launch_bounds__(kThreads, 1)
fp8_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_row,
           const __grid_constant__ CUtensorMap map_x, const Params p) {
  constexpr int kHalves = PAIR ? 2 : 1;         // CTAs of a unit, 128 table rows each
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw_addr = ptx::smem_u32(smem_raw);
  const uint32_t base_addr = (raw_addr + 1023) & ~1023u;
  uint8_t* base = smem_raw + (base_addr - raw_addr);
  uint64_t* full = reinterpret_cast<uint64_t*>(base + (size_t)p.stages * p.stage_bytes);
  uint64_t* empty = full + kMaxStages;
  uint64_t* acc_full = empty + kMaxStages;      // [2]
  uint64_t* acc_empty = acc_full + 2;           // [2]
  uint64_t* sx_full = acc_empty + 2;            // [kSxSlots]
  uint64_t* sx_empty = sx_full + kSxSlots;      // [kSxSlots]
  uint32_t* holder = reinterpret_cast<uint32_t*>(sx_empty + kSxSlots);
  volatile int* s_abort = reinterpret_cast<volatile int*>(holder + 1);
  float* sx_ring = reinterpret_cast<float*>(base + (size_t)p.stages * p.stage_bytes + kBarBytes);
  // (from lane 0, so that the compiler knows that a warp takes one branch and can
  // keep its loop's counters and descriptors in uniform registers)
  const int warp = __shfl_sync(0xFFFFFFFFu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  const Fp8Gemm& g = p.g;
  const int half = PAIR ? __shfl_sync(0xFFFFFFFFu, (int)ptx::cluster_ctarank(), 0) : 0;
  const int unit = (int)blockIdx.x / kHalves, units = (int)gridDim.x / kHalves;
  const bool gather = g.ids != nullptr;
  const bool pieces = gather && !PAIR;          // scattered rows by cp.async
  const int bnc = p.bn / kHalves;               // rows of X's codes in this CTA
  const int x_bytes = bnc * kFp8Block;

  if (threadIdx.x == 0) {
    for (int s = 0; s < p.stages; ++s) {
      // W and X codes of each CTA, scattered rows of W
      ptx::mbar_init(&full[s], 2 * kHalves + (pieces ? 32 : 0));
      ptx::mbar_init(&empty[s], 1);
    }
    for (int a = 0; a < 2; ++a) {
      ptx::mbar_init(&acc_full[a], 1);
      ptx::mbar_init(&acc_empty[a], 4 * H * kHalves);
    }
    for (int s = 0; s < kSxSlots; ++s) {
      ptx::mbar_init(&sx_full[s], 1);
      ptx::mbar_init(&sx_empty[s], 4 * H);
    }
    *s_abort = 0;
    ptx::fence_mbar_init();
  }
  if (warp == kWarpMma) {
    if constexpr (PAIR) ptx::tmem_alloc_pair(holder, kTmemCols);
    else ptx::tmem_alloc(holder, kTmemCols);
  }
  ptx::tc_fence_before();
  if constexpr (PAIR) ptx::cluster_sync();
  else __syncthreads();
  ptx::tc_fence_after();
  const uint32_t tmem = __shfl_sync(0xFFFFFFFFu, *holder, 0);
  // (after the allocation, so that no later kernel's CTA takes the tensor memory first)
  ptx::griddep_launch_dependents();

  // A wait that gives up after spin_limit cycles, or once another warp has; the
  // whole warp gets one answer.  at_once: asked first without suspension, so that a limit
  // of a cycle or two runs out where the phase is not complete yet.
  auto wait = [&](uint64_t* bar, uint32_t parity, bool at_once = false) {
    if (__all_sync(0xFFFFFFFFu,
                   at_once ? ptx::mbar_test(bar, parity) : ptx::mbar_try_wait(bar, parity)))
      return true;
    const long long t0 = clock64();
    do {
      const bool late = clock64() - t0 > p.spin_limit;
      if (__any_sync(0xFFFFFFFFu, late || *s_abort)) {
        if (late) atomicOr(g.status, ERR_TIMEOUT);
        *s_abort = 1;
        return false;
      }
    } while (!__all_sync(0xFFFFFFFFu, ptx::mbar_try_wait(bar, parity)));
    return true;
  };
  // the even CTA's barrier, which the MMA warp waits on
  auto leader = [&](uint64_t* bar) {
    return PAIR ? ptx::mapa(ptx::smem_u32(bar), 0) : ptx::smem_u32(bar);
  };
  auto arrive = [&](uint64_t* bar) {
    if constexpr (PAIR) arrive_at(leader(bar));
    else ptx::mbar_arrive(bar);
  };
  auto expect = [&](uint64_t* bar, uint32_t bytes) {
    if constexpr (PAIR) expect_at(leader(bar), bytes);
    else ptx::mbar_expect_tx(bar, bytes);
  };
  auto commit = [&](uint64_t* bar) {
    if constexpr (PAIR) ptx::umma_commit_pair(bar);
    else ptx::umma_commit(bar);
  };
  // first table row (as an index into the kept ones) of a tile in this CTA
  auto first_row = [&](int tile) { return (tile / p.row_tiles * kHalves + half) * kM; };
  int stage = 0;
  uint32_t phase = 0;
  auto advance = [&] {
    if (++stage == p.stages) { stage = 0; phase ^= 1; }
  };
  bool ok = true;

  if (warp == kWarpW) {
    // ---- W codes -----------------------------------------------------------
    // Groups of 32 consecutive ids are one box.  Rows of others come as 16-byte pieces by
    // cp.async, four rows an instruction, each piece where the 128-byte swizzle has it; on
    // pairs, whose barriers wait for no generic writes (arrive_at), four rows a copy.
    for (int tile = unit; ok && tile < p.tiles; tile += units) {
      const int j0 = first_row(tile), last = g.n - 1;
      int4 id = make_int4(0, 0, 0, 0);
      unsigned solid = 0;
      // where rows lane / 8, lane / 8 + 4, ... begin (ids outside the table, which are the
      // caller's mistake, take a row of it)
      const uint8_t* from[PAIR ? 1 : 32];
      if (gather) {
        // the ids of rows 4 lane .. 4 lane + 3, rows past the last kept id repeating it, and
        // which 32-row groups are consecutive ids
        const int j = j0 + 4 * lane;
        id = make_int4(g.ids[min(j, last)], g.ids[min(j + 1, last)], g.ids[min(j + 2, last)],
                       g.ids[min(j + 3, last)]);
        const bool own = id.y == id.x + 1 && id.z == id.x + 2 && id.w == id.x + 3;
        const int next = __shfl_down_sync(0xFFFFFFFFu, id.x, 1);
        const unsigned four = __ballot_sync(0xFFFFFFFFu, own);
        const unsigned link = __ballot_sync(0xFFFFFFFFu, next == id.w + 1);
#pragma unroll
        for (int q = 0; q < 4; ++q)
          if ((four >> 8 * q & 0xFFu) == 0xFFu && (link >> 8 * q & 0x7Fu) == 0x7Fu) solid |= 1u << q;
        if constexpr (!PAIR) {
          if (solid != 0xFu) {
#pragma unroll
            for (int i = 0; i < 32; ++i) {
              const int row = g.ids[min(j0 + 4 * i + (lane >> 3), last)];
              from[i] = g.w_codes + max(0, min(row, (int)g.V - 1)) * g.ld_codes;
            }
          }
        }
      }
      for (int k = 0; k < p.kt; ++k) {
        if (!wait(&empty[stage], phase ^ 1, true)) { ok = false; break; }
        uint8_t* a = base + (size_t)stage * p.stage_bytes;
        const uint32_t bar = leader(&full[stage]);
        const int x = k * kFp8Block;
        if (lane == 0) expect(&full[stage], pieces ? __popc(solid) * (kABytes / 4) : kABytes);
        __syncwarp();
        auto box = [&](uint8_t* dst, int row) {
          if constexpr (PAIR) ptx::tma_load_2d_pair(dst, &map_w, x, row, bar);
          else ptx::tma_load_2d(dst, &map_w, x, row, &full[stage]);
        };
        if (gather) {
          if (solid >> (lane >> 3) & 1) {
            if ((lane & 7) == 0) box(a + lane * 512, id.x);
          } else if constexpr (PAIR) {
            tma_gather4(a + lane * 512, &map_row, x, id, bar);
          }
          if constexpr (!PAIR) {
            const int piece = lane & 7, row = lane >> 3;
            const int at = min(x + 16 * piece, g.d - 1) & ~15;
            const int size = max(0, min(16, g.d - (x + 16 * piece)));
            const uint32_t even = ptx::smem_u32(a) + row * 128 + (piece ^ row) * 16;
            const uint32_t odd = ptx::smem_u32(a) + row * 128 + (piece ^ (row + 4)) * 16;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              if (solid >> q & 1) continue;
#pragma unroll
              for (int i = 8 * q; i < 8 * q + 8; ++i)
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(
                                 (i % 2 ? odd : even) + i * 512),
                             "l"(from[i] + at), "r"(size)
                             : "memory");
            }
            asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(
                             ptx::smem_u32(&full[stage]))
                         : "memory");
          }
        } else if (lane == 0) {
          // (a pair's second half may lie past the last row: any rows of the table do,
          // for a box starts inside it)
          box(a, min(j0, (int)g.V - 1));
        }
        advance();
      }
    }
  } else if (warp == kWarpX) {
    // ---- X codes and scales ------------------------------------------------
    ptx::griddep_wait();
    int slot = 0;
    uint32_t slot_phase = 0;
    for (int tile = unit; ok && tile < p.tiles; tile += units) {
      const int r0 = tile % p.row_tiles * p.bn;
      for (int k = 0; k < p.kt; ++k) {
        if (!wait(&empty[stage], phase ^ 1)) { ok = false; break; }
        if (lane == 0) {
          uint8_t* s = base + (size_t)stage * p.stage_bytes + kABytes;
          expect(&full[stage], (uint32_t)x_bytes);
          if constexpr (PAIR)
            ptx::tma_load_2d_pair(s, &map_x, k * kFp8Block, r0 + half * bnc, leader(&full[stage]));
          else
            ptx::tma_load_2d(s, &map_x, k * kFp8Block, r0, &full[stage]);
        }
        __syncwarp();
        if (!wait(&sx_empty[slot], slot_phase ^ 1)) { ok = false; break; }
        if (lane == 0) {
          ptx::mbar_expect_tx(&sx_full[slot], (uint32_t)p.bn * 4);
          bulk_load(sx_ring + slot * kSxRow, p.x_scales + (int64_t)k * p.ld_xs + r0,
                    (uint32_t)p.bn * 4, &sx_full[slot]);
        }
        __syncwarp();
        if (++slot == kSxSlots) { slot = 0; slot_phase ^= 1; }
        advance();
      }
    }
  } else if (warp == kWarpMma && half == 0) {
    // ---- MMA ---------------------------------------------------------------
    int acc = 0;
    uint32_t acc_phase = 0;
    const uint32_t idesc = ptx::idesc_e4m3_f32(kHalves * kM, p.bn);
    for (int tile = unit; ok && tile < p.tiles; tile += units) {
      for (int k = 0; k < p.kt; ++k) {
        if (!wait(&acc_empty[acc], acc_phase ^ 1) || !wait(&full[stage], phase)) { ok = false; break; }
        // (what cp.async wrote is there for the MMAs' reads)
        if (pieces) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        ptx::tc_fence_after();
        const uint32_t s = base_addr + stage * p.stage_bytes, d = tmem + acc * kAccCols;
        const uint32_t ad = ptx::sdesc_k128(s), bd = ptx::sdesc_k128(s + kABytes);
        // steps of 32 columns, none past the last column
        const int steps = min(4, (g.d - k * kFp8Block + 31) / 32);
        for (int j = 0; j < steps; ++j) {
          if constexpr (PAIR) ptx::umma_f8_pair(d, ad + 2 * j, bd + 2 * j, idesc, j > 0);
          else ptx::umma_f8(d, ad + 2 * j, bd + 2 * j, idesc, j > 0);
        }
        commit(&empty[stage]);
        commit(&acc_full[acc]);
        advance();
        if (++acc == 2) { acc = 0; acc_phase ^= 1; }
      }
    }
  } else if (warp >= kWarpOut && warp < kWarpOut + 4 * H) {
    // ---- accumulators to sums, sums to y -------------------------------------
    constexpr int G = NC < 32 ? NC : 32;         // columns a load
    const int quarter = warp & 3;                // (the lanes that a warp may read)
    const int col0 = (warp - kWarpOut) / 4 * NC; // the warp's first column
    ptx::griddep_wait();
    int acc = 0, slot = 0;
    uint32_t acc_phase = 0, slot_phase = 0;
    const int groups = max(0, min(NC / G, (p.bn - col0 + G - 1) / G));
    for (int tile = unit; ok && tile < p.tiles; tile += units) {
      const int r0 = tile % p.row_tiles * p.bn, rows = min(p.bn, g.rows - r0);
      const int j = first_row(tile) + quarter * 32 + lane;
      const bool live = j < g.n;
      int64_t id = !live ? -1 : gather ? g.ids[j] : j;
      const bool there = id >= 0 && id < g.V;
      const float* ws = g.w_scales + (there ? id / g.block_rows : 0) * g.ld_scales;
      const float b = there && g.bias ? g.bias[id] : 0.f;
      float next = ws[0];
      uint64_t sum[NC / 2];
#pragma unroll
      for (int i = 0; i < NC / 2; ++i) sum[i] = 0;
      for (int k = 0; k < p.kt; ++k) {
        float sw = next;
        next = ws[min(k + 1, p.kt - 1)];
        // A block's sum times sw stays within fp32's range for sw between 2^-100 and 2^100
        // (it is a multiple of 2^-18 below 2^25).  Where a lane's lies outside, a factor of
        // 2^64 goes from one scale to the other.
        const float mag = fabsf(sw);
        float lift = 1.f;
        if (mag > 0x1p100f) { lift = 0x1p64f; sw *= 0x1p-64f; }
        else if (mag < 0x1p-100f && mag > 0.f) { lift = 0x1p-64f; sw *= 0x1p64f; }
        const bool far = __any_sync(0xFFFFFFFFu, lift != 1.f);
        const uint64_t sw2 = pack2(sw, sw);
        if (!wait(&sx_full[slot], slot_phase) || !wait(&acc_full[acc], acc_phase, true)) {
          ok = false;
          break;
        }
        ptx::tc_fence_after();
        const uint32_t t = tmem + acc * kAccCols + col0 + ((uint32_t)(quarter * 32) << 16);
        const float* sx = sx_ring + slot * kSxRow + col0;
#pragma unroll
        for (int q = 0; q < NC / G; ++q) {
          if (q >= groups) break;
          float v[G];
          if constexpr (G == 32) ptx::tmem_ld32(t + q * G, v);
          else ptx::tmem_ld16(t + q * G, v);
          if (!far) {
#pragma unroll
            for (int i = 0; i < G / 4; ++i) {
              const ulonglong2 s = *reinterpret_cast<const ulonglong2*>(sx + q * G + 4 * i);
              uint64_t& lo = sum[(q * G + 4 * i) / 2];
              uint64_t& hi = sum[(q * G + 4 * i) / 2 + 1];
              lo = fma2(mul2(pack2(v[4 * i], v[4 * i + 1]), sw2), s.x, lo);
              hi = fma2(mul2(pack2(v[4 * i + 2], v[4 * i + 3]), sw2), s.y, hi);
            }
          } else {
#pragma unroll
            for (int i = 0; i < G / 2; ++i) {
              // (a product past the range has to stay finite for a sum of zero)
              const float s0 = fminf(sx[q * G + 2 * i] * lift, 3.402823466e38f);
              const float s1 = fminf(sx[q * G + 2 * i + 1] * lift, 3.402823466e38f);
              uint64_t& at = sum[(q * G + 2 * i) / 2];
              at = fma2(mul2(pack2(v[2 * i], v[2 * i + 1]), sw2), pack2(s0, s1), at);
            }
          }
        }
        ptx::tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          arrive(&acc_empty[acc]);
          ptx::mbar_arrive(&sx_empty[slot]);
        }
        if (++acc == 2) { acc = 0; acc_phase ^= 1; }
        if (++slot == kSxSlots) { slot = 0; slot_phase ^= 1; }
      }
      if (!ok) break;
      // (values first, then their stores in one block without conditions)
      auto store = [&](auto* y) {
#pragma unroll
        for (int q = 0; q < NC / G; ++q) {
          float v[G];
#pragma unroll
          for (int i = 0; i < G / 2; ++i) {
            const uint64_t s = sum[q * (G / 2) + i];
            v[2 * i] = __uint_as_float((uint32_t)s) + b;
            v[2 * i + 1] = __uint_as_float((uint32_t)(s >> 32)) + b;
          }
          const int c = col0 + q * G;
          auto* o = y + (int64_t)(r0 + c) * g.ld_out + j;
          if (live && rows - c >= G) {
#pragma unroll
            for (int i = 0; i < G; ++i) store_value(o + i * g.ld_out, v[i]);
          } else if (live) {
#pragma unroll
            for (int i = 0; i < G; ++i)
              if (c + i < rows) store_value(o + i * g.ld_out, v[i]);
          }
        }
      };
      if (g.out_type == TAB_FP32) store(static_cast<float*>(g.out));
      else store(static_cast<__nv_bfloat16*>(g.out));
    }
  }

  __syncwarp();
  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
  if (*s_abort) {      // copies and MMAs of the stages given up end within this
    const long long t0 = clock64();
    while (clock64() - t0 < kDrainCycles) {}
  }
  // (pair: neither CTA leaves, or frees its tensor memory, before the other is done)
  if constexpr (PAIR) ptx::cluster_sync();
  else __syncthreads();
  if (warp == kWarpMma) {
    if constexpr (PAIR) ptx::tmem_dealloc_pair(tmem, kTmemCols);
    else ptx::tmem_dealloc(tmem, kTmemCols);
  }
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
// Codes [rows][d bytes], boxes of 128 bytes by box_rows; zeros past the last column and row.
bool code_map(CUtensorMap* m, const void* ptr, uint64_t d, uint64_t rows, uint64_t ld,
              uint32_t box_rows) {
  EncodeFn fn = encode_fn();
  if (!fn) return false;
  const cuuint64_t dims[2] = {d, rows}, strides[1] = {ld};
  const cuuint32_t box[2] = {kFp8Block, box_rows}, es[2] = {1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(ptr), dims, strides, box, es,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

size_t up256(size_t x) { return (x + 255) / 256 * 256; }

struct Plan {
  int pair, bn, row_tiles, tiles, kt, stages, stage_bytes, units;
};
// As many equal tiles of hidden-state rows as these need.
Plan plan_of(const Fp8Plan& a) {
  Plan pl{};
  pl.pair = a.pair_units > 0 && a.pair_mode == 2;
  const int unit = pl.pair ? 32 : 16;
  const int64_t count = (a.rows + kMaxBn - 1) / kMaxBn;
  pl.bn = (int)(((a.rows + count - 1) / count + unit - 1) / unit * unit);
  pl.row_tiles = (int)((a.rows + pl.bn - 1) / pl.bn);
  const int64_t m = pl.pair ? 2 * kM : kM;
  pl.tiles = (int)((a.n + m - 1) / m) * pl.row_tiles;
  pl.kt = (a.d + kFp8Block - 1) / kFp8Block;
  pl.stage_bytes = (kABytes + pl.bn / (pl.pair ? 2 : 1) * kFp8Block + 1023) / 1024 * 1024;
  pl.stages = (kSmemMax - kExtraBytes) / pl.stage_bytes;
  if (pl.stages > kMaxStages) pl.stages = kMaxStages;
  const int most = pl.pair ? a.pair_units : a.sm_count;
  pl.units = pl.tiles < most ? pl.tiles : most;
  return pl;
}

struct Scratch {        // X
  int64_t ld, ld_scales;
  size_t scales, bytes;
};
Scratch scratch_of(const Plan& pl, int64_t rows, int d) {
  Scratch o{};
  o.ld = (d + 15) / 16 * 16;
  o.ld_scales = (int64_t)pl.row_tiles * pl.bn;
  o.scales = up256((size_t)(rows * o.ld));
  o.bytes = o.scales + up256((size_t)pl.kt * o.ld_scales * 4);
  return o;
}

struct Maps {
  CUtensorMap w, row, x;
};
template <int NC, int H, bool PAIR>
cudaError_t launch(const Maps& m, const Params& p, int units, cudaStream_t st) {
  const size_t smem = (size_t)p.stages * p.stage_bytes + kExtraBytes;
  auto kernel = fp8_kernel<NC, H, PAIR>;
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemMax);
  if (e != cudaSuccess) return e;
  if constexpr (PAIR)
    return launch_pdl_cluster(kernel, dim3((unsigned)(2 * units)), dim3(kThreads), smem, st, 2, m.w,
                              m.row, m.x, p);
  else
    return launch_pdl(kernel, dim3((unsigned)units), dim3(kThreads), smem, st, m.w, m.row, m.x, p);
}
template <bool PAIR>
cudaError_t launch_bn(const Maps& m, const Params& p, int units, cudaStream_t st) {
  if (p.bn <= 16) return launch<16, 1, PAIR>(m, p, units, st);
  if (p.bn <= 32) return launch<32, 1, PAIR>(m, p, units, st);
  if (p.bn <= 64) return launch<32, 2, PAIR>(m, p, units, st);
  if (p.bn <= 128) return launch<64, 2, PAIR>(m, p, units, st);
  return launch<96, 2, PAIR>(m, p, units, st);
}

}  // namespace

size_t fp8_gemm_scratch_bytes(const Fp8Plan& a) { return scratch_of(plan_of(a), a.rows, a.d).bytes; }

// At least what any call of up to `rows` rows and d columns takes: tiles cover at most 32
// more rows each, and one that is not the only one has at least 64.
size_t fp8_gemm_reserve_bytes(int64_t rows, int64_t d) {
  const size_t padded = 2 * (size_t)rows + 64, kt = (size_t)((d + kFp8Block - 1) / kFp8Block);
  return up256((size_t)rows * ((size_t)(d + 15) / 16 * 16)) + up256(kt * padded * 4);
}

cudaError_t launch_fp8_gemm(const Fp8Gemm& g, const Fp8Plan& a, void* scratch, long long spin_limit,
                            cudaStream_t st) {
  const Plan pl = plan_of(a);
  const Scratch o = scratch_of(pl, g.rows, g.d);
  char* at = static_cast<char*>(scratch);
  Params p{};
  p.g = g;
  p.x_scales = reinterpret_cast<float*>(at + o.scales);
  p.ld_xs = o.ld_scales;
  p.bn = pl.bn; p.row_tiles = pl.row_tiles; p.tiles = pl.tiles; p.kt = pl.kt;
  p.stages = pl.stages; p.stage_bytes = pl.stage_bytes;
  p.spin_limit = spin_limit;
  Maps m;
  if (!code_map(&m.x, at, (uint64_t)g.d, (uint64_t)g.rows, (uint64_t)o.ld,
                (uint32_t)(pl.bn / (pl.pair ? 2 : 1))) ||
      !code_map(&m.w, g.w_codes, (uint64_t)g.d, (uint64_t)g.V, (uint64_t)g.ld_codes, g.ids ? 32 : kM))
    return cudaErrorInvalidValue;
  m.row = m.w;
  if (g.ids && !code_map(&m.row, g.w_codes, (uint64_t)g.d, (uint64_t)g.V, (uint64_t)g.ld_codes, 1))
    return cudaErrorInvalidValue;

  Fp8Quant q{};
  q.x = g.x; q.ld_x = g.ld_x; q.rows = g.rows; q.d = g.d; q.block_rows = 1;
  q.codes = reinterpret_cast<uint8_t*>(at); q.ld_codes = o.ld;
  q.scales = reinterpret_cast<float*>(at + o.scales);
  q.row_step = 1; q.col_step = o.ld_scales;
  cudaError_t e = launch_fp8_quant(q, g.x_type, st);
  if (e != cudaSuccess) return e;
  return pl.pair ? launch_bn<true>(m, p, pl.units, st) : launch_bn<false>(m, p, pl.units, st);
}

}  // namespace sph
