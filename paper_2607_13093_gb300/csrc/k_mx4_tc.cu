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
// A CTA keeps a ring of stages of 256 columns, 128 bytes of codes a row: W's codes
// by TMA, whole boxes where the kept ids are consecutive and four gathered rows a
// copy elsewhere; X's codes and scales by TMA; W's scales by cp.async.  Four warps
// move a stage's scales from shared memory to tensor memory (in the quarter of
// the lanes that each may write), into one of several sets of columns; one warp
// issues the MMAs; four read the accumulator, double-buffered in tensor memory,
// and store.  (Scales by tcgen05.cp took some 80 cycles a copy of four columns in
// the MMAs' own queue: 1024 rows x 256000 ids x 4608 907 us.)
#include <cuda.h>
#include <cuda_bf16.h>

#include <mutex>

#include "mx4.cuh"
#include "sm100_ptx.cuh"
#include "sph_internal.h"

namespace sph {
namespace {

constexpr int kM = 128;                  // table rows of a tile
constexpr int kCols = 256;               // columns of a stage: 128 bytes of codes
constexpr int kABytes = kM * kCols / 2;
constexpr int kThreads = 384;            // 12 warps
constexpr int kWarpW = 0, kWarpMma = 1, kWarpX = 2, kWarpRaw = 3, kWarpScale = 4, kWarpOut = 8;
constexpr int kMaxSets = 8;              // sets of scale columns in tensor memory
constexpr int kMaxStages = 12;
constexpr int kMaxBn = 256;              // hidden-state rows of a tile
constexpr int kSmemMax = 227 * 1024;
constexpr int kBarBytes = 1024;
constexpr uint32_t kTmemCols = 512;
constexpr long long kDrainCycles = 1ll << 20;

// groups of four scale bytes a stage and row
__host__ __device__ constexpr int groups_of(int fmt) { return fmt == MX4_E4M3 ? 4 : 2; }

// ---- instructions ------------------------------------------------------------
// N columns of this warp's lanes of tensor memory.
template <int N>
__device__ __forceinline__ void tmem_st(uint32_t taddr, const uint32_t (&r)[N]) {
  static_assert(N == 8 || N == 16 || N == 32, "column count");
  if constexpr (N == 8)
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"r"(taddr),
                 "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
                 : "memory");
  else if constexpr (N == 16)
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
        "{%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(taddr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
        "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
  else
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
        "{%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,"
        "%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};" ::"r"(taddr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
        "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]),
        "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]),
        "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]),
        "r"(r[30]), "r"(r[31])
        : "memory");
}
// Scales of a stage, one row after another in shared memory (4 G bytes each), to
// tensor memory: word q of row r goes to lane r % 32 of column q * 4 C + r / 32.
// (What rows past `rows` get is read by no MMA.)
template <int G, int C>
__device__ __forceinline__ void put_scales(uint32_t taddr, const uint8_t* src, int rows, int lane) {
  uint32_t w[G * 4 * C];
#pragma unroll
  for (int i = 0; i < 4 * C; ++i) {
    uint4 v = make_uint4(0, 0, 0, 0);
    if (32 * i < rows) {
      if constexpr (G == 4) {
        v = reinterpret_cast<const uint4*>(src)[32 * i + lane];
      } else {
        const uint2 h = reinterpret_cast<const uint2*>(src)[32 * i + lane];
        v.x = h.x;
        v.y = h.y;
      }
    }
    w[i] = v.x;
    w[4 * C + i] = v.y;
    if constexpr (G == 4) {
      w[8 * C + i] = v.z;
      w[12 * C + i] = v.w;
    }
  }
  tmem_st(taddr, w);
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

__device__ __forceinline__ void store_value(float* p, float v) { *p = v; }
__device__ __forceinline__ void store_value(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }

struct Params {
  Mx4Gemm g;
  const uint8_t* x_scales;      // [plane][row tile][stage][bn][scale bytes of a stage]
  int64_t x_scale_plane;        // bytes
  const float* x_row;           // [row tiles * bn], e4m3 only
  int bn, row_tiles, tiles, kt; // row tiles are the fast index of a tile
  int stages, stage_bytes, chunks, sf_col, sf_cols, sf_sets;
  long long spin_limit;
};

template <int FMT, bool GATHER, class OT>
__global__ void __launch_bounds__(kThreads, 1)
mx4_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_row,
           const __grid_constant__ CUtensorMap map_x, const Params p) {
  constexpr int kGroups = groups_of(FMT);
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = ptx::smem_u32(smem_raw);
  const uint32_t base_addr = (raw + 1023) & ~1023u;
  uint8_t* base = smem_raw + (base_addr - raw);
  uint64_t* full = reinterpret_cast<uint64_t*>(base + (size_t)p.stages * p.stage_bytes);
  uint64_t* empty = full + kMaxStages;
  uint64_t* acc_full = empty + kMaxStages;      // [2]
  uint64_t* acc_empty = acc_full + 2;           // [2]
  uint64_t* sf_full = acc_empty + 2;            // [kMaxSets]
  uint64_t* sf_empty = sf_full + kMaxSets;      // [kMaxSets]
  uint32_t* holder = reinterpret_cast<uint32_t*>(sf_empty + kMaxSets);
  volatile int* s_abort = reinterpret_cast<volatile int*>(holder + 1);
  // (from lane 0, so that the compiler knows that a warp takes one branch and can
  // keep its loop's counters and descriptors in uniform registers)
  const int warp = __shfl_sync(0xFFFFFFFFu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  const Mx4Gemm& g = p.g;
  constexpr int kRow = 4 * kGroups;             // scale bytes of a row and stage
  // a stage: W codes, X codes (a term after the other), W scales, X scales
  const int x_bytes = p.bn * (kCols / 2), xs_bytes = p.bn * kRow;
  const int off_ws = kABytes + g.planes * x_bytes, off_xs = off_ws + kM * kRow;

  if (threadIdx.x == 0) {
    for (int s = 0; s < p.stages; ++s) {
      ptx::mbar_init(&full[s], 1 + 1 + 32);     // W codes, X, the lanes that copy W's scales
      ptx::mbar_init(&empty[s], 1);
    }
    for (int a = 0; a < 2; ++a) {
      ptx::mbar_init(&acc_full[a], 1);
      ptx::mbar_init(&acc_empty[a], 4);
    }
    for (int s = 0; s < p.sf_sets; ++s) {
      ptx::mbar_init(&sf_full[s], 4);
      ptx::mbar_init(&sf_empty[s], 1);
    }
    *s_abort = 0;
    ptx::fence_mbar_init();
  }
  if (warp == kWarpMma) ptx::tmem_alloc(holder, kTmemCols);
  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
  const uint32_t tmem = __shfl_sync(0xFFFFFFFFu, *holder, 0);
  // (after the allocation, so that no later kernel's CTA takes the tensor memory first)
  ptx::griddep_launch_dependents();

  // A wait that gives up after spin_limit cycles, or once another warp has; the
  // whole warp gets one answer.
  auto wait = [&](uint64_t* bar, uint32_t parity) {
    if (__all_sync(0xFFFFFFFFu, ptx::mbar_try_wait(bar, parity))) return true;
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
  int stage = 0;
  uint32_t phase = 0;
  auto advance = [&] {
    if (++stage == p.stages) { stage = 0; phase ^= 1; }
  };
  int set = 0;
  uint32_t set_phase = 0;
  auto next_set = [&] {
    if (++set == p.sf_sets) { set = 0; set_phase ^= 1; }
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
    bool ok = true;
    int acc = 0;
    uint32_t acc_phase = 0;
    for (int tile = blockIdx.x; ok && tile < p.tiles; tile += gridDim.x) {
      if (!wait(&acc_empty[acc], acc_phase ^ 1)) break;
      ptx::tc_fence_after();
      const uint32_t d = tmem + acc * p.bn;
      for (int k = 0; k < p.kt; ++k) {
        if (!wait(&full[stage], phase) || !wait(&sf_full[set], set_phase)) { ok = false; break; }
        ptx::tc_fence_after();
        const uint32_t s = base_addr + stage * p.stage_bytes;
        const uint32_t sfa = tmem + p.sf_col + set * p.sf_cols;
        uint32_t sfb = sfa + 4 * kGroups, bd = ptx::sdesc_k128(s + kABytes);
        const uint32_t ad = ptx::sdesc_k128(s);
        // steps of 64 columns, none past the last column
        const int steps = min(4, (g.d - k * kCols + 63) / 64);
        for (int t = 0; t < g.planes; ++t) {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            if (j >= steps) break;
            const int q = FMT == MX4_E4M3 ? j : j / 2;
            mma_mx4<FMT>(d, ad + 2 * j, bd + 2 * j,
                         idesc_mx4<FMT>(p.bn, FMT == MX4_E4M3 ? 0 : j % 2), sfa + 4 * q,
                         sfb + q * p.chunks * 4, k > 0 || t > 0 || j > 0);
          }
          sfb += kGroups * p.chunks * 4;
          bd += (uint32_t)x_bytes >> 4;
        }
        ptx::umma_commit(&empty[stage]);
        ptx::umma_commit(&sf_empty[set]);
        advance();
        next_set();
      }
      if (!ok) break;
      ptx::umma_commit(&acc_full[acc]);
      acc ^= 1;
      if (acc == 0) acc_phase ^= 1;
    }
  } else if (warp >= kWarpScale && warp < kWarpScale + 4) {
    // ---- scales to tensor memory ---------------------------------------------
    const uint32_t lanes = (uint32_t)((warp - kWarpScale) * 32) << 16;
    bool ok = true;
    for (int tile = blockIdx.x; ok && tile < p.tiles; tile += gridDim.x) {
      for (int k = 0; k < p.kt; ++k) {
        if (!wait(&full[stage], phase) || !wait(&sf_empty[set], set_phase ^ 1)) { ok = false; break; }
        ptx::tc_fence_after();
        const uint8_t* s = base + (size_t)stage * p.stage_bytes;
        uint32_t to = tmem + lanes + p.sf_col + set * p.sf_cols;
        put_scales<kGroups, 1>(to, s + off_ws, kM, lane);
        to += 4 * kGroups;
        for (int t = 0; t < g.planes; ++t) {
          if (p.chunks == 1) put_scales<kGroups, 1>(to, s + off_xs + t * xs_bytes, p.bn, lane);
          else put_scales<kGroups, 2>(to, s + off_xs + t * xs_bytes, p.bn, lane);
          to += kGroups * p.chunks * 4;
        }
        asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
        ptx::tc_fence_before();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(&sf_full[set]);
        advance();
        next_set();
      }
    }
  } else if (warp == kWarpRaw) {
    // ---- W scales --------------------------------------------------------------
    // Lane l copies rows l, l + 32, l + 64 and l + 96 of the tile; rows past the last
    // kept id and bytes past the last scale become zeros.
    const int bytes = (g.d + Mx4<FMT>::kBlock - 1) / Mx4<FMT>::kBlock;
    bool ok = true;
    for (int tile = blockIdx.x; ok && tile < p.tiles; tile += gridDim.x) {
      const uint8_t* row[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int j = tile / p.row_tiles * kM + 32 * i + lane;
        row[i] = j < g.n ? g.w_scales + (int64_t)(GATHER ? g.ids[j] : j) * g.ld_scales : nullptr;
      }
      for (int k = 0; k < p.kt; ++k) {
        if (!wait(&empty[stage], phase ^ 1)) { ok = false; break; }
        uint8_t* dst = base + (size_t)stage * p.stage_bytes + off_ws;
        const int left = min(kRow, bytes - k * kRow);
#pragma unroll
        for (int i = 0; i < 4; ++i)
          asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"(
                           ptx::smem_u32(dst + (32 * i + lane) * kRow)),
                       "l"(row[i] ? row[i] + k * kRow : g.w_scales), "n"(kRow),
                       "r"(row[i] ? left : 0)
                       : "memory");
        asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(
                         ptx::smem_u32(&full[stage]))
                     : "memory");
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
      // the X row scales of the tile, 32 columns a register, handed out by shuffles
      // (loaded where they are used, each one would wait for the stores before it)
      float xs[kMaxBn / 32];
      if constexpr (FMT == MX4_E4M3) {
#pragma unroll
        for (int m = 0; m < kMaxBn / 32; ++m)
          xs[m] = 32 * m + lane < rows ? p.x_row[r0 + 32 * m + lane] : 0.f;
      }
      if (!wait(&acc_full[acc], acc_phase)) break;
      ptx::tc_fence_after();
      const uint32_t t = tmem + acc * p.bn + ((uint32_t)(quarter * 32) << 16);
      OT* y = static_cast<OT*>(g.out) + (int64_t)r0 * g.ld_out + j;
#pragma unroll
      for (int m = 0; m < kMaxBn / 32; ++m) {
        if (32 * m >= rows) break;
        float v[32];
        ptx::tmem_ld32(t + 32 * m, v);
        // (values first, then their stores in one block without conditions: with a
        // condition a value each waits for the one before, some 100 cycles a column)
#pragma unroll
        for (int i = 0; i < 32; ++i) {
          v[i] *= ws;
          if constexpr (FMT == MX4_E4M3) v[i] *= __shfl_sync(0xFFFFFFFFu, xs[m], i);
          v[i] += b;
        }
        OT* q = y + (int64_t)(32 * m) * g.ld_out;
        if (live && rows - 32 * m >= 32) {
#pragma unroll
          for (int i = 0; i < 32; ++i) store_value(q + i * g.ld_out, v[i]);
        } else if (live) {
#pragma unroll
          for (int i = 0; i < 32; ++i)
            if (32 * m + i < rows) store_value(q + i * g.ld_out, v[i]);
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
  int bn, row_tiles, tiles, kt, stages, stage_bytes, chunks, sf_col, sf_cols, sf_sets;
};
int stage_bytes_of(int bn, int planes, int fmt) {
  const int row = groups_of(fmt) * 4;
  return (kABytes + planes * bn * (kCols / 2) + (kM + planes * bn) * row + 1023) / 1024 * 1024;
}
int sf_col_of(int bn) { return (2 * bn + 31) / 32 * 32; }
int sf_cols_of(int bn, int planes, int fmt) {
  return 4 * groups_of(fmt) * (1 + planes * ((bn + 127) / 128));
}
constexpr int kExtraBytes = 1024 + kBarBytes;     // shared memory beside the stages
// The largest tile of hidden-state rows of which three stages fit, and two
// accumulators with a stage's scales; then as many equal tiles as the rows need.
Plan plan_of(int64_t rows, int64_t n, int d, int planes, int fmt) {
  Plan pl{};
  int most = 16;
  for (int bn = 16; bn <= kMaxBn; bn += 16) {
    if (3 * stage_bytes_of(bn, planes, fmt) + kExtraBytes > kSmemMax ||
        sf_col_of(bn) + sf_cols_of(bn, planes, fmt) > (int)kTmemCols)
      break;
    most = bn;
  }
  const int64_t count = (rows + most - 1) / most;
  pl.bn = (int)(((rows + count - 1) / count + 15) / 16 * 16);
  pl.row_tiles = (int)((rows + pl.bn - 1) / pl.bn);
  pl.tiles = (int)((n + kM - 1) / kM) * pl.row_tiles;
  pl.kt = (d + kCols - 1) / kCols;
  pl.stage_bytes = stage_bytes_of(pl.bn, planes, fmt);
  pl.stages = (kSmemMax - kExtraBytes) / pl.stage_bytes;
  if (pl.stages > kMaxStages) pl.stages = kMaxStages;
  pl.chunks = (pl.bn + 127) / 128;
  pl.sf_col = sf_col_of(pl.bn);
  pl.sf_cols = sf_cols_of(pl.bn, planes, fmt);
  pl.sf_sets = ((int)kTmemCols - pl.sf_col) / pl.sf_cols;
  if (pl.sf_sets > kMaxSets) pl.sf_sets = kMaxSets;
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
  o.scale_plane = (int64_t)up256((size_t)pl.row_tiles * pl.kt * pl.bn * groups_of(fmt) * 4);
  o.scales = (size_t)(planes * o.plane);
  o.row = o.scales + (size_t)(planes * o.scale_plane);
  o.bytes = o.row + up256((size_t)pl.row_tiles * pl.bn * 4);
  return o;
}

template <int FMT, bool GATHER, class OT>
cudaError_t launch(const CUtensorMap& w, const CUtensorMap& row, const CUtensorMap& x,
                   const Params& p, int sm_count, cudaStream_t st) {
  const size_t smem = (size_t)p.stages * p.stage_bytes + kExtraBytes;
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

// At least what any call of up to `rows` rows and d columns takes: tiles cover at
// most 16 more rows each, and one that is not the only one has at least 32.
size_t mx4_gemm_reserve_bytes(int64_t rows, int64_t d) {
  const size_t r = (size_t)rows, padded = 2 * r + 64, kt = (size_t)((d + kCols - 1) / kCols);
  return 4 * (up256(r * ((size_t)(d + 31) / 32 * 16)) +
              up256(padded * kt * groups_of(MX4_E4M3) * 4)) +
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
  p.stages = pl.stages; p.stage_bytes = pl.stage_bytes; p.chunks = pl.chunks;
  p.sf_col = pl.sf_col; p.sf_cols = pl.sf_cols; p.sf_sets = pl.sf_sets;
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
  q.tile_rows = pl.bn; q.tile_words = groups_of(g.fmt);
  q.tile_bytes = (int64_t)pl.kt * pl.bn * groups_of(g.fmt) * 4;
  cudaError_t e = launch_mx4_quant(q, g.fmt, g.x_type, true, st);
  if (e != cudaSuccess) return e;
  if (g.fmt == MX4_E4M3)
    return g.ids ? launch_o<MX4_E4M3, true>(mw, mr, mx, p, sm_count, st)
                 : launch_o<MX4_E4M3, false>(mw, mr, mx, p, sm_count, st);
  return g.ids ? launch_o<MX4_E8M0, true>(mw, mr, mx, p, sm_count, st)
               : launch_o<MX4_E8M0, false>(mw, mr, mx, p, sm_count, st);
}

}  // namespace sph
