// Product of many hidden states and the kept rows of a table in e4m3 whose scales belong to
// blocks of 128 rows by 128 columns:
//
//   y[r, j] = sum over blocks b of sx[r, b] * sw[id_j / 128, b] * (qx[r, b] . qw[id_j, b])  (+ bias)
//
// The hidden states are the MMA's M, 256 rows over a pair of CTAs (cta_group::2), table rows
// its N, 256 too, half of them in each CTA's shared memory; a stage is a block of 128 columns.
//
// The scales differ from block to block and are no powers of two, so a block's sums leave the
// tensor core before they are scaled: the MMA warp fills two accumulators in tensor memory in
// turn, and eight warps add the full one, scaled, to sums in their registers.  A thread has a
// hidden state and 128 table rows, which share one scale (a kept subset's in runs of 32 do
// mostly): its factor is one number a block, and a value costs one fused multiply-add.  (With
// table rows in the lanes, as few hidden states need it, each thread reads a factor a column
// from shared memory, which gives 128 bytes a cycle and takes twice the MMAs' time: 1024
// rows x 256000 ids x 4608 1197 us, so 953 to 1026: 2.4 PFLOP/s, where MMAs and copies alone take
// 678.)  What is left is the additions' latency: eight warps, two a scheduler, read 128 columns
// of an accumulator and add them (tensor pipe active 44 % of the time, issue slots 42 %); more
// warps have too few registers for their sums (232 a thread now).
//
// Tiles that one factor a block does not serve are computed again by a second kernel, which scales
// each value by its own table scale: those with a scale outside [2^-50, 2^50] (a block of zeros
// has 2^-126: with a hidden state of zeros in each 256, 1024 x 256000 x 4608 takes 2091 us), and
// those with a group of 32 kept ids that meets three blocks of 128 rows or more (1024 x 30412 of
// 152064 ids x 3584: the first ones 145 us, random ones 3782; with table rows as M, k_fp8_tc.cu
// without pairs, 171 and 220).
#include "fp8_tc.cuh"
#include "rows.cuh"

namespace sph {
namespace {

constexpr int kM = 128;                  // hidden states of a CTA
constexpr int kN = 256;                  // table rows of a tile, kN / 2 copied by each CTA
constexpr int kHalfBytes = 128 * kFp8Block, kStageBytes = 2 * kHalfBytes;
constexpr int kWarpW = 0, kWarpMma = 1, kWarpX = 2, kWarpOut = 4;
constexpr int kStages = 6;
constexpr int kBarBytes = 1024;
constexpr int kGroup = 32, kGroups = 4;  // table rows a thread adds together, groups of them
constexpr int kTurnRow = kGroup + 1;     // words a row of the turned group (below)
constexpr int kTurnBytes = 8 * 32 * kTurnRow * 4;
constexpr int kSmem = kStages * kStageBytes + kBarBytes + kTurnBytes + 1024;
static_assert(kSmem <= kSmemMax, "shared memory");
constexpr int kRegsFew = 40, kRegsMany = 232;    // (of 168 a thread at the launch)
static_assert(kRegsFew + 2 * kRegsMany <= 3 * 168, "more registers than the launch has");

struct Params {
  Fp8Gemm g;
  const float* x_scales;        // [rows][ld_xs], 16-byte rows of whole fours of blocks
  int64_t ld_xs;
  int row_tiles, tiles, kt;     // row tiles are the fast index of a tile
  int out32;                    // rows of out are on 32 bytes
  int* far;                     // [tiles] those whose scales are far from 1; zero before
  long long spin_limit;
};

// Two scales in this range multiply without leaving fp32's, times a block's sum too.
__device__ __forceinline__ bool in_range(float s) { return fabsf(s) >= 0x1p-50f && fabsf(s) <= 0x1p50f; }

// 16 values to a row's 32 bytes, or 8.
__device__ __forceinline__ void store_line(float* p, const float (&v)[8]) { store_v8(p, v); }
__device__ __forceinline__ void store_line(__nv_bfloat16* p, const float (&v)[16]) {
  uint32_t w[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
    w[i] = *reinterpret_cast<const uint32_t*>(&h);
  }
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(w[0]),
               "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
               : "memory");
}

// FAR: the tiles of p.far, with scales one after another (below).
template <bool GATHER, bool FAR>
__global__ void __launch_bounds__(kThreads, 1)
fp8_rows_as_m_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_row,
                     const __grid_constant__ CUtensorMap map_x, const Params p) {
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw_addr = ptx::smem_u32(smem_raw);
  const uint32_t base_addr = (raw_addr + 1023) & ~1023u;
  uint8_t* base = smem_raw + (base_addr - raw_addr);
  uint64_t* full = reinterpret_cast<uint64_t*>(base + kStages * kStageBytes);
  uint64_t* empty = full + kStages;
  uint64_t* acc_full = empty + kStages;         // [2]
  uint64_t* acc_empty = acc_full + 2;           // [2]
  uint32_t* holder = reinterpret_cast<uint32_t*>(acc_empty + 2);
  volatile int* s_abort = reinterpret_cast<volatile int*>(holder + 1);
  const int warp = __shfl_sync(0xFFFFFFFFu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  const Fp8Gemm& g = p.g;
  const int half = __shfl_sync(0xFFFFFFFFu, (int)ptx::cluster_ctarank(), 0);
  const int unit = (int)blockIdx.x / 2, units = (int)gridDim.x / 2;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      ptx::mbar_init(&full[s], 4);              // W and X of each CTA
      ptx::mbar_init(&empty[s], 1);
    }
    for (int a = 0; a < 2; ++a) {
      ptx::mbar_init(&acc_full[a], 1);
      ptx::mbar_init(&acc_empty[a], 16);
    }
    *s_abort = 0;
    ptx::fence_mbar_init();
  }
  if (warp == kWarpMma) ptx::tmem_alloc_pair(holder, kTmemCols);
  ptx::tc_fence_before();
  ptx::cluster_sync();
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
  auto leader = [&](uint64_t* bar) { return ptx::mapa(ptx::smem_u32(bar), 0); };
  int stage = 0;
  uint32_t phase = 0;
  auto advance = [&] {
    if (++stage == kStages) { stage = 0; phase ^= 1; }
  };
  bool ok = true;
  if (warp < kWarpOut) {
    give_registers<kRegsFew>();
    if (warp == kWarpW) {
      // ---- W codes: groups of 32 consecutive ids by one box, others four rows a copy ----
      if constexpr (FAR) ptx::griddep_wait();
      for (int tile = unit; ok && tile < p.tiles; tile += units) {
        if (FAR && !p.far[tile]) continue;
        const int j0 = tile / p.row_tiles * kN + half * (kN / 2), last = g.n - 1;
        int4 id = make_int4(0, 0, 0, 0);
        unsigned solid = 0;
        if constexpr (GATHER) {
          // rows past the last kept id repeat it
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
        }
        for (int k = 0; k < p.kt; ++k) {
          if (!wait(&empty[stage], phase ^ 1, true)) { ok = false; break; }
          uint8_t* b = base + stage * kStageBytes + kHalfBytes;
          const uint32_t bar = leader(&full[stage]);
          const int x = k * kFp8Block;
          if (lane == 0) expect_at(bar, kHalfBytes);
          __syncwarp();
          if constexpr (GATHER) {
            if (solid >> (lane >> 3) & 1) {
              if ((lane & 7) == 0) ptx::tma_load_2d_pair(b + lane * 512, &map_w, x, id.x, bar);
            } else {
              tma_gather4(b + lane * 512, &map_row, x, id, bar);
            }
          } else if (lane == 0) {
            // (the last tile's second half may lie past the last row: a box starts inside)
            ptx::tma_load_2d_pair(b, &map_w, x, min(j0, (int)g.V - 1), bar);
          }
          advance();
        }
      }
    } else if (warp == kWarpX) {
      // ---- X codes -----------------------------------------------------------
      ptx::griddep_wait();
      for (int tile = unit; ok && tile < p.tiles; tile += units) {
        if (FAR && !p.far[tile]) continue;
        // (rows past the last one come as zeros)
        const int r0 = (tile % p.row_tiles * 2 + half) * kM;
        for (int k = 0; k < p.kt; ++k) {
          if (!wait(&empty[stage], phase ^ 1)) { ok = false; break; }
          if (lane == 0) {
            const uint32_t bar = leader(&full[stage]);
            expect_at(bar, kHalfBytes);
            ptx::tma_load_2d_pair(base + stage * kStageBytes, &map_x, k * kFp8Block, r0, bar);
          }
          __syncwarp();
          advance();
        }
      }
    } else if (warp == kWarpMma && half == 0) {
      // ---- MMA ---------------------------------------------------------------
      if constexpr (FAR) ptx::griddep_wait();
      int acc = 0;
      uint32_t acc_phase = 0;
      const uint32_t idesc = ptx::idesc_e4m3_f32(2 * kM, kN);
      for (int tile = unit; ok && tile < p.tiles; tile += units) {
        if (FAR && !p.far[tile]) continue;
        for (int k = 0; k < p.kt; ++k) {
          if (!wait(&acc_empty[acc], acc_phase ^ 1) || !wait(&full[stage], phase)) { ok = false; break; }
          ptx::tc_fence_after();
          const uint32_t s = base_addr + stage * kStageBytes, d = tmem + acc * kAccCols;
          const uint32_t ad = ptx::sdesc_k128(s), bd = ptx::sdesc_k128(s + kHalfBytes);
          // steps of 32 columns, none past the last column
          const int steps = min(4, (g.d - k * kFp8Block + 31) / 32);
          for (int i = 0; i < steps; ++i) ptx::umma_f8_pair(d, ad + 2 * i, bd + 2 * i, idesc, i > 0);
          ptx::umma_commit_pair(&empty[stage]);
          ptx::umma_commit_pair(&acc_full[acc]);
          advance();
          if (++acc == 2) { acc = 0; acc_phase ^= 1; }
        }
      }
    }
  } else {
    take_registers<kRegsMany>();
    // ---- accumulators to sums, sums to y -------------------------------------
    const int quarter = warp & 3;                // (the lanes that a warp may read)
    const int side = (warp - kWarpOut) >> 2;     // which half of the tile's table rows
    float* turn = reinterpret_cast<float*>(base + kStages * kStageBytes + kBarBytes) +
                  (warp - kWarpOut) * 32 * kTurnRow;
    ptx::griddep_wait();
    int acc = 0;
    uint32_t acc_phase = 0;
    for (int tile = unit; ok && tile < p.tiles; tile += units) {
      if (FAR && !p.far[tile]) continue;
      const int r = (tile % p.row_tiles * 2 + half) * kM + quarter * 32 + lane;
      const int j0 = tile / p.row_tiles * kN + side * (kN / 2);
      const bool live = r < g.rows;
      // Scales come four blocks at a time, four blocks ahead (one ahead, their way from the L2
      // was twice a block's time: 1163 us).  A thread holds its row's; the table's are a warp's:
      // lane 8 q + 4 e + i has block i of the four for group q, of its first rows (e = 0) or its
      // last ones.
      const float4* xs = reinterpret_cast<const float4*>(p.x_scales + (int64_t)(live ? r : 0) * p.ld_xs);
      const int own = lane >> 3, own_end = lane >> 2 & 1;
      int64_t own_block = min(j0, g.n - 1) / kFp8Block;
      // kept rows in runs: a group's first `split[q]` rows have one block's scale, the others
      // another's; more: groups that three blocks or more meet
      int split[kGroups] = {kGroup, kGroup, kGroup, kGroup};
      unsigned more = 0;
      if constexpr (GATHER) {
#pragma unroll
        for (int q = 0; q < kGroups; ++q) {
          const int at = min(j0 + q * kGroup + lane, g.n - 1);
          const int block = (int)(min((int64_t)max(g.ids[at], 0), g.V - 1) / kFp8Block);
          const int first = __shfl_sync(0xFFFFFFFFu, block, 0), end = __shfl_sync(0xFFFFFFFFu, block, 31);
          const unsigned a = __ballot_sync(0xFFFFFFFFu, block == first);
          const unsigned z = __ballot_sync(0xFFFFFFFFu, block == end);
          if (first != end) split[q] = __ffs(z) - 1;
          if ((a | z) != 0xFFFFFFFFu) more |= 1u << q;
          if (own == q) own_block = own_end ? end : first;
        }
      }
      const float* ws = g.w_scales + own_block * g.ld_scales;
      auto w_of = [&](int k) { return ws[min(k + (lane & 3), p.kt - 1)]; };
      float sum[kN / 2];
#pragma unroll
      for (int i = 0; i < kN / 2; ++i) sum[i] = 0.f;
      constexpr int kScales = GATHER ? kGroups : 1, kEnds = GATHER ? 2 : 1;
      float4 sx = xs[0], sx_next = sx;
      float sw = w_of(0), sw_next = sw;
      // The product of the two scales serves unless one is far from 1; such tiles, and those of
      // groups with more than two scales, are done again by the FAR kernel.  (With its code
      // here 1147 to 1422 us, without 982.)
      bool far = more != 0;
      for (int k0 = 0; ok && k0 < p.kt; k0 += 4) {
        if (k0 + 4 < p.kt) {
          sx_next = xs[k0 / 4 + 1];
          sw_next = w_of(k0 + 4);
        }
        const float x4[4] = {live ? sx.x : 1.f, live ? sx.y : 1.f, live ? sx.z : 1.f, live ? sx.w : 1.f};
        if constexpr (!FAR) {
          far |= sw != 0.f && !in_range(sw);
#pragma unroll
          for (int u = 0; u < 4; ++u) far |= k0 + u < p.kt && !in_range(x4[u]);
        }
#pragma unroll 1
        for (int u = 0; u < 4 && k0 + u < p.kt; ++u) {
          const float x = u & 2 ? (u & 1 ? x4[3] : x4[2]) : (u & 1 ? x4[1] : x4[0]);
          if (!wait(&acc_full[acc], acc_phase, true)) { ok = false; break; }
          ptx::tc_fence_after();
          const uint32_t t = tmem + acc * kAccCols + side * (kN / 2) + ((uint32_t)(quarter * 32) << 16);
          uint32_t v[2][kGroup];
          tmem_request(t, v[0]);
          tmem_request(t + kGroup, v[1]);
          float w[kScales][kEnds];
#pragma unroll
          for (int q = 0; q < kScales; ++q)
#pragma unroll
            for (int e = 0; e < kEnds; ++e) w[q][e] = __shfl_sync(0xFFFFFFFFu, sw, 8 * q + 4 * e + u);
          auto add = [&](int q, uint32_t (&of)[kGroup]) {
            const float w0 = w[GATHER ? q : 0][0], w1 = w[GATHER ? q : 0][kEnds - 1];
            if constexpr (FAR) {
              // where W's scale is far from 1 a factor of 2^64 goes from it to X's
#pragma unroll
              for (int i = 0; i < kGroup; ++i) {
                float s = GATHER && i >= split[q] ? w1 : w0, lift = 1.f;
                if (GATHER && (more >> q & 1)) {
                  const int64_t id = min((int64_t)max(g.ids[min(j0 + q * kGroup + i, g.n - 1)], 0), g.V - 1);
                  s = g.w_scales[id / kFp8Block * g.ld_scales + k0 + u];
                }
                if (fabsf(s) > kFar) { lift = 0x1p64f; s *= 0x1p-64f; }
                else if (fabsf(s) < kNear && s != 0.f) { lift = 0x1p-64f; s *= 0x1p64f; }
                const float part = __fmul_rn(__uint_as_float(of[i]), s);
                sum[q * kGroup + i] = __fmaf_rn(part, bounded(x * lift), sum[q * kGroup + i]);
              }
            } else {
              const float f0 = x * w0, f1 = x * w1;
              if (!GATHER || split[q] == kGroup) {
#pragma unroll
                for (int i = 0; i < kGroup; ++i)
                  sum[q * kGroup + i] = __fmaf_rn(__uint_as_float(of[i]), f0, sum[q * kGroup + i]);
              } else {
#pragma unroll
                for (int i = 0; i < kGroup; ++i)
                  sum[q * kGroup + i] = fma_here(__uint_as_float(of[i]), i < split[q] ? f0 : f1, sum[q * kGroup + i]);
              }
            }
          };
          tmem_wait();
          arrived(v[0]);
          arrived(v[1]);
          add(0, v[0]);
          tmem_request(t + 2 * kGroup, v[0]);
          add(1, v[1]);
          tmem_request(t + 3 * kGroup, v[1]);
          tmem_wait();
          // (the accumulator goes back as soon as its last columns have come)
          ptx::tc_fence_before();
          __syncwarp();
          if (lane == 0) arrive_at(leader(&acc_empty[acc]));
          arrived(v[0]);
          arrived(v[1]);
          add(2, v[0]);
          add(3, v[1]);
          if (++acc == 2) { acc = 0; acc_phase ^= 1; }
        }
        sx = sx_next;
        sw = sw_next;
      }
      if (!FAR && far) p.far[tile] = 1;
      if (!ok) break;
      auto store = [&](auto* y) {
        using T = std::remove_pointer_t<decltype(y)>;
        constexpr int kLine = 32 / (int)sizeof(T);
        const int row0 = r - lane;
#pragma unroll
        for (int q = 0; q < kGroups; ++q) {
          const int j = j0 + q * kGroup;
          float v[kGroup];
#pragma unroll
          for (int i = 0; i < kGroup; ++i) v[i] = sum[q * kGroup + i];
          if (g.bias) {
            const int at = min(j + lane, g.n - 1);
            const int64_t id = GATHER ? g.ids[at] : at;
            const float b = id >= 0 && id < g.V ? g.bias[id] : 0.f;
#pragma unroll
            for (int i = 0; i < kGroup; ++i) v[i] += __shfl_sync(0xFFFFFFFFu, b, i);
          }
          if (p.out32 && j + kGroup <= g.n) {
            T* o = y + (int64_t)r * g.ld_out + j;
            if (live) {
#pragma unroll
              for (int i = 0; i < kGroup; i += kLine) {
                float line[kLine];
#pragma unroll
                for (int e = 0; e < kLine; ++e) line[e] = v[i + e];
                store_line(o + i, line);
              }
            }
          } else {
            // turned over in shared memory, so that a warp stores a row's 32 values at once
#pragma unroll
            for (int i = 0; i < kGroup; ++i) turn[lane * kTurnRow + i] = v[i];
            __syncwarp();
            const int rows = min(32, g.rows - row0);
            if (j + lane < g.n) {
              T* o = y + (int64_t)row0 * g.ld_out + j + lane;
              for (int i = 0; i < rows; ++i) store_value(o + i * g.ld_out, turn[i * kTurnRow + lane]);
            }
            __syncwarp();
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
  // (neither CTA leaves, or frees its tensor memory, before the other is done)
  ptx::cluster_sync();
  if (warp == kWarpMma) ptx::tmem_dealloc_pair(tmem, kTmemCols);
}

}  // namespace

cudaError_t launch_fp8_rows_as_m(const Fp8Gemm& g, const uint8_t* x_codes, int64_t ld_x,
                                 const float* x_scales, int64_t ld_xs, int* far, int pair_units,
                                 long long spin_limit, cudaStream_t st) {
  Params p{};
  p.g = g;
  p.x_scales = x_scales;
  p.ld_xs = ld_xs;
  p.row_tiles = (g.rows + 2 * kM - 1) / (2 * kM);
  p.tiles = (int)fp8_rows_as_m_tiles(g.rows, g.n);
  p.kt = (g.d + kFp8Block - 1) / kFp8Block;
  p.out32 = ((uintptr_t)g.out & 31) == 0 && g.ld_out * (g.out_type == TAB_FP32 ? 4 : 2) % 32 == 0;
  p.far = far;
  p.spin_limit = spin_limit;
  CUtensorMap w, row, x;
  if (!code_map(&x, x_codes, (uint64_t)g.d, (uint64_t)g.rows, (uint64_t)ld_x, kM) ||
      !code_map(&w, g.w_codes, (uint64_t)g.d, (uint64_t)g.V, (uint64_t)g.ld_codes, g.ids ? 32 : kN / 2))
    return cudaErrorInvalidValue;
  row = w;
  if (g.ids && !code_map(&row, g.w_codes, (uint64_t)g.d, (uint64_t)g.V, (uint64_t)g.ld_codes, 1))
    return cudaErrorInvalidValue;
  const int units = p.tiles < pair_units ? p.tiles : pair_units;
  auto go = [&](auto kernel) {
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
    if (e != cudaSuccess) return e;
    return launch_pdl_cluster(kernel, dim3((unsigned)(2 * units)), dim3(kThreads), kSmem, st, 2, w, row, x, p);
  };
  const cudaError_t e = g.ids ? go(fp8_rows_as_m_kernel<true, false>) : go(fp8_rows_as_m_kernel<false, false>);
  if (e != cudaSuccess) return e;
  return g.ids ? go(fp8_rows_as_m_kernel<true, true>) : go(fp8_rows_as_m_kernel<false, true>);
}

int64_t fp8_rows_as_m_tiles(int64_t rows, int64_t n) {
  return (n + kN - 1) / kN * ((rows + 2 * kM - 1) / (2 * kM));
}

}  // namespace sph
