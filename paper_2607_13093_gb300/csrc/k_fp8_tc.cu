// Product of hidden states and the kept rows of a table in e4m3 with a scale for each block
// of 128 columns:
//
//   y[r, j] = sum over blocks b of sx[r, b] * sw[id_j, b] * (qx[r, b] . qw[id_j, b])  (+ bias)
//
// where qx, sx are the hidden states in the same form, a scale for each row and block
// (k_fp8.cu).  W's rows are the MMA's M = 128 (256 over a pair of CTAs), the hidden states its N;
// a stage is one block: 128 columns, a 128-byte row of codes.
//
// The scales differ from block to block and are no powers of two, so a block's sums leave
// the tensor core before they are scaled: the MMA warp fills two accumulators in tensor
// memory in turn, one block each, and eight warps (four for few rows) read the one that is
// full and add it, scaled, to sums in their registers: a multiplication and a fused
// multiply-add a value, two values an instruction.  W's scales come four blocks ahead (one
// block ahead the L2's latency was the block's time).
//
// Few rows are bound by W's codes: 8 rows x 152064 ids x 7168 169 us (6.6 TB/s), 64 x 128256 x
// 4096 92 us (5.9 TB/s), 32 x 12000 x 3840 12.3 us; many by the additions, 1024 x 256000 x 4608
// with scales of one row 1343 us (1.8 PFLOP/s).  Many rows and scales of 128 rows: k_fp8_rows.cu.
#include "fp8_tc.cuh"

namespace sph {
namespace {

constexpr int kM = 128;                  // table rows of a tile (of a CTA)
constexpr int kABytes = kM * kFp8Block;
constexpr int kWarpW = 0, kWarpMma = 1, kWarpX = 2, kWarpScale = 3, kWarpOut = 4;
constexpr int kMaxStages = 12;
constexpr int kMaxBn = 256;              // hidden-state rows of a tile
// A block's factors (X's scales): a slot for each block on its way.  One is written
// again once the MMAs of `stages` blocks ago are done, which began when all warps had read the
// accumulator two before that; so no slot that is still read is, with three more than stages.
constexpr int kSxSlots = 16;
static_assert(kSxSlots >= kMaxStages + 3, "slots of factors");
constexpr int kLag = 3, kMinStages = 4;
static_assert(kLag < kMinStages, "a block's stage is free before its factors are announced");
constexpr int kBarBytes = 1024;
constexpr int kSxBytes = kSxSlots * kMaxBn * 4 + 1024;     // (groups of 32 are read whole)
constexpr int kExtraBytes = 1024 + kBarBytes + kSxBytes;   // beside the stages

struct Params {
  Fp8Gemm g;
  const float* x_scales;        // [block][row tiles * bn]
  int64_t ld_xs;
  int bn, row_tiles, tiles, kt; // row tiles are the fast index of a tile
  int stages, stage_bytes;
  int ws16;                     // rows of w_scales are on 16 bytes
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
  uint32_t* holder = reinterpret_cast<uint32_t*>(acc_empty + 2);
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
      // W and X codes of each CTA, X's scales, scattered rows of W
      ptx::mbar_init(&full[s], 2 * kHalves + (PAIR ? 2 : 32) + (pieces ? 32 : 0));
      ptx::mbar_init(&empty[s], 1);
    }
    for (int a = 0; a < 2; ++a) {
      ptx::mbar_init(&acc_full[a], 1);
      ptx::mbar_init(&acc_empty[a], 4 * H * kHalves);
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
  if (warp < kWarpOut) {
    if constexpr (NC >= 96) give_registers<Regs<PAIR>::kFew>();
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
      // ---- X codes -------------------------------------------------------------
      ptx::griddep_wait();
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
    } else if (warp == kWarpScale) {
      // ---- X's scales ----------------------------------------------------------
      // By cp.async, which arrives by itself; not at the even CTA's barrier of a pair, so there
      // kLag blocks are on their way before the first one has to have come.
      ptx::griddep_wait();
      int slot = 0, behind = 0, done = 0, total = 0;       // (pair: the block to announce, its stage)
      auto announce = [&] {
        if (lane == 0) arrive(&full[behind]);
        if (++behind == p.stages) behind = 0;
        ++done;
      };
      for (int tile = unit; ok && tile < p.tiles; tile += units) {
        const float* xs = p.x_scales + tile % p.row_tiles * p.bn;
        for (int k = 0; k < p.kt; ++k) {
          if (!wait(&empty[stage], phase ^ 1)) { ok = false; break; }
          for (int i = lane * 4; i < p.bn; i += 128)
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(
                             ptx::smem_u32(sx_ring + slot * p.bn + i)),
                         "l"(xs + (int64_t)k * p.ld_xs + i)
                         : "memory");
          if constexpr (PAIR) {
            asm volatile("cp.async.commit_group;" ::: "memory");
            if (++total > kLag) {
              asm volatile("cp.async.wait_group %0;" ::"n"(kLag) : "memory");
              __syncwarp();
              announce();
            }
          } else {
            asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(
                             ptx::smem_u32(&full[stage]))
                         : "memory");
          }
          advance();
          if (++slot == kSxSlots) slot = 0;
        }
      }
      if constexpr (PAIR) {
        asm volatile("cp.async.wait_group 0;" ::: "memory");
        __syncwarp();
        while (ok && done < total) announce();
      }
    }
  } else if (warp < kWarpOut + 4 * H) {
    if constexpr (NC >= 96) take_registers<Regs<PAIR>::kMany>();
    // ---- accumulators to sums, sums to y -------------------------------------
    // A thread has a table row and NC columns.  Two groups of columns are requested together,
    // the next two as their registers come free; the accumulator goes back to the MMAs as soon
    // as its last columns have come, before they are added.
    constexpr int G = NC < 32 ? NC : 32;         // columns a group
    constexpr int NG = NC / G;
    const int quarter = warp & 3;                // (the lanes that a warp may read)
    const int col0 = (warp - kWarpOut) / 4 * NC; // the warp's first column
    ptx::griddep_wait();
    int acc = 0, slot = 0;
    uint32_t acc_phase = 0;
    for (int tile = unit; ok && tile < p.tiles; tile += units) {
      const int r0 = tile % p.row_tiles * p.bn, rows = min(p.bn, g.rows - r0);
      const int j = first_row(tile) + quarter * 32 + lane;
      const bool live = j < g.n;
      const int64_t id = !live ? -1 : gather ? g.ids[j] : j;
      const bool there = id >= 0 && id < g.V;
      const float* ws = g.w_scales + (there ? id / g.block_rows : 0) * g.ld_scales;
      const float b = there && g.bias ? g.bias[id] : 0.f;
      // (four blocks' scales at a time, four blocks ahead: one ahead, their way from the L2 took
      // longer than a block)
      auto scales = [&](int k) {
        if (p.ws16 && k + 4 <= p.kt) return *reinterpret_cast<const float4*>(ws + k);
        const int last = p.kt - 1;
        return make_float4(ws[min(k, last)], ws[min(k + 1, last)], ws[min(k + 2, last)], ws[min(k + 3, last)]);
      };
      float4 four = scales(0), ahead = four;
      uint64_t sum[NC / 2];
#pragma unroll
      for (int i = 0; i < NC / 2; ++i) sum[i] = 0;
      for (int k = 0; k < p.kt; ++k) {
        if ((k & 3) == 0) {
          if (k > 0) four = ahead;
          if (k + 4 < p.kt) ahead = scales(k + 4);
        }
        float sw = (k & 2) ? ((k & 1) ? four.w : four.z) : ((k & 1) ? four.y : four.x);
        // Where a scale is far from 1 a factor of 2^64 goes from it to the other one.
        float lift = 1.f;
        const float mag = fabsf(sw);
        if (mag > kFar) { lift = 0x1p64f; sw *= 0x1p-64f; }
        else if (mag < kNear && mag > 0.f) { lift = 0x1p-64f; sw *= 0x1p64f; }
        const bool far = __any_sync(0xFFFFFFFFu, lift != 1.f);
        if (!wait(&acc_full[acc], acc_phase, true)) { ok = false; break; }
        ptx::tc_fence_after();
        const uint32_t t = tmem + acc * kAccCols + col0 + ((uint32_t)(quarter * 32) << 16);
        uint32_t v[2][G];
        tmem_request(t, v[0]);
        if constexpr (NG > 1) tmem_request(t + G, v[1]);
        const float* sx = sx_ring + slot * p.bn + col0;
        const uint64_t sw2 = pack2(sw, sw);
        auto add = [&](int q, uint32_t (&of)[G]) {
          if (!far) {
#pragma unroll
            for (int i = 0; i < G / 4; ++i) {
              const ulonglong2 s = *reinterpret_cast<const ulonglong2*>(sx + q * G + 4 * i);
              uint64_t& lo = sum[(q * G + 4 * i) / 2];
              uint64_t& hi = sum[(q * G + 4 * i) / 2 + 1];
              const uint64_t t0 = pack2(of[4 * i], of[4 * i + 1]), t1 = pack2(of[4 * i + 2], of[4 * i + 3]);
              lo = fma2(mul2(t0, sw2), s.x, lo);
              hi = fma2(mul2(t1, sw2), s.y, hi);
            }
          } else {
#pragma unroll
            for (int i = 0; i < G / 2; ++i) {
              const float s0 = bounded(sx[q * G + 2 * i] * lift), s1 = bounded(sx[q * G + 2 * i + 1] * lift);
              uint64_t& at = sum[(q * G + 2 * i) / 2];
              at = fma2_here(mul2(pack2(of[2 * i], of[2 * i + 1]), sw2), pack2(s0, s1), at);
            }
          }
        };
        auto release = [&] {
          ptx::tc_fence_before();
          __syncwarp();
          if (lane == 0) arrive(&acc_empty[acc]);
        };
        tmem_wait();
        if constexpr (NG <= 2) release();
        arrived(v[0]);
        if constexpr (NG > 1) arrived(v[1]);
        add(0, v[0]);
        if constexpr (NG > 2) tmem_request(t + 2 * G, v[0]);
        if constexpr (NG > 1) add(1, v[1]);
        if constexpr (NG > 3) tmem_request(t + 3 * G, v[1]);
        if constexpr (NG > 2) {
          tmem_wait();
          release();
          arrived(v[0]);
          if constexpr (NG > 3) arrived(v[1]);
          add(2, v[0]);
          if constexpr (NG > 3) add(3, v[1]);
        }
        if (++acc == 2) { acc = 0; acc_phase ^= 1; }
        if (++slot == kSxSlots) slot = 0;
      }
      if (!ok) break;
      // (values first, then their stores in one block without conditions)
      auto store = [&](auto* y) {
#pragma unroll
        for (int q = 0; q < NG; ++q) {
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
size_t up256(size_t x) { return (x + 255) / 256 * 256; }

struct Plan {
  int rows_as_m;                // the other kernel (k_fp8_rows.cu)
  int pair, bn, row_tiles, tiles, kt, stages, stage_bytes, units;
};
// As many equal tiles of hidden-state rows as these need.
Plan plan_of(const Fp8Plan& a) {
  Plan pl{};
  // The other kernel where its 256 rows are at most a fifth padding (single CTAs here / that
  // kernel, us: 256 rows x 152064 ids x 7168 383 / 253, 1024 x 256000 x 4608 1636 / 965; 128 x
  // 128256 x 4096 109 / 136, 320 x 51302 kept ids x 3584 117 / 138).  Pairs for row tiles above
  // 192 (scales of one row, single CTAs / pairs: 256 x 152064 x 7168 404 / 330, 1024 x 256000 x
  // 4608 1690 / 1343; tiles of 160, 320 x 51302 112 / 120).
  const int64_t count = (a.rows + kMaxBn - 1) / kMaxBn;
  pl.rows_as_m = a.pair_units > 0 && a.block_rows == kFp8Block &&
                 (a.pair_mode == 2 ? a.rows > 64 : a.pair_mode == 1 && 5 * a.rows >= 4 * 256 * count);
  pl.pair = a.pair_units > 0 && (a.pair_mode == 2 || (a.pair_mode == 1 && a.rows > 192 * count));
  const int unit = pl.pair ? 32 : 16;
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

struct Scratch {        // X: codes, and scales [block][ld_scales], or [row][ld_scales]
  int64_t ld, ld_scales, tiles;
  size_t scales, far, bytes;    // (far: a word for each of the other kernel's tiles)
};
Scratch scratch_of(const Plan& pl, int64_t rows, int64_t n, int d) {
  Scratch o{};
  o.ld = (d + 15) / 16 * 16;
  o.ld_scales = pl.rows_as_m ? (pl.kt + 3) / 4 * 4 : (int64_t)pl.row_tiles * pl.bn;
  o.scales = up256((size_t)(rows * o.ld));
  o.far = o.scales + up256((size_t)(pl.rows_as_m ? rows : pl.kt) * o.ld_scales * 4);
  o.tiles = pl.rows_as_m ? fp8_rows_as_m_tiles(rows, n) : 0;
  o.bytes = o.far + up256((size_t)o.tiles * 4);
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
  if (p.bn <= 192) return launch<96, 2, PAIR>(m, p, units, st);
  return launch<128, 2, PAIR>(m, p, units, st);
}
}  // namespace

size_t fp8_gemm_scratch_bytes(const Fp8Plan& a) { return scratch_of(plan_of(a), a.rows, a.n, a.d).bytes; }

// At least what any call of up to so many rows, kept ids and columns takes: tiles cover at
// most 32 more rows each, and one that is not the only one has at least 64.
size_t fp8_gemm_reserve_bytes(int64_t rows, int64_t n, int64_t d) {
  const size_t padded = 2 * (size_t)rows + 64, kt = (size_t)((d + kFp8Block - 1) / kFp8Block);
  return up256((size_t)rows * ((size_t)(d + 15) / 16 * 16)) + up256((kt + 3) * padded * 4) +
         up256((size_t)fp8_rows_as_m_tiles(rows, n) * 4);
}

cudaError_t launch_fp8_gemm(const Fp8Gemm& g, const Fp8Plan& a, void* scratch, long long spin_limit,
                            cudaStream_t st) {
  const Plan pl = plan_of(a);
  const Scratch o = scratch_of(pl, g.rows, g.n, g.d);
  char* at = static_cast<char*>(scratch);
  Params p{};
  p.g = g;
  p.x_scales = reinterpret_cast<float*>(at + o.scales);
  p.ld_xs = o.ld_scales;
  p.bn = pl.bn; p.row_tiles = pl.row_tiles; p.tiles = pl.tiles; p.kt = pl.kt;
  p.stages = pl.stages; p.stage_bytes = pl.stage_bytes;
  p.spin_limit = spin_limit;
  p.ws16 = ((uintptr_t)g.w_scales & 15) == 0 && g.ld_scales % 4 == 0;
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
  q.row_step = pl.rows_as_m ? o.ld_scales : 1;
  q.col_step = pl.rows_as_m ? 1 : o.ld_scales;
  q.zero = reinterpret_cast<int*>(at + o.far);
  q.zeros = o.tiles;
  cudaError_t e = launch_fp8_quant(q, g.x_type, st);
  if (e != cudaSuccess) return e;
  if (pl.rows_as_m)
    return launch_fp8_rows_as_m(g, q.codes, o.ld, p.x_scales, o.ld_scales, q.zero, a.pair_units,
                                spin_limit, st);
  return pl.pair ? launch_bn<true>(m, p, pl.units, st) : launch_bn<false>(m, p, pl.units, st);
}

}  // namespace sph
