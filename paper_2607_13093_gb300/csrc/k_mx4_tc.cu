// Product of hidden states and the kept rows of a table held in 4 bits:
//
//   y[r, j] = sum_c X[r, c] * W[ids[j], c] (+ bias[ids[j]])
//
// with X the sum of `planes` terms in the table's own format (k_mx4.cu).  Both
// operands go to the tensor cores in 4 bits with their block scales
// (tcgen05.mma kind::mxf4nvf4): W's rows are the MMA's M = 128, the hidden
// states its N, and all terms of X meet a stage of W, so a term costs its MMAs
// and no traffic of W.  The first two terms add into one accumulator, the third and
// fourth into another: an MMA drops what lies below its accumulator's 24 bits, which
// two terms mostly fit and four do not (300 rows x 4608, four terms in one accumulator:
// 3e-6 off in norm, in two 5e-8).
//
// A CTA keeps a ring of stages of 256 columns, 128 bytes of codes a row: codes by
// TMA, rows of W whose kept ids are not consecutive by cp.async; X's scales by TMA,
// W's by cp.async.  Eight warps move a
// stage's scales from shared memory to tensor memory (in the quarter of the lanes
// that each may write), into one of several sets of columns; one warp issues the
// MMAs; four read the accumulator and store it, while the next tile's is computed (three
// or four terms of more rows than fit twice have one accumulator, and wait).
// (Scales by tcgen05.cp took some 80 cycles a copy of four columns in the MMAs' own
// queue: 1024 rows x 256000 ids x 4608 907 us.)
//
// Few rows are bound by the stream of W: 8 rows x 152064 ids x 7168 take 91.5 us,
// 6.7 TB/s of the table's 4.5 bits an element.  Many rows are bound by what an SM gets
// from the L2, some 54 bytes a cycle: 1024 rows x 256000 ids x 4608 in one term come in
// tiles of 208 rows, whose stages of 48 KB, more than half of it X, take some 900 cycles
// each; the call takes 526 us, 4.6 PFLOP/s.  The MMA warp's own time a stage, some 560
// cycles whatever the rows (waits, descriptors, the commit), lies behind that, and shows
// where a stage is small (32 rows x 12000 ids x 3840 9.9 us: 15 stages one after another).
// So that warp has one barrier to wait for and one to signal, issues a stage's MMAs in
// one piece, and takes the terms of few rows as more rows of one MMA.
//
// PAIR: two CTAs share a tile of 256 table rows (cta_group::2): each holds its 128
// rows of W and half of X's codes, so that a stage costs each SM half the traffic of X.
// The even CTA issues the MMAs for both.
//
// Work is whole tiles in turn, or, where these would leave SMs idle, equal ranges of
// all tiles' stages: tiles cut by a range's end leave fp32 parts, and the last CTA
// to count in adds them in the order of the ranges.
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
constexpr int kThreads = 512;            // 16 warps
constexpr int kWarpW = 0, kWarpMma = 1, kWarpX = 2, kWarpRaw = 3, kWarpScale = 4, kWarpOut = 8;
constexpr int kWarpScale2 = 12;          // (the second four of them)
constexpr int kMaxSets = 8;              // sets of scale columns in tensor memory
constexpr int kWsRow = 64;               // bytes of a table row's scales copied together
constexpr int kWsSlots = 3, kWsBytes = kM * kWsRow;
constexpr int kMaxStages = 12;
constexpr int kMaxBn = 256;              // hidden-state rows of a tile
constexpr int kPairRows = 96;            // more rows than these may take CTA pairs
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
// One column of this warp's lanes, read and written.
__device__ __forceinline__ float tmem_ld1(uint32_t taddr) {
  uint32_t r;
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x1.b32 {%0}, [%1];" : "=r"(r) : "r"(taddr));
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
  return __uint_as_float(r);
}
__device__ __forceinline__ void tmem_st1(uint32_t taddr, float v) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x1.b32 [%0], {%1};" ::"r"(taddr), "r"(__float_as_uint(v))
               : "memory");
  asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
}
// X's scales of a stage, one row after another in shared memory (4 G bytes each), to
// tensor memory: word q of row r goes to lane r % 32 of column q * 4 C + r / 32.
// (What rows past `rows` get is read by no MMA.)
template <int G, int C>
__device__ __forceinline__ void load_scales(uint32_t (&w)[G * 4 * C], const uint8_t* src, int rows,
                                            int lane) {
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
}
// W's, from the 64-byte rows of several stages (kWsRow).
template <int G>
__device__ __forceinline__ void load_w_scales(uint32_t (&w)[G * 4], const uint8_t* src, int in_slot,
                                              int lane) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = 32 * i + lane, piece = G == 4 ? in_slot : in_slot / 2;
    const uint8_t* at = src + r * kWsRow + (piece ^ (r >> 1 & 3)) * 16;
    if constexpr (G == 4) {
      const uint4 v = *reinterpret_cast<const uint4*>(at);
      w[i] = v.x; w[4 + i] = v.y; w[8 + i] = v.z; w[12 + i] = v.w;
    } else {
      const uint2 v = reinterpret_cast<const uint2*>(at)[in_slot & 1];
      w[i] = v.x; w[4 + i] = v.y;
    }
  }
}
// e2m1 operands, K-major, fp32 accumulator: N, M / 16, and the scales' format
// (bit 23: e8m0).  With 32-column blocks an MMA's two scales are the low or the
// high half of a scale word (the ids in bits 4 and 29).
template <int FMT>
__host__ __device__ constexpr uint32_t idesc_mx4(int M, int N, int half) {
  return (1u << 7) | (1u << 10) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24) |
         (FMT == MX4_E8M0 ? 1u << 23 : 0u) | ((uint32_t)(2 * half) << 4) |
         ((uint32_t)(2 * half) << 29);
}
// One MMA of 64 columns, or (mma4) the four of a stage, issued by one elected lane:
// the operands advance by 32 bytes, the scales by a column group an MMA (e4m3) or
// every other one (e8m0: `other` is the descriptor of the second half).
#define SPH_MMA_MX4(group, vec)                                                              \
  asm volatile(                                                                              \
      "{\n .reg .pred p, q;\n .reg .b64 a, b;\n elect.sync _|q, 0xFFFFFFFF;\n"               \
      " setp.ne.b32 p, %4, 0;\n mov.b64 a, {%1, %5};\n mov.b64 b, {%2, %5};\n"               \
      " @q tcgen05.mma.cta_group::" group ".kind::mxf4nvf4.block_scale.scale_vec::" vec      \
      " [%0], a, b, %3, [%6], [%7], p;\n}\n" ::"r"(d),                                       \
      "r"(adesc), "r"(bdesc), "r"(idesc), "r"(accumulate), "r"(ptx::kSdescHi), "r"(sfa),     \
      "r"(sfb)                                                                               \
      : "memory")
template <int FMT, bool PAIR>
__device__ __forceinline__ void mma_mx4(uint32_t d, uint32_t adesc, uint32_t bdesc, uint32_t idesc,
                                        uint32_t sfa, uint32_t sfb, uint32_t accumulate) {
  if constexpr (FMT == MX4_E4M3 && PAIR) SPH_MMA_MX4("2", "4X");
  else if constexpr (FMT == MX4_E4M3) SPH_MMA_MX4("1", "4X");
  else if constexpr (PAIR) SPH_MMA_MX4("2", "2X");
  else SPH_MMA_MX4("1", "2X");
}
#undef SPH_MMA_MX4
#define SPH_STEP(group, vec, desc, sa, sb, acc)                                              \
  " mov.b64 a, {x, %5};\n mov.b64 b, {y, %5};\n"                                             \
  " @q tcgen05.mma.cta_group::" group ".kind::mxf4nvf4.block_scale.scale_vec::" vec          \
  " [%0], a, b, " desc ", [" sa "], [" sb "], " acc ";\n add.u32 x, x, 2;\n add.u32 y, y, 2;\n"
#define SPH_MMA4_HEAD                                                                        \
  "{\n .reg .pred p, q, t;\n .reg .b64 a, b;\n .reg .b32 x, y, u, v;\n"                      \
  " elect.sync _|q, 0xFFFFFFFF;\n setp.ne.b32 p, %4, 0;\n setp.eq.b32 t, 0, 0;\n"            \
  " mov.b32 x, %1;\n mov.b32 y, %2;\n mov.b32 u, %6;\n mov.b32 v, %7;\n"
#define SPH_NEXT " add.u32 u, u, 4;\n add.u32 v, v, %8;\n"
#define SPH_MMA4_E4M3(group)                                                                 \
  asm volatile(SPH_MMA4_HEAD SPH_STEP(group, "4X", "%3", "u", "v", "p")                      \
                   SPH_NEXT SPH_STEP(group, "4X", "%3", "u", "v", "t")                       \
                       SPH_NEXT SPH_STEP(group, "4X", "%3", "u", "v", "t")                   \
                           SPH_NEXT SPH_STEP(group, "4X", "%3", "u", "v", "t") "}\n" ::"r"(d), \
               "r"(adesc), "r"(bdesc), "r"(idesc), "r"(accumulate), "r"(ptx::kSdescHi),      \
               "r"(sfa), "r"(sfb), "r"(sfb_step)                                             \
               : "memory")
#define SPH_MMA4_E8M0(group)                                                                 \
  asm volatile(SPH_MMA4_HEAD SPH_STEP(group, "2X", "%3", "u", "v", "p")                      \
                   SPH_STEP(group, "2X", "%9", "u", "v", "t")                                \
                       SPH_NEXT SPH_STEP(group, "2X", "%3", "u", "v", "t")                   \
                           SPH_STEP(group, "2X", "%9", "u", "v", "t") "}\n" ::"r"(d),        \
               "r"(adesc), "r"(bdesc), "r"(idesc), "r"(accumulate), "r"(ptx::kSdescHi),      \
               "r"(sfa), "r"(sfb), "r"(sfb_step), "r"(other)                                 \
               : "memory")
template <int FMT, bool PAIR>
__device__ __forceinline__ void mma4_mx4(uint32_t d, uint32_t adesc, uint32_t bdesc, uint32_t idesc,
                                         uint32_t other, uint32_t sfa, uint32_t sfb,
                                         uint32_t sfb_step, uint32_t accumulate) {
  if constexpr (FMT == MX4_E4M3 && PAIR) SPH_MMA4_E4M3("2");
  else if constexpr (FMT == MX4_E4M3) SPH_MMA4_E4M3("1");
  else if constexpr (PAIR) SPH_MMA4_E8M0("2");
  else SPH_MMA4_E8M0("1");
}
#undef SPH_STEP
#undef SPH_NEXT
#undef SPH_MMA4_HEAD
#undef SPH_MMA4_E4M3
#undef SPH_MMA4_E8M0
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

// Arrivals at a barrier of either CTA of a pair (a shared::cluster address).  What
// they announce is in tensor memory (complete, by tcgen05.wait, before) or comes by
// TMA: no generic writes that a release at cluster scope would have to wait for.
__device__ __forceinline__ void arrive_at(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void expect_at(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cluster.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes)
               : "memory");
}
// Whether `ok` holds in all of the barrier's threads.
__device__ __forceinline__ bool all_of(int barrier, int threads, bool ok) {
  uint32_t r;
  asm volatile(
      "{\n .reg .pred p, q;\n setp.ne.u32 q, %1, 0;\n bar.red.and.pred p, %2, %3, q;\n"
      " selp.u32 %0, 1, 0, p;\n}\n"
      : "=r"(r)
      : "r"((uint32_t)ok), "r"(barrier), "r"(threads)
      : "memory");
  return r != 0;
}

__device__ __forceinline__ void store_value(float* p, float v) { *p = v; }
__device__ __forceinline__ void store_value(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }

struct Params {
  Mx4Gemm g;
  const uint8_t* x_scales;      // [row tile][stage][term][bn][scale bytes of a stage]
  const float* x_row;           // [row tiles * bn], e4m3 only
  int bn, row_tiles, tiles, kt; // row tiles are the fast index of a tile
  int mma_n, terms;             // an MMA's N, and MMAs a step: bn and `planes`, or (few
                                // rows) the terms' rows one after another and 1
  int accs, acc_cols;           // accumulators of a tile: buffers, columns of each
  int low_col;                  // where the third and fourth term's sums start (0: none)
  int stages, stage_bytes, chunks, sf_col, sf_cols, sf_sets;
  int ranges;                   // 1: equal ranges of stages, 0: whole tiles in turn
  float* parts;                 // [unit][2][half][bn][128] of tiles that a range's end cuts
  unsigned* counts;             // [tile][half], zero
  long long spin_limit;
};

// The same value as lane 0's, which the compiler then knows to be one for the warp.
__device__ __forceinline__ long long uniform(long long v) {
  const uint32_t lo = __shfl_sync(0xFFFFFFFFu, (uint32_t)v, 0);
  const uint32_t hi = __shfl_sync(0xFFFFFFFFu, (uint32_t)((unsigned long long)v >> 32), 0);
  return (long long)((unsigned long long)hi << 32 | lo);
}

// A unit's work: whole tiles unit, unit + units, ..., or the stages of a range, tile by
// tile.  Its results are uniform: a division's are not for the compiler, and loops over
// them would cost the MMA warp its uniform registers.
struct Work {
  int ranges, kt, tiles, units;
  long long at, end;
  __device__ Work(const Params& p, int unit, int n)
      : ranges(p.ranges), kt(p.kt), tiles(p.tiles), units(n) {
    at = ranges ? uniform(start(unit)) : unit;
    end = ranges ? uniform(start(unit + 1)) : tiles;
  }
  __device__ long long start(int unit) const { return (long long)tiles * kt * unit / units; }
  // the unit whose range holds stage `it`
  __device__ int holder(long long it) const {
    return (int)(((it + 1) * units - 1) / ((long long)tiles * kt));
  }
  __device__ bool next(int& tile, int& k0, int& k1) {
    if (at >= end) return false;
    if (!ranges) {
      tile = (int)at;
      k0 = 0;
      k1 = kt;
      at += units;
    } else {
      tile = __shfl_sync(0xFFFFFFFFu, (int)(at / kt), 0);
      k0 = (int)(at - (long long)tile * kt);
      k1 = (int)min((long long)kt, k0 + end - at);
      at += k1 - k0;
    }
    return true;
  }
};

// The row scales of W and X may be as far apart as 2^116 and 2^-110, and a sum is a multiple
// of 2^-20 below 2^45: times a W scale above this it may pass fp32's range where the logit
// does not.
constexpr float kFarScale = 0x1p80f;
// A warp that has such a row of W scales its tile's sums here, where they are, the further
// terms' added (W scales above 1 after X's, others before: exactly, as 2^-130 is a step of
// fp32), and goes on with scales of 1; what a cut tile leaves is scaled then.  Not in the
// unrolled code of every tile: the choice there, or one product more a value, made all calls
// longer (1024 rows x 256000 ids x 4608 525 us, 562 and 547).
__device__ __noinline__ void scale_far_sums(uint32_t t, int bn, int acc_cols, int rows, float ws,
                                            const float* x_row) {
  for (int i = 0; i < rows; ++i) {
    float v = tmem_ld1(t + i);
    for (int c = bn; c < acc_cols; c += bn) {
      v += tmem_ld1(t + c + i);
      tmem_st1(t + c + i, 0.f);
    }
    tmem_st1(t + i, v * (ws < 1.f ? ws : 1.f) * x_row[i] * (ws < 1.f ? 1.f : ws));
  }
}

template <int FMT, bool GATHER, bool PAIR, class OT>
__global__ void __launch_bounds__(kThreads, 1)
mx4_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_row,
           const __grid_constant__ CUtensorMap map_x, const Params p) {
  constexpr int kGroups = groups_of(FMT);
  constexpr int kHalves = PAIR ? 2 : 1;         // CTAs of a unit, 128 table rows each
  constexpr bool kPieces = GATHER && !PAIR;     // scattered rows by cp.async
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw_addr = ptx::smem_u32(smem_raw);
  const uint32_t base_addr = (raw_addr + 1023) & ~1023u;
  uint8_t* base = smem_raw + (base_addr - raw_addr);
  uint64_t* full = reinterpret_cast<uint64_t*>(base + (size_t)p.stages * p.stage_bytes);
  uint64_t* raw = full + kMaxStages;            // X's scales of a stage are there
  uint64_t* empty = raw + kMaxStages;
  uint64_t* acc_full = empty + kMaxStages;      // [2]
  uint64_t* acc_empty = acc_full + 2;           // [2]
  uint64_t* sf_full = acc_empty + 2;            // [kMaxSets]
  uint64_t* ws_full = sf_full + kMaxSets;       // [kWsSlots]
  uint64_t* ws_empty = ws_full + kWsSlots;      // [kWsSlots]
  uint32_t* holder = reinterpret_cast<uint32_t*>(ws_empty + kWsSlots);
  volatile int* s_abort = reinterpret_cast<volatile int*>(holder + 1);
  volatile unsigned* s_count = reinterpret_cast<volatile unsigned*>(holder + 2);
  // (from lane 0, so that the compiler knows that a warp takes one branch and can
  // keep its loop's counters and descriptors in uniform registers)
  const int warp = __shfl_sync(0xFFFFFFFFu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  const Mx4Gemm& g = p.g;
  const int half = PAIR ? __shfl_sync(0xFFFFFFFFu, (int)ptx::cluster_ctarank(), 0) : 0;
  const int unit = (int)blockIdx.x / kHalves, units = (int)gridDim.x / kHalves;
  constexpr int kRow = 4 * kGroups;             // scale bytes of a row and stage
  // W's scales, 64 bytes a row: those of several stages
  uint8_t* ws_ring = base + (size_t)p.stages * p.stage_bytes + kBarBytes;
  constexpr int kWsStages = kWsRow / kRow;
  // a stage: W codes, X codes (a term after the other), X scales
  const int bnc = p.bn / kHalves;               // rows of X's codes in this CTA
  const int x_bytes = bnc * (kCols / 2), xs_bytes = p.bn * kRow;
  const int off_xs = kABytes + g.planes * x_bytes;

  if (threadIdx.x == 0) {
    for (int s = 0; s < p.stages; ++s) {
      // W and X codes of each CTA, scattered rows of W
      ptx::mbar_init(&full[s], 2 * kHalves + (kPieces ? 32 : 0));
      ptx::mbar_init(&raw[s], 1);
      ptx::mbar_init(&empty[s], 1);
    }
    for (int a = 0; a < 2; ++a) {
      ptx::mbar_init(&acc_full[a], 1);
      ptx::mbar_init(&acc_empty[a], 4 * kHalves);
    }
    for (int s = 0; s < p.sf_sets; ++s) ptx::mbar_init(&sf_full[s], 4 * kHalves);
    for (int s = 0; s < kWsSlots; ++s) {
      ptx::mbar_init(&ws_full[s], 32);
      ptx::mbar_init(&ws_empty[s], 8);
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
  // whole warp gets one answer.
  // at_once: asked first without suspension, so that a limit of a cycle or two runs
  // out where the phase is not complete yet (the accumulator's readers and the
  // producer of W's codes; elsewhere it would only delay the end of a wait).
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
  // the ids of rows 4 lane .. 4 lane + 3, rows past the last kept id repeating it, and
  // which 32-row groups are consecutive ids
  auto ids_of = [&](int tile, unsigned& solid) {
    const int j = first_row(tile) + 4 * lane, last = g.n - 1;
    const int4 id = make_int4(g.ids[min(j, last)], g.ids[min(j + 1, last)], g.ids[min(j + 2, last)],
                              g.ids[min(j + 3, last)]);
    const bool own = id.y == id.x + 1 && id.z == id.x + 2 && id.w == id.x + 3;
    const int next = __shfl_down_sync(0xFFFFFFFFu, id.x, 1);
    const unsigned four = __ballot_sync(0xFFFFFFFFu, own);
    const unsigned link = __ballot_sync(0xFFFFFFFFu, next == id.w + 1);
    solid = 0;
#pragma unroll
    for (int q = 0; q < 4; ++q)
      if ((four >> 8 * q & 0xFFu) == 0xFFu && (link >> 8 * q & 0x7Fu) == 0x7Fu) solid |= 1u << q;
    return id;
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
  Work work(p, unit, units);
  int tile, k0, k1;
  bool ok = true;

  if (warp == kWarpW) {
    // ---- W codes -----------------------------------------------------------
    // Groups of 32 consecutive ids are one box.  Rows of others come as 16-byte pieces
    // by cp.async, four rows an instruction, each piece where the 128-byte swizzle has
    // it; on pairs, whose barriers wait for no generic writes (arrive_at), four rows a
    // copy.  (32 rows x 12000 of 32000 ids x 3840: all ids 9.9 us, scattered ones 11.1 by
    // cp.async, 20.6 by such copies on single CTAs.)
    const int bytes = (g.d + 31) / 32 * 16;
    while (ok && work.next(tile, k0, k1)) {
      const int j0 = first_row(tile);
      int4 id;
      unsigned solid = 0;
      // where rows lane / 8, lane / 8 + 4, ... begin (ids outside the table, which are the
      // caller's mistake, take the codes of a row of it, with scale bytes of 0: 0 in e4m3,
      // 2^-127 in e8m0)
      const uint8_t* from[kPieces ? 32 : 1];
      if constexpr (GATHER) id = ids_of(tile, solid);
      if constexpr (kPieces) {
        if (solid != 0xFu) {
#pragma unroll
          for (int i = 0; i < 32; ++i) {
            const int row = g.ids[min(j0 + 4 * i + (lane >> 3), (int)g.n - 1)];
            from[i] = g.w_codes + max(0, min(row, (int)g.V - 1)) * g.ld_codes;
          }
        }
      }
      for (int k = k0; k < k1; ++k) {
        if (!wait(&empty[stage], phase ^ 1, true)) { ok = false; break; }
        uint8_t* a = base + (size_t)stage * p.stage_bytes;
        const uint32_t bar = leader(&full[stage]);
        const int x = k * (kCols / 2);
        if (lane == 0) expect(&full[stage], kPieces ? __popc(solid) * (kABytes / 4) : kABytes);
        __syncwarp();
        auto box = [&](uint8_t* dst, int row) {
          if constexpr (PAIR) ptx::tma_load_2d_pair(dst, &map_w, x, row, bar);
          else ptx::tma_load_2d(dst, &map_w, x, row, &full[stage]);
        };
        if constexpr (GATHER) {
          if (solid >> (lane >> 3) & 1) {
            if ((lane & 7) == 0) box(a + lane * 512, id.x);
          } else if constexpr (!kPieces) {
            tma_gather4(a + lane * 512, &map_row, x, id, bar);
          }
          if constexpr (kPieces) {
            const int piece = lane & 7, row = lane >> 3;
            const int size = x + 16 * piece < bytes ? 16 : 0;
            const int at = size ? x + 16 * piece : 0;
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
    // (One copy each for all terms: each one that a producer's thread issues takes it
    // some 150 cycles.)
    ptx::griddep_wait();
    while (ok && work.next(tile, k0, k1)) {
      const int rt = tile % p.row_tiles, r0 = rt * p.bn + half * bnc;
      for (int k = k0; k < k1; ++k) {
        if (!wait(&empty[stage], phase ^ 1)) { ok = false; break; }
        if (lane == 0) {
          uint8_t* s = base + (size_t)stage * p.stage_bytes + kABytes;
          expect(&full[stage], (uint32_t)(g.planes * x_bytes));
          if constexpr (PAIR)
            ptx::tma_load_3d_pair(s, &map_x, k * (kCols / 2), r0, 0, leader(&full[stage]));
          else
            ptx::tma_load_3d(s, &map_x, k * (kCols / 2), r0, 0, &full[stage]);
          const uint32_t size = (uint32_t)(g.planes * xs_bytes);
          ptx::mbar_expect_tx(&raw[stage], size);
          bulk_load(s - kABytes + off_xs, p.x_scales + ((int64_t)rt * p.kt + k) * size, size,
                    &raw[stage]);
        }
        __syncwarp();
        advance();
      }
    }
  } else if (warp == kWarpRaw) {
    // ---- W scales to shared memory -----------------------------------------
    // By cp.async, 64 bytes a row (four or eight stages' worth) by four lanes, so that
    // an instruction touches 8 rows.  (16 bytes of 32 rows an instruction cost the
    // shared memory some 50 cycles each, a quarter of what a stage has; boxes of 16
    // bytes by 128 rows by TMA took longer still.)  The 16-byte piece c of row r lies
    // at place c ^ (r / 2 % 4), so that lanes that read a piece of 32 rows meet no bank
    // twice.  Rows past the last kept id and bytes past the last scale become zeros.
    const int bytes = (g.d + Mx4<FMT>::kBlock - 1) / Mx4<FMT>::kBlock;
    const int sub = lane >> 2, piece = lane & 3;
    int slot = 0;
    uint32_t slot_phase = 0;
    while (ok && work.next(tile, k0, k1)) {
      const int j0 = first_row(tile) + sub;
      int id[kM / 8];
#pragma unroll
      for (int i = 0; i < kM / 8; ++i) {
        const int j = j0 + 8 * i;
        id[i] = j < g.n ? (GATHER ? g.ids[j] : j) : -1;
        if (GATHER && (uint32_t)id[i] >= (uint32_t)g.V) id[i] = -1;
      }
      for (int w = k0 / kWsStages; w * kWsStages < k1; ++w) {
        if (!wait(&ws_empty[slot], slot_phase ^ 1)) { ok = false; break; }
        const int at = w * kWsRow + 16 * piece, left = min(16, max(0, bytes - at));
        const uint32_t dst = ptx::smem_u32(ws_ring + slot * kWsBytes);
#pragma unroll
        for (int i = 0; i < kM / 8; ++i) {
          const int r = 8 * i + sub;
          const bool there = id[i] >= 0 && left > 0;
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(
                           dst + r * kWsRow + (piece ^ (r >> 1 & 3)) * 16),
                       "l"(there ? g.w_scales + (int64_t)id[i] * g.ld_scales + at : g.w_scales),
                       "r"(there ? left : 0)
                       : "memory");
        }
        asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(
                         ptx::smem_u32(&ws_full[slot]))
                     : "memory");
        if (++slot == kWsSlots) { slot = 0; slot_phase ^= 1; }
      }
    }
  } else if ((warp >= kWarpScale && warp < kWarpScale + 4) || warp >= kWarpScale2) {
    // ---- scales to tensor memory -------------------------------------------
    // Two groups of four warps take the stages in turn.  A set of columns is free once
    // the MMAs of the stage that had it last are done, which is when that stage's
    // shared memory is (there are no more sets than stages).  The group signals the
    // MMA warp once the stage's codes are there too, so that it waits once.
    const uint32_t lanes = (uint32_t)(warp % 4 * 32) << 16;
    bool turn = warp < kWarpScale2;
    int had = 0, behind = -p.sf_sets;         // the stage that had the set, its use
    uint32_t had_phase = 0;
    int slot = 0;
    uint32_t slot_phase = 0;
    while (ok && work.next(tile, k0, k1)) {
      for (int k = k0; k < k1; ++k, turn = !turn) {
        const int in_slot = k % kWsStages;
        if ((k == k0 || in_slot == 0) && !wait(&ws_full[slot], slot_phase)) { ok = false; break; }
        if (turn) {
          if (!wait(&raw[stage], phase)) { ok = false; break; }
          // (in registers before the set is free: what comes after that delays the MMAs)
          uint32_t w[4 * kGroups];
          load_w_scales<kGroups>(w, ws_ring + slot * kWsBytes, in_slot, lane);
          const uint8_t* xs = base + (size_t)stage * p.stage_bytes + off_xs;
          const uint32_t to = tmem + lanes + p.sf_col + set * p.sf_cols;
          auto move = [&](auto chunks) {
            constexpr int C = decltype(chunks)::value;
            uint32_t x[4 * kGroups * C];
            load_scales<kGroups, C>(x, xs, p.mma_n, lane);
            if (behind >= 0 && !wait(&empty[had], had_phase)) return false;
            ptx::tc_fence_after();
            tmem_st(to, w);
            tmem_st(to + 4 * kGroups, x);
            for (int t = 1; t < p.terms; ++t) {
              load_scales<kGroups, C>(x, xs + t * p.mma_n * kRow, p.mma_n, lane);
              tmem_st(to + 4 * kGroups * (1 + t * C), x);
            }
            return true;
          };
          if (!(p.chunks == 1 ? move(std::integral_constant<int, 1>())
                              : move(std::integral_constant<int, 2>()))) {
            ok = false;
            break;
          }
          asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
          ptx::tc_fence_before();
          if (half == 0 && !wait(&full[stage], phase)) { ok = false; break; }
          // (what cp.async wrote is there for the MMAs' reads)
          if constexpr (kPieces) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          __syncwarp();
          if (lane == 0) arrive(&sf_full[set]);
        }
        if (in_slot == kWsStages - 1 || k == k1 - 1) {
          __syncwarp();
          if (lane == 0) ptx::mbar_arrive(&ws_empty[slot]);
          if (++slot == kWsSlots) { slot = 0; slot_phase ^= 1; }
        }
        advance();
        if (++set == p.sf_sets) set = 0;
        if (++behind > 0 && ++had == p.stages) { had = 0; had_phase ^= 1; }
      }
    }
  } else if (warp == kWarpMma && half == 0) {
    // ---- MMA ---------------------------------------------------------------
    int acc = 0;
    uint32_t acc_phase = 0;
    const uint32_t idesc = idesc_mx4<FMT>(kHalves * kM, p.mma_n, 0);
    const uint32_t other = idesc_mx4<FMT>(kHalves * kM, p.mma_n, FMT == MX4_E8M0 ? 1 : 0);
    auto tile_mmas = [&](int from, int to) {
      if (!wait(&acc_empty[acc], acc_phase ^ 1)) return false;
      ptx::tc_fence_after();
      const uint32_t d = tmem + acc * p.acc_cols;
      for (int k = from; k < to; ++k) {
        if (!wait(&sf_full[set], set_phase)) return false;
        ptx::tc_fence_after();
        const uint32_t s = base_addr + stage * p.stage_bytes;
        const uint32_t sfa = tmem + p.sf_col + set * p.sf_cols;
        uint32_t sfb = sfa + 4 * kGroups, bd = ptx::sdesc_k128(s + kABytes);
        const uint32_t ad = ptx::sdesc_k128(s);
        // steps of 64 columns, none past the last column
        const int steps = min(4, (g.d - k * kCols + 63) / 64);
        for (int t = 0; t < p.terms; ++t) {
          const uint32_t dt = t < 2 ? d : d + p.low_col;
          const bool add = k > from || (t > 0 && (t != 2 || p.low_col == 0));
          if (steps == 4) {
            mma4_mx4<FMT, PAIR>(dt, ad, bd, idesc, other, sfa, sfb, 4 * p.chunks, add);
          } else {
            for (int j = 0; j < steps; ++j) {
              const int q = FMT == MX4_E4M3 ? j : j / 2;
              mma_mx4<FMT, PAIR>(dt, ad + 2 * j, bd + 2 * j, FMT == MX4_E8M0 && j % 2 ? other : idesc,
                                 sfa + 4 * q, sfb + q * p.chunks * 4, add || j > 0);
            }
          }
          sfb += kGroups * p.chunks * 4;
          bd += (uint32_t)x_bytes >> 4;
        }
        commit(&empty[stage]);
        advance();
        next_set();
      }
      commit(&acc_full[acc]);
      if (++acc == p.accs) { acc = 0; acc_phase ^= 1; }
      return true;
    };
    if (p.ranges) {
      while (work.next(tile, k0, k1) && tile_mmas(k0, k1)) {}
    } else {
      for (int t = unit; t < p.tiles && tile_mmas(0, p.kt); t += units) {}
    }
  } else if (warp >= kWarpOut && warp < kWarpOut + 4) {
    // ---- accumulator to y --------------------------------------------------
    const int quarter = warp - kWarpOut;         // (warp % 4: the lanes it may read)
    const int in_tile = quarter * 32 + lane;     // table row of the tile in this CTA
    ptx::griddep_wait();
    int acc = 0;
    uint32_t acc_phase = 0;
    while (work.next(tile, k0, k1)) {
      const int r0 = tile % p.row_tiles * p.bn, rows = min(p.bn, g.rows - r0);
      const int j = first_row(tile) + in_tile;
      const bool live = j < g.n;
      float ws = 1.f, b = 0.f;
      const int64_t id = !live ? -1 : GATHER ? g.ids[j] : j;
      if (id >= 0 && id < g.V) {
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
      OT* y = static_cast<OT*>(g.out) + (int64_t)r0 * g.ld_out + j;
      // columns 32 m .. 32 m + 31 of the sums, scaled and stored
      auto finish = [&](int m, float xm, float (&v)[32]) {
        // (values first, then their stores in one block without conditions: with a
        // condition a value each waits for the one before, some 100 cycles a column)
#pragma unroll
        for (int i = 0; i < 32; ++i) {
          v[i] *= ws;
          if constexpr (FMT == MX4_E4M3) v[i] *= __shfl_sync(0xFFFFFFFFu, xm, i);
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
      };
      ok = wait(&acc_full[acc], acc_phase, true);
      // (the barriers below are for all four warps: they give up together)
      if (p.ranges) ok = all_of(1, 128, ok);
      if (!ok) break;
      ptx::tc_fence_after();
      const uint32_t t = tmem + acc * p.acc_cols + ((uint32_t)(quarter * 32) << 16);
      const bool whole = k0 == 0 && k1 == p.kt;
      const int64_t part_size = (int64_t)kHalves * p.bn * kM;
      // (slot 0 of a unit: the tile its range begins in)
      float* part = p.parts + half * p.bn * kM + in_tile;
      float* mine = part + (2 * unit + (k0 > 0 || work.start(unit) == (long long)tile * p.kt ? 0 : 1)) *
                               part_size;
      if (FMT == MX4_E4M3 && __any_sync(0xFFFFFFFFu, ws > kFarScale)) {
        scale_far_sums(t, p.bn, p.acc_cols, rows, ws, p.x_row + r0);
        ws = 1.f;
#pragma unroll
        for (int m = 0; m < kMaxBn / 32; ++m) xs[m] = 1.f;
      }
#pragma unroll
      for (int m = 0; m < kMaxBn / 32; ++m) {
        if (32 * m >= rows) break;
        float v[32];
        ptx::tmem_ld32(t + 32 * m, v);
        for (int c = p.bn; c < p.acc_cols; c += p.bn) {  // the further terms' columns
          float w[32];
          ptx::tmem_ld32(t + c + 32 * m, w);
#pragma unroll
          for (int i = 0; i < 32; ++i) v[i] += w[i];
        }
        if (whole) {
          finish(m, xs[m], v);
        } else {
#pragma unroll
          for (int i = 0; i < 32; ++i)
            if (32 * m + i < p.bn) mine[(32 * m + i) * kM] = v[i];
        }
      }
      ptx::tc_fence_before();
      __syncwarp();
      if (lane == 0) arrive(&acc_empty[acc]);
      if (++acc == p.accs) { acc = 0; acc_phase ^= 1; }
      if (!whole) {
        // the unit that counts in last adds the tile's parts
        const long long first = (long long)tile * p.kt;
        const int c0 = work.holder(first), c1 = work.holder(first + p.kt - 1);
        __threadfence();
        ptx::named_bar_sync(1, 128);
        if (threadIdx.x == kWarpOut * 32)
          *s_count = atomicAdd(&p.counts[tile * kHalves + half], 1u);
        ptx::named_bar_sync(1, 128);
        if (*s_count == (unsigned)(c1 - c0)) {
          __threadfence();
#pragma unroll
          for (int m = 0; m < kMaxBn / 32; ++m) {
            if (32 * m >= rows) break;
            float v[32];
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = 0.f;
            for (int c = c0; c <= c1; ++c) {
              const float* q = part + (2 * c + (work.start(c) >= first ? 0 : 1)) * part_size;
#pragma unroll
              for (int i = 0; i < 32; ++i)
                v[i] += 32 * m + i < p.bn ? __ldcg(q + (32 * m + i) * kM) : 0.f;
            }
            finish(m, xs[m], v);
          }
        }
        ptx::named_bar_sync(1, 128);      // (s_count is free again)
      }
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
// Byte matrix [planes][rows][bytes a row] (planes 0: of two dimensions), boxes of 128
// bytes by box_rows by box_planes.
bool byte_map(CUtensorMap* m, const void* ptr, uint64_t bytes, uint64_t rows, uint64_t ld,
              uint64_t planes, uint64_t plane_ld, uint32_t box_rows, uint32_t box_planes) {
  EncodeFn fn = encode_fn();
  if (!fn) return false;
  const cuuint64_t dims[3] = {bytes, rows, planes};
  const cuuint64_t strides[2] = {ld, plane_ld};
  const cuuint32_t box[3] = {128, box_rows, box_planes};
  const cuuint32_t es[3] = {1, 1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, planes ? 3 : 2, const_cast<void*>(ptr), dims, strides,
            box, es, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

size_t up256(size_t x) { return (x + 255) / 256 * 256; }

struct Plan {
  int pair, bn, mma_n, terms, accs, acc_cols, low_col, row_tiles, tiles, kt, stages, stage_bytes, chunks, sf_col, sf_cols, sf_sets;
  int units, ranges;
};
int stage_bytes_of(int bn, int planes, int fmt, int pair) {
  const int x = planes * bn / (pair ? 2 : 1) * (kCols / 2);
  return (kABytes + x + planes * bn * groups_of(fmt) * 4 + 1023) / 1024 * 1024;
}
int sf_col_of(int acc_cols, int accs) { return (accs * acc_cols + 31) / 32 * 32; }
int sf_cols_of(int bn, int planes, int fmt) {
  return 4 * groups_of(fmt) * (1 + planes * ((bn + 127) / 128));
}
constexpr int kExtraBytes = 1024 + kBarBytes + kWsSlots * kWsBytes;   // beside the stages
// Columns of an accumulator: the rows' (stacked: the terms' one after another), twice
// from three terms on.
int acc_cols_of(int bn, int planes, bool stacked) {
  return stacked ? planes * bn : planes > 2 ? 2 * bn : bn;
}
// Whether tiles of bn rows fit: three stages, `accs` accumulators and two sets of scales.
bool fits(int bn, int planes, int fmt, int pair, bool stacked, int accs) {
  const int n = stacked ? planes * bn : bn;
  return n <= kMaxBn && 3 * stage_bytes_of(bn, planes, fmt, pair) + kExtraBytes <= kSmemMax &&
         sf_col_of(acc_cols_of(bn, planes, stacked), accs) +
                 2 * sf_cols_of(n, stacked ? 1 : planes, fmt) <= (int)kTmemCols;
}
int largest(int unit, int planes, int fmt, int pair, int accs) {
  int most = unit;
  for (int bn = unit; bn <= kMaxBn && fits(bn, planes, fmt, pair, false, accs); bn += unit) most = bn;
  return most;
}
// The largest tile of hidden-state rows that fits, then as many equal tiles as the rows
// need.  Pairs where several terms make X's codes the larger part of a stage (single CTAs
// / pairs, us, all ids: 1024 rows x 38912 ids x 4608, one term 97.5 / 107, two 158 / 140,
// four 372 / 260; 320 x 51302 x 3584, two 72.3 / 70.9; 100 x 20000 x 2000, three 25.7 / 22.8;
// 32 x 12000 x 3840, two, with the terms side by side, 12.3 / 13.4).  With kept ids only
// for four terms, as pairs fetch scattered rows at half the rate (1024 x 51302 of 128256 x
// 4608, ids in runs of 64 / scattered: two terms 209 / 213 on single CTAs, 235 / 463 on pairs;
// three 360 / 367, 294 / 472; four 476 / 480, 342 / 480).  On pairs a tile of
// more than 128 rows, whose scales take twice the columns, costs a third more a stage:
// it is taken only where that saves more (the 1024 rows, two terms, in 8 tiles of 128 140
// us, in 7 of 160 162; the 320 rows in 3 and 2 76.3 and 70.5).
Plan plan_of(const Mx4Plan& a) {
  Plan pl{};
  pl.pair = a.pair_units > 0 &&
            (a.pair_mode == 2 || (a.pair_mode == 1 && a.planes > (a.gather ? 3 : 1) && a.rows > kPairRows));
  const int unit = pl.pair ? 32 : 16;         // rows a tile is a multiple of
  // two accumulators, so that a tile is stored while the next is computed; one where
  // that halves the tile's rows (three and four terms of more rows than fit so)
  pl.accs = 2;
  int most = largest(unit, a.planes, a.fmt, pl.pair, 2);
  if (a.planes > 2 && a.rows > most) {
    pl.accs = 1;
    most = largest(unit, a.planes, a.fmt, pl.pair, 1);
  }
  int64_t count = (a.rows + most - 1) / most;
  if (pl.pair && most > 128 && (a.rows + 127) / 128 * 3 < count * 4) count = (a.rows + 127) / 128;
  pl.bn = (int)(((a.rows + count - 1) / count + unit - 1) / unit * unit);
  // one row tile whose terms fit side by side: one MMA a step instead of one a term
  // (not on pairs, whose CTAs hold half of an MMA's columns each)
  const bool stacked =
      a.planes > 1 && count == 1 && !pl.pair && fits(pl.bn, a.planes, a.fmt, 0, true, 2);
  if (stacked) pl.accs = 2;
  pl.acc_cols = acc_cols_of(pl.bn, a.planes, stacked);
  pl.low_col = !stacked && a.planes > 2 ? pl.bn : 0;
  pl.mma_n = stacked ? a.planes * pl.bn : pl.bn;
  pl.terms = stacked ? 1 : a.planes;
  pl.row_tiles = (int)((a.rows + pl.bn - 1) / pl.bn);
  const int64_t m = pl.pair ? 2 * kM : kM;
  pl.tiles = (int)((a.n + m - 1) / m) * pl.row_tiles;
  pl.kt = (a.d + kCols - 1) / kCols;
  pl.stage_bytes = stage_bytes_of(pl.bn, a.planes, a.fmt, pl.pair);
  pl.stages = (kSmemMax - kExtraBytes) / pl.stage_bytes;
  if (pl.stages > kMaxStages) pl.stages = kMaxStages;
  pl.chunks = (pl.mma_n + 127) / 128;
  pl.sf_col = sf_col_of(pl.acc_cols, pl.accs);
  pl.sf_cols = sf_cols_of(pl.mma_n, pl.terms, a.fmt);
  pl.sf_sets = ((int)kTmemCols - pl.sf_col) / pl.sf_cols;
  if (pl.sf_sets > kMaxSets) pl.sf_sets = kMaxSets;
  if (pl.sf_sets > pl.stages) pl.sf_sets = pl.stages;
  // Whole tiles, or equal ranges of stages where few tiles of a long hidden dimension
  // would leave most SMs idle: the parts' way through memory costs more than it saves
  // below some 40 stages, and with many rows (whole tiles / ranges, us, two terms: 1 row x
  // 5000 ids x 14336, 40 tiles of 56 stages, 22.8 / 17.3; 32 x 2000 x 14336 22.8 / 19.8;
  // 1 x 12000 x 14336, 94 tiles, 23.6 / 22.6; 1 x 2000 x 7168 13.3 / 14.4; 32 x 5000 x 7168
  // 13.4 / 15.5; 320 x 2000 x 3584 17.9 / 34.6).  A unit gets two stages at least.
  const int64_t most_units = pl.pair ? a.pair_units : a.sm_count;
  const int64_t stages = (int64_t)pl.tiles * pl.kt;
  pl.ranges = a.schedule == 2 || (a.schedule == 0 && pl.kt > 40 && a.rows <= 32 &&
                                  3 * (int64_t)pl.tiles <= most_units);
  if (pl.ranges) {
    const int64_t by_two = stages / 2 > 1 ? stages / 2 : 1;
    pl.units = (int)(by_two < most_units ? by_two : most_units);
    // (equal ranges of whole tiles are whole tiles)
    if (stages % pl.units == 0 && stages / pl.units % pl.kt == 0) pl.ranges = 0;
  }
  if (!pl.ranges) pl.units = (int)(pl.tiles < most_units ? pl.tiles : most_units);
  return pl;
}

struct Scratch {        // X, and what tiles cut by ranges leave
  int64_t ld, plane;
  size_t scales, row, counts, parts, bytes;
};
Scratch scratch_of(const Plan& pl, int64_t rows, int d, int planes, int fmt) {
  Scratch o{};
  const int halves = pl.pair ? 2 : 1;
  o.ld = (d + 31) / 32 * 16;
  o.plane = (int64_t)up256((size_t)(rows * o.ld));
  o.scales = (size_t)(planes * o.plane);
  o.row = o.scales + up256((size_t)pl.row_tiles * pl.kt * planes * pl.bn * groups_of(fmt) * 4);
  o.counts = o.row + up256((size_t)pl.row_tiles * pl.bn * 4);
  o.parts = o.counts + (pl.ranges ? up256((size_t)pl.tiles * halves * 4) : 0);
  o.bytes = o.parts + (pl.ranges ? (size_t)pl.units * 2 * halves * pl.bn * kM * 4 : 0);
  return o;
}

struct Maps {
  CUtensorMap w, row, x;
};
template <int FMT, bool GATHER, bool PAIR, class OT>
cudaError_t launch(const Maps& m, const Params& p, int units, cudaStream_t st) {
  const size_t smem = (size_t)p.stages * p.stage_bytes + kExtraBytes;
  auto kernel = mx4_kernel<FMT, GATHER, PAIR, OT>;
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemMax);
  if (e != cudaSuccess) return e;
  if constexpr (PAIR)
    return launch_pdl_cluster(kernel, dim3((unsigned)(2 * units)), dim3(kThreads), smem, st, 2, m.w,
                              m.row, m.x, p);
  else
    return launch_pdl(kernel, dim3((unsigned)units), dim3(kThreads), smem, st, m.w, m.row, m.x, p);
}
template <int FMT, bool GATHER, bool PAIR>
cudaError_t launch_o(const Maps& m, const Params& p, int units, cudaStream_t st) {
  return p.g.out_type == TAB_FP32 ? launch<FMT, GATHER, PAIR, float>(m, p, units, st)
                                  : launch<FMT, GATHER, PAIR, __nv_bfloat16>(m, p, units, st);
}
template <int FMT>
cudaError_t launch_f(const Maps& m, const Params& p, bool pair, int units, cudaStream_t st) {
  if (pair)
    return p.g.ids ? launch_o<FMT, true, true>(m, p, units, st)
                   : launch_o<FMT, false, true>(m, p, units, st);
  return p.g.ids ? launch_o<FMT, true, false>(m, p, units, st)
                 : launch_o<FMT, false, false>(m, p, units, st);
}

}  // namespace

size_t mx4_gemm_scratch_bytes(const Mx4Plan& a) {
  return scratch_of(plan_of(a), a.rows, a.d, a.planes, a.fmt).bytes;
}

// At least what any call of up to `rows` rows and d columns takes: tiles cover at
// most 32 more rows each, and one that is not the only one has at least 32; an SM
// leaves two parts of a tile at most.
size_t mx4_gemm_reserve_bytes(int64_t rows, int64_t n, int64_t d, int sm_count) {
  const size_t r = (size_t)rows, padded = 2 * r + 64, kt = (size_t)((d + kCols - 1) / kCols);
  const size_t tiles = (size_t)((n + kM - 1) / kM + 1) * (r / 32 + 1);
  return 4 * (up256(r * ((size_t)(d + 31) / 32 * 16)) +
              up256(padded * kt * groups_of(MX4_E4M3) * 4)) +
         up256(padded * 4) + up256(tiles * 4) +
         (size_t)sm_count * 2 * (r < kMaxBn ? (r + 31) / 32 * 32 : kMaxBn) * kM * 4;
}

cudaError_t launch_mx4_gemm(const Mx4Gemm& g, const Mx4Plan& a, void* scratch, long long spin_limit,
                            cudaStream_t st) {
  const Plan pl = plan_of(a);
  const Scratch o = scratch_of(pl, g.rows, g.d, g.planes, g.fmt);
  char* at = static_cast<char*>(scratch);
  Params p{};
  p.g = g;
  p.x_scales = reinterpret_cast<uint8_t*>(at + o.scales);
  p.x_row = reinterpret_cast<float*>(at + o.row);
  p.bn = pl.bn; p.row_tiles = pl.row_tiles; p.tiles = pl.tiles; p.kt = pl.kt;
  p.stages = pl.stages; p.stage_bytes = pl.stage_bytes; p.chunks = pl.chunks;
  p.sf_col = pl.sf_col; p.sf_cols = pl.sf_cols; p.sf_sets = pl.sf_sets;
  p.ranges = pl.ranges; p.mma_n = pl.mma_n; p.terms = pl.terms;
  p.accs = pl.accs; p.acc_cols = pl.acc_cols; p.low_col = pl.low_col;
  p.counts = reinterpret_cast<unsigned*>(at + o.counts);
  p.parts = reinterpret_cast<float*>(at + o.parts);
  p.spin_limit = spin_limit;
  Maps m;
  const uint64_t bytes = (uint64_t)(g.d + 31) / 32 * 16;
  const uint64_t V = (uint64_t)g.V;
  if (!byte_map(&m.x, at, bytes, (uint64_t)g.rows, (uint64_t)o.ld, (uint64_t)g.planes,
                (uint64_t)o.plane, (uint32_t)(pl.bn / (pl.pair ? 2 : 1)), (uint32_t)g.planes) ||
      !byte_map(&m.w, g.w_codes, bytes, V, (uint64_t)g.ld_codes, 0, 0, g.ids ? 32 : kM, 1))
    return cudaErrorInvalidValue;
  m.row = m.w;
  if (g.ids && !byte_map(&m.row, g.w_codes, bytes, V, (uint64_t)g.ld_codes, 0, 0, 1, 1))
    return cudaErrorInvalidValue;

  Mx4Quant q{};
  q.x = g.x; q.ld_x = g.ld_x; q.rows = g.rows; q.d = g.d;
  q.codes = reinterpret_cast<uint8_t*>(at); q.ld_codes = o.ld; q.plane_codes = o.plane;
  q.scales = reinterpret_cast<uint8_t*>(at + o.scales); q.plane_scales = (int64_t)pl.bn * groups_of(g.fmt) * 4;
  q.row_scale = g.fmt == MX4_E4M3 ? reinterpret_cast<float*>(at + o.row) : nullptr;
  q.planes = g.planes; q.scale_cols = pl.kt * kCols;
  q.tile_rows = pl.bn; q.tile_words = groups_of(g.fmt);
  q.stage_bytes = g.planes * q.plane_scales;
  q.tile_bytes = pl.kt * q.stage_bytes;
  q.zero = p.counts; q.zeros = pl.ranges ? pl.tiles * (pl.pair ? 2 : 1) : 0;
  cudaError_t e = launch_mx4_quant(q, g.fmt, g.x_type, true, st);
  if (e != cudaSuccess) return e;
  return g.fmt == MX4_E4M3 ? launch_f<MX4_E4M3>(m, p, pl.pair, pl.units, st)
                           : launch_f<MX4_E8M0>(m, p, pl.pair, pl.units, st);
}

}  // namespace sph
