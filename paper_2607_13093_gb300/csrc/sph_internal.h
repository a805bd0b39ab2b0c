// Internal interfaces between the C-ABI layer (sph_api.cu) and the kernel
// translation units.  Not part of the public ABI.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include <utility>

namespace sph {

enum Epilogue : int {
  EPI_CLOUD = 0,     // +bias, optional unclipped store, clip, row |max|
  EPI_ENDPOINT = 1,  // + code * row_scale (dequantized cloud partial)
  EPI_FUSED = 2,     // endpoint that quantizes the cloud's clipped partials
                     // itself: code = Q(yc), written out as the payload,
                     // then + code * row_scale as EPI_ENDPOINT
};

enum WDtype : int { W_BF16 = 0, W_FP8 = 1 };

// Device-side error bits (OR-ed into the context's status word).
enum : unsigned int {
  ERR_TIMEOUT = 1u,     // a bounded wait gave up
  ERR_BAD_INDEX = 2u,   // a token outside its table (kept ids are not checked on the device)
};

// Kernels launched by this thread (read by the tracing layer).
extern thread_local long long launch_count;

// Launch with programmatic stream serialization: the kernel may start while
// the previous kernel of the stream is still running, and must call
// griddepcontrol.wait (ptx::griddep_wait) before it touches memory that an
// earlier kernel writes or reads.  Every kernel of this library does so.  The
// earlier kernel may be the caller's, which writes anything the call is given,
// ids and weights too, and may let its dependents start early itself: the
// first kernel that an API call launches on a stream waits before it reads
// anything and before it lets its own dependents start.  The later ones of
// the call start only after that wait, so they may read the caller's ids and
// weights (not what kernels of the call write) before their own.
// What is read behind the wait is read with coherent loads: a non-coherent one
// (__ldg, or a const __restrict__ parameter) is free to move before it, and is
// only for memory whose writer had finished before the kernel could start --
// for the kernels that follow an operand split or a statistics pass of their
// own call, what the call was given or wrote before that pass.
template <typename... KArgs, typename... Args>
cudaError_t launch_pdl(void (*kernel)(KArgs...), dim3 grid, dim3 block, size_t smem,
                       cudaStream_t st, Args&&... args) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  ++launch_count;
  return cudaLaunchKernelEx(&cfg, kernel, std::forward<Args>(args)...);
}
// launch_pdl with thread-block clusters of `cluster_x` CTAs along x
template <typename... KArgs, typename... Args>
cudaError_t launch_pdl_cluster(void (*kernel)(KArgs...), dim3 grid, dim3 block, size_t smem,
                               cudaStream_t st, int cluster_x, Args&&... args) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)cluster_x;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  ++launch_count;
  return cudaLaunchKernelEx(&cfg, kernel, std::forward<Args>(args)...);
}

// One gathered contraction  acc[r, j] = sum_c h[r, c] * W[ids[j], c]
// followed by an epilogue.  Pointers are device pointers.
struct GatherGemm {
  const float* h;          // [rows, K] fp32, row stride ld_h
  int64_t ld_h;
  int rows;
  const void* W;           // [V, K] bf16 or e4m3, row stride ld_w elements
  int64_t ld_w;
  int w_dtype;             // WDtype
  const float* w_scale;    // [V] (fp8 only)
  int K;
  int64_t V;               // rows of W
  const int32_t* ids;      // [n] sorted ids or nullptr (identity)
  int n;
  int act_bf16;            // round h to bf16 first
  int epilogue;            // Epilogue
  // EPI_CLOUD
  const float* bias;       // [V] or nullptr
  float clip;
  float* partial_out;      // [rows, n] unclipped, or nullptr
  float* Y;                // [rows, n] clipped (cloud) / fused z (endpoint)
  unsigned* rowmax;        // [rows] bits of max |clipped y|, zeroed by caller
  // EPI_ENDPOINT
  const int8_t* codes;     // [rows, n]
  const float* row_scale;  // [rows]
  float inv_tau;           // 1 / temperature (softmax statistics)
  int64_t ldy = 0;         // row stride of Y (z) in elements; 0: n
  // EPI_FUSED: the cloud's clipped partials and row maxima in, the payload out
  const float* yc = nullptr;            // [rows, n] clipped cloud partials
  const unsigned* rowmax_in = nullptr;  // [rows] bits of their row |max|
  int8_t* codes_out = nullptr;          // [rows, n] int8 codes (Eq. 18)
  float* scale_out = nullptr;           // [rows] row scales
  unsigned* status;        // device error word
  long long finish_wait = 1ll << 15;   // split-tile finisher poll (cycles; 0: none)
  bool no_stats = false;   // endpoint: skip the softmax statistics (Gumbel-max draw)
  bool after_own = false;  // the kernel before it on its stream is of the same API call
  // cloud GEMV in one launch: the last block to arrive (q_ticket, which it
  // resets) quantizes every row (Eq. 18) into q_codes / q_scale and clears
  // the row maxima for the next call; nullptr: the quantize pass does it
  unsigned* q_ticket = nullptr;
  int8_t* q_codes = nullptr;
  float* q_scale = nullptr;
};

// CUDA-core gathered GEMV (few rows); returns a cudaError_t.
cudaError_t launch_gemv(const GatherGemm& g, int sm_count, cudaStream_t st);
// Largest K the GEMV supports for a given row count.
int gemv_max_k();
// Hidden-state rows one GEMV launch covers (1, 2, 4 or 8).
int gemv_rows_per_launch(int rows, int K);
// Most rows x kept ids the cloud GEMV quantizes in its last block (two
// batches of eight loads a thread; measured: at 25,600 entries the one
// block took longer than a separate quantize pass over the whole grid)
constexpr int64_t kGemvQuantizeMax = 1 << 12;
// Whether the cloud GEMV can quantize in its last block (one launch covers
// the rows, at most kGemvQuantizeMax entries).
inline bool gemv_can_quantize(int64_t rows, int64_t n, int K) {
  return gemv_rows_per_launch((int)rows, K) >= rows && rows * n <= kGemvQuantizeMax;
}

// Tensor-core path (k_tc.cu): sizes, work split and scratch of one call.
struct TcPlan {
  int hilo, RB, BN, Rp, KB, Kp, NT, G, stages, whole_tiles, na, fp8;
  int pg;          // groups the h planes are taken in, one a k-block (KB counts them)
  int pair;        // CTA pairs (clusters of two) share each 256-id tile; G counts CTAs
  int tm;          // vocabulary rows per tile: 128 or 256
  int single_acc;  // one TMEM accumulator (256-id tiles over > 128 rows)
  int nseg;        // endpoint statistics: 32-id segments per row, NT * tm / 32
  int epi_stats;   // endpoint: softmax statistics in the epilogue (else a pass over z)
  int rm;          // endpoint on CTA pairs with rows as M (256-row blocks, whole tiles)
  int epi_t;       // endpoint: the epilogue may finish through a shared-memory transpose
                   // (where rows are 2-element aligned; shared memory reserved for it)
  long long T;
  size_t hs_bytes, p_bytes, cnt_bytes, stats_bytes, scratch_bytes, smem_bytes;
  bool ok;
};
// `endpoint` reserves the per-segment softmax statistics; schedule 0/1/2 =
// automatic / whole tiles / stream-K; max_stages 0 = automatic; block_k =
// hidden elements per pipeline stage (64, 128 or 256; 0 = automatic);
// gather = the kept-id subset path (keep_ids given); fp8 = e4m3 weights;
// max_bn = most hidden-state rows per tile (0 = automatic); tile_m =
// vocabulary rows per tile (128, 256 = two M = 128 halves, 0 = automatic);
// pair_mode = CTA pairs on 256-id tiles: 0 never, 1 where the row blocks are
// long enough (SPH_OPT_TC_PAIR has the rows), 2 always; max_pairs caps the
// pairs (0: no cap); rm_mode = the endpoint on pairs with rows as M: 0 where
// the 256-row blocks pad little, 1 always (where the call pairs), 2 never.
TcPlan tc_plan(int rows, int n, int K, int act_bf16, int sm_count, int endpoint,
               int schedule, int max_stages, int block_k, int gather, int fp8, int max_bn,
               int tile_m, int pair_mode = 0, int max_pairs = 0, int rm_mode = 0);
// CTA pairs of the pair kernel that can run at once on `device` (0 when the
// query fails): tc_plan's max_pairs.
int tc_pair_max_units(int device);
// Launch the operand split and the tcgen05 kernel; `scratch` holds
// plan.scratch_bytes bytes.  bf16 weights only.
cudaError_t launch_tc(const GatherGemm& g, const TcPlan& plan, void* scratch,
                      long long spin_limit, cudaStream_t st);
// Few-row endpoint contraction over a short hidden dimension (k_few.cu): one
// CTA per SM takes tiles of at most 128 kept ids, the hidden states of all
// rows stay in its shared memory.
constexpr int kFewMaxRows = 32;
constexpr int kFewMaxK = 512;
struct FewPlan {
  int pitch;       // kept ids of a tile: 32, 64, 96 or 128
  int na, KB;      // 64-column atoms of a stage, stages of a tile
  int tiles;
  int grid;        // persistent CTAs, one per SM at most
  int stages, lag; // ring depth; stages copied before a tile's epilogue waits
  int nseg;        // 32-id segments per row of the statistics
  size_t smem_bytes;
  bool ok;
};
FewPlan few_plan(int rows, int n, int K, int sm_count);
// What the kernel takes: EPI_ENDPOINT or EPI_FUSED, bf16 weights with 16-byte
// aligned rows.
bool few_operands(const GatherGemm& g);
// seg_stats receives, unless g.no_stats, the statistics [rows][plan.nseg].
cudaError_t launch_few(const GatherGemm& g, const FewPlan& plan, float2* seg_stats,
                       long long spin_limit, cudaStream_t st);

// Where a draw finds the fused logits of the ids it visits (the 32 ids of
// the segment it lands in): stored in Z (fp32 [rows, n]), or, with Z null,
// recomputed for just those ids from the endpoint call's own inputs (Eq. 13),
//   z[r, j] = codes[r, j] * row_scale[r] + sum_{c < K} h[r, c] * W[ids[j], c]
// with bf16 W (16-byte aligned rows), fp32 h, fp32 accumulation; codes null:
// the local part alone.
struct ZSource {
  const float* Z = nullptr;
  const float* h = nullptr;
  int64_t ld_h = 0;
  int K = 0;
  const void* W = nullptr;
  int64_t ld_w = 0;
  const int32_t* ids = nullptr;
  const int8_t* codes = nullptr;
  const float* row_scale = nullptr;
};
// One inverse-CDF draw per row after an endpoint launch_tc: from the segment
// statistics its epilogue left in `scratch` (plan.epi_stats), else from a
// statistics pass over the stored z into the same area (a z that is not
// stored needs plan.epi_stats); `cstats` receives the chunk statistics on
// the way (at most rows * (n / 1024 + 2)).
cudaError_t launch_sample_from_stats(const ZSource& zs, int rows, int n,
                                     const TcPlan& plan, const void* scratch,
                                     float2* cstats, const int32_t* ids,
                                     float inv_tau, uint64_t seed, uint64_t offset,
                                     int sm_count, int32_t* tokens, cudaStream_t st,
                                     int greedy = 0);

// codes/row_scale from the clipped partials and their row maxima
cudaError_t launch_quantize(const float* Y, const unsigned* rowmax, int rows,
                            int n, int8_t* codes, float* row_scale,
                            cudaStream_t st);

// Row kernels over fused logits Z (fp32 [rows, n]), k_rows.cu.
// Segment statistics: stats[r * nseg + s] = (max of z over the ids
// 32s..32s+31 of row r, sum of exp((z - max) * inv_tau) over them), nseg =
// seg_count(n); chunk statistics cstats[r * nchunk + c], nchunk =
// chunk_count(nseg), the same pair over the 32 segments 32c..32c+31.
int seg_count(int n);
int chunk_count(int nseg);
cudaError_t launch_seg_stats(const float* Z, int rows, int n, float inv_tau,
                             float2* stats, float2* cstats, int sm_count,
                             cudaStream_t st);
// chunk statistics from segment statistics with nseg segments per row
cudaError_t launch_chunk_stats(const float2* stats, int rows, int nseg,
                               float inv_tau, float2* cstats, int sm_count,
                               cudaStream_t st);
// Gumbel-max draw per row over Z (fp32 [rows, n]): the first index of the
// largest z * inv_tau - log(-log u) with per-(row, index) Philox uniforms.
cudaError_t launch_gumbel(const float* Z, int rows, int n, const int32_t* ids, float inv_tau,
                          uint64_t seed, uint64_t offset, int32_t* tokens, cudaStream_t st);
// One inverse-CDF draw per row from segment statistics alone (nseg per row):
// a block per row makes the chunk statistics in shared memory first.
// cudaErrorNotSupported (nothing launched) past 4096 chunks per row.
cudaError_t launch_sample_rows(const ZSource& zs, int rows, int n, const float2* stats,
                               int nseg, const int32_t* ids, float inv_tau, uint64_t seed,
                               uint64_t offset, int32_t* tokens, cudaStream_t st);
// One inverse-CDF draw per row from segment and chunk statistics with nseg
// segments per row (nseg * 32 >= n; segments past n hold zero weight);
// greedy: the first id of the row maximum (segment maxima, then the ids of
// the segment that holds it).
cudaError_t launch_sample_segments(const ZSource& zs, int rows, int n,
                                   const float2* stats, int nseg,
                                   const float2* cstats, const int32_t* ids,
                                   float inv_tau, uint64_t seed, uint64_t offset,
                                   int32_t* tokens, cudaStream_t st, int greedy = 0);
inline cudaError_t launch_sample_segments(const float* Z, int rows, int n,
                                          const float2* stats, int nseg,
                                          const float2* cstats, const int32_t* ids,
                                          float inv_tau, uint64_t seed, uint64_t offset,
                                          int32_t* tokens, cudaStream_t st, int greedy = 0) {
  ZSource zs;
  zs.Z = Z;
  return launch_sample_segments(zs, rows, n, stats, nseg, cstats, ids, inv_tau, seed, offset,
                                tokens, st, greedy);
}
// One draw per row (greedy: the argmax) from segment statistics a
// contraction's epilogue made: the fused sampler, or past its 4096 chunks a
// chunk-statistics pass into cstats and the segment sampler.
cudaError_t launch_sample_made_stats(const ZSource& zs, int rows, int n, const float2* stats,
                                     int nseg, float2* cstats, const int32_t* ids,
                                     float inv_tau, uint64_t seed, uint64_t offset,
                                     int sm_count, int32_t* tokens, cudaStream_t st,
                                     int greedy);
// One draw per row (greedy: the argmax) of a short stored row, statistics and
// draw in one launch (sample_is_short: at most 16 rows of at most 8192 ids).
bool sample_is_short(int rows, int n);
cudaError_t launch_sample_short(const float* Z, int rows, int n, const int32_t* ids, float inv_tau,
                                uint64_t seed, uint64_t offset, int32_t* tokens, cudaStream_t st,
                                int greedy);
int sample_max_n();
int verify_max_k();

// Speculative verification (four launches; greedy: three); `scratch` holds
// verify_scratch_bytes(sessions, k, n) bytes.
size_t verify_scratch_bytes(int sessions, int k, int n);
cudaError_t launch_verify(const float* Z, int sessions, int k, int n,
                          const int32_t* ids, int V, float inv_tau,
                          const int32_t* draft, const float* q,
                          uint64_t seed, uint64_t offset, int32_t* n_acc,
                          int32_t* next_token, void* scratch, int sm_count,
                          cudaStream_t st, int greedy = 0);

// ---- operators on a vocabulary table ---------------------------------------
// Element types of their rows (sph_tab_type).
enum TabType : int { TAB_BF16 = 0, TAB_FP32 = 1, TAB_FP16 = 2, TAB_E8M0 = 3, TAB_E4M3 = 4 };

// Rows to 4 bits (k_mx4.cu).
struct Mx4Quant {
  const void* x;            // [rows, d], row stride ld_x elements
  int64_t ld_x;
  int rows, d;
  uint8_t* codes;           // row stride ld_codes bytes; columns d up to a whole 32 are zeros
  int64_t ld_codes;
  uint8_t* scales;          // table form: row stride ld_scales bytes
  int64_t ld_scales;
  float* row_scale;         // [rows] 2^k, or nullptr
  int scale_cols;           // columns whose scale bytes are written (zeros past d)
  int planes;               // terms; 1 in the table form
  // operand form
  int64_t plane_codes, plane_scales;    // bytes between terms
  int tile_rows;            // rows of a tile; its scales are [stage][term][tile_rows]
  int tile_words;           // [tile_words] 4-byte words
  int64_t stage_bytes, tile_bytes;
  unsigned* zero;           // words to clear
  int zeros;
  int aligned;              // set by the launch: rows start on 16 bytes
};
cudaError_t launch_mx4_quant(Mx4Quant a, int fmt, int x_type, bool operand, cudaStream_t st);

// Product with a table held in 4 bits (k_mx4_tc.cu).
struct Mx4Gemm {
  const void* x;            // [rows, d], row stride ld_x elements of x_type
  int64_t ld_x;
  int rows, d, x_type, planes, fmt;
  const uint8_t* w_codes;   // [V], row stride ld_codes bytes
  int64_t ld_codes;
  const uint8_t* w_scales;  // [V], row stride ld_scales bytes
  int64_t ld_scales;
  const float* w_row;       // [V], e4m3 only
  int64_t V;
  const float* bias;        // [V] or nullptr
  const int32_t* ids;       // [n] or nullptr (identity)
  int n;
  void* out;                // [rows, n], row stride ld_out elements of out_type
  int64_t ld_out;
  int out_type;             // TAB_FP32 or TAB_BF16
  unsigned* status;
};
// What its work split depends on.
struct Mx4Plan {
  int64_t rows, n;
  int d, planes, fmt;
  int sm_count, pair_units;     // SMs, CTA pairs that fit at once
  int pair_mode;                // 0 never, 1 where it pays, 2 always
  int schedule;                 // 0 automatic, 1 whole tiles, 2 ranges of stages
  int gather;                   // kept ids are given
};
size_t mx4_gemm_scratch_bytes(const Mx4Plan& a);
size_t mx4_gemm_reserve_bytes(int64_t rows, int64_t n, int64_t d, int sm_count);
cudaError_t launch_mx4_gemm(const Mx4Gemm& g, const Mx4Plan& a, void* scratch, long long spin_limit,
                            cudaStream_t st);

// Lookup of table rows (k_table.cu).
struct Lookup {
  const int32_t* tokens;    // [n], or nullptr: rows 0 .. n - 1
  int64_t n;
  const void* table;        // [V, d], row stride ld_table elements (4-bit codes: bytes)
  int64_t ld_table;
  const uint8_t* scales;    // 4-bit tables: scale bytes, and row scales for e4m3
  int64_t ld_scales;
  const float* row_scale;
  int64_t V;
  int d;
  float scale;
  int64_t padding;          // the id that stands for a row of zeros
  void* out;                // [n, d], row stride ld_out elements
  int64_t ld_out;
  unsigned* status;
  int blocks, turns;        // set by the launch: blocks a token, spans of columns a block
};
cudaError_t launch_lookup(Lookup a, int table_type, int out_type, int sm_count, cudaStream_t st);

// Gradient of a table (k_table.cu).
struct TableGrad {
  const int32_t* tokens;    // [n]
  int n;
  const void* d_out;        // [n, d], row stride ld_d_out elements
  int64_t ld_d_out;
  int32_t V;
  int d;
  float scale;
  int64_t padding;
  int add;                  // 1: added to what out holds
  void* out;                // [V, d], row stride ld_out elements
  int64_t ld_out;
  unsigned* status;
  // set by the launch
  int32_t* keys[2];         // ids and positions; sorted in [0]
  int32_t* pos[2];
  float* partial;           // [ranges][2][ld_partial]
  int64_t ld_partial;
  int range, groups;        // sorted positions a range, column groups
};
size_t grad_scratch_bytes(int64_t n, int d, int sm_count);
size_t grad_reserve_bytes(int64_t n, int64_t d, int sm_count);
cudaError_t launch_table_grad(TableGrad a, int src_type, int out_type, void* scratch, int sm_count,
                              cudaStream_t st);

// ---- layer norm (k_norm.cu) -----------------------------------------------
struct Norm {
  const void* x;            // [rows, d], row stride ld_x elements
  int64_t ld_x, rows;
  int d;
  const void* weight;       // [d] of param_type, or nullptr
  const void* bias;
  int param_type;
  float eps;
  int centre;               // 0: the mean is not taken off
  void* out;                // [rows, d], row stride ld_out elements of out_type
  int out_type;
  int64_t ld_out;
  float* mean;              // [rows] or nullptr
  float* rstd;
};
cudaError_t launch_norm(const Norm& a, int x_type, int sm_count, cudaStream_t st);

struct NormGrad {
  const void* dy;           // [rows, d], row stride ld_dy elements
  int64_t ld_dy;
  const void* x;
  int64_t ld_x, rows;
  int d;
  const void* weight;       // [d] of weight_type, or nullptr
  int weight_type;
  const float* mean;        // [rows], or nullptr: not centred
  const float* rstd;
  void* dx;                 // [rows, d], row stride ld_dx elements of dx_type
  int dx_type;
  int64_t ld_dx;
  void* dw;                 // [d] or nullptr
  void* db;
  int accumulate;           // 1: added to what dw and db hold
  // set by the launch
  int parts;
  float* partial;           // [parts][2][ld_partial], or nullptr
  int64_t ld_partial;
};
size_t norm_grad_scratch_bytes(int64_t rows, int d, int x_type, int dy_type, int sm_count);
size_t norm_grad_reserve_bytes(int64_t rows, int64_t d, int sm_count);
cudaError_t launch_norm_grad(NormGrad a, int x_type, int dy_type, int grad_type, void* scratch,
                             int sm_count, cudaStream_t st);

// ---- rows in e4m3 with block scales (k_fp8.cu) ------------------------------
constexpr int kFp8Block = 128;           // columns of a scale, and rows where they share one
struct Fp8Quant {
  const void* x;            // [rows, d], row stride ld_x elements
  int64_t ld_x, rows;
  int d, block_rows;        // 1 or 128
  uint8_t* codes;           // row stride ld_codes bytes
  int64_t ld_codes;
  float* scales;            // of block (i, b) at i * row_step + b * col_step
  int64_t row_step, col_step;
  int* zero;                // words to clear (blocks of one row only)
  int64_t zeros;
  int aligned, spans;       // set by the launch
};
cudaError_t launch_fp8_quant(Fp8Quant a, int x_type, cudaStream_t st);

struct Fp8Lookup {
  const int32_t* tokens;    // [n], or nullptr: rows 0 .. n - 1
  int64_t n;
  const uint8_t* codes;     // [V, d], row stride ld_codes bytes
  int64_t ld_codes;
  const float* scales;      // row stride ld_scales
  int64_t ld_scales, V;
  int d, block_rows;
  float scale;
  int64_t padding;          // the id that stands for a row of zeros
  void* out;                // [n, d], row stride ld_out elements
  int64_t ld_out;
  unsigned* status;
  int spans;                // set by the launch
};
cudaError_t launch_fp8_lookup(const Fp8Lookup& a, int out_type, cudaStream_t st);

// Product with such a table (k_fp8_tc.cu).
struct Fp8Gemm {
  const void* x;            // [rows, d], row stride ld_x elements of x_type
  int64_t ld_x;
  int rows, d, x_type;
  const uint8_t* w_codes;   // [V], row stride ld_codes bytes
  int64_t ld_codes;
  const float* w_scales;    // row stride ld_scales
  int64_t ld_scales;
  int block_rows;
  int64_t V;
  const float* bias;        // [V] or nullptr
  const int32_t* ids;       // [n] or nullptr (identity)
  int n;
  void* out;                // [rows, n], row stride ld_out elements of out_type
  int64_t ld_out;
  int out_type;             // TAB_FP32 or TAB_BF16
  unsigned* status;
};
// What its work split depends on.
struct Fp8Plan {
  int64_t rows, n;
  int d, block_rows;
  int sm_count, pair_units;     // SMs, CTA pairs that fit at once
  int pair_mode;                // 0 never, 1 where it pays, 2 always
};
// The kernel for many hidden states and scales of 128 rows, on x's codes and scales [rows][ld_xs]
// (k_fp8_rows.cu).
cudaError_t launch_fp8_rows_as_m(const Fp8Gemm& g, const uint8_t* x_codes, int64_t ld_x,
                                 const float* x_scales, int64_t ld_xs, int* far, int pair_units,
                                 long long spin_limit, cudaStream_t st);
// Its tiles: `far` has a word for each, zero before.
int64_t fp8_rows_as_m_tiles(int64_t rows, int64_t n);
size_t fp8_gemm_scratch_bytes(const Fp8Plan& a);
size_t fp8_gemm_reserve_bytes(int64_t rows, int64_t n, int64_t d);
cudaError_t launch_fp8_gemm(const Fp8Gemm& g, const Fp8Plan& a, void* scratch, long long spin_limit,
                            cudaStream_t st);

// ---- logits with penalties, biases and masks (k_shape.cu) -------------------
struct Shape {
  const void* z;            // [rows, n], row stride ld_z elements
  int64_t ld_z, rows;
  int n;
  int64_t V;
  const int32_t* ids;       // [n] or nullptr (identity)
  const int32_t* history;   // [rows, max_tokens], row stride ld_history, or nullptr
  int64_t ld_history;
  int max_tokens;
  const int32_t* lengths;   // [rows] or nullptr: max_tokens
  const int32_t* prompts;   // [rows] or nullptr: 0
  const float* repetition;  // [rows] or nullptr, each
  const float* frequency;
  const float* presence;
  const int32_t* bias_ids;  // [rows, n_bias], row stride ld_bias_ids
  int64_t ld_bias_ids;
  const float* bias_values;
  int64_t ld_bias_values;
  int n_bias;
  const uint32_t* mask;     // [n_masks, ceil(V / 32)], row stride ld_mask, or nullptr
  int64_t ld_mask, n_masks;
  const int32_t* mask_rows; // [rows] or nullptr: the row's own
  void* out;                // [rows, n], row stride ld_out elements
  int64_t ld_out;
  int draw, greedy;
  float inv_tau;
  uint64_t seed, offset;
  int32_t* tokens;          // [rows]
  unsigned* status;
  // set by the launch
  int cols, chunks, vec;    // columns of a warp, warps a row, rows on 16 bytes
  float l2t;
  float4* stats;            // [rows][chunks]
  // columns that anything sparse befalls, in ascending order: column (as bits) and logit
  float2* pairs;            // [rows][ranges][most_marks]
  uint32_t* marks;          // [rows][ld_marks] of each 256 columns: first pair, pairs << 16; or nullptr
  int64_t ld_marks;
  int ranges, most_marks;   // blocks of the sparse part a row, marks one may have
  int wide, sparse_threads; // these blocks' columns are many; they have 1024 threads
};
// entries: tokens and biases that a row may have
size_t shape_scratch_bytes(int64_t rows, int n, bool draw, int64_t entries, int sm_count);
size_t shape_reserve_bytes(int64_t rows, int64_t n);
int64_t shape_blocks(int64_t rows, int n, int sm_count);
cudaError_t launch_shape(Shape a, int z_type, int out_type, void* scratch, int sm_count,
                         cudaStream_t st);

}  // namespace sph
