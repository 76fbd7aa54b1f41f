// bf16 loss forward / backward on the 5th-generation tensor cores (sm_100a).
//
// One persistent, warp-specialised kernel template does every contraction of the path:
//   FWD : S = H W^T tile by tile; epilogue keeps an online (max, sum-exp, target logit)
//         per token row in registers across the vocabulary tiles of its split.
//   G   : the same contraction for one chunk of token rows; epilogue turns each logit
//         into g = c_t (1[v=y_t] - e^{z-lse_t}) and writes it as bf16 into the chunk buffer.
//   E   : the same contraction again, for the one-pass forward+backward: epilogue sums the
//         row's exponentials AND writes every logit of the chunk as e = 2^(z log2e - ref_t),
//         bf16, against one reference exponent per token row that is fixed before the sweep.
//         With l_t = sum_v e the softmax is p = e / l_t, so the logit gradient factors as
//         g[t,v] = rowscale_t * (e[t,v] - l_t 1[v = y_t]): the finalisation kernel patches the
//         one target entry per row, and a per-row scale (in DH's epilogue, and applied to the
//         rows of H that DW reads) does the rest -- the stored chunk is never rewritten and the
//         backward needs no second logits contraction.
//   DH  : dH_chunk = G W        (A = G, K-major;  B = W read as an N-major operand)
//   DW  : dW (+)= G^T H_chunk   (A = G read as an M-major operand; B = H, N-major)
//
// CTAs run as pairs (a cluster of two SMs, tcgen05 cta_group::2).  A pair owns a
// 256 x 512 output tile: per 64-deep k-block each CTA stages 128 rows of A and its
// half (2 x 128 columns) of B, and the leader issues two 256x256x16 MMAs per k-step
// that share the A operand and fill the two 256-column halves of tensor memory.
// The wide tile is what keeps the L2 -> shared-memory traffic (48 KB per 256x256x64
// block of MACs) under the L2 bandwidth; the price is that the accumulator is not
// double-buffered, so the epilogue is kept short: eight warps drain it in parallel.
//
// Pipeline per CTA (one CTA per SM, 352 threads):
//   warp 0 : allocates tensor memory; lane 0 issues the TMA loads (128-byte swizzle)
//            of this CTA's operand parts into its 4-stage shared-memory ring; completion
//            is signalled on the "full" mbarrier of the pair's leader CTA.
//   warp 1 : (leader CTA only) lane 0 issues tcgen05.mma (bf16 -> fp32);
//            tcgen05.commit, multicast to both CTAs, releases the stage ("empty") and,
//            after the last k-block, publishes the accumulator ("tfull").
//   warps 2-9 : epilogue; each owns the 32 accumulator lanes its warp id selects and one
//            256-column half, reads them with tcgen05.ld and applies the mode's fused
//            epilogue, then releases the accumulator ("tempty", on the leader).
//   warp 10 : (leader CTA only) pacer: publishes how many k-blocks the pair has loaded, reads the
//            other pairs' counts and tells warp 0 how far it may run ahead of the slowest, so
//            that pairs sweeping the same operand tiles find them in L2.
// Every mbarrier wait is bounded: when it runs out the CTA raises SPO_DEV_TIMEOUT,
// all roles leave their loops, tensor memory is released and the kernel returns.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <math_constants.h>
#include <stdint.h>

#include <atomic>

#include "spo_internal.h"
#include "spo_ptx.cuh"

namespace spo {

namespace {

constexpr int CG = 2;                   // CTAs per MMA group (cluster size)
constexpr int BM = 128;                 // rows of A (and accumulator lanes) per CTA
constexpr int GROUP_M = BM * CG;        // rows of one output tile
constexpr int HALF_N = 256;             // columns of one MMA / one accumulator half
constexpr int BN = 2 * HALF_N;          // columns of one output tile
constexpr int BK = 64;
constexpr int STAGES = 4;
constexpr int A_BYTES = BM * BK * 2;                 // 16 KB
constexpr int BSUB_ROWS = HALF_N / CG;               // B columns per CTA per half (128)
constexpr int BSUB_BYTES = BSUB_ROWS * BK * 2;       // 16 KB
constexpr int STAGE_BYTES = A_BYTES + 2 * BSUB_BYTES;  // 48 KB
constexpr int RING_BYTES = STAGES * STAGE_BYTES;
constexpr int kWideStages = STAGES;
constexpr int kNarrowStages = RING_BYTES / (A_BYTES + BSUB_BYTES);   // 256-column tiles
constexpr int EPI_WARPS = 8;
constexpr int PACER_WARP = 2 + EPI_WARPS;              // last warp: keeps the pairs' loads close together in time
constexpr int NUM_THREADS = 32 * (3 + EPI_WARPS);
constexpr int TMEM_COLS = 512;
constexpr int STAGING_BYTES = 4096;                    // per epilogue warp: 32 rows x 128 bytes, for coalesced stores
constexpr int SMEM_BYTES = STAGES * STAGE_BYTES + 1024 + 256 + EPI_WARPS * STAGING_BYTES;
constexpr int kEpilogueSleepNs = 64;
constexpr int kProducerSleepNs = 32;
// Between two looks at the other pairs' progress.  The 74 counters share three cache lines that every
// pacer reads and writes, i.e. one L2 slice serves them all beside its share of the operand traffic:
// looks every 32 ns cost 4 % of the step and a loop with its loads issued back to back 50 %; 256, 1024 and
// 4096 ns agree within 0.2 %; 16 384 ns (longer than the window lasts) stalls the pairs.
constexpr int kPacerSleepNs = 1024;                     // between two looks at the other pairs' progress
constexpr uint32_t kPacerMaxSpins = 1u << 24;          // the pacer gives up (and lets everyone run free) after this many looks
constexpr int kLagCut = 8;                             // pairs more than this many windows behind are not waited for
constexpr int kHoldTries = 2048;                       // x 64 ns: longest time a producer holds back for the slowest pair

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kRefMargin = 40.0f;     // binary orders between a row's reference exponent and its first tile's maximum

enum : int { MODE_FWD = 0, MODE_G = 1, MODE_DH = 2, MODE_DW = 3, MODE_E = 4 };
constexpr int kMaxDwShards = SPO_MAX_DW_SHARDS;

struct GemmParams {
  int m_tiles, n_tiles, nsplit, per_split;   // work decomposition: unit = (row tile, split of the column tiles)
  int k_blocks;                              // K / 64, rounded up
  int a_row0;                                // added to A's row coordinate (K-major A) or k coordinate (M-major A)
  int b_k0;                                  // added to B's k coordinate (N-major B)
  int64_t rows_valid;                        // rows of the output that exist (tokens or vocabulary rows)
  int32_t cols_valid;                        // columns of the output that exist (V or d)
  int64_t out_row0;                          // first output row of tile row 0 (token offset of the chunk)
  // FWD / G
  const int32_t* y;
  const float* lse;
  const float* coef;
  float grad_loss;
  FwdPartial* partials;
  int64_t T;                                 // stride between the splits' partials (rows they cover)
  int64_t part_row0;                         // global row that partial 0 of a split belongs to
  __nv_bfloat16* G;
  int64_t ldg;
  const FwdPartial* pre;                     // E: statistics of every row's first vocabulary tile, [2][pre_ld] (both halves)
  int64_t pre_ld;
  const float* rowscale;                     // DH (one-pass): factor of each output row, indexed like the output; NULL = none
  int m_tile0;                               // added to every unit's row tile (a launch that covers a slab of row tiles)
  // DW, reduce-scatter form: instead of going to `out`, every tile (plus what `out` holds, when accumulating)
  // is ADDED into the shard that owns its vocabulary rows; shard k = rows [k shard_rows, (k+1) shard_rows)
  float* shard[kMaxDwShards];
  int n_shards;                              // 0: plain output
  int64_t shard_rows;
  // DH / DW
  void* out;
  int out_bf16;
  int64_t ldo;
  int accumulate;
  int32_t* d_status;
  // Soft lock-step between CTA pairs: progress[g] = k-blocks whose loads pair g has issued, ~0u when done;
  // a pair holds its loads back while it is more than `window` k-blocks ahead of the slowest pair.
  uint32_t* progress;
  int window;
  // Log-probability operators (template argument LP >= 0)
  float sc2;                                 // FWD / G: log2(e) / temperature
  float* cand;                               // FWD: logits of the listed column groups, [list][cand_ld][cand_slots][32]
  float2* cand_max;                          // FWD: (group maximum, group and slot) of the listed groups, [list][cand_ld][LP]
  int64_t cand_ld;                           // rows between two lists
  int cand_slots;                            // places of a list: LP, or as many groups as its columns have
  const uint8_t* mask;                       // G: rows with mask 0 get g = 0
  const float *ent, *g_logp, *g_lse, *g_ent; // G: entropy and upstream gradients per row (g_lse, g_ent + ent optional)
  float inv_t;                               // G: 1 / temperature
  const float* partial;                      // DW: fp32 sum of the earlier chunks, added before the rounding; NULL = none
  int k_splits, k_per;                       // DH: the contraction cut into k_splits parts of k_per k-blocks, each with an
                                             // fp32 result of its own in `out`, [part][rows_valid][ldo]
  TargetRest rest;                           // G: rest is stored;  DH (one part), DW: it is added to the result
  int n_rest;                                // DH: V
  const __nv_bfloat16* w_rows;               // DH: W, [vocabulary row][ldo]
};

// g = c_t (1[v = y_t] - 2^(z log2e - lse_t log2e)) for 32 consecutive columns, packed to bf16.
__device__ __forceinline__ void g_values(const uint32_t (&v)[32], int col0, float c, float lse2, int yt,
                                         int cols_valid, uint4* out4) {
  float g[32];
  if (c != 0.0f) {
    const float nc = -c;
#pragma unroll
    for (int j = 0; j < 32; ++j) g[j] = nc * fast_exp2(fmaf(__uint_as_float(v[j]), kLog2e, -lse2));
    if (yt >= col0 && yt < col0 + 32) {
      const int jj = yt - col0;
#pragma unroll
      for (int j = 0; j < 32; ++j) if (j == jj) g[j] += c;
    }
    if (col0 + 32 > cols_valid) {
#pragma unroll
      for (int j = 0; j < 32; ++j) if (col0 + j >= cols_valid) g[j] = 0.0f;
    }
  } else {
#pragma unroll
    for (int j = 0; j < 32; ++j) g[j] = 0.0f;
  }
#pragma unroll
  for (int q = 0; q < 4; ++q)
    out4[q] = make_uint4(pack_bf16(g[8 * q + 0], g[8 * q + 1]), pack_bf16(g[8 * q + 2], g[8 * q + 3]),
                         pack_bf16(g[8 * q + 4], g[8 * q + 5]), pack_bf16(g[8 * q + 6], g[8 * q + 7]));
}

// Gradient of a row's logits for upstream gradients of its log-prob, log-sum-exp and entropy:
// with u = log2 p = z sc2 - lse2, g = 2^u (a + b u) + tgt 1[v = y_t] (a, b, tgt: see the row setup), packed to bf16.
// p log p is zero where p is: kNoChance stands for u there (a logit of -inf gives 0 x inf otherwise; a NaN still comes through 2^u).
__device__ __forceinline__ void g_values_lp(const uint32_t (&v)[32], int col0, bool live, float sc2, float lse2, float a,
                                            float b, float tgt, int yt, int cols_valid, uint4* out4, float* rest) {
  float g[32];
  if (live) {
#pragma unroll
    for (int j = 0; j < 32; ++j) {
      const float u = fmaf(__uint_as_float(v[j]), sc2, -lse2);
      g[j] = fast_exp2(u) * fmaf(b, fmaxf(u, kNoChance), a);
    }
    if (yt >= col0 && yt < col0 + 32) {
      const int jj = yt - col0;
      float t = 0.0f;
#pragma unroll
      for (int j = 0; j < 32; ++j) if (j == jj) { g[j] += tgt; t = g[j]; }
      if (rest) {                                  // what the rounding takes off the target's entry (see TargetRest)
        const float r = t - __bfloat162float(__float2bfloat16_rn(t));
        *rest = isfinite(r) ? r : 0.0f;
      }
    }
    if (col0 + 32 > cols_valid) {
#pragma unroll
      for (int j = 0; j < 32; ++j) if (col0 + j >= cols_valid) g[j] = 0.0f;
    }
  } else {
#pragma unroll
    for (int j = 0; j < 32; ++j) g[j] = 0.0f;
  }
#pragma unroll
  for (int q = 0; q < 4; ++q)
    out4[q] = make_uint4(pack_bf16(g[8 * q + 0], g[8 * q + 1]), pack_bf16(g[8 * q + 2], g[8 * q + 3]),
                         pack_bf16(g[8 * q + 4], g[8 * q + 5]), pack_bf16(g[8 * q + 6], g[8 * q + 7]));
}

// v += r x the 32 bf16 values of `row`
__device__ __forceinline__ void add_row(uint32_t (&v)[32], const uint4 (&row)[4], float r) {
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const uint32_t x[4] = {row[q].x, row[q].y, row[q].z, row[q].w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      v[8 * q + 2 * k] = __float_as_uint(fmaf(r, __uint_as_float(x[k] << 16), __uint_as_float(v[8 * q + 2 * k])));
      v[8 * q + 2 * k + 1] = __float_as_uint(fmaf(r, __uint_as_float(x[k] & 0xFFFF0000u), __uint_as_float(v[8 * q + 2 * k + 1])));
    }
  }
}

// Two floats to a bf16 pair, infinities replaced by the largest finite value (stored exponentials
// of a row whose logits outrun the reference must not become Inf: Inf times a zero row scale is NaN).
__device__ __forceinline__ uint32_t pack_bf16_finite(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.satfinite.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

__device__ __forceinline__ void bf16_values_finite(const uint32_t (&v)[32], uint4* out4) {
#pragma unroll
  for (int q = 0; q < 4; ++q)
    out4[q] = make_uint4(pack_bf16_finite(__uint_as_float(v[8 * q + 0]), __uint_as_float(v[8 * q + 1])),
                         pack_bf16_finite(__uint_as_float(v[8 * q + 2]), __uint_as_float(v[8 * q + 3])),
                         pack_bf16_finite(__uint_as_float(v[8 * q + 4]), __uint_as_float(v[8 * q + 5])),
                         pack_bf16_finite(__uint_as_float(v[8 * q + 6]), __uint_as_float(v[8 * q + 7])));
}

__device__ __forceinline__ void bf16_values(const uint32_t (&v)[32], uint4* out4) {
#pragma unroll
  for (int q = 0; q < 4; ++q)
    out4[q] = make_uint4(pack_bf16(__uint_as_float(v[8 * q + 0]), __uint_as_float(v[8 * q + 1])),
                         pack_bf16(__uint_as_float(v[8 * q + 2]), __uint_as_float(v[8 * q + 3])),
                         pack_bf16(__uint_as_float(v[8 * q + 4]), __uint_as_float(v[8 * q + 5])),
                         pack_bf16(__uint_as_float(v[8 * q + 6]), __uint_as_float(v[8 * q + 7])));
}


// Instruction descriptor for kind::f16: fp32 accumulate, bf16 A and B, M = 256 over the pair, N = 256.
__host__ __device__ constexpr uint32_t instr_desc(bool a_mn, bool b_mn) {
  return (1u << 4) | (1u << 7) | (1u << 10) | ((a_mn ? 1u : 0u) << 15) | ((b_mn ? 1u : 0u) << 16) |
         ((uint32_t)(HALF_N >> 3) << 17) | ((uint32_t)(GROUP_M >> 4) << 24);
}


struct Unit { int m_tile, n_begin, n_end; };
__device__ __forceinline__ Unit unit_of(int u, const GemmParams& p) {
  Unit r;
  const int split = u % p.nsplit;
  r.m_tile = u / p.nsplit + p.m_tile0;
  r.n_begin = split * p.per_split;
  r.n_end = min(r.n_begin + p.per_split, p.n_tiles);
  return r;
}

// ---------------------------------------------------------------------------
// the kernel
// ---------------------------------------------------------------------------
// ENT (FWD / E): also accumulate sum_v e z per row, from which the finalisation forms the entropy of
// the row's softmax, lse - sum_v p z (one more multiply-add per logit; a separate instantiation so that
// the kernels without it stay as they are).
// LP: the log-probability operators' variants.  -1: none (the policy loss).  FWD: logits carry a
// temperature, and LP > 0 also lists, per row, vocabulary split and column half, the LP column groups (32
// columns each) with the largest maxima: the K largest logits of a row lie in its K groups of largest
// maximum, so a merge over the lists finds the row's top K.  The group maximum falls out of the online
// softmax; the list is kept sorted in registers by LP compare-exchanges that the warp skips when none of its
// rows has a group above its last entry, and a listed group's 32 logits are stored once, when it enters.
// (A list of the logits themselves would be touched by nearly every group of 32 rows x 32 columns, in a
// scan of every logit.)  G: general upstream gradients.  DW: bf16 result.  DH: the contraction split along k.
// NARROW (log-probability operators): tiles of 256 x 256 with two accumulators and six stages, so that a tile's epilogue
// runs under the next one's products, for contractions too short to carry it otherwise (see lp_narrow).
template <int MODE, bool ENT = false, int LP = -1, bool NARROW = false>
__global__ void __launch_bounds__(NUM_THREADS, 1)
spo_gemm_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB, const GemmParams p) {
  constexpr bool A_MN = (MODE == MODE_DW);
  constexpr bool B_MN = (MODE == MODE_DH || MODE == MODE_DW);
  constexpr int MMAS = NARROW ? 1 : 2;                        // products of 256 columns per k-step
  constexpr int BN = MMAS * HALF_N;                           // columns of a tile
  constexpr int EPI_N = BN / 2;                               // columns of an epilogue warp
  constexpr int BUFS = NARROW ? 2 : 1;                        // accumulators
  constexpr int STAGE_BYTES = A_BYTES + MMAS * BSUB_BYTES;
  constexpr int STAGES = NARROW ? kNarrowStages : kWideStages;
  static_assert(STAGES * STAGE_BYTES == RING_BYTES && 16 * STAGES + 80 <= 256, "shared memory");

  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t base = (raw + 1023u) & ~1023u;
  uint8_t* gen = smem_raw + (base - raw);
  const uint32_t bars = base + STAGES * STAGE_BYTES;
  const uint32_t full0 = bars, empty0 = bars + 8 * STAGES, tfull0 = bars + 16 * STAGES, tempty0 = tfull0 + 8 * BUFS;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(gen + RING_BYTES + 16 * STAGES + 16 * BUFS);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(gen + RING_BYTES + 16 * STAGES + 16 * BUFS + 8);
  volatile uint32_t* pace_mine = reinterpret_cast<volatile uint32_t*>(gen + RING_BYTES + 16 * STAGES + 16 * BUFS + 16);
  volatile uint32_t* pace_limit = pace_mine + 1;   // k-blocks this pair's producer may have issued (pacer -> producer)

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank();                    // 0 = leader of the pair
  const int group = blockIdx.x / CG, n_groups = gridDim.x / CG;
  constexpr bool KS = MODE == MODE_DH && LP >= 0;             // units are (tile, part of the contraction)
  const int total_units = p.m_tiles * p.nsplit * (KS ? p.k_splits : 1);

  if (MODE == MODE_G && LP >= 0 && p.rest.rest) {
    for (int i = blockIdx.x * NUM_THREADS + threadIdx.x; i < p.cols_valid; i += gridDim.x * NUM_THREADS) p.rest.slot[i] = -1;
  }
  if (threadIdx.x == 0) {
    for (int s = 0; s < STAGES; ++s) { mbar_init(full0 + 8 * s, 1); mbar_init(empty0 + 8 * s, 1); }
    for (int b = 0; b < BUFS; ++b) { mbar_init(tfull0 + 8 * b, 1); mbar_init(tempty0 + 8 * b, EPI_WARPS * CG); }
    *abort_flag = 0;
    *pace_mine = 0;
    *pace_limit = p.progress ? (uint32_t)p.window : 0xFFFFFFFFu;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 0) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(TMEM_COLS) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();                       // the peer's barriers exist before anything signals them
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;

  if (warp == 0) {
    // ------------------------------------------------------------------ TMA producer
    // Lane 0 issues the loads.  Before each k-block it tells the pacer warp how far it is and holds
    // back while it is ahead of what the pacer allows (the slowest pair's count plus `window`
    // k-blocks): pairs that sweep the same operand tiles then stay close enough in time for those
    // tiles to be served from L2 instead of being streamed from HBM once per pair (without any pacing
    // the forward at 244k tokens read 0.8 TB from HBM per launch, with it 0.12 TB; dH at one look per
    // tile read 17 GB per chunk, at a window of 32 k-blocks 8 GB).  Both words are in shared memory,
    // so the loop pays two shared-memory accesses per k-block; the looks at the other pairs are the
    // pacer's.  The hold is bounded and advisory (after ~0.13 ms the pair goes on regardless), so
    // it cannot dead-lock, and finished pairs publish ~0u so that they never hold anyone back.
    uint32_t it = 0;
    int ok = 1;
    const bool paced = (rank == 0) && p.progress != nullptr;
    for (int u = group; u < total_units; u += n_groups) {
      const Unit un = unit_of(KS ? u / p.k_splits : u, p);
      const int kb0 = KS ? (u % p.k_splits) * p.k_per : 0, kb1 = KS ? min(kb0 + p.k_per, p.k_blocks) : p.k_blocks;
      const int row_base = un.m_tile * GROUP_M + (int)rank * BM;       // this CTA's rows of the tile
      for (int n = un.n_begin; n < un.n_end; ++n) {
        const int col_base = n * BN + (int)rank * BSUB_ROWS;           // this CTA's columns of half 0
        for (int kb = kb0; kb < kb1; ++kb, ++it) {
          if (paced && lane == 0 && ok) {
            *pace_mine = it;
            for (int tries = 0; tries < kHoldTries && it > *pace_limit; ++tries) __nanosleep(64);
          }
          if (lane == 0 && ok) {
            const uint32_t s = it % STAGES, ph = (it / STAGES) & 1u;
            if (!mbar_wait<kProducerSleepNs>(empty0 + 8 * s, ph ^ 1u, abort_flag, p.d_status)) {
              ok = 0;
            } else {
              const uint32_t sa = base + s * STAGE_BYTES, sb = sa + A_BYTES;
              if (rank == 0) mbar_expect_tx(full0 + 8 * s, CG * STAGE_BYTES);   // both CTAs' bytes land on the leader's barrier
              const uint32_t fb = map_to_cta(full0 + 8 * s, 0);
              if (!A_MN) {
                tma_load_2d(sa, &tmA, kb * BK, p.a_row0 + row_base, fb);
              } else {
#pragma unroll
                for (int b = 0; b < BM / 64; ++b)
                  tma_load_2d(sa + b * 8192, &tmA, row_base + b * 64, p.a_row0 + kb * BK, fb);
              }
#pragma unroll
              for (int h = 0; h < MMAS; ++h) {
                const uint32_t sbh = sb + h * BSUB_BYTES;
                const int col = col_base + h * HALF_N;
                if (!B_MN) {
                  tma_load_2d(sbh, &tmB, kb * BK, col, fb);
                } else {
#pragma unroll
                  for (int b = 0; b < BSUB_ROWS / 64; ++b)
                    tma_load_2d(sbh + b * 8192, &tmB, col + b * 64, p.b_k0 + kb * BK, fb);
                }
              }
            }
          }
        }
      }
    }
    __syncwarp();
    if (paced && lane == 0) *pace_mine = 0xFFFFFFFFu;                  // done: the pacer publishes it and stops
  } else if (warp == 1) {
    // ------------------------------------------------------------------ MMA issuer (leader CTA)
    if (lane == 0 && rank == 0) {
      constexpr uint32_t idesc = instr_desc(A_MN, B_MN);
      uint32_t it = 0, tile = 0;
      bool ok = true;
      for (int u = group; u < total_units && ok; u += n_groups) {
        const Unit un = unit_of(KS ? u / p.k_splits : u, p);
        const int kb0 = KS ? (u % p.k_splits) * p.k_per : 0, kb1 = KS ? min(kb0 + p.k_per, p.k_blocks) : p.k_blocks;
        for (int n = un.n_begin; n < un.n_end && ok; ++n, ++tile) {
          const uint32_t buf = tile % BUFS;
          if (!mbar_wait(tempty0 + 8 * buf, ((tile / BUFS) & 1u) ^ 1u, abort_flag, p.d_status)) { ok = false; break; }
          tc_fence_after();
          for (int kb = kb0; kb < kb1; ++kb, ++it) {
            const uint32_t s = it % STAGES, ph = (it / STAGES) & 1u;
            if (!mbar_wait(full0 + 8 * s, ph, abort_flag, p.d_status)) { ok = false; break; }
            tc_fence_after();
            const uint32_t sa = base + s * STAGE_BYTES, sb = sa + A_BYTES;
#pragma unroll
            for (int j = 0; j < BK / 16; ++j) {
              const uint64_t da = A_MN ? smem_desc(sa + j * 2048, 8192, 1024) : smem_desc(sa + j * 32, 16, 1024);
#pragma unroll
              for (int h = 0; h < MMAS; ++h) {
                const uint32_t sbh = sb + h * BSUB_BYTES;
                const uint64_t db = B_MN ? smem_desc(sbh + j * 2048, 8192, 1024) : smem_desc(sbh + j * 32, 16, 1024);
                umma_bf16(tmem_base + (buf + h) * HALF_N, da, db, idesc, ((kb - kb0) | j) != 0 ? 1u : 0u);
              }
            }
            umma_commit(empty0 + 8 * s);
          }
          if (ok) umma_commit(tfull0 + 8 * buf);
        }
      }
    }
  } else if (warp < 2 + EPI_WARPS) {
    // ------------------------------------------------------------------ epilogue (warps 2..9)
    const int quarter = warp & 3;                            // tensor-memory lanes this warp may read
    const int half = (warp - 2) >> 2;                        // which half of the tile's columns
    const int row = (int)rank * BM + quarter * 32 + lane;    // row of the pair's tile
    const int warp_row0 = (int)rank * BM + quarter * 32;     // tile row of the warp's first lane
    uint8_t* stage = gen + RING_BYTES + 256 + (warp - 2) * STAGING_BYTES;
    const uint32_t tempty_leader = map_to_cta(tempty0, 0);
    uint32_t tile = 0;
    bool ok = true;
    auto slot_of = [&](int unit) {                       // DW with LP: of this lane's row in a unit
      if (MODE != MODE_DW || LP < 0 || p.rest.rest == nullptr || unit >= total_units) return -1;
      const int64_t r = p.out_row0 + (int64_t)unit_of(unit, p).m_tile * GROUP_M + row;
      return r < p.rows_valid ? p.rest.slot[r] : -1;
    };
    int32_t slot_next = slot_of(group);
    for (int u = group; u < total_units && ok; u += n_groups) {
      const Unit un = unit_of(KS ? u / p.k_splits : u, p);
      const int64_t grow = p.out_row0 + (int64_t)un.m_tile * GROUP_M + row;   // global output row of this lane
      const int64_t grow_warp0 = grow - lane;                                  // ... and of the warp's first lane
      const bool row_ok = grow < p.rows_valid;
      // per-row state
      float m2 = -CUDART_INF_F, l = 0.0f, zt = -CUDART_INF_F;             // FWD
      float ez = 0.0f;                                                     // ENT: sum e z relative to m2
      int32_t yt = -1;
      float c = 0.0f, lse2 = 0.0f;                                         // G
      constexpr int LIST = (MODE == MODE_FWD && LP > 0) ? LP : 1;
      float top_v[LIST];                                                   // FWD with lists: group maxima, descending,
      uint32_t top_p[LIST];                                                // ... and (group << 8 | slot)
      if (MODE == MODE_FWD && LP > 0) {
#pragma unroll
        for (int i = 0; i < LIST; ++i) {                                 // (slots are taken from the end: 0, 1, ..)
          top_v[i] = -CUDART_INF_F;
          top_p[i] = 0xFFFFFF00u | (uint32_t)(LIST - 1 - i);
        }
      }
      const float sc2 = (MODE == MODE_FWD && LP >= 0) ? p.sc2 : kLog2e;
      bool live = false;                                                   // G with LP: coefficients of g
      float ga = 0.0f, gb = 0.0f, gt = 0.0f;
      if (MODE == MODE_G && LP >= 0 && row_ok) {
        // d logp: gl (1[v=y] - p);  d lse: glse p;  d entropy: -ge p (log p + ent);  all times 1/temperature
        live = p.mask == nullptr || p.mask[grow] != 0;
        float gl = p.g_logp ? p.g_logp[grow] : 0.0f;
        const int32_t yy = p.y ? p.y[grow] : -1;
        if (p.g_logp && (yy < 0 || yy >= p.cols_valid)) {                  // no such target: its log-prob is the constant -inf
          if (live && p.d_status) atomicOr(p.d_status, SPO_DEV_ID_OUT_OF_RANGE);
          gl = 0.0f;
        }
        const float ge = p.g_ent ? p.g_ent[grow] : 0.0f;
        const float gs = p.g_lse ? p.g_lse[grow] : 0.0f;
        gt = p.inv_t * gl;
        ga = p.inv_t * (gs - gl - (p.g_ent ? ge * p.ent[grow] : 0.0f));
        gb = -p.inv_t * ge * 0.69314718055994531f;
        lse2 = p.lse[grow] * kLog2e;
      }
      float* const rest_at = MODE == MODE_G && LP >= 0 && p.rest.rest ? p.rest.rest + (grow - p.out_row0) : nullptr;
      // DH, DW with LP: what the row's targets are still owed (see TargetRest), `owed` times a bf16 row, which is fetched one
      // step of 64 columns ahead, the first one before the tile's products are waited for
      constexpr bool OWED = (MODE == MODE_DH || MODE == MODE_DW) && LP >= 0;
      float owed = 0.0f;
      const uint4* owed_row = nullptr;
      uint4 owed0[4], owed1[4];
      if (MODE == MODE_DH && OWED && p.rest.rest && row_ok) {
        const int32_t yy = p.rest.y[grow];
        if (yy >= 0 && yy < p.n_rest && (p.rest.mask == nullptr || p.rest.mask[grow] != 0)) {
          owed = p.rest.rest[grow];
          owed_row = reinterpret_cast<const uint4*>(p.w_rows + (int64_t)yy * p.ldo);
        }
      }
      if (MODE == MODE_DW && OWED) {
        const int32_t s = slot_next;
        slot_next = slot_of(u + n_groups);
        if (s >= 0) {
          owed = 1.0f;
          owed_row = reinterpret_cast<const uint4*>(p.rest.rows + (int64_t)s * p.ldo);
        }
      }
      const bool any_owed = OWED && __any_sync(0xffffffffu, owed != 0.0f);
      auto fetch_owed = [&](int col0) {
        if constexpr (OWED) {
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const bool on = owed != 0.0f && col0 < p.cols_valid;
            owed0[q] = on ? __ldg(owed_row + col0 / 8 + q) : make_uint4(0u, 0u, 0u, 0u);
            owed1[q] = on && col0 + 32 < p.cols_valid ? __ldg(owed_row + col0 / 8 + 4 + q) : make_uint4(0u, 0u, 0u, 0u);
          }
        }
      };
      float rs = 1.0f;                                                     // DH: factor of this lane's output row
      if (MODE == MODE_FWD || MODE == MODE_G || MODE == MODE_E) {
        if (row_ok && (LP < 0 || p.y)) yt = p.y[grow];
        if (MODE == MODE_G && LP < 0 && row_ok) { c = p.grad_loss * p.coef[grow]; lse2 = p.lse[grow] * kLog2e; }
        if (MODE == MODE_E) {
          // Reference exponent of the row: the largest logit of its first vocabulary tile (found by a
          // short launch beforehand) plus a margin, the same for every pair and column half that works
          // on the row.  Exponentials are taken against it without a running maximum: bf16 and fp32
          // keep their relative precision at any magnitude, so all that matters is that nothing
          // overflows (row maximum up to kRefMargin + 109 binary orders above the first tile's) and
          // that entries worth keeping do not underflow (anything within 126 - kRefMargin orders
          // below the first tile's maximum survives).
          m2 = row_ok ? fmaxf(p.pre[grow].m2, p.pre[p.pre_ld + grow].m2) + kRefMargin : 0.0f;
        }
      }
      if (MODE == MODE_DH && p.rowscale && row_ok) rs = p.rowscale[grow];
      for (int n = un.n_begin; n < un.n_end && ok; ++n, ++tile) {
        if (OWED && any_owed) fetch_owed(n * BN + half * EPI_N);
        {                                   // one lane polls (with backoff); the warp reconverges on the outcome
          int good = 1;
          if (lane == 0)
            good = mbar_wait<kEpilogueSleepNs>(tfull0 + 8 * (tile % BUFS), (tile / BUFS) & 1u, abort_flag, p.d_status) ? 1 : 0;
          good = __shfl_sync(0xffffffffu, good, 0);
          if (!good) { ok = false; break; }
        }
        tc_fence_after();
        const int col_half = n * BN + half * EPI_N;
        const uint32_t taddr = tmem_base + ((uint32_t)(quarter * 32) << 16) + (tile % BUFS) * HALF_N + half * EPI_N;
        if (MODE == MODE_FWD) {
#pragma unroll 1
          for (int ch = 0; ch < EPI_N / 32; ++ch) {
            const int col0 = col_half + ch * 32;
            if (col0 >= p.cols_valid) break;                           // nothing valid further right
            uint32_t v[32];
            tmem_ld32(taddr + ch * 32, v);
            if (col0 + 32 > p.cols_valid) {                            // ragged last chunk of the vocabulary
              // (with ENT a large finite value instead of -inf: its e is 0 either way and 0 * z stays 0.  LP takes -inf, which no
              // logit of a banned token is below, so that the lists are right among those too)
              const float fill = ENT && LP < 0 ? -1.0e30f : -CUDART_INF_F;
#pragma unroll
              for (int j = 0; j < 32; ++j)
                if (col0 + j >= p.cols_valid) v[j] = __float_as_uint(fill);
            }
            float mx0 = __uint_as_float(v[0]), mx1 = __uint_as_float(v[1]);
#pragma unroll
            for (int j = 2; j < 32; j += 2) {
              mx0 = fmaxf(mx0, __uint_as_float(v[j]));
              mx1 = fmaxf(mx1, __uint_as_float(v[j + 1]));
            }
            if (MODE == MODE_FWD && LP > 0) {
              const float mx = row_ok ? fmaxf(mx0, mx1) : -CUDART_INF_F;
              const bool enters = mx > top_v[LIST - 1];
              if (__any_sync(0xffffffffu, enters)) {
                const uint32_t slot = top_p[LIST - 1] & 255u;
                float x = enters ? mx : -CUDART_INF_F;
                uint32_t px = ((uint32_t)(col0 >> 5) << 8) | slot;
                bool above = false;
#pragma unroll
                for (int i = 0; i < LIST; ++i) {                       // from its place on everything moves down one:
                  above = above || x > top_v[i];                       // equal maxima keep their order of arrival
                  const float tv = top_v[i];
                  const uint32_t tp = top_p[i];
                  top_v[i] = above ? x : tv;
                  top_p[i] = above ? px : tp;
                  x = above ? tv : x;
                  px = above ? tp : px;
                }
                if (enters) {
                  float4* dst = reinterpret_cast<float4*>(
                      p.cand + (((int64_t)((u % p.nsplit) * 2 + half) * p.cand_ld + (grow - p.part_row0)) * p.cand_slots + slot) * 32);
#pragma unroll
                  for (int q = 0; q < 8; ++q)
                    dst[q] = make_float4(__uint_as_float(v[4 * q]), __uint_as_float(v[4 * q + 1]),
                                         __uint_as_float(v[4 * q + 2]), __uint_as_float(v[4 * q + 3]));
                }
              }
            }
            float mn = fmaxf(m2, fmaxf(mx0, mx1) * sc2);
            if (LP >= 0) mn = fmaxf(mn, kMaxFloor);
            const float neg = -mn;
            float s0 = 0.0f, s1 = 0.0f, t0 = 0.0f, t1 = 0.0f;
#pragma unroll
            for (int j = 0; j < 32; j += 2) {
              const float e0 = fast_exp2(fmaf(__uint_as_float(v[j]), sc2, neg));
              const float e1 = fast_exp2(fmaf(__uint_as_float(v[j + 1]), sc2, neg));
              s0 += e0;
              s1 += e1;
              if (ENT) {
                const float z0 = __uint_as_float(v[j]), z1 = __uint_as_float(v[j + 1]);
                t0 = fmaf(e0, LP >= 0 ? fmaxf(z0, kFarBelow) : z0, t0);
                t1 = fmaf(e1, LP >= 0 ? fmaxf(z1, kFarBelow) : z1, t1);
              }
            }
            const float down = fast_exp2(m2 - mn);
            l = fmaf(l, down, s0 + s1);
            if (ENT) ez = fmaf(ez, down, t0 + t1);
            m2 = mn;
            if (yt >= col0 && yt < col0 + 32) {
              const int jj = yt - col0;
#pragma unroll
              for (int j = 0; j < 32; ++j) if (j == jj) zt = __uint_as_float(v[j]);
            }
          }
        } else if (MODE == MODE_E) {
          // Sum of the row's exponentials (and sum e z with ENT) and the stored exponentials in one
          // pass, all against the row's fixed reference m2: no running maximum, no rescaling.
          __nv_bfloat16* obase = p.G + ((int64_t)(un.m_tile - p.m_tile0) * GROUP_M + warp_row0) * p.ldg;
          const float neg = -m2;
#pragma unroll 1
          for (int r2 = 0; r2 < EPI_N / 64; ++r2) {
            const int col0 = col_half + r2 * 64;
            uint4 piece[8];
            if (col0 < p.cols_valid) {
              uint32_t v0[32], v1[32];
              tmem_ld32_nowait(taddr + r2 * 64, v0);
              tmem_ld32_nowait(taddr + r2 * 64 + 32, v1);
              tmem_wait_ld(v0);
              tmem_wait_ld(v1);
              if (col0 + 64 > p.cols_valid) {                          // ragged end of the vocabulary: e = 0
#pragma unroll
                for (int j = 0; j < 32; ++j) {
                  // (with ENT a large finite value instead of -inf: its e is 0 either way and 0 * z stays 0)
                  const float fill = ENT ? -1.0e30f : -CUDART_INF_F;
                  if (col0 + j >= p.cols_valid) v0[j] = __float_as_uint(fill);
                  if (col0 + 32 + j >= p.cols_valid) v1[j] = __float_as_uint(fill);
                }
              }
              if (yt >= col0 && yt < col0 + 64) {
                const int jj = yt - col0;
#pragma unroll
                for (int j = 0; j < 32; ++j) {
                  if (j == jj) zt = __uint_as_float(v0[j]);
                  if (j + 32 == jj) zt = __uint_as_float(v1[j]);
                }
              }
              float s0 = 0.0f, s1 = 0.0f, s2 = 0.0f, s3 = 0.0f, t0 = 0.0f, t1 = 0.0f;
#pragma unroll
              for (int j = 0; j < 32; j += 2) {
                const float e0 = fast_exp2(fmaf(__uint_as_float(v0[j]), kLog2e, neg));
                const float e1 = fast_exp2(fmaf(__uint_as_float(v0[j + 1]), kLog2e, neg));
                const float e2 = fast_exp2(fmaf(__uint_as_float(v1[j]), kLog2e, neg));
                const float e3 = fast_exp2(fmaf(__uint_as_float(v1[j + 1]), kLog2e, neg));
                s0 += e0; s1 += e1; s2 += e2; s3 += e3;
                if (ENT) {
                  t0 = fmaf(e0, __uint_as_float(v0[j]), fmaf(e1, __uint_as_float(v0[j + 1]), t0));
                  t1 = fmaf(e2, __uint_as_float(v1[j]), fmaf(e3, __uint_as_float(v1[j + 1]), t1));
                }
                v0[j] = __float_as_uint(e0); v0[j + 1] = __float_as_uint(e1);
                v1[j] = __float_as_uint(e2); v1[j + 1] = __float_as_uint(e3);
              }
              l += (s0 + s1) + (s2 + s3);
              if (ENT) ez += t0 + t1;
              bf16_values_finite(v0, piece);
              bf16_values_finite(v1, piece + 4);
            } else {                                                   // pad columns: e = 0
#pragma unroll
              for (int q = 0; q < 8; ++q) piece[q] = make_uint4(0u, 0u, 0u, 0u);
            }
            stage_put(stage, lane, piece);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              int r, cc;
              const uint4 val = stage_get(stage, lane, i, r, cc);
              if (grow_warp0 + r < p.rows_valid) {
                // streaming store: the chunk buffer is next read by another launch, and lines that stayed in
                // L2 would push out the row strips of H that every tile of this sweep re-reads
                __stcs(reinterpret_cast<uint4*>(obase + (int64_t)r * p.ldg + col0 + cc * 8), val);
              }
            }
          }
        } else if (MODE == MODE_G || (MODE == MODE_DH && p.out_bf16) ||
                   (MODE == MODE_DW && LP >= 0 && !p.partial && !p.accumulate)) {
          // bf16 outputs: 64 columns (128 bytes per row) per staging round
          __nv_bfloat16* obase = MODE == MODE_G
              ? p.G + ((int64_t)un.m_tile * GROUP_M + warp_row0) * p.ldg
              : reinterpret_cast<__nv_bfloat16*>(p.out) + grow_warp0 * p.ldo;
          const int64_t ld = MODE == MODE_G ? p.ldg : p.ldo;
#pragma unroll 1
          for (int r2 = 0; r2 < EPI_N / 64; ++r2) {
            const int col0 = col_half + r2 * 64;
            if (MODE != MODE_G && col0 >= p.cols_valid) break;
            uint32_t v0[32], v1[32];
            tmem_ld32_nowait(taddr + r2 * 64, v0);
            tmem_ld32_nowait(taddr + r2 * 64 + 32, v1);
            tmem_wait_ld(v0);
            tmem_wait_ld(v1);
            uint4 piece[8];
            if (MODE == MODE_G) {
              if (LP >= 0) {
                g_values_lp(v0, col0, live, p.sc2, lse2, ga, gb, gt, yt, p.cols_valid, piece, rest_at);
                g_values_lp(v1, col0 + 32, live, p.sc2, lse2, ga, gb, gt, yt, p.cols_valid, piece + 4, rest_at);
              } else {
                g_values(v0, col0, c, lse2, yt, p.cols_valid, piece);
                g_values(v1, col0 + 32, c, lse2, yt, p.cols_valid, piece + 4);
              }
            } else {
              if (MODE == MODE_DH && p.rowscale) {                    // one-pass path: the row's factor (a zero factor gives exact zeros)
#pragma unroll
                for (int j = 0; j < 32; ++j) {
                  v0[j] = __float_as_uint(rs == 0.0f ? 0.0f : __uint_as_float(v0[j]) * rs);
                  v1[j] = __float_as_uint(rs == 0.0f ? 0.0f : __uint_as_float(v1[j]) * rs);
                }
              }
              if (OWED && any_owed) {
                add_row(v0, owed0, owed);
                add_row(v1, owed1, owed);
                if (r2 + 1 < EPI_N / 64) fetch_owed(col0 + 64);
              }
              bf16_values(v0, piece);
              bf16_values(v1, piece + 4);
            }
            stage_put(stage, lane, piece);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              int r, cc;
              const uint4 val = stage_get(stage, lane, i, r, cc);
              if (grow_warp0 + r < p.rows_valid) {
                uint4* dst = reinterpret_cast<uint4*>(obase + (int64_t)r * ld + col0 + cc * 8);
                if (MODE == MODE_G) __stcs(dst, val);        // chunk buffer: streaming, as in the E epilogue
                else *dst = val;
              }
            }
          }
        } else {
          // fp32 outputs: 32 columns (128 bytes per row) per staging round; dW may accumulate
          float* obase = reinterpret_cast<float*>(p.out) + grow_warp0 * p.ldo + (KS ? (u % p.k_splits) * p.rows_valid * p.ldo : 0);
#pragma unroll 1
          for (int ch = 0; ch < EPI_N / 32; ++ch) {
            const int col0 = col_half + ch * 32;
            if (col0 >= p.cols_valid) break;
            uint32_t v[32];
            tmem_ld32(taddr + ch * 32, v);
            if (MODE == MODE_DH && p.rowscale) {
#pragma unroll
              for (int j = 0; j < 32; ++j) v[j] = __float_as_uint(rs == 0.0f ? 0.0f : __uint_as_float(v[j]) * rs);
            }
            if (OWED && any_owed) {
              if (ch & 1) {
                add_row(v, owed1, owed);
                if (ch + 1 < EPI_N / 32) fetch_owed(col0 + 32);
              } else {
                add_row(v, owed0, owed);
              }
            }
            uint4 piece[8];
#pragma unroll
            for (int q = 0; q < 8; ++q) piece[q] = make_uint4(v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]);
            stage_put(stage, lane, piece);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              int r, cc;
              const uint4 raw4 = stage_get(stage, lane, i, r, cc);
              if (grow_warp0 + r < p.rows_valid) {
                if (MODE == MODE_DW && LP >= 0) {
                  // bf16 result: this launch's term, the earlier chunks' fp32 sum and (accumulating) the old
                  // value are added in fp32 and rounded once
                  const int64_t at = (grow_warp0 + r) * p.ldo + col0 + cc * 4;
                  float4 val = make_float4(__uint_as_float(raw4.x), __uint_as_float(raw4.y), __uint_as_float(raw4.z),
                                           __uint_as_float(raw4.w));
                  if (p.partial) {
                    const float4 old = *reinterpret_cast<const float4*>(p.partial + at);
                    val.x += old.x; val.y += old.y; val.z += old.z; val.w += old.w;
                  }
                  uint2* dst16 = reinterpret_cast<uint2*>(reinterpret_cast<__nv_bfloat16*>(p.out) + at);
                  if (p.accumulate) {
                    const uint2 old = *dst16;
                    val.x += __uint_as_float(old.x << 16); val.y += __uint_as_float(old.x & 0xFFFF0000u);
                    val.z += __uint_as_float(old.y << 16); val.w += __uint_as_float(old.y & 0xFFFF0000u);
                  }
                  *dst16 = make_uint2(pack_bf16(val.x, val.y), pack_bf16(val.z, val.w));
                  continue;
                }
                float* dst = obase + (int64_t)r * p.ldo + col0 + cc * 4;
                if (MODE == MODE_DW && p.n_shards > 0) {
                  // reduce-scatter form: this tile, plus the sum of the earlier chunks' tiles held in `out`,
                  // goes to the owner of the vocabulary row (its memory may be another GPU's: a plain
                  // peer store-reduction over NVLink, no load from there and nothing to wait for)
                  float4 val = make_float4(__uint_as_float(raw4.x), __uint_as_float(raw4.y), __uint_as_float(raw4.z),
                                           __uint_as_float(raw4.w));
                  if (p.accumulate) {
                    const float4 old = *reinterpret_cast<const float4*>(dst);
                    val.x += old.x; val.y += old.y; val.z += old.z; val.w += old.w;
                  }
                  const int64_t vrow = grow_warp0 + r;
                  const int owner = (int)(vrow / p.shard_rows);
                  float* sdst = p.shard[owner] + (vrow - (int64_t)owner * p.shard_rows) * p.ldo + col0 + cc * 4;
                  asm volatile("red.global.add.v4.f32 [%0], {%1, %2, %3, %4};"
                               ::"l"(sdst), "f"(val.x), "f"(val.y), "f"(val.z), "f"(val.w) : "memory");
                } else if (p.accumulate) {
                  // Added in L2, nothing comes back: no load latency in this (un-overlapped) epilogue.
                  // Each element receives exactly one addend per launch and launches are ordered on
                  // the stream, so the summation order is fixed.
                  asm volatile("red.global.add.v4.f32 [%0], {%1, %2, %3, %4};"
                               ::"l"(dst), "f"(__uint_as_float(raw4.x)), "f"(__uint_as_float(raw4.y)),
                                 "f"(__uint_as_float(raw4.z)), "f"(__uint_as_float(raw4.w))
                               : "memory");
                } else {
                  *reinterpret_cast<uint4*>(dst) = raw4;
                }
              }
            }
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster(tempty_leader + 8 * (tile % BUFS));
      }
      if ((MODE == MODE_FWD || MODE == MODE_E) && ok && row_ok) {
        FwdPartial part;
        part.m2 = m2; part.l = l; part.zt = zt; part.pad = ez;
        p.partials[(int64_t)((u % p.nsplit) * 2 + half) * p.T + (grow - p.part_row0)] = part;
        if (MODE == MODE_FWD && LP > 0) {
          float2* dst = p.cand_max + ((int64_t)((u % p.nsplit) * 2 + half) * p.cand_ld + (grow - p.part_row0)) * LIST;
#pragma unroll
          for (int i = 0; i < LIST; ++i) dst[i] = make_float2(top_v[i], __uint_as_float(top_p[i]));
        }
      }
    }
  }

  else if (warp == PACER_WARP && rank == 0 && p.progress != nullptr) {
    // ------------------------------------------------------------------ pacer (leader CTA)
    // Publishes this pair's k-block count, reads every pair's, and hands the producer its limit.  A
    // few loads and one sleep per turn; it ends when the producer has, or after kPacerMaxSpins turns
    // (then with the limit lifted, so that nobody waits for a pacer that has gone).
    volatile uint32_t* progress = p.progress;
    for (uint32_t spins = 0;; ++spins) {
      const uint32_t mine = *pace_mine;
      if (lane == 0) progress[group] = mine;
      if (mine == 0xFFFFFFFFu) break;
      if (spins >= kPacerMaxSpins) {
        if (lane == 0) { *pace_limit = 0xFFFFFFFFu; progress[group] = 0xFFFFFFFFu; }
        break;
      }
      // The slowest pair that is still within reach: one that is more than kLagCut windows behind this
      // pair (its CTAs started late because another kernel held their SMs, say) cannot share L2
      // lines with it any more, and waiting for it would only pass its delay on to everybody.
      const uint32_t reach = (uint32_t)kLagCut * (uint32_t)p.window;
      uint32_t mn = 0xFFFFFFFFu;
      for (int g = lane; g < n_groups; g += 32) {
        const uint32_t v = progress[g];
        if (v >= mine || mine - v <= reach) mn = min(mn, v);
      }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) mn = min(mn, __shfl_xor_sync(0xffffffffu, mn, o));
      if (lane == 0) *pace_limit = (mn > 0xFFFFFFFFu - (uint32_t)p.window) ? 0xFFFFFFFFu : mn + (uint32_t)p.window;
      __nanosleep(kPacerSleepNs);
    }
  }

  // ------------------------------------------------------------------ teardown
  __syncwarp();
  if (*abort_flag) {                       // let copies still in flight land before the CTA retires
    for (int i = 0; i < 200; ++i) __nanosleep(1000);
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();                       // the peer may still be reading this CTA's shared / tensor memory
  if (warp == 0)
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(TMEM_COLS) : "memory");
}

// A wait that nothing ever satisfies, through the same bounded-wait routine the pipeline uses:
// checks that a stuck barrier ends in SPO_DEV_TIMEOUT and a clean return instead of a hang.
__global__ void bounded_wait_probe_kernel(int32_t* d_status, unsigned long long limit_ns, int* reached_end) {
  __shared__ uint64_t bar;
  __shared__ int abort_flag;
  if (threadIdx.x == 0) {
    abort_flag = 0;
    mbar_init(smem_u32(&bar), 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncthreads();
  bool ok = true;
  if (threadIdx.x == 0) ok = mbar_wait<64>(smem_u32(&bar), 0, &abort_flag, d_status, limit_ns);
  __syncthreads();
  if (threadIdx.x == 0 && reached_end) *reached_end = ok ? 2 : 1;
}

// ---------------------------------------------------------------------------
// host side: tensor maps and launches
// ---------------------------------------------------------------------------
// How many k-blocks a CTA pair may run ahead of the slowest pair before it holds back.
#ifndef SPO_TUNE_WINDOW_SWEEP
#define SPO_TUNE_WINDOW_SWEEP 32
#endif
#ifndef SPO_TUNE_WINDOW_STREAM
#define SPO_TUNE_WINDOW_STREAM 16
#endif
constexpr int kWindowSweep = SPO_TUNE_WINDOW_SWEEP;
constexpr int kWindowStream = SPO_TUNE_WINDOW_STREAM;

// CTA pairs that can be resident at once (one CTA per SM).
int group_count() { return sm_count() / CG; }

// CTA pairs of this instantiation that can be resident together on a device (0 = not yet asked).
// The kernel is persistent and its pairs pace one another, so a grid must not exceed it.  One slot
// per device, filled once; concurrent first calls compute the same value (atomic stores).
template <int MODE, bool ENT, int LP, bool NARROW>
cudaError_t resident_groups(int* out) {
  static std::atomic<int> cached[64];
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
  int n = cached[dev].load(std::memory_order_acquire);
  if (n == 0) {
    e = cudaFuncSetAttribute(spo_gemm_kernel<MODE, ENT, LP, NARROW>, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM_BYTES);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t q = {};
    q.gridDim = dim3(group_count() * CG, 1, 1);
    q.blockDim = dim3(NUM_THREADS, 1, 1);
    q.dynamicSmemBytes = SMEM_BYTES;
    cudaLaunchAttribute qa[1];
    qa[0].id = cudaLaunchAttributeClusterDimension;
    qa[0].val.clusterDim.x = CG;
    qa[0].val.clusterDim.y = 1;
    qa[0].val.clusterDim.z = 1;
    q.attrs = qa;
    q.numAttrs = 1;
    e = cudaOccupancyMaxActiveClusters(&n, spo_gemm_kernel<MODE, ENT, LP, NARROW>, &q);
    if (e != cudaSuccess) return e;
    if (n < 1) return cudaErrorLaunchOutOfResources;
    if (n > group_count()) n = group_count();
    cached[dev].store(n, std::memory_order_release);
  }
  *out = n;
  return cudaSuccess;
}

template <int MODE, bool ENT = false, int LP = -1, bool NARROW = false>
cudaError_t launch_gemm(const CUtensorMap& a, const CUtensorMap& b, const GemmParams& p_in, uint32_t* progress,
                        cudaStream_t st) {
  int max_groups = 0;
  cudaError_t e0 = resident_groups<MODE, ENT, LP, NARROW>(&max_groups);
  if (e0 != cudaSuccess) return e0;
  const int units = p_in.m_tiles * p_in.nsplit * (MODE == MODE_DH && LP >= 0 ? p_in.k_splits : 1);
  if (units <= 0) return cudaSuccess;
  GemmParams p = p_in;
  // k-blocks a pair may run ahead of the slowest one.  E / FWD / G sweep short tiles (d / 64 k-blocks) and
  // re-read their row strip per tile; dH / dW stream both operands through one long tile.
  p.window = (MODE == MODE_DH || MODE == MODE_DW) ? kWindowStream : kWindowSweep;
  p.progress = nullptr;
  if (p.window > 0 && progress) {
    cudaError_t e = cudaMemsetAsync(progress, 0, kProgressBytes, st);
    if (e != cudaSuccess) return e;
    p.progress = progress;
  }
  const int groups = units < max_groups ? units : max_groups;
  if ((size_t)groups * 4 > kProgressBytes) p.progress = nullptr;       // more pairs than progress words: run unpaced
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(groups * CG, 1, 1);
  cfg.blockDim = dim3(NUM_THREADS, 1, 1);
  cfg.dynamicSmemBytes = SMEM_BYTES;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = CG;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, spo_gemm_kernel<MODE, ENT, LP, NARROW>, a, b, p);
}

// Operand box heights (rows per TMA box) for K-major operands.
constexpr uint32_t kBoxA = BM;
constexpr uint32_t kBoxB = BSUB_ROWS;

// How many splits of the column tiles a FWD / G launch uses.  All pairs running at one time form
// a rectangle of (pairs / nsplit) row tiles x nsplit column positions; per sweep step L2 has to hold
// that many A tiles (re-read every step) plus nsplit B tiles (streamed).  Fewer splits mean fewer
// re-reads of W from HBM; the choice also avoids a short last split (pairs would fall out of step)
// and a nearly empty last round of units.
int pick_fwd_split(int64_t m_tiles, int n_tiles, int d) {
#ifdef SPO_TUNE_NSPLIT
  if (m_tiles > 8) return SPO_TUNE_NSPLIT < n_tiles ? SPO_TUNE_NSPLIT : n_tiles;
#endif
  const int groups = group_count();
  const double a_tile = (double)GROUP_M * d * 2, b_tile = (double)BN * d * 2;
  const double l2_budget = 56e6;
  int best = 1;
  double best_score = -1.0;
  for (int ns = 1; ns <= n_tiles && ns <= 256; ++ns) {
    const int per = (int)ceil_div(n_tiles, ns);
    if ((int)ceil_div(n_tiles, per) != ns) continue;               // not a distinct partition
    const double ragged = (double)(ns * per - n_tiles) / (double)(ns * per);
    const int64_t units = m_tiles * ns;
    const int64_t rounds = ceil_div(units, groups);
    const double fill = (double)units / (double)(rounds * groups);
    const double rows_live = (double)(m_tiles < (groups + ns - 1) / ns ? m_tiles : (groups + ns - 1) / ns);
    const double footprint = rows_live * a_tile + ns * b_tile;
    double score = fill * (1.0 - ragged) / (1.0 + 0.01 * ns);
    if (footprint > l2_budget) score *= l2_budget / footprint;
    if (score > best_score) { best_score = score; best = ns; }
  }
  return best;
}

// Splits of the vocabulary tiles actually used for a given shape.
int fwd_unit_splits(int64_t T, int32_t d, int32_t V) {
  const int64_t m_tiles = ceil_div(T, GROUP_M);
  const int n_tiles = (int)ceil_div(V, BN);
  return pick_fwd_split(m_tiles, n_tiles, d);
}

}  // namespace

// Number of forward partials per token row (two column halves per vocabulary split);
// the workspace layout depends on it.
int fwd_bf16_nsplit(int64_t T, int32_t d, int32_t V) { return 2 * fwd_unit_splits(T, d, V); }

cudaError_t launch_fwd_bf16(const void* H, const void* W, const int32_t* y, int64_t T, int32_t d, int32_t V,
                            FwdPartial* partials, int nsplit, int want_entropy, uint32_t* progress, int32_t* d_status,
                            cudaStream_t st) {
  if (T == 0) return cudaSuccess;
  CUtensorMap ma, mb;
  if (!make_map(&ma, H, d, T, d, kBoxA) || !make_map(&mb, W, d, V, d, kBoxB)) return cudaErrorInvalidValue;
  GemmParams p{};
  p.m_tiles = (int)ceil_div(T, GROUP_M);
  p.n_tiles = (int)ceil_div(V, BN);
  p.nsplit = nsplit / 2;
  p.per_split = (int)ceil_div(p.n_tiles, p.nsplit);
  p.k_blocks = (int)ceil_div(d, BK);
  p.rows_valid = T;
  p.cols_valid = V;
  p.out_row0 = 0;
  p.y = y;
  p.partials = partials;
  p.T = T;
  p.d_status = d_status;
  if (want_entropy) return launch_gemm<MODE_FWD, true>(ma, mb, p, progress, st);
  return launch_gemm<MODE_FWD>(ma, mb, p, progress, st);
}

BwdWs bwd_ws_layout(int64_t T, int32_t d, int32_t V) {
  BwdWs L{};
  // Token rows per chunk: half as many row tiles as there are CTA pairs.  With d/512 column
  // tiles (a multiple of 2 for the usual hidden sizes) the dH tiles of a full chunk then fill the
  // pairs a whole number of times, and the chunk buffer stays at a few GB.
  const int groups = group_count();
  int64_t m_tiles = groups / 2 > 0 ? groups / 2 : 1;
  int64_t rows = m_tiles * GROUP_M;
  const int64_t t_pad = ceil_div(T > 0 ? T : 1, GROUP_M) * GROUP_M;
  if (rows > t_pad) rows = t_pad;
  L.chunk_rows = rows;
  L.ldg = ceil_div(V, BN) * BN;
  L.g = 0;
  L.progress = align_up((size_t)rows * (size_t)L.ldg * 2, 256);
  L.total = L.progress + kProgressBytes;
  return L;
}

namespace {

// dH rows [t0, t0 + rows) = G W, where G is the chunk buffer (one-pass path: times `rowscale`, indexed by
// token row, in the epilogue).
cudaError_t launch_dh(const CUtensorMap& mG_k, const CUtensorMap& mW_mn, int64_t t0, int64_t rows, int64_t T,
                      int32_t d, int32_t V, void* dH, int32_t dH_dtype, const float* rowscale, uint32_t* progress,
                      int32_t* d_status, cudaStream_t st) {
  const int n_tiles_d = (int)ceil_div(d, BN);
  GemmParams p{};
  p.m_tiles = (int)ceil_div(rows, GROUP_M);
  p.n_tiles = n_tiles_d;
  p.nsplit = n_tiles_d;
  p.per_split = 1;
  p.k_blocks = (int)ceil_div(V, BK);
  p.rows_valid = T;
  p.cols_valid = d;
  p.out_row0 = t0;
  p.out = dH; p.out_bf16 = (dH_dtype == SPO_DTYPE_BF16); p.ldo = d; p.accumulate = 0;
  p.rowscale = rowscale;
  p.d_status = d_status;
  return launch_gemm<MODE_DH>(mG_k, mW_mn, p, progress, st);
}

// dW (+)= G^T Hk over `rows` token rows: G is the chunk buffer read as an M-major operand, Hk the
// matching rows of the hidden states (read from row `h_row0` of their tensor map).  `tile0`, `tiles`:
// the slab of 256-row vocabulary tiles this launch covers (the whole vocabulary: 0, all of them).
cudaError_t launch_dw(const CUtensorMap& mG_mn, const CUtensorMap& mH_mn, int64_t h_row0, int64_t rows, int32_t d,
                      int32_t V, float* dW, int dw_accumulate, int tile0, int tiles, uint32_t* progress,
                      int32_t* d_status, cudaStream_t st, const spo_dw_shards* shards = nullptr) {
  const int n_tiles_d = (int)ceil_div(d, BN);
  GemmParams p{};
  p.m_tiles = tiles;
  p.m_tile0 = tile0;
  p.n_tiles = n_tiles_d;
  p.nsplit = n_tiles_d;
  p.per_split = 1;
  p.k_blocks = (int)ceil_div(rows, BK);
  p.b_k0 = (int)h_row0;
  p.rows_valid = V;
  p.cols_valid = d;
  p.out_row0 = 0;
  p.out = dW; p.out_bf16 = 0; p.ldo = d; p.accumulate = dw_accumulate;
  if (shards) {
    p.n_shards = shards->n_shards;
    p.shard_rows = shards->rows_per_shard;
    for (int k = 0; k < shards->n_shards; ++k) p.shard[k] = shards->shard[k];
  }
  p.d_status = d_status;
  return launch_gemm<MODE_DW>(mG_mn, mH_mn, p, progress, st);
}

}  // namespace

cudaError_t launch_bwd_bf16(const void* H, const void* W, const int32_t* y, const float* lse,
                            const float* coef, float grad_loss, int64_t T, int32_t d, int32_t V,
                            void* dH, int32_t dH_dtype, float* dW, int accumulate,
                            char* ws, const BwdWs& L, int32_t* d_status, cudaStream_t st) {
  __nv_bfloat16* G = reinterpret_cast<__nv_bfloat16*>(ws + L.g);
  uint32_t* progress = reinterpret_cast<uint32_t*>(ws + L.progress);
  if (T == 0) {
    if (!accumulate) return cudaMemsetAsync(dW, 0, sizeof(float) * (size_t)V * d, st);
    return cudaSuccess;
  }
  CUtensorMap mH_k, mW_k, mW_mn, mH_mn;
  if (!make_map(&mH_k, H, d, T, d, kBoxA) || !make_map(&mW_k, W, d, V, d, kBoxB) ||
      !make_map(&mW_mn, W, d, V, d, 64) || !make_map(&mH_mn, H, d, T, d, 64))
    return cudaErrorInvalidValue;
  const int n_tiles_v = (int)ceil_div(V, BN);
  cudaError_t e;
  int chunk = 0;
  for (int64_t t0 = 0; t0 < T; t0 += L.chunk_rows, ++chunk) {
    const int64_t rows = (T - t0) < L.chunk_rows ? (T - t0) : L.chunk_rows;
    const int m_tiles = (int)ceil_div(rows, GROUP_M);
    CUtensorMap mG_k, mG_mn;
    if (!make_map(&mG_k, G, V, rows, L.ldg, kBoxA) || !make_map(&mG_mn, G, V, rows, L.ldg, 64))
      return cudaErrorInvalidValue;
    // 1) logits of the chunk, rewritten in place as g (bf16)
    {
      GemmParams p{};
      p.m_tiles = m_tiles;
      p.n_tiles = n_tiles_v;
      p.nsplit = pick_fwd_split(m_tiles, n_tiles_v, d);
      p.per_split = (int)ceil_div(n_tiles_v, p.nsplit);
      p.k_blocks = (int)ceil_div(d, BK);
      p.a_row0 = (int)t0;
      p.rows_valid = T;
      p.cols_valid = V;
      p.out_row0 = t0;
      p.y = y; p.lse = lse; p.coef = coef; p.grad_loss = grad_loss;
      p.T = T;
      p.G = G; p.ldg = L.ldg;
      p.d_status = d_status;
      if ((e = launch_gemm<MODE_G>(mH_k, mW_k, p, progress, st)) != cudaSuccess) return e;
    }
    // 2) dH rows of the chunk = G W;  3) dW (+)= G^T H_chunk
    if ((e = launch_dh(mG_k, mW_mn, t0, rows, T, d, V, dH, dH_dtype, nullptr, progress, d_status, st)) != cudaSuccess)
      return e;
    if ((e = launch_dw(mG_mn, mH_mn, t0, rows, d, V, dW, (accumulate || chunk > 0) ? 1 : 0, 0,
                       (int)ceil_div(V, GROUP_M), progress, d_status, st)) != cudaSuccess)
      return e;
  }
  return cudaSuccess;
}

// ---------------------------------------------------------------------------
// Log-probability operators: the forward's contraction with a temperature and lists of the largest
// column groups, and the chunked backward for general upstream gradients.
// ---------------------------------------------------------------------------
int lp_list_len(int top_k) { return top_k == 0 ? 0 : top_k <= 8 ? 8 : kMaxTopK; }

#ifndef SPO_TUNE_LP_NARROW
#define SPO_TUNE_LP_NARROW 1024
#endif
// Splits of the vocabulary tiles of `bn` columns.  A few row tiles stream W once whatever the split (its tiles are not read
// again), so only the number of tiles that the busiest pair gets counts; with many row tiles the pairs re-read W and
// pick_fwd_split weighs the L2 footprint.  (129 rows at d = 4096, V = 151936: 1001 us with the latter's 12 splits, which
// leave 62 pairs idle, 263 us with 60.)
static int lp_split(int64_t rows, int32_t d, int32_t V, int bn) {
  const int64_t m_tiles = ceil_div(rows, GROUP_M);
  const int n_tiles = (int)ceil_div(V, bn), groups = group_count();
  if (m_tiles * 4 > groups) {
    const int ns = pick_fwd_split(m_tiles, n_tiles, d);
    if (ns <= 80) return ns;                                       // (a row's partials: at most 160)
  }
  int best = 1;
  int64_t best_cost = INT64_MAX;
  for (int ns = 1; ns <= n_tiles && ns <= groups && ns <= 80; ++ns) {
    const int64_t per = ceil_div(n_tiles, ns);
    if (ceil_div(n_tiles, per) != ns) continue;                    // not a distinct partition
    const int64_t cost = per * ceil_div(m_tiles * ns, groups);
    if (cost < best_cost) { best_cost = cost; best = ns; }
  }
  return best;
}

// Tiles of 256 columns instead of 512 for a contraction of `k` products: an epilogue of a 512-column tile takes 5 us
// (statistics) to 10 us (stored gradient), its products k / 64 x 0.61 us.  Up to k = 1024 hiding the epilogue is worth the
// narrow tile's third more operand traffic: forward of 3000 rows at V = 32000, d = 512 120 us wide, 90 narrow; d = 1024
// 170 / 157; forward and backward of 1531 rows at V = 151936, d = 1024 366 / 368 and 1133 / 1109; d = 2048 677 / 724 and 2110 / 2230.
static bool lp_narrow(int64_t k) { return k <= SPO_TUNE_LP_NARROW; }
static int lp_tile_cols(int64_t k) { return lp_narrow(k) ? HALF_N : BN; }

int lp_fwd_lists(int64_t rows, int32_t d, int32_t V) { return 2 * lp_split(rows, d, V, lp_tile_cols(d)); }
int lp_fwd_slots(int lists, int32_t d, int32_t V, int top_k) {
  const int bn = lp_tile_cols(d), len = lp_list_len(top_k);
  const int64_t groups = ceil_div(ceil_div(V, bn), lists / 2) * (bn / 2 / 32);    // of a split's column half
  return len < groups ? len : (int)groups;
}

// With one or two row tiles the pairs share nothing but those rows, which stay in L2: no pacing, and no launch that
// zeroes its counters (2 us of some 25).
static bool lp_paced(int64_t rows) { return rows > 2 * GROUP_M; }

template <bool NARROW>
static cudaError_t launch_lp_fwd(int list, bool ent, const CUtensorMap& ma, const CUtensorMap& mb, const GemmParams& p,
                                 uint32_t* progress, cudaStream_t st) {
  if (list == 0) return ent ? launch_gemm<MODE_FWD, true, 0, NARROW>(ma, mb, p, progress, st)
                            : launch_gemm<MODE_FWD, false, 0, NARROW>(ma, mb, p, progress, st);
  if (list == 8) return ent ? launch_gemm<MODE_FWD, true, 8, NARROW>(ma, mb, p, progress, st)
                            : launch_gemm<MODE_FWD, false, 8, NARROW>(ma, mb, p, progress, st);
  return ent ? launch_gemm<MODE_FWD, true, kMaxTopK, NARROW>(ma, mb, p, progress, st)
             : launch_gemm<MODE_FWD, false, kMaxTopK, NARROW>(ma, mb, p, progress, st);
}

cudaError_t launch_lp_fwd_bf16(const LpFwd& a, int64_t t0, int64_t rows, FwdPartial* partials, float* cand,
                               float2* cand_max, uint32_t* progress, cudaStream_t st) {
  CUtensorMap ma, mb;
  if (!make_map(&ma, a.H, a.d, a.T, a.ldh, kBoxA) || !make_map(&mb, a.W, a.d, a.V, a.d, kBoxB))
    return cudaErrorInvalidValue;
  GemmParams p{};
  p.m_tiles = (int)ceil_div(rows, GROUP_M);
  p.n_tiles = (int)ceil_div(a.V, lp_tile_cols(a.d));
  p.nsplit = lp_split(rows, a.d, a.V, lp_tile_cols(a.d));
  p.per_split = (int)ceil_div(p.n_tiles, p.nsplit);
  p.k_blocks = (int)ceil_div(a.d, BK);
  p.a_row0 = (int)t0;
  p.rows_valid = t0 + rows;
  p.cols_valid = a.V;
  p.out_row0 = t0;
  p.y = a.y;
  p.partials = partials;
  p.T = rows;
  p.part_row0 = t0;
  p.d_status = a.d_status;
  p.sc2 = kLog2e * a.inv_t;
  p.cand = cand;
  p.cand_max = cand_max;
  p.cand_ld = rows;
  p.cand_slots = lp_fwd_slots(2 * p.nsplit, a.d, a.V, a.top_k);
  const int list = lp_list_len(a.top_k);
  const bool ent = a.entropy != nullptr;
  if (!lp_paced(rows)) progress = nullptr;
  return lp_narrow(a.d) ? launch_lp_fwd<true>(list, ent, ma, mb, p, progress, st)
                        : launch_lp_fwd<false>(list, ent, ma, mb, p, progress, st);
}

// Parts that dH's contraction over the vocabulary is cut into when its tiles leave pairs idle: the one that minimises
// the k-blocks of a part (0.61 us each) plus the writing and summing of the parts' fp32 results (8 bytes per element at 4 TB/s,
// and a launch).  203 rows, d = 1024, V = 32000: 2 tiles, 286 us in one part, 26 + 4 us in 25 parts and their sum.
int lp_dh_splits(int64_t rows, int32_t d, int32_t V) {
  const int64_t units = ceil_div(rows, GROUP_M) * ceil_div(d, BN);
  const int k_blocks = (int)ceil_div(V, BK), most = (int)(group_count() / units);
  int best = 1;
  double best_t = 0.61 * k_blocks;
  for (int s = 2; s <= most && s <= k_blocks; ++s) {
    const int per = (int)ceil_div(k_blocks, s);
    if ((int)ceil_div(k_blocks, per) != s) continue;
    const double t = 0.61 * per + 4.0 + s * (double)rows * d * 2.0e-6;
    if (t < best_t) { best_t = t; best = s; }
  }
  return best;
}

// Room for those parts, for a launch over any number of rows up to `rows`: s parts take at most the pairs, s x row tiles x
// column tiles <= pairs, so neither more than pairs / column tiles of them nor more than a tile for each pair.
size_t lp_dh_split_bytes(int64_t rows, int32_t d) {
  const int64_t cols = ceil_div(d, BN), most = group_count() / cols;
  if (most < 2) return 0;
  const int64_t by_rows = most * rows * d, by_tiles = group_count() * (int64_t)GROUP_M * BN;
  return (size_t)(by_rows < by_tiles ? by_rows : by_tiles) * 4;
}

// bf16 backward for general upstream gradients, chunk by chunk as launch_bwd_bf16: the chunk's logit
// gradient, dH = G W, dW (+)= G^T H.  A bf16 dW over several chunks is summed in fp32 (`partial`) and
// rounded once, in the last chunk's epilogue.
cudaError_t launch_lp_bwd_bf16(const LpBwd& a, const LpBwdScratch& w, cudaStream_t st) {
  __nv_bfloat16* const G = w.g;
  const int64_t chunk_rows = w.chunk, ldg = w.ldg;
  uint32_t* progress = w.progress;
  CUtensorMap mH_k, mW_k, mW_mn, mH_mn;
  if (!make_map(&mH_k, a.H, a.d, a.T, a.ldh, kBoxA) || !make_map(&mW_k, a.W, a.d, a.V, a.d, kBoxB) ||
      !make_map(&mW_mn, a.W, a.d, a.V, a.d, 64))
    return cudaErrorInvalidValue;
  const int tiles_v = (int)ceil_div(a.V, GROUP_M);
  uint32_t* const all_progress = progress;
  cudaError_t e;
  for (int64_t t0 = 0; t0 < a.T; t0 += chunk_rows) {
    const int64_t rows = (a.T - t0) < chunk_rows ? (a.T - t0) : chunk_rows;
    progress = lp_paced(rows) ? all_progress : nullptr;
    const bool rounded = a.dW_dtype == SPO_DTYPE_BF16 && t0 + rows >= a.T;       // dW's final rounding is this chunk's
    TargetRest rest{};
    if (a.g_logp) {
      rest.y = a.y + t0;
      rest.mask = a.mask ? a.mask + t0 : nullptr;
      rest.rest = w.rest; rest.slot = w.slot; rest.rows = w.rest_rows;
    }
    const int m_tiles = (int)ceil_div(rows, GROUP_M);
    CUtensorMap mG_k, mG_mn;
    if (!make_map(&mG_k, G, a.V, rows, ldg, kBoxA) || !make_map(&mG_mn, G, a.V, rows, ldg, 64))
      return cudaErrorInvalidValue;
    {
      GemmParams p{};
      p.m_tiles = m_tiles;
      p.n_tiles = (int)ceil_div(a.V, lp_tile_cols(a.d));
      p.nsplit = lp_split(rows, a.d, a.V, lp_tile_cols(a.d));
      p.per_split = (int)ceil_div(p.n_tiles, p.nsplit);
      p.k_blocks = (int)ceil_div(a.d, BK);
      p.a_row0 = (int)t0;
      p.rows_valid = a.T;
      p.cols_valid = a.V;
      p.out_row0 = t0;
      p.y = a.y; p.lse = a.lse; p.mask = a.mask; p.ent = a.ent;
      p.g_logp = a.g_logp; p.g_lse = a.g_lse; p.g_ent = a.g_ent;
      p.inv_t = a.inv_t; p.sc2 = kLog2e * a.inv_t;
      p.G = G; p.ldg = ldg;
      p.rest = rest;
      p.d_status = a.d_status;
      e = lp_narrow(a.d) ? launch_gemm<MODE_G, false, 0, true>(mH_k, mW_k, p, progress, st)
                         : launch_gemm<MODE_G, false, 0, false>(mH_k, mW_k, p, progress, st);
      if (e != cudaSuccess) return e;
    }
    const int k_splits = lp_dh_splits(rows, a.d, a.V);
    const int64_t dh_bytes = a.dH_dtype == SPO_DTYPE_BF16 ? 2 : 4;
    void* const dH = (char*)a.dH + t0 * a.d * dh_bytes;
    {
      GemmParams p{};
      p.m_tiles = m_tiles;
      p.n_tiles = (int)ceil_div(a.d, BN);
      p.nsplit = p.n_tiles;
      p.per_split = 1;
      p.k_blocks = (int)ceil_div(a.V, BK);
      p.k_splits = k_splits;
      p.k_per = (int)ceil_div(p.k_blocks, k_splits);
      p.rows_valid = rows;
      p.cols_valid = a.d;
      p.ldo = a.d;
      p.d_status = a.d_status;
      if (k_splits == 1) {
        p.out = dH; p.out_bf16 = a.dH_dtype == SPO_DTYPE_BF16;
        p.rest = rest; p.n_rest = a.V; p.w_rows = reinterpret_cast<const __nv_bfloat16*>(a.W);
      } else {
        p.out = w.split;
      }
      e = launch_gemm<MODE_DH, false, 0>(mG_k, mW_mn, p, progress, st);
      if (e != cudaSuccess) return e;
    }
    const __nv_bfloat16* const H = reinterpret_cast<const __nv_bfloat16*>(a.H) + t0 * a.ldh;
    e = launch_lp_rest(w.split, k_splits == 1 ? 0 : k_splits, rows, a.d, a.V, dH, a.dH_dtype, a.W, H, a.ldh, rest, rounded,
                       nullptr, a.mask ? a.mask + t0 : nullptr, a.mask ? w.h_clean : nullptr, st);
    if (e != cudaSuccess) return e;
    // The gradient of a masked row is zero, but zero times a NaN in that row of H is not: with a mask the
    // dW contraction reads a copy of the chunk's rows in which the masked ones are zero.
    int64_t h_row0 = t0;
    if (a.mask) {
      h_row0 = 0;
      if (!make_map(&mH_mn, w.h_clean, a.d, rows, a.d, 64)) return cudaErrorInvalidValue;
    } else if (!make_map(&mH_mn, a.H, a.d, a.T, a.ldh, 64)) {
      return cudaErrorInvalidValue;
    }
    if (!rounded) {
      float* const sum = a.dW_dtype == SPO_DTYPE_F32 ? (float*)a.dW : w.partial;
      const bool add = t0 > 0 || (a.dW_dtype == SPO_DTYPE_F32 && a.accumulate);
      e = launch_dw(mG_mn, mH_mn, h_row0, rows, a.d, a.V, sum, add ? 1 : 0, 0, tiles_v, progress, a.d_status, st);
      if (e == cudaSuccess)
        e = launch_lp_rest(nullptr, 0, rows, a.d, a.V, nullptr, a.dH_dtype, a.W, H, a.ldh, rest, true, sum,
                           nullptr, nullptr, st);
    } else {
      GemmParams p{};
      p.m_tiles = tiles_v;
      p.n_tiles = (int)ceil_div(a.d, lp_tile_cols(rows));
      p.nsplit = p.n_tiles;
      p.per_split = 1;
      p.k_blocks = (int)ceil_div(rows, BK);
      p.b_k0 = (int)h_row0;
      p.rows_valid = a.V;
      p.cols_valid = a.d;
      p.out = a.dW; p.out_bf16 = 1; p.ldo = a.d; p.accumulate = a.accumulate;
      p.partial = t0 > 0 ? w.partial : nullptr;
      p.rest = rest;
      p.d_status = a.d_status;
      e = lp_narrow(rows) ? launch_gemm<MODE_DW, false, 0, true>(mG_mn, mH_mn, p, progress, st)
                          : launch_gemm<MODE_DW, false, 0, false>(mG_mn, mH_mn, p, progress, st);
    }
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

// ---------------------------------------------------------------------------
// One-pass forward+backward: three contractions per token instead of the four of
// forward-then-backward.
//   PRE      the logits of the first vocabulary tile for all rows (0.3 % of one contraction): their
//            row maxima fix every row's reference exponent
//   per chunk c of token rows, into slot c % slots of the chunk buffers:
//     E(c)     logits contraction; epilogue: sum of exponentials, target logit, e = 2^(z log2e - ref) as bf16
//     fin(c)   lse, logp, ratio, surrogate, coef, loss terms; row scale; the target entry of e patched
//     scale(c) the chunk's rows of H times their row scale (bf16), the operand of the dW contraction
//     DH(c)    dH rows = rowscale * (e W)
//   per group of `slots` chunks:  DW   dW (+)= e^T (rowscale H) over the rows of the whole group
// Contracting dW over several chunks at once divides its read-modify-write passes over the
// [V x d] fp32 matrix (and its accumulator drains) by that number.
// ---------------------------------------------------------------------------
#ifndef SPO_DW_CHUNK_GROUP
#define SPO_DW_CHUNK_GROUP 2
#endif
constexpr int kDwChunkGroup = SPO_DW_CHUNK_GROUP;

FusedWs fused_ws_layout(int64_t T, int32_t d, int32_t V, int32_t S) {
  FusedWs L{};
  const BwdWs b = bwd_ws_layout(T, d, V);
  L.chunk_rows = b.chunk_rows;
  L.ldg = b.ldg;
  const int n_tiles_v = (int)ceil_div(V, BN);
  const int64_t t_eff = T > 0 ? T : 1;
  const int64_t n_chunks = ceil_div(t_eff, L.chunk_rows);
  L.slots = (int)(n_chunks < kDwChunkGroup ? n_chunks : kDwChunkGroup);
  // partials: the full chunk and the (shorter) last chunk may pick different split counts
  const int64_t full_rows = t_eff < L.chunk_rows ? ceil_div(t_eff, GROUP_M) * GROUP_M : L.chunk_rows;
  size_t part_elems = (size_t)2 * pick_fwd_split(full_rows / GROUP_M, n_tiles_v, d) * (size_t)full_rows;
  const int64_t tail = t_eff % L.chunk_rows;
  if (t_eff > L.chunk_rows && tail > 0) {
    const int64_t tail_rows = ceil_div(tail, GROUP_M) * GROUP_M;
    const size_t e2 = (size_t)2 * pick_fwd_split(tail_rows / GROUP_M, n_tiles_v, d) * (size_t)tail_rows;
    if (e2 > part_elems) part_elems = e2;
  }
  L.fin_blocks = ceil_div(t_eff, kFinalizeThreads);
  size_t off = 0;
  L.g = off;          off = align_up(off + (size_t)L.slots * (size_t)L.chunk_rows * (size_t)L.ldg * 2, 256);
  L.hs = off;         off = align_up(off + (size_t)L.slots * (size_t)L.chunk_rows * (size_t)d * 2, 256);
  L.pre = off;        off = align_up(off + sizeof(FwdPartial) * 2 * (size_t)t_eff, 256);
  L.rowscale = off;   off = align_up(off + sizeof(float) * (size_t)t_eff, 256);
  L.partials = off;   off = align_up(off + sizeof(FwdPartial) * part_elems, 256);
  L.progress = off;   off = align_up(off + kProgressBytes, 256);
  L.block_sums = off; off = align_up(off + sizeof(double) * (size_t)L.fin_blocks, 256);
  L.counters = off;   off = align_up(off + 4 * sizeof(int32_t), 256);
  L.seq_cnt = off;    off = align_up(off + sizeof(int32_t) * (size_t)(S > 0 ? S : 1), 256);
  L.total = off;
  return L;
}

namespace {
// Row tiles (of GROUP_M vocabulary rows) per slab: whole rounds of units, so that no slab ends on a
// partly filled round of CTA pairs.
int slab_tiles(int32_t V, int32_t d, int n_wanted, int* n_out) {
  const int tiles = (int)ceil_div(V, GROUP_M), n_tiles_d = (int)ceil_div(d, BN), groups = group_count();
  int g = groups, b = n_tiles_d;                       // gcd
  while (b) { const int t = g % b; g = b; b = t; }
  const int quantum = groups / g;                      // row tiles whose units fill the pairs a whole number of times
  if (n_wanted < 1) n_wanted = 1;
  int per = tiles / n_wanted / quantum * quantum;      // rounded down: the last slab takes what is left over
  if (per < quantum) per = quantum;
  const int n = (int)ceil_div(tiles, per);
  *n_out = n < n_wanted ? n : n_wanted;
  return per;
}
}  // namespace

int dw_slab_rows(int32_t V, int32_t d, int n_wanted, int64_t* row_begin) {
  int n = 1;
  const int per = slab_tiles(V, d, n_wanted, &n);
  for (int k = 0; k < n; ++k) row_begin[k] = (int64_t)k * per * GROUP_M;
  row_begin[n] = V;                                    // slab n-1 runs to the end of the vocabulary
  return n;
}

cudaError_t launch_fused_bf16(const FusedArgs& a, char* ws, const FusedWs& L, cudaStream_t st) {
  FwdPartial* partials = reinterpret_cast<FwdPartial*>(ws + L.partials);
  FwdPartial* pre = reinterpret_cast<FwdPartial*>(ws + L.pre);
  float* rowscale = reinterpret_cast<float*>(ws + L.rowscale);
  uint32_t* progress = reinterpret_cast<uint32_t*>(ws + L.progress);
  double* block_sums = reinterpret_cast<double*>(ws + L.block_sums);
  int32_t* counters = reinterpret_cast<int32_t*>(ws + L.counters);
  int32_t* seq_cnt = reinterpret_cast<int32_t*>(ws + L.seq_cnt);
  __nv_bfloat16* gbuf = reinterpret_cast<__nv_bfloat16*>(ws + L.g);
  __nv_bfloat16* hsbuf = reinterpret_cast<__nv_bfloat16*>(ws + L.hs);
  const spo_params& pr = *a.params;
  const int64_t T = a.T;
  const int32_t d = a.d, V = a.V;
  cudaError_t e = launch_fwd_prepare(a.mask, T, a.cu_seqlens, a.S, pr.agg_mode != 0, seq_cnt, counters, st);
  if (e != cudaSuccess) return e;
  if (T == 0) {
    e = launch_fwd_finalize(partials, 0, a.y, a.logp_old, a.mask, a.cu_seqlens, a.a_norm, 0, V, a.S, a.loss, a.logp,
                            a.lse, a.coef, a.seq_sums, a.entropy, block_sums, counters, seq_cnt, pr, L.fin_blocks,
                            a.d_status, st);
    if (e != cudaSuccess) return e;
    if (!a.accumulate && (e = cudaMemsetAsync(a.dW, 0, sizeof(float) * (size_t)V * d, st)) != cudaSuccess) return e;
    if (a.shards && a.accumulate && (e = launch_dw_scatter_add(a.dW, V, d, *a.shards, st)) != cudaSuccess) return e;
    if (a.n_slabs > 0 && a.events) {              // nothing to contract: every slab is final at once
      int n = 1;
      slab_tiles(V, d, a.n_slabs, &n);
      for (int k = 0; k < n; ++k)
        if ((e = cudaEventRecord(a.events[k], st)) != cudaSuccess) return e;
    }
    return cudaSuccess;
  }
  CUtensorMap mH_k, mW_k, mW_mn;
  if (!make_map(&mH_k, a.H, d, T, d, kBoxA) || !make_map(&mW_k, a.W, d, V, d, kBoxB) ||
      !make_map(&mW_mn, a.W, d, V, d, 64))
    return cudaErrorInvalidValue;
  const int n_tiles_v = (int)ceil_div(V, BN);
  const int n_chunks = (int)ceil_div(T, L.chunk_rows);
  const bool ent = a.entropy != nullptr;

  // PRE: first vocabulary tile of every row (the forward's kernel on one column tile)
  {
    GemmParams p{};
    p.m_tiles = (int)ceil_div(T, GROUP_M);
    p.n_tiles = 1;
    p.nsplit = 1;
    p.per_split = 1;
    p.k_blocks = (int)ceil_div(d, BK);
    p.rows_valid = T;
    p.cols_valid = V;
    p.y = a.y;
    p.partials = pre;
    p.T = T;
    p.d_status = a.d_status;
    if ((e = launch_gemm<MODE_FWD>(mH_k, mW_k, p, progress, st)) != cudaSuccess) return e;
  }

  for (int c0 = 0; c0 < n_chunks; c0 += L.slots) {
    int64_t group_rows = 0;
    for (int c = c0; c < n_chunks && c < c0 + L.slots; ++c) {
      const int slot = c - c0;
      const int64_t t0 = (int64_t)c * L.chunk_rows;
      const int64_t rows = (T - t0) < L.chunk_rows ? (T - t0) : L.chunk_rows;
      const int m_tiles = (int)ceil_div(rows, GROUP_M);
      const int64_t rows_pad = (int64_t)m_tiles * GROUP_M;
      __nv_bfloat16* G = gbuf + (size_t)slot * (size_t)L.chunk_rows * (size_t)L.ldg;
      // E: logits of chunk c
      const int nsplit = pick_fwd_split(m_tiles, n_tiles_v, d);
      {
        GemmParams p{};
        p.m_tiles = m_tiles;
        p.n_tiles = n_tiles_v;
        p.nsplit = nsplit;
        p.per_split = (int)ceil_div(n_tiles_v, p.nsplit);
        p.k_blocks = (int)ceil_div(d, BK);
        p.a_row0 = (int)t0;
        p.rows_valid = T;
        p.cols_valid = V;
        p.out_row0 = t0;
        p.y = a.y;
        p.partials = partials;
        p.T = rows_pad;
        p.part_row0 = t0;
        p.G = G; p.ldg = L.ldg;
        p.pre = pre; p.pre_ld = T;
        p.d_status = a.d_status;
        e = ent ? launch_gemm<MODE_E, true>(mH_k, mW_k, p, progress, st)
                : launch_gemm<MODE_E, false>(mH_k, mW_k, p, progress, st);
        if (e != cudaSuccess) return e;
      }
      // fin: per-token outputs of chunk c's rows, loss terms per block, row scale, patched target entries
      {
        FinalizeRange rg;
        rg.t_begin = t0;
        rg.part_ld = rows_pad;
        rg.block0 = (int)(t0 / kFinalizeThreads);
        rg.total_blocks = (int)L.fin_blocks;
        rg.last = (c == n_chunks - 1) ? 1 : 0;
        OnePassFix fix;
        fix.G = reinterpret_cast<uint16_t*>(G);
        fix.ldg = L.ldg;
        fix.g_row0 = t0;
        fix.rowscale = rowscale;
        fix.grad_loss = a.grad_loss;
        e = launch_fwd_finalize(partials, 2 * nsplit, a.y, a.logp_old, a.mask, a.cu_seqlens, a.a_norm, t0 + rows, V,
                                a.S, a.loss, a.logp, a.lse, a.coef, a.seq_sums, a.entropy, block_sums, counters, seq_cnt,
                                pr, L.fin_blocks, a.d_status, st, &rg, &fix);
        if (e != cudaSuccess) return e;
      }
      // the chunk's rows of H times their row scale, behind the rows of the group's earlier chunks
      e = launch_scale_rows(a.H, rowscale, t0, rows, d * 2, hsbuf + (size_t)slot * (size_t)L.chunk_rows * (size_t)d, st);
      if (e != cudaSuccess) return e;
      // DH: rows of chunk c
      {
        CUtensorMap mG_k;
        if (!make_map(&mG_k, G, V, rows, L.ldg, kBoxA)) return cudaErrorInvalidValue;
        e = launch_dh(mG_k, mW_mn, t0, rows, T, d, V, a.dH, a.dH_dtype, rowscale, progress, a.d_status, st);
        if (e != cudaSuccess) return e;
      }
      group_rows += rows;        // only the group's last chunk can be short, so the rows stay contiguous
    }
    // DW over the group's rows
    CUtensorMap mG_mn, mHs_mn;
    if (!make_map(&mG_mn, gbuf, V, group_rows, L.ldg, 64) || !make_map(&mHs_mn, hsbuf, d, group_rows, d, 64))
      return cudaErrorInvalidValue;
    const int tiles = (int)ceil_div(V, GROUP_M);
    const int dw_acc = (a.accumulate || c0 > 0) ? 1 : 0;
    if (a.n_slabs > 0 && a.events && c0 + L.slots >= n_chunks) {
      // the last contraction of dW, slab by slab: behind each slab its rows are final
      int n = 1;
      const int per = slab_tiles(V, d, a.n_slabs, &n);
      for (int k = 0; k < n; ++k) {
        const int t_begin = k * per, t_count = k == n - 1 ? tiles - t_begin : per;
        e = launch_dw(mG_mn, mHs_mn, 0, group_rows, d, V, a.dW, dw_acc, t_begin, t_count, progress, a.d_status, st);
        if (e != cudaSuccess) return e;
        if ((e = cudaEventRecord(a.events[k], st)) != cudaSuccess) return e;
      }
    } else {
      // reduce-scatter form: the call's last contraction sends the finished tiles to their owners
      const spo_dw_shards* sh = (a.shards && c0 + L.slots >= n_chunks) ? a.shards : nullptr;
      e = launch_dw(mG_mn, mHs_mn, 0, group_rows, d, V, a.dW, dw_acc, 0, tiles, progress, a.d_status, st, sh);
      if (e != cudaSuccess) return e;
    }
  }
  return cudaSuccess;
}

cudaError_t launch_bounded_wait_probe(int32_t* d_status, uint32_t limit_us, int32_t* reached_end, cudaStream_t st) {
  bounded_wait_probe_kernel<<<1, 32, 0, st>>>(d_status, (unsigned long long)limit_us * 1000ull, reached_end);
  return cudaGetLastError();
}

}  // namespace spo
