// Orthogonalised weight updates (spo_orthogonalize, spo_muon_update): Newton-Schulz iteration
//   X <- a X + (b A + c A A) X,   A = X X^T,   X_0 = U / (|U|_F + eps)
// on the tensor cores, with momentum in front and the weight update behind it in the same call.
// (Taller than wide: A = X^T X and X <- a X + X (b A + c A A), so the square products are over the smaller side
// and nothing is ever transposed.)
//
// Numbers.  The iteration multiplies small singular values by a per step (a^5 = 485), and with them
// every rounding made in X while they are small.  So X is held twice, in fp32 for the term a X and in fp16
// for the products, whose spectrum is small where X's is; both times s = 2^round(log2 sqrt(max(m, n))), which
// puts the entries of an orthogonal matrix near one.  Errors against 64 bits for a 512 x 512 update of rank 16
// under no noise: this 8e-4, fp16 alone 4e-2, bf16 alone 0.33 (a full-rank Gaussian: 8e-4, 1.3e-3, 1.1e-2).  fp16
// rather than bf16 because everything here is bounded by about 10 in magnitude and fp16 has 8 times finer steps.
// A and b A + c A A are rounded to fp16 once each, but for the diagonal of the latter: near convergence it is -2.7 and
// the rest almost nothing, so it stays in fp32 and multiplies X in fp32 (19 x 183: error of the iteration 8e-4; rounded
// with the rest 1.7e-3).  All sums are fp32.
//
// Work.  A and A A are symmetric: only the blocks on and above the diagonal are computed and stored (a block below it
// is read as the transposed operand of its mirror image), 3 m^2 n + m^3 operations a step for m <= n instead of
// 4 m^2 n + 2 m^3.  Five steps of a 4096 x 4096 matrix are 1.37 TFLOP: tensor-bound from a few hundred rows on,
// launch-bound below.
#include <cuda.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <math_constants.h>
#include <stdint.h>

#include <atomic>

#include "spo_internal.h"
#include "spo_ptx.cuh"

namespace spo {

namespace {

constexpr int NS_BM = 128;                      // rows of A per CTA; a pair's tile has 256
constexpr int NS_EPI_WARPS = 8;
constexpr int NS_THREADS = 32 * (2 + NS_EPI_WARPS);
constexpr int NS_STAGING = 4096;
constexpr int NS_RING = 192 * 1024;             // operand stages
constexpr int NS_BARS = 512;                    // barriers of the two kinds of product, tensor-memory address, flags
constexpr int NS_SMEM = NS_RING + 1024 + NS_BARS + NS_EPI_WARPS * NS_STAGING;

template <int BN>
struct NsCfg {
  static constexpr int mmas = BN > 256 ? 2 : 1;          // products per step of 16 in k, sharing A
  static constexpr int n_mma = BN / mmas;                // columns of one
  static constexpr int b_rows = n_mma / 2;               // B columns per CTA and product
  static constexpr int a_bytes = NS_BM * 64 * 2;
  static constexpr int b_bytes = b_rows * 64 * 2;
  static constexpr int stage_bytes = a_bytes + mmas * b_bytes;
  static constexpr int stages = NS_RING / stage_bytes;
  static constexpr int bufs = BN > 256 ? 1 : 2;          // accumulators in tensor memory
  static constexpr int tmem_cols = bufs * BN;
  static constexpr int bar_bytes = 16 * stages + 32;
};
// Barriers of one kind of product: stages full / empty, accumulators full / empty.
struct NsBars { uint32_t full0, empty0, tfull0, tempty0; };
template <int BN>
__device__ __forceinline__ NsBars ns_bars(uint32_t at) {
  constexpr int S = NsCfg<BN>::stages;
  return {at, at + 8 * S, at + 16 * S, at + 16 * S + 16};
}

enum : int { OUT_BF16 = 1, OUT_F32 = 2, OUT_W_BF16 = 3, OUT_W_F32 = 4 };

struct NsMaps { CUtensorMap x128[2], x64[2], gram128, gram64, poly128, poly64; };   // by box height

struct NsParams {
  int batch, steps, tall;
  int m, n, mm;                                // matrix, and its smaller side
  int64_t ld, gld;                             // pitch of X and of the square matrices
  int sym_tiles, sym_n, upd_tiles, upd_n;      // tiles per matrix and column tiles of the two kinds of product
  int kb_long, kb_short;                       // k-blocks along the longer / the smaller side
  __half *hi[2], *gram, *poly;                 // X in fp16 (two, written in turn), A, b A + c A A; row-major
  float* x32;                                  // X in fp32, in blocks of 32 x 32 (see ns_block)
  __half* gram_blk;                            // A once more, in blocks
  float* diag;                                 // [batch][mm] the diagonal of b A + c A A (zero in poly)
  float inv_s2, a, b, c;
  int out_mode;
  void* out;                                   // result or weights, pitch n
  float out_scale, decay;                      // result: x out_scale;  weights: w decay - x out_scale
  const int32_t* bad;                          // [batch]: the matrix held a NaN or an infinity: leave its weights alone
  uint32_t* arrivals;                          // CTAs that have finished a product, over all products; zero at the start
  int32_t* d_status;
};

__device__ __forceinline__ void tma_load_3d_pair(uint32_t dst, const CUtensorMap* map, int c0, int c1, int c2, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
      ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(c0), "r"(c1), "r"(c2), "r"(bar)
      : "memory");
}
// Orders this thread's plain accesses to global memory against TMA accesses (the asynchronous proxy).
__device__ __forceinline__ void fence_proxy_async() { asm volatile("fence.proxy.async.global;" ::: "memory"); }

__device__ __forceinline__ uint32_t pack_half(float lo, float hi) {
  const __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ float2 unpack_half(uint32_t v) { return __half22float2(*reinterpret_cast<const __half2*>(&v)); }

// What only epilogues read (X in fp32, the copy of A) is kept in blocks of 32 x 32 in the order in which tensor
// memory hands out an accumulator: lane = row, 16 bytes of each lane side by side, so that a warp's access
// is 512 consecutive bytes and nothing passes through shared memory.
__device__ __forceinline__ int64_t ns_block(int b, int row, int col, int rows, int cols) {
  const int64_t rb = (rows + 31) >> 5, cb = (cols + 31) >> 5;
  return (((int64_t)b * rb + (row >> 5)) * cb + (col >> 5)) * 1024;
}

// Storage of an operand: with k contiguous, with the M / N index contiguous, or a symmetric matrix of which the
// 256-blocks on and above the diagonal are stored.
enum : int { OP_K = 0, OP_MN = 1, OP_SYM = 2 };
// Whether the 64-deep k-block kb of the rows from `row` on is fetched with the M / N index contiguous.
template <int OP>
__device__ __forceinline__ bool ns_is_mn(int row, int kb) { return OP == OP_MN || (OP == OP_SYM && (kb >> 2) < (row >> 8)); }

struct NsTile { int b, i, j; };
// Tile `t` of a product: row tile i, column tile j of matrix b.  SYM: row tile i has the column tiles that
// reach to or past its diagonal block (row i starts with column tile 256 i / BN).
template <bool SYM, int BN>
__device__ __forceinline__ NsTile ns_tile(int t, int tiles, int n_tiles) {
  NsTile r;
  r.b = t / tiles;
  int q = t - r.b * tiles;
  if (SYM) {
    int i = 0, first = 0;
    while (q >= n_tiles - first) { q -= n_tiles - first; ++i; first = i * 256 / BN; }
    r.i = i;
    r.j = first + q;
  } else {
    r.i = q / n_tiles;
    r.j = q - r.i * n_tiles;
  }
  return r;
}

// Waits until `goal` CTAs have arrived (bounded).  Called by one lane.
__device__ __forceinline__ bool ns_grid_wait(const NsParams& p, uint32_t goal, volatile int* abort_flag) {
  unsigned long long t0 = 0;
  for (uint32_t spins = 0;; ++spins) {
    uint32_t v;
    asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(v) : "l"(p.arrivals) : "memory");
    if (v >= goal) return true;
    __nanosleep(40);
    if ((spins & 255u) == 255u) {
      if (*abort_flag) return false;
      const unsigned long long now = global_timer_ns();
      if (t0 == 0) {
        t0 = now;
      } else if (now - t0 > kWaitLimitNs) {
        *abort_flag = 1;
        if (p.d_status) atomicOr(p.d_status, SPO_DEV_TIMEOUT);
        return false;
      }
    }
  }
}

// ---- roles.  Each walks this pair's tiles of one product; `it` and `n` run on over all products. ----

template <bool SYM, int A, int B, int BN>
__device__ __forceinline__ bool ns_produce(const CUtensorMap* a128, const CUtensorMap* a64, const CUtensorMap* b128,
                                           const CUtensorMap* b64, int total, int tiles, int n_tiles, int k_blocks,
                                           uint32_t base, const NsBars& bars, uint32_t rank, uint32_t& it,
                                           volatile int* abort_flag, int32_t* d_status) {
  const uint32_t full0 = bars.full0, empty0 = bars.empty0;
  using C = NsCfg<BN>;
  for (int t = blockIdx.x / 2; t < total; t += gridDim.x / 2) {
    const NsTile tl = ns_tile<SYM, BN>(t, tiles, n_tiles);
    const int row = tl.i * 256 + (int)rank * NS_BM, col = tl.j * BN + (int)rank * C::b_rows;
    for (int kb = 0; kb < k_blocks; ++kb, ++it) {
      const uint32_t s = it % C::stages, ph = (it / C::stages) & 1u;
      if (!mbar_wait<20>(empty0 + 8 * s, ph ^ 1u, abort_flag, d_status)) return false;
      const uint32_t sa = base + s * C::stage_bytes, sb = sa + C::a_bytes;
      if (rank == 0) mbar_expect_tx(full0 + 8 * s, 2 * C::stage_bytes);
      const uint32_t fb = map_to_cta(full0 + 8 * s, 0);
      if (!ns_is_mn<A>(row, kb)) {
        tma_load_3d_pair(sa, a128, kb * 64, row, tl.b, fb);
      } else {
#pragma unroll
        for (int x = 0; x < NS_BM / 64; ++x) tma_load_3d_pair(sa + x * 8192, a64, row + x * 64, kb * 64, tl.b, fb);
      }
#pragma unroll
      for (int h = 0; h < C::mmas; ++h) {
        const int c = col + h * C::n_mma;
        if (!ns_is_mn<B>(c, kb)) {
          tma_load_3d_pair(sb + h * C::b_bytes, C::b_rows == 64 ? b64 : b128, kb * 64, c, tl.b, fb);
        } else {
#pragma unroll
          for (int x = 0; x < C::b_rows / 64; ++x)
            tma_load_3d_pair(sb + h * C::b_bytes + x * 8192, b64, c + x * 64, kb * 64, tl.b, fb);
        }
      }
    }
  }
  return true;
}

template <bool SYM, int A, int B, int BN>
__device__ __forceinline__ bool ns_multiply(int total, int tiles, int n_tiles, int k_blocks, uint32_t base, uint32_t tmem_base,
                                            const NsBars& bars, uint32_t& it, uint32_t& n, volatile int* abort_flag,
                                            int32_t* d_status) {
  const uint32_t full0 = bars.full0, empty0 = bars.empty0, tfull0 = bars.tfull0, tempty0 = bars.tempty0;
  using C = NsCfg<BN>;
  // fp32 accumulate, fp16 A and B, M = 256 over the pair
  constexpr uint32_t idesc0 = (1u << 4) | ((uint32_t)(C::n_mma >> 3) << 17) | (16u << 24);
  for (int t = blockIdx.x / 2; t < total; t += gridDim.x / 2, ++n) {
    const NsTile tl = ns_tile<SYM, BN>(t, tiles, n_tiles);
    const uint32_t b = n % C::bufs;
    if (!mbar_wait(tempty0 + 8 * b, ((n / C::bufs) & 1u) ^ 1u, abort_flag, d_status)) return false;
    tc_fence_after();
    for (int kb = 0; kb < k_blocks; ++kb, ++it) {
      const uint32_t s = it % C::stages, ph = (it / C::stages) & 1u;
      if (!mbar_wait(full0 + 8 * s, ph, abort_flag, d_status)) return false;
      tc_fence_after();
      const uint32_t sa = base + s * C::stage_bytes, sb = sa + C::a_bytes;
      const bool a_mn = ns_is_mn<A>(tl.i * 256, kb);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint64_t da = a_mn ? smem_desc(sa + j * 2048, 8192, 1024) : smem_desc(sa + j * 32, 16, 1024);
#pragma unroll
        for (int h = 0; h < C::mmas; ++h) {
          const uint32_t sbh = sb + h * C::b_bytes;
          const bool b_mn = ns_is_mn<B>(tl.j * BN + h * C::n_mma, kb);
          const uint64_t db = b_mn ? smem_desc(sbh + j * 2048, 8192, 1024) : smem_desc(sbh + j * 32, 16, 1024);
          umma_bf16(tmem_base + b * BN + h * C::n_mma, da, db, idesc0 | ((a_mn ? 1u : 0u) << 15) | ((b_mn ? 1u : 0u) << 16),
                    (kb | j) != 0 ? 1u : 0u);
        }
      }
      umma_commit(empty0 + 8 * s);
    }
    umma_commit(tfull0 + 8 * b);
  }
  return true;
}

// Epilogues.  On small matrices a product lasts as long as its code takes to arrive: each of them runs once between two
// barriers, so the 32-column steps are loops that are not unrolled (unrolled in pairs: 128 x 512 106 us for 96, four
// 1000 x 2730 568 for 540).
// What the epilogue warps share: barriers, tensor memory, staging buffer.
struct NsEpi {
  uint32_t tmem_base, rank;
  uint8_t* stage;
  int quarter, half, lane;
  volatile int* abort_flag;
  int32_t* d_status;
};
template <int BN>
__device__ __forceinline__ bool ns_tile_ready(const NsEpi& e, const NsBars& bars, uint32_t n) {
  using C = NsCfg<BN>;
  int good = 1;
  if (e.lane == 0) good = mbar_wait<20>(bars.tfull0 + 8 * (n % C::bufs), (n / C::bufs) & 1u, e.abort_flag, e.d_status) ? 1 : 0;
  good = __shfl_sync(0xffffffffu, good, 0);
  tc_fence_after();
  return good != 0;
}
template <int BN>
__device__ __forceinline__ void ns_tile_done(const NsEpi& e, const NsBars& bars, uint32_t n) {
  tc_fence_before();
  __syncwarp();
  if (e.lane == 0) mbar_arrive_cluster(map_to_cta(bars.tempty0 + 8 * (n % NsCfg<BN>::bufs), 0));
}

// A = acc / s^2, or b A + c acc (POLY); A is also kept in blocks, from which POLY reads it.  POLY keeps the diagonal
// apart, in fp32, and leaves zeros in its place: see the numbers above.  What a tile reads is fetched before its
// products are waited for, then one step of 64 columns ahead.
template <int BN, bool POLY>
__device__ __forceinline__ bool ns_store_sym(const NsEpi& e, const NsBars& bars, const NsParams& p, int total, __half* S, float alpha, float beta,
                                             uint32_t& n) {
  const int lane = e.lane, rows = p.mm;
  const int64_t ld = p.gld;
  for (int t = blockIdx.x / 2; t < total; t += gridDim.x / 2, ++n) {
    const NsTile tl = ns_tile<true, BN>(t, p.sym_tiles, p.sym_n);
    const int row0 = tl.i * 256 + (int)e.rank * NS_BM + e.quarter * 32;
    // Columns left of the diagonal block (512-wide tiles of odd row blocks) are the mirror of another tile.  The
    // two warps of a quarter take alternate steps of 64 columns, so that a narrow matrix occupies both.
    const int tile_col = tl.j * BN;
    const int64_t mat = (int64_t)tl.b * rows * ld;
    const int col_begin = (tile_col < tl.i * 256 ? tl.i * 256 : tile_col) + e.half * 64;
    const int col_end = row0 >= rows ? 0 : tile_col + BN < rows ? tile_col + BN : rows;
    uint4 next[4];
    auto fetch = [&](int c0) {
      const uint4* src = reinterpret_cast<const uint4*>(p.gram_blk + ns_block(tl.b, row0, c0, rows, rows)) + lane;
#pragma unroll
      for (int q = 0; q < 4; ++q) next[q] = __ldcg(src + 32 * q);
    };
    if (POLY && col_begin < col_end) fetch(col_begin);
    if (!ns_tile_ready<BN>(e, bars, n)) return false;
    const uint32_t taddr = e.tmem_base + ((uint32_t)(e.quarter * 32) << 16) + (n % NsCfg<BN>::bufs) * BN;
#pragma unroll 1
    for (int col0 = col_begin; col0 < col_end; col0 += 128) {
      __syncwarp();                                       // earlier read-backs of the staging buffer are done
#pragma unroll 1
      for (int h = 0; h < 2 && col0 + 32 * h < col_end; ++h) {
        const int c0 = col0 + 32 * h;
        uint32_t v[32];
        float x[32];
        tmem_ld32(taddr + (c0 - tile_col), v);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const uint32_t cw[4] = {next[q].x, next[q].y, next[q].z, next[q].w};
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const int at = 8 * q + 2 * k;
            x[at] = alpha * __uint_as_float(v[at]);
            x[at + 1] = alpha * __uint_as_float(v[at + 1]);
            if (POLY) {
              const float2 f = unpack_half(cw[k]);
              x[at] = fmaf(beta, f.x, x[at]);
              x[at + 1] = fmaf(beta, f.y, x[at + 1]);
            }
          }
        }
        if (POLY && h == 0 && c0 + 32 < col_end) fetch(c0 + 32);
        if (POLY && h == 1 && c0 + 96 < col_end) fetch(c0 + 96);
        if (POLY && c0 == row0) {                         // the block on the diagonal: lane's own column
          float d = 0.0f;
#pragma unroll
          for (int k = 0; k < 32; ++k) {
            d = k == lane ? x[k] : d;
            x[k] = k == lane ? 0.0f : x[k];
          }
          if (row0 + lane < rows) p.diag[(int64_t)tl.b * rows + row0 + lane] = d;
        }
        uint4* dst = reinterpret_cast<uint4*>(p.gram_blk + ns_block(tl.b, row0, c0, rows, rows)) + lane;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const uint4 piece = make_uint4(pack_half(x[8 * q], x[8 * q + 1]), pack_half(x[8 * q + 2], x[8 * q + 3]),
                                         pack_half(x[8 * q + 4], x[8 * q + 5]), pack_half(x[8 * q + 6], x[8 * q + 7]));
          if (!POLY) dst[32 * q] = piece;
          stage_put_piece(e.stage, lane, 4 * h + q, piece);
        }
      }
      __syncwarp();
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        int r, cc;
        const uint4 val = stage_get(e.stage, lane, i, r, cc);
        const int c = col0 + cc * 8;
        // the pitch is a multiple of 8, so a piece that begins inside the row may be stored whole
        if (row0 + r < rows && c < rows) *reinterpret_cast<uint4*>(S + mat + (int64_t)(row0 + r) * ld + c) = val;
      }
    }
    ns_tile_done<BN>(e, bars, n);
  }
  return true;
}

// Four columns of the last x: the result, or the weights with the step taken.  `left`: columns to the row's end.
__device__ __forceinline__ void ns_emit(const NsParams& p, const uint4& acc, int64_t at, int left, int vec) {
  float x[4] = {__uint_as_float(acc.x), __uint_as_float(acc.y), __uint_as_float(acc.z), __uint_as_float(acc.w)};
  if (p.out_mode == OUT_W_BF16 || p.out_mode == OUT_W_F32) {
    float w[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if (p.out_mode == OUT_W_F32) {
      const float* W = reinterpret_cast<const float*>(p.out) + at;
      if (vec == 4) {
        const float4 q = *reinterpret_cast<const float4*>(W);
        w[0] = q.x; w[1] = q.y; w[2] = q.z; w[3] = q.w;
      } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) if (k < left) w[k] = W[k];
      }
    } else {
      const __nv_bfloat16* W = reinterpret_cast<const __nv_bfloat16*>(p.out) + at;
      if (vec == 4) {
        const uint2 q = *reinterpret_cast<const uint2*>(W);
        w[0] = __uint_as_float(q.x << 16); w[1] = __uint_as_float(q.x & 0xFFFF0000u);
        w[2] = __uint_as_float(q.y << 16); w[3] = __uint_as_float(q.y & 0xFFFF0000u);
      } else if (vec == 2) {
        const uint32_t q0 = *reinterpret_cast<const uint32_t*>(W);
        w[0] = __uint_as_float(q0 << 16); w[1] = __uint_as_float(q0 & 0xFFFF0000u);
        if (left > 2) {
          const uint32_t q1 = *reinterpret_cast<const uint32_t*>(W + 2);
          w[2] = __uint_as_float(q1 << 16); w[3] = __uint_as_float(q1 & 0xFFFF0000u);
        }
      } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) if (k < left) w[k] = __bfloat162float(W[k]);
      }
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) x[k] = fmaf(w[k], p.decay, -p.out_scale * x[k]);
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k) x[k] *= p.out_scale;
  }
  if (p.out_mode == OUT_F32 || p.out_mode == OUT_W_F32) {
    float* W = reinterpret_cast<float*>(p.out) + at;
    if (vec == 4) {
      *reinterpret_cast<float4*>(W) = make_float4(x[0], x[1], x[2], x[3]);
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k) if (k < left) W[k] = x[k];
    }
  } else {
    __nv_bfloat16* W = reinterpret_cast<__nv_bfloat16*>(p.out) + at;
    if (vec == 4) {
      *reinterpret_cast<uint2*>(W) = make_uint2(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]));
    } else if (vec == 2) {
      *reinterpret_cast<uint32_t*>(W) = pack_bf16(x[0], x[1]);
      if (left > 2) *reinterpret_cast<uint32_t*>(W + 2) = pack_bf16(x[2], x[3]);
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k) if (k < left) W[k] = __float2bfloat16_rn(x[k]);
    }
  }
}

// x = (a + diagonal) X + acc (the diagonal's entry of the row, TALL: of the column), stored as the next X (fp32 blocks
// and fp16 rows), as the result, or applied to the weights.  The last x is looked at for NaN and infinities: whatever
// overflows on the way (coefficients under which X grows without bound) ends in one, as inf - inf or inf x 0 at the latest.
template <bool TALL, int BN, bool LAST>
__device__ __forceinline__ bool ns_store_update(const NsEpi& e, const NsBars& bars, const NsParams& p, int total, __half* hi_out, uint32_t& n) {
  const int lane = e.lane, rows = p.m, cols = p.n;
  const int vec = (cols & 3) == 0 ? 4 : (cols & 1) == 0 ? 2 : 1;
  for (int t = blockIdx.x / 2; t < total; t += gridDim.x / 2, ++n) {
    const NsTile tl = ns_tile<false, BN>(t, p.upd_tiles, p.upd_n);
    const int row0 = tl.i * 256 + (int)e.rank * NS_BM + e.quarter * 32;
    const int col_first = tl.j * BN;                      // alternate steps of 64 columns, as above
    const int64_t mat = (int64_t)tl.b * rows * p.ld, umat = (int64_t)tl.b * rows * cols;
    const bool skip = LAST && (p.out_mode == OUT_W_BF16 || p.out_mode == OUT_W_F32) && p.bad[tl.b] != 0;
    const int col_end = row0 >= rows ? 0 : col_first + BN < cols ? col_first + BN : cols;
    float4* blk = reinterpret_cast<float4*>(p.x32 + ns_block(tl.b, row0, col_first, rows, cols)) + lane;   // + 256 per 32 columns
    const float* diag = p.diag + (int64_t)tl.b * p.mm;
    const float row_a = TALL || row0 + lane >= rows ? 0.0f : p.a + __ldcg(diag + row0 + lane);
    float4 next[8];
    float next_a = 0.0f;                                  // TALL: of column `lane` of the step
    auto fetch = [&](int step) {
#pragma unroll
      for (int q = 0; q < 8; ++q) next[q] = __ldcg(blk + step * 256 + 32 * q);
      const int c = col_first + 32 * step + lane;
      if (TALL) next_a = c < cols ? p.a + __ldcg(diag + c) : 0.0f;
    };
    float odd = 0.0f;                                     // LAST: NaN once an x is not finite
    if (col_first + e.half * 64 < col_end) fetch(2 * e.half);
    if (!ns_tile_ready<BN>(e, bars, n)) return false;
    const uint32_t taddr = e.tmem_base + ((uint32_t)(e.quarter * 32) << 16) + (n % NsCfg<BN>::bufs) * BN;
#pragma unroll 1
    for (int step = 2 * e.half; col_first + 32 * step < col_end; step += 4) {
      if (!LAST) __syncwarp();                            // earlier read-backs of the staging buffer are done
#pragma unroll 1
      for (int h = 0; h < 2 && col_first + 32 * (step + h) < col_end; ++h) {
        const int col0 = col_first + 32 * (step + h);
        float4 x32[8];
        uint32_t v[32];
        tmem_ld32(taddr + 32 * (step + h), v);
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          auto factor = [&](int c) { return TALL ? __shfl_sync(0xffffffffu, next_a, c) : row_a; };
          x32[q].x = fmaf(factor(4 * q), next[q].x, __uint_as_float(v[4 * q]));
          x32[q].y = fmaf(factor(4 * q + 1), next[q].y, __uint_as_float(v[4 * q + 1]));
          x32[q].z = fmaf(factor(4 * q + 2), next[q].z, __uint_as_float(v[4 * q + 2]));
          x32[q].w = fmaf(factor(4 * q + 3), next[q].w, __uint_as_float(v[4 * q + 3]));
        }
        if (h == 0 ? col0 + 32 < col_end : col0 + 96 < col_end) fetch(h == 0 ? step + 1 : step + 4);
        if constexpr (!LAST) {
#pragma unroll
          for (int q = 0; q < 8; ++q) blk[(step + h) * 256 + 32 * q] = x32[q];
#pragma unroll
          for (int q = 0; q < 4; ++q)
            stage_put_piece(e.stage, lane, 4 * h + q,
                            make_uint4(pack_half(x32[2 * q].x, x32[2 * q].y), pack_half(x32[2 * q].z, x32[2 * q].w),
                                       pack_half(x32[2 * q + 1].x, x32[2 * q + 1].y), pack_half(x32[2 * q + 1].z, x32[2 * q + 1].w)));
        } else {
          uint4 piece[8];
#pragma unroll
          for (int q = 0; q < 8; ++q) {
            piece[q] = make_uint4(__float_as_uint(x32[q].x), __float_as_uint(x32[q].y), __float_as_uint(x32[q].z), __float_as_uint(x32[q].w));
            odd = fmaf(x32[q].x, 0.0f, fmaf(x32[q].y, 0.0f, fmaf(x32[q].z, 0.0f, fmaf(x32[q].w, 0.0f, odd))));
          }
          stage_put(e.stage, lane, piece);
#pragma unroll 1
          for (int i = 0; i < 8; ++i) {
            int rr, cc;
            const uint4 acc = stage_get(e.stage, lane, i, rr, cc);
            const int r = row0 + rr, c = col0 + cc * 4;
            if (r < rows && c < cols && !skip) ns_emit(p, acc, umat + (int64_t)r * cols + c, cols - c, vec);
          }
        }
      }
      if constexpr (!LAST) {
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          int r, cc;
          const uint4 val = stage_get(e.stage, lane, i, r, cc);
          const int c = col_first + 32 * step + cc * 8;
          // the pitch is a multiple of 8: whole pieces; columns past the end are never read as operands
          if (row0 + r < rows && c < cols) *reinterpret_cast<uint4*>(hi_out + mat + (int64_t)(row0 + r) * p.ld + c) = val;
        }
      }
    }
    if (LAST && odd != odd && p.d_status) atomicOr(p.d_status, SPO_DEV_NONFINITE);
    ns_tile_done<BN>(e, bars, n);
  }
  return true;
}

// All products of the iteration in one cooperative launch: 3 steps products with a grid-wide barrier after each
// (a counter in global memory; every wait is bounded).  A launch per product cost 10 to 17 us on a single
// tile, most of it launching, filling the pipeline and draining one epilogue; here it is 6.
// CTA pairs (cta_group::2) own 256 x BN tiles, BS columns for the symmetric products, BU for the update.  512: two
// products per k-step share A, which takes the L2 -> SM traffic from 64 to 48 bytes per SM and clock (64 is all there
// is: a k-block of 256 x 256 takes 1.25 times its clocks), but fills tensor memory, so every epilogue is exposed (9 us on a
// 4096 x 4096 matrix).  256 and 128: two accumulators, the epilogue runs under the next tile.
template <bool TALL, int BS, int BU>
__global__ void __launch_bounds__(NS_THREADS, 1)
ns_iterate_kernel(const __grid_constant__ NsMaps maps, const __grid_constant__ NsParams p) {
  using CS = NsCfg<BS>;
  using CU = NsCfg<BU>;
  static_assert(CS::bar_bytes + CU::bar_bytes + 16 <= NS_BARS, "barriers");
  constexpr int kTmemCols = CS::tmem_cols > CU::tmem_cols ? CS::tmem_cols : CU::tmem_cols;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t base = (raw + 1023u) & ~1023u;
  uint8_t* gen = smem_raw + (base - raw);
  const NsBars bs = ns_bars<BS>(base + NS_RING), bu = ns_bars<BU>(base + NS_RING + CS::bar_bytes);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(gen + NS_RING + CS::bar_bytes + CU::bar_bytes);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  uint32_t* warps_done = tmem_slot + 2;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank();
  const int sym_total = p.batch * p.sym_tiles, upd_total = p.batch * p.upd_tiles;
  const int products = 3 * p.steps;

  if (threadIdx.x == 0) {
    for (int s = 0; s < CS::stages; ++s) { mbar_init(bs.full0 + 8 * s, 1); mbar_init(bs.empty0 + 8 * s, 1); }
    for (int s = 0; s < CU::stages; ++s) { mbar_init(bu.full0 + 8 * s, 1); mbar_init(bu.empty0 + 8 * s, 1); }
    for (int b = 0; b < 2; ++b) {
      mbar_init(bs.tfull0 + 8 * b, 1);
      mbar_init(bu.tfull0 + 8 * b, 1);
      mbar_init(bs.tempty0 + 8 * b, 2 * NS_EPI_WARPS);
      mbar_init(bu.tempty0 + 8 * b, 2 * NS_EPI_WARPS);
    }
    *abort_flag = 0;
    *warps_done = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 0) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(kTmemCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;

  // The stages of both kinds of product share the ring, the accumulators tensor memory: between two products
  // everything is drained (the barrier comes after the last epilogue).
  if (warp == 0) {
    if (lane == 0) {
      uint32_t its = 0, itu = 0;
      for (int q = 0; q < products; ++q) {
        if (q > 0 && !ns_grid_wait(p, (uint32_t)q * gridDim.x, abort_flag)) break;
        fence_proxy_async();                        // the operands were written by plain stores
        const int k = q / 3, kind = q - 3 * k, x = k & 1;
        bool ok;
        if (kind == 0)
          ok = ns_produce<true, TALL ? OP_MN : OP_K, TALL ? OP_MN : OP_K, BS>(
              &maps.x128[x], &maps.x64[x], &maps.x128[x], &maps.x64[x], sym_total, p.sym_tiles, p.sym_n, p.kb_long, base, bs, rank,
              its, abort_flag, p.d_status);
        else if (kind == 1)
          ok = ns_produce<true, OP_SYM, OP_SYM, BS>(&maps.gram128, &maps.gram64, &maps.gram128, &maps.gram64, sym_total,
                                                    p.sym_tiles, p.sym_n, p.kb_short, base, bs, rank, its, abort_flag, p.d_status);
        else if (TALL)
          ok = ns_produce<false, OP_K, OP_SYM, BU>(&maps.x128[x], &maps.x64[x], &maps.poly128, &maps.poly64, upd_total,
                                                   p.upd_tiles, p.upd_n, p.kb_short, base, bu, rank, itu, abort_flag, p.d_status);
        else
          ok = ns_produce<false, OP_SYM, OP_MN, BU>(&maps.poly128, &maps.poly64, &maps.x128[x], &maps.x64[x], upd_total,
                                                    p.upd_tiles, p.upd_n, p.kb_short, base, bu, rank, itu, abort_flag, p.d_status);
        if (!ok) break;
      }
    }
  } else if (warp == 1) {
    if (lane == 0 && rank == 0) {
      uint32_t its = 0, itu = 0, ns = 0, nu = 0;
      for (int q = 0; q < products; ++q) {
        const int kind = q % 3;
        bool ok;
        if (kind == 0)
          ok = ns_multiply<true, TALL ? OP_MN : OP_K, TALL ? OP_MN : OP_K, BS>(sym_total, p.sym_tiles, p.sym_n, p.kb_long, base,
                                                                               tmem_base, bs, its, ns, abort_flag, p.d_status);
        else if (kind == 1)
          ok = ns_multiply<true, OP_SYM, OP_SYM, BS>(sym_total, p.sym_tiles, p.sym_n, p.kb_short, base, tmem_base, bs, its, ns,
                                                     abort_flag, p.d_status);
        else
          ok = ns_multiply<false, TALL ? OP_K : OP_SYM, TALL ? OP_SYM : OP_MN, BU>(upd_total, p.upd_tiles, p.upd_n, p.kb_short,
                                                                                   base, tmem_base, bu, itu, nu, abort_flag,
                                                                                   p.d_status);
        if (!ok) break;
      }
    }
  } else {
    NsEpi e;
    e.tmem_base = tmem_base; e.rank = rank;
    e.stage = gen + NS_RING + NS_BARS + (warp - 2) * NS_STAGING;
    e.quarter = warp & 3; e.half = (warp - 2) >> 2; e.lane = lane;
    e.abort_flag = abort_flag; e.d_status = p.d_status;
    uint32_t ns = 0, nu = 0;
    for (int q = 0; q < products; ++q) {
      if (q > 0) {
        int good = 1;
        if (lane == 0) good = ns_grid_wait(p, (uint32_t)q * gridDim.x, abort_flag) ? 1 : 0;
        if (!__shfl_sync(0xffffffffu, good, 0)) break;
      }
      const int k = q / 3, kind = q - 3 * k;
      bool ok;
      if (kind == 0)
        ok = ns_store_sym<BS, false>(e, bs, p, sym_total, p.gram, p.inv_s2, 0.0f, ns);
      else if (kind == 1)
        ok = ns_store_sym<BS, true>(e, bs, p, sym_total, p.poly, p.c, p.b, ns);
      else if (k < p.steps - 1)
        ok = ns_store_update<TALL, BU, false>(e, bu, p, upd_total, p.hi[(k + 1) & 1], nu);
      else
        ok = ns_store_update<TALL, BU, true>(e, bu, p, upd_total, nullptr, nu);
      if (!ok) break;
      if (q + 1 < products) {                       // this CTA's part of the product is in memory: count it
        // (no barrier among the warps: one that gave up must not leave the others waiting)
        fence_proxy_async();
        __syncwarp();
        if (lane == 0) {
          __threadfence();
          if (atomicAdd(warps_done, 1u) % NS_EPI_WARPS == NS_EPI_WARPS - 1)
            asm volatile("red.release.gpu.global.add.u32 [%0], 1;" ::"l"(p.arrivals) : "memory");
        }
      }
    }
  }

  __syncwarp();
  if (*abort_flag) {                       // let copies still in flight land before the CTA retires
    for (int i = 0; i < 200; ++i) __nanosleep(1000);
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();
  if (warp == 0)
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(kTmemCols) : "memory");
}

// ---------------------------------------------------------------------------
// The pass in front: U = G, or with momentum M' = mu M + G and U = G + mu M' (Nesterov) or M'.
// ---------------------------------------------------------------------------
struct NsInput {
  const void* G;
  int g_bf16;
  float* momentum;                         // NULL: U = G
  float mu;
  int nesterov;
  int64_t m, n, ld;                        // ld: pitch of hi
  int blocks;                              // blocks (and norm partials) per matrix
  double* partials;                        // [batch][blocks]
  float eps, scale;
  __half* hi;
  float* x32;
  int32_t *bad, *d_status;
  uint32_t* arrivals;                      // the iteration's barrier counter, zeroed here
};

__device__ __forceinline__ float ns_load(const NsInput& p, int64_t at) {
  return p.g_bf16 ? __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(p.G)[at])
                  : reinterpret_cast<const float*>(p.G)[at];
}
__device__ __forceinline__ void ns_load4(const NsInput& p, int64_t at, float (&g)[4]) {
  if (p.g_bf16) {
    const uint2 q = *reinterpret_cast<const uint2*>(reinterpret_cast<const __nv_bfloat16*>(p.G) + at);
    g[0] = __uint_as_float(q.x << 16); g[1] = __uint_as_float(q.x & 0xFFFF0000u);
    g[2] = __uint_as_float(q.y << 16); g[3] = __uint_as_float(q.y & 0xFFFF0000u);
  } else {
    const float4 q = *reinterpret_cast<const float4*>(reinterpret_cast<const float*>(p.G) + at);
    g[0] = q.x; g[1] = q.y; g[2] = q.z; g[3] = q.w;
  }
}
__device__ __forceinline__ float ns_momentum(const NsInput& p, float g, float m, float* m_new) {
  *m_new = fmaf(p.mu, m, g);
  return p.nesterov ? fmaf(p.mu, *m_new, g) : *m_new;
}

// Sum of squares of U, one partial per block: fixed order, so the same bits every time.
__global__ void __launch_bounds__(256)
ns_norm_kernel(const NsInput p) {
  const int64_t count = p.m * p.n, mat = (int64_t)blockIdx.y * count;
  double acc = 0.0;
  if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *p.arrivals = 0;
  if ((count & 3) == 0) {
    for (int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4; i < count; i += (int64_t)p.blocks * 1024) {
      float g[4], u[4];
      ns_load4(p, mat + i, g);
      if (p.momentum) {
        const float4 q = *reinterpret_cast<const float4*>(p.momentum + mat + i);
        const float mo[4] = {q.x, q.y, q.z, q.w};
        float mn;
#pragma unroll
        for (int k = 0; k < 4; ++k) u[k] = ns_momentum(p, g[k], mo[k], &mn);
      } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) u[k] = g[k];
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) acc += (double)u[k] * (double)u[k];
    }
  } else {
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < count; i += (int64_t)p.blocks * 256) {
      float u = ns_load(p, mat + i), mn;
      if (p.momentum) u = ns_momentum(p, u, p.momentum[mat + i], &mn);
      acc += (double)u * (double)u;
    }
  }
  __shared__ double s[8];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) acc += __shfl_xor_sync(0xffffffffu, acc, o);
  if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = acc;
  __syncthreads();
  if (threadIdx.x == 0) {
    double tot = 0.0;
    for (int w = 0; w < 8; ++w) tot += s[w];
    p.partials[(int64_t)blockIdx.y * p.blocks + blockIdx.x] = tot;
  }
}

// Momentum, and U / (|U|_F + eps) times the scale, in fp32 blocks and fp16 rows.
__global__ void __launch_bounds__(256)
ns_split_kernel(const NsInput p) {
  const int64_t count = p.m * p.n, mat = (int64_t)blockIdx.y * count, xmat = (int64_t)blockIdx.y * p.m * p.ld;
  __shared__ double s[8];
  double acc = 0.0;
  for (int i = threadIdx.x; i < p.blocks; i += 256) acc += p.partials[(int64_t)blockIdx.y * p.blocks + i];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) acc += __shfl_xor_sync(0xffffffffu, acc, o);
  if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = acc;
  __syncthreads();
  double tot = 0.0;
#pragma unroll
  for (int w = 0; w < 8; ++w) tot += s[w];
  const bool bad = !(tot < (double)CUDART_INF);
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    p.bad[blockIdx.y] = bad;
    if (bad && p.d_status) atomicOr(p.d_status, SPO_DEV_NONFINITE);
  }
  // scale / (|U|_F + eps) may be past fp32's range (a zero matrix with a tiny eps), or so small that fp32 has few bits left:
  // multiplied in two steps then, the second an exact power of two (1 otherwise), U f up being at most the scale.
  double factor = bad ? 0.0 : (double)p.scale / (sqrt(tot) + (double)p.eps);
  float up = 1.0f;
  if (factor > 0x1p100) { factor *= 0x1p-64; up = 0x1p64f; }
  else if (factor < 0x1p-100) { factor *= 0x1p64; up = 0x1p-64f; }
  const float f = (float)factor;
  const int64_t cbs = (p.n + 31) >> 5, tasks = ((p.m + 31) >> 5) * cbs;
  const int lane = threadIdx.x & 31;
  const bool quads = (p.n & 3) == 0;
  for (int64_t task = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); task < tasks; task += (int64_t)gridDim.x * 8) {
    const int64_t rb = task / cbs, c0 = (task - rb * cbs) * 32;
    float* blk = p.x32 + ((int64_t)blockIdx.y * tasks + task) * 1024;
    if (quads) {
      // a warp takes a block of 32 x 32: eight lanes a row, four rows an access
      const int64_t c = c0 + (lane & 7) * 4;
#pragma unroll 4
      for (int i = 0; i < 8; ++i) {
        const int rr = 4 * i + (lane >> 3);
        const int64_t r = rb * 32 + rr, at = mat + r * p.n + c;
        float u[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        if (r < p.m && c < p.n && !bad) {
          ns_load4(p, at, u);
          if (p.momentum) {
            float4* mp = reinterpret_cast<float4*>(p.momentum + at);
            const float4 q = *mp;
            const float mo[4] = {q.x, q.y, q.z, q.w};
            float mn[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) u[k] = ns_momentum(p, u[k], mo[k], &mn[k]);
            *mp = make_float4(mn[0], mn[1], mn[2], mn[3]);
          }
#pragma unroll
          for (int k = 0; k < 4; ++k) u[k] = u[k] * f * up;
        }
        *reinterpret_cast<float4*>(blk + (lane & 7) * 128 + rr * 4) = make_float4(u[0], u[1], u[2], u[3]);
        if (r < p.m && c < p.n)                           // the pitch is a multiple of 8: whole pieces
          *reinterpret_cast<uint2*>(p.hi + xmat + r * p.ld + c) = make_uint2(pack_half(u[0], u[1]), pack_half(u[2], u[3]));
      }
    } else {
      // rows that do not begin on 16 bytes: a lane a column, a row an access
      const int64_t c = c0 + lane;
#pragma unroll 8
      for (int rr = 0; rr < 32; ++rr) {
        const int64_t r = rb * 32 + rr, at = mat + r * p.n + c;
        float u = 0.0f;
        if (r < p.m && c < p.n && !bad) {
          u = ns_load(p, at);
          if (p.momentum) {
            float mn;
            u = ns_momentum(p, u, p.momentum[at], &mn);
            p.momentum[at] = mn;
          }
          u = u * f * up;
        }
        blk[(lane >> 2) * 128 + rr * 4 + (lane & 3)] = u;
        if (r < p.m && c < p.n) p.hi[xmat + r * p.ld + c] = __float2half_rn(u);
      }
    }
  }
}

// ---------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------
struct NsWs { size_t hi[2], x32, gram, gram_blk, poly, diag, partials, bad, arrivals, total; int64_t ld, mm, gld; int blocks; };

constexpr int kNormBlocks = 592;

NsWs ns_layout(int64_t m, int64_t n, int64_t batch) {
  NsWs L{};
  L.ld = (n + 63) / 64 * 64;                  // rows begin on 128 bytes: a row of a TMA box is one line, not parts of two
  L.mm = m < n ? m : n;
  L.gld = (L.mm + 63) / 64 * 64;
  const int64_t want = ceil_div(m * n, 4096);
  L.blocks = (int)(want < kNormBlocks ? want : kNormBlocks);
  const size_t x = (size_t)batch * m * L.ld * 2, g = (size_t)batch * L.mm * L.gld * 2;
  size_t off = 0;
  for (int i = 0; i < 2; ++i) { L.hi[i] = off; off = align_up(off + x, 256); }
  L.x32 = off;      off = align_up(off + (size_t)batch * ceil_div(m, 32) * ceil_div(n, 32) * 4096, 256);
  L.gram = off;     off = align_up(off + g, 256);
  L.gram_blk = off; off = align_up(off + (size_t)batch * ceil_div(L.mm, 32) * ceil_div(L.mm, 32) * 2048, 256);
  L.poly = off;     off = align_up(off + g, 256);
  L.diag = off;     off = align_up(off + (size_t)batch * L.mm * 4, 256);
  L.partials = off; off = align_up(off + (size_t)batch * L.blocks * 8, 256);
  L.bad = off;      off = align_up(off + (size_t)batch * 4, 256);
  L.arrivals = off; off = align_up(off + 4, 256);
  L.total = off;
  return L;
}

// fp16 [batch][rows][cols] with row pitch ld; box {64, box_rows, 1}, 128-byte swizzle, zeros outside
bool make_map3(CUtensorMap* m, const void* ptr, int64_t cols, int64_t rows, int64_t batch, int64_t ld, uint32_t box_rows) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return false;
  cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)batch};
  cuuint64_t strides[2] = {(cuuint64_t)ld * 2, (cuuint64_t)rows * ld * 2};
  cuuint32_t box[3] = {64, box_rows, 1};
  cuuint32_t estr[3] = {1, 1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, const_cast<void*>(ptr), dims, strides, box, estr,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// CTA pairs of an instantiation that can be resident together (0 = not yet asked); one slot per device.
template <bool TALL, int BS, int BU>
cudaError_t ns_resident(int* out) {
  static std::atomic<int> cached[64];
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
  int n = cached[dev].load(std::memory_order_acquire);
  if (n == 0) {
    auto kern = ns_iterate_kernel<TALL, BS, BU>;
    e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, NS_SMEM);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t q = {};
    q.gridDim = dim3((unsigned)(sm_count() / 2 * 2), 1, 1);
    q.blockDim = dim3(NS_THREADS, 1, 1);
    q.dynamicSmemBytes = NS_SMEM;
    cudaLaunchAttribute qa[1];
    qa[0].id = cudaLaunchAttributeClusterDimension;
    qa[0].val.clusterDim.x = 2;
    qa[0].val.clusterDim.y = 1;
    qa[0].val.clusterDim.z = 1;
    q.attrs = qa;
    q.numAttrs = 1;
    e = cudaOccupancyMaxActiveClusters(&n, kern, &q);
    if (e != cudaSuccess) return e;
    if (n < 1) return cudaErrorLaunchOutOfResources;
    if (n > sm_count() / 2) n = sm_count() / 2;
    cached[dev].store(n, std::memory_order_release);
  }
  *out = n;
  return cudaSuccess;
}

int64_t sym_tile_count(int64_t mm, int bn) {
  const int64_t mt = ceil_div(mm, 256), nt = ceil_div(mm, bn);
  int64_t tiles = 0;
  for (int64_t i = 0; i < mt; ++i) tiles += nt - i * 256 / bn;
  return tiles;
}

template <bool TALL, int BS, int BU>
cudaError_t launch_iterate_t(const NsMaps& maps, NsParams p, cudaStream_t st) {
  int pairs = 0;
  cudaError_t e = ns_resident<TALL, BS, BU>(&pairs);
  if (e != cudaSuccess) return e;
  const int64_t sym = sym_tile_count(p.mm, BS), un = ceil_div(p.n, BU), upd = ceil_div(p.m, 256) * un;
  const int64_t most = (sym > upd ? sym : upd) * p.batch;
  if (most > 0x7FFFFFFF) return cudaErrorInvalidValue;
  p.sym_tiles = (int)sym; p.sym_n = (int)ceil_div(p.mm, BS);
  p.upd_tiles = (int)upd; p.upd_n = (int)un;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(2 * (most < pairs ? most : pairs)), 1, 1);
  cfg.blockDim = dim3(NS_THREADS, 1, 1);
  cfg.dynamicSmemBytes = NS_SMEM;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = 2;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeCooperative;               // all CTAs resident, or the launch fails
  attr[1].val.cooperative = 1;
  cfg.attrs = attr;
  cfg.numAttrs = most > 1 ? 2 : 1;                           // (the CTAs of a single pair, a cluster, always are)
  return cudaLaunchKernelEx(&cfg, ns_iterate_kernel<TALL, BS, BU>, maps, p);
}

template <int BS, int BU>
cudaError_t launch_iterate(const NsMaps& maps, const NsParams& p, cudaStream_t st) {
  return p.tall ? launch_iterate_t<true, BS, BU>(maps, p, st) : launch_iterate_t<false, BS, BU>(maps, p, st);
}

// Column widths of the tiles.  128 instead of 256 where that takes no more rounds over the pairs: more pairs have work and an
// epilogue is shorter (us; symmetric products 128 against 256 columns, update 256: 512 x 2048 179 / 193, 1000 x 2730 240 / 254, 2048 x 2048
// 291 / 298; update 128 against 256, symmetric 128: 128 x 512 104 / 116, 512 x 2048 169 / 179, 3 x 4000 x 300 248 / 271).  With one
// round more they lose by what their operands cost in traffic (symmetric: 16 x 1024 x 1024 718 / 593, 4 x 1000 x 2730 514 / 436,
// 80 x 2056 x 130 863 / 803; update: 1000 x 2730 265 / 240, 2 x 1500 x 1500 298 / 271, 2048 x 2048 334 / 291).
int64_t rounds_of(int64_t tiles) { return ceil_div(tiles, sm_count() / 2); }
bool narrow_symmetric(const NsParams& p) {
  return rounds_of(sym_tile_count(p.mm, 128) * p.batch) <= rounds_of(sym_tile_count(p.mm, 256) * p.batch);
}
bool narrow_update(const NsParams& p) {
  const int64_t rows = ceil_div(p.m, 256) * p.batch;
  return rounds_of(rows * ceil_div(p.n, 128)) <= rounds_of(rows * ceil_div(p.n, 256));
}
// 512 or 256 for the other symmetric products: rounds of tiles x k-blocks x the nanoseconds of a k-block (610 and 380: 1.0 and
// 1.25 times the clocks of its products, the narrower one waiting for L2) and the exposed epilogues, one a round for 512, the
// last one for 256.  An ordering, not a time: barriers, fills and fences are left out.  512 against 256: 4096 x 4096 1217 and
// 1352 us, 12 x 1000 x 2600 905 / 993; 4 x 1000 x 2730 529 / 436, 16 x 1024 x 1024 688 / 593, 2048 x 8192 930 / 715.
double sym_time(const NsParams& p, int bn) {
  const double pairs = sm_count() / 2, rounds = ceil((double)sym_tile_count(p.mm, bn) * p.batch / pairs);
  const double kb = p.kb_long + p.kb_short;
  return bn == 512 ? rounds * (kb * 610.0 + 2 * 9000.0) : rounds * kb * 380.0 + 2 * 5000.0;
}

}  // namespace

size_t muon_ws_bytes(int64_t m, int64_t n, int64_t batch) { return ns_layout(m, n, batch).total; }

cudaError_t muon_run(const MuonArgs& a, char* ws, cudaStream_t st) {
  if (a.batch == 0) return cudaSuccess;
  const NsWs L = ns_layout(a.m, a.n, a.batch);
  const spo_muon_params& pr = *a.params;
  NsInput in{};
  in.G = a.G; in.g_bf16 = a.G_dtype == SPO_DTYPE_BF16;
  in.momentum = a.momentum; in.mu = pr.momentum; in.nesterov = pr.nesterov;
  in.m = a.m; in.n = a.n; in.ld = L.ld; in.blocks = L.blocks;
  in.partials = reinterpret_cast<double*>(ws + L.partials);
  in.eps = pr.eps;
  const int64_t longer = a.m > a.n ? a.m : a.n;
  int ex = 0;                                                    // s = 2^ex, ex = round(log2 sqrt(longer))
  while (ex < 14 && ((int64_t)1 << (2 * ex + 1)) < longer) ++ex;
  const float s = (float)(1 << ex);
  in.scale = s;
  in.hi = reinterpret_cast<__half*>(ws + L.hi[0]);
  in.x32 = reinterpret_cast<float*>(ws + L.x32);
  in.bad = reinterpret_cast<int32_t*>(ws + L.bad);
  in.d_status = a.d_status;
  in.arrivals = reinterpret_cast<uint32_t*>(ws + L.arrivals);
  const dim3 grid((unsigned)L.blocks, (unsigned)a.batch);
  ns_norm_kernel<<<grid, 256, 0, st>>>(in);
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  ns_split_kernel<<<grid, 256, 0, st>>>(in);
  if ((e = cudaGetLastError()) != cudaSuccess) return e;

  NsParams p{};
  p.batch = a.batch; p.steps = pr.steps; p.tall = a.m > a.n;
  p.m = (int)a.m; p.n = (int)a.n; p.mm = (int)L.mm;
  p.ld = L.ld; p.gld = L.gld;
  p.kb_long = (int)ceil_div(longer, 64); p.kb_short = (int)ceil_div(L.mm, 64);
  p.hi[0] = in.hi; p.hi[1] = reinterpret_cast<__half*>(ws + L.hi[1]);
  p.x32 = in.x32;
  p.gram_blk = reinterpret_cast<__half*>(ws + L.gram_blk);
  p.gram = reinterpret_cast<__half*>(ws + L.gram);
  p.poly = reinterpret_cast<__half*>(ws + L.poly);
  p.diag = reinterpret_cast<float*>(ws + L.diag);
  p.inv_s2 = 1.0f / (s * s);
  p.a = pr.coef_a; p.b = pr.coef_b; p.c = pr.coef_c;
  p.out = a.out;
  p.bad = in.bad;
  p.arrivals = in.arrivals;
  p.d_status = a.d_status;
  if (a.update) {
    p.out_mode = a.out_dtype == SPO_DTYPE_BF16 ? OUT_W_BF16 : OUT_W_F32;
    p.out_scale = pr.lr * a.update_scale / s;
    p.decay = 1.0f - pr.lr * pr.weight_decay;
  } else {
    p.out_mode = a.out_dtype == SPO_DTYPE_BF16 ? OUT_BF16 : OUT_F32;
    p.out_scale = 1.0f / s;
  }
  NsMaps maps;
  for (int x = 0; x < 2; ++x)
    if (!make_map3(&maps.x128[x], p.hi[x], a.n, a.m, a.batch, L.ld, 128) ||
        !make_map3(&maps.x64[x], p.hi[x], a.n, a.m, a.batch, L.ld, 64))
      return cudaErrorInvalidValue;
  if (!make_map3(&maps.gram128, p.gram, L.mm, L.mm, a.batch, L.gld, 128) ||
      !make_map3(&maps.gram64, p.gram, L.mm, L.mm, a.batch, L.gld, 64) ||
      !make_map3(&maps.poly128, p.poly, L.mm, L.mm, a.batch, L.gld, 128) ||
      !make_map3(&maps.poly64, p.poly, L.mm, L.mm, a.batch, L.gld, 64))
    return cudaErrorInvalidValue;
  // (Where the update is narrow and the symmetric products are not, these are one round of 256 columns, and 512 never less: the
  // update has as many tiles at least, and for two rounds of 256 to hold the 128-column ones too there have to be few of them.)
  const bool narrow = narrow_update(p);
  if (narrow_symmetric(p)) return narrow ? launch_iterate<128, 128>(maps, p, st) : launch_iterate<128, 256>(maps, p, st);
  if (narrow) return launch_iterate<256, 128>(maps, p, st);
  if (sym_time(p, 512) < sym_time(p, 256)) return launch_iterate<512, 256>(maps, p, st);
  return launch_iterate<256, 256>(maps, p, st);
}

}  // namespace spo
