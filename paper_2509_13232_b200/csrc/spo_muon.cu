// Orthogonalised weight updates (spo_orthogonalize, spo_muon_update): Newton-Schulz iteration
//   X <- a X + (b A + c A A) X,   A = X X^T,   X_0 = U / (|U|_F + eps)
// on the tensor cores, with momentum in front and the weight update behind it in the same call.
// (Taller than wide: A = X^T X and X <- a X + X (b A + c A A), so the square products are over the smaller side
// and nothing is ever transposed.)
//
// Numbers.  The iteration multiplies small singular values by a per step (a^5 = 485), and with them
// every rounding made in X while they are small.  So X is held as a pair of fp16 numbers, hi + lo
// (22 bits), times s = 2^round(log2 sqrt(max(m, n))), which puts the entries of an orthogonal matrix near one: the
// term a X is formed from the pair in fp32, and only hi enters the products, whose spectrum is small where X's
// is.  Measured against 64 bits for a 512 x 512 update of rank 16 under no noise: pair 4e-4, fp16 without lo
// 4e-2, bf16 0.33 (a full-rank Gaussian: 1.5e-3, 1.3e-3, 1.1e-2).  fp16 rather than bf16 because everything
// here is bounded by about 10 in magnitude and fp16 has 8 times finer steps.  A and b A + c A A are rounded
// to fp16 once each; all sums are fp32.
//
// Work.  A and A A are symmetric: only the tiles on and above the diagonal are computed and stored twice,
// 3 m^2 n + m^3 operations a step for m <= n instead of 4 m^2 n + 2 m^3.  Five steps of a 4096 x 4096
// matrix are 1.37 TFLOP: tensor-bound from a few hundred rows on, launch-bound below.
#include <cuda.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
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

template <int BN>
struct NsCfg {
  static constexpr int a_bytes = NS_BM * 64 * 2;
  static constexpr int b_bytes = BN / 2 * 64 * 2;
  static constexpr int stage_bytes = a_bytes + b_bytes;
  static constexpr int stages = 192 * 1024 / stage_bytes;
  static constexpr int smem = stages * stage_bytes + 1024 + 256 + NS_EPI_WARPS * NS_STAGING;
  static constexpr int tmem_cols = 2 * BN;
};

enum : int { OUT_PAIR = 0, OUT_BF16 = 1, OUT_F32 = 2, OUT_W_BF16 = 3, OUT_W_F32 = 4 };

struct NsParams {
  int batch, m_tiles, n_tiles, tiles;          // tiles per matrix (symmetric product: on and above the diagonal)
  int k_blocks;
  int rows, cols;                              // of the result
  // symmetric product: S = alpha acc + beta Cin (fp16, pitch ld, both triangles)
  __half* S;
  const __half* Cin;
  int64_t ld;
  float alpha, beta;
  // update: x = a (hi + lo) + acc
  const __half* hi;
  __half *lo, *hi_out;
  float a;
  int out_mode;
  void* out;                                   // result or weights, pitch cols
  float out_scale, decay;                      // result: x out_scale;  weights: w decay - x out_scale
  const int32_t* bad;                          // [batch]: the matrix held a NaN or an infinity: leave its weights alone
  int32_t* d_status;
};

__device__ __forceinline__ void tma_load_3d_pair(uint32_t dst, const CUtensorMap* map, int c0, int c1, int c2, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
      ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(c0), "r"(c1), "r"(c2), "r"(bar)
      : "memory");
}

__device__ __forceinline__ uint32_t pack_half(float lo, float hi) {
  const __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}

struct NsTile { int b, i, j; };
// Tile `t` of the launch: row tile i, column tile j of matrix b.  SYM: row i has the column tiles
// from the diagonal on (R = 256 / BN column tiles per row tile).
template <bool SYM, int BN>
__device__ __forceinline__ NsTile ns_tile(int t, const NsParams& p) {
  NsTile r;
  r.b = t / p.tiles;
  int q = t - r.b * p.tiles;
  if (SYM) {
    constexpr int R = 256 / BN;
    int i = 0;
    while (q >= p.n_tiles - R * i) { q -= p.n_tiles - R * i; ++i; }
    r.i = i;
    r.j = R * i + q;
  } else {
    r.i = q / p.n_tiles;
    r.j = q - r.i * p.n_tiles;
  }
  return r;
}

// One product of the iteration.  CTA pairs (cta_group::2) own 256 x BN tiles; two accumulators in tensor
// memory, so that a tile's epilogue runs under the next tile's products.  A_MN / B_MN: the operand is stored
// with the M / N index contiguous.
template <bool SYM, bool A_MN, bool B_MN, int BN>
__global__ void __launch_bounds__(NS_THREADS, 1)
ns_gemm_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB, const NsParams p) {
  using C = NsCfg<BN>;
  constexpr int S = C::stages;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t base = (raw + 1023u) & ~1023u;
  uint8_t* gen = smem_raw + (base - raw);
  const uint32_t bars = base + S * C::stage_bytes;
  const uint32_t full0 = bars, empty0 = bars + 8 * S, tfull0 = bars + 16 * S, tempty0 = tfull0 + 16;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(gen + S * C::stage_bytes + 16 * S + 32);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank();
  const int group = blockIdx.x / 2, n_groups = gridDim.x / 2;
  const int total = p.batch * p.tiles;

  if (threadIdx.x == 0) {
    for (int s = 0; s < S; ++s) { mbar_init(full0 + 8 * s, 1); mbar_init(empty0 + 8 * s, 1); }
    for (int b = 0; b < 2; ++b) { mbar_init(tfull0 + 8 * b, 1); mbar_init(tempty0 + 8 * b, 2 * NS_EPI_WARPS); }
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 0) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(C::tmem_cols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;

  if (warp == 0) {
    if (lane == 0) {
      uint32_t it = 0;
      bool ok = true;
      for (int t = group; t < total && ok; t += n_groups) {
        const NsTile tl = ns_tile<SYM, BN>(t, p);
        const int row = tl.i * 256 + (int)rank * NS_BM, col = tl.j * BN + (int)rank * (BN / 2);
        for (int kb = 0; kb < p.k_blocks; ++kb, ++it) {
          const uint32_t s = it % S, ph = (it / S) & 1u;
          if (!mbar_wait<20>(empty0 + 8 * s, ph ^ 1u, abort_flag, p.d_status)) { ok = false; break; }
          const uint32_t sa = base + s * C::stage_bytes, sb = sa + C::a_bytes;
          if (rank == 0) mbar_expect_tx(full0 + 8 * s, 2 * C::stage_bytes);
          const uint32_t fb = map_to_cta(full0 + 8 * s, 0);
          if (!A_MN) {
            tma_load_3d_pair(sa, &tmA, kb * 64, row, tl.b, fb);
          } else {
#pragma unroll
            for (int x = 0; x < NS_BM / 64; ++x) tma_load_3d_pair(sa + x * 8192, &tmA, row + x * 64, kb * 64, tl.b, fb);
          }
          if (!B_MN) {
            tma_load_3d_pair(sb, &tmB, kb * 64, col, tl.b, fb);
          } else {
#pragma unroll
            for (int x = 0; x < BN / 128; ++x) tma_load_3d_pair(sb + x * 8192, &tmB, col + x * 64, kb * 64, tl.b, fb);
          }
        }
      }
    }
  } else if (warp == 1) {
    if (lane == 0 && rank == 0) {
      // fp32 accumulate, fp16 A and B, M = 256 over the pair, N = BN
      constexpr uint32_t idesc = (1u << 4) | ((A_MN ? 1u : 0u) << 15) | ((B_MN ? 1u : 0u) << 16) |
                                 ((uint32_t)(BN >> 3) << 17) | (16u << 24);
      uint32_t it = 0, n = 0;
      bool ok = true;
      for (int t = group; t < total && ok; t += n_groups, ++n) {
        const uint32_t b = n & 1u;
        if (!mbar_wait(tempty0 + 8 * b, ((n >> 1) & 1u) ^ 1u, abort_flag, p.d_status)) { ok = false; break; }
        tc_fence_after();
        for (int kb = 0; kb < p.k_blocks; ++kb, ++it) {
          const uint32_t s = it % S, ph = (it / S) & 1u;
          if (!mbar_wait(full0 + 8 * s, ph, abort_flag, p.d_status)) { ok = false; break; }
          tc_fence_after();
          const uint32_t sa = base + s * C::stage_bytes, sb = sa + C::a_bytes;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const uint64_t da = A_MN ? smem_desc(sa + j * 2048, 8192, 1024) : smem_desc(sa + j * 32, 16, 1024);
            const uint64_t db = B_MN ? smem_desc(sb + j * 2048, 8192, 1024) : smem_desc(sb + j * 32, 16, 1024);
            umma_bf16(tmem_base + b * BN, da, db, idesc, (kb | j) != 0 ? 1u : 0u);
          }
          umma_commit(empty0 + 8 * s);
        }
        if (ok) umma_commit(tfull0 + 8 * b);
      }
    }
  } else {
    const int quarter = warp & 3, half = (warp - 2) >> 2;
    uint8_t* stage = gen + S * C::stage_bytes + 256 + (warp - 2) * NS_STAGING;
    uint32_t n = 0;
    for (int t = group; t < total; t += n_groups, ++n) {
      const NsTile tl = ns_tile<SYM, BN>(t, p);
      const uint32_t b = n & 1u;
      int good = 1;
      if (lane == 0) good = mbar_wait<20>(tfull0 + 8 * b, (n >> 1) & 1u, abort_flag, p.d_status) ? 1 : 0;
      good = __shfl_sync(0xffffffffu, good, 0);
      if (!good) break;
      tc_fence_after();
      const int row0 = tl.i * 256 + (int)rank * NS_BM + quarter * 32;      // result row of the warp's lane 0
      const int row = row0 + lane;
      const int col_first = tl.j * BN + half * (BN / 2);
      const uint32_t taddr = tmem_base + ((uint32_t)(quarter * 32) << 16) + b * BN + half * (BN / 2);
      if (SYM) {
        const int64_t mat = (int64_t)tl.b * p.rows * p.ld;
        const bool mirror = tl.j >= (256 / BN) * (tl.i + 1);                // the diagonal block is computed whole
#pragma unroll 1
        for (int r2 = 0; r2 < BN / 2; r2 += 64) {
          const int col0 = col_first + r2;
          if (col0 >= p.cols) break;
          uint4 piece[8];
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const int c0 = col0 + h * 32;
            float cin[32];
            // Cin is symmetric: its element (row, c) is read from (c, row), 32 consecutive rows per access
            if (p.Cin) {
#pragma unroll
              for (int j = 0; j < 32; ++j)
                cin[j] = row < p.rows && c0 + j < p.cols ? __half2float(p.Cin[mat + (int64_t)(c0 + j) * p.ld + row]) : 0.0f;
            }
            uint32_t v[32];
            tmem_ld32(taddr + r2 + h * 32, v);
            uint32_t o[16];
#pragma unroll
            for (int j = 0; j < 32; ++j) {
              float x = p.alpha * __uint_as_float(v[j]);
              if (p.Cin) x = fmaf(p.beta, cin[j], x);
              v[j] = __float_as_uint(x);
            }
#pragma unroll
            for (int j = 0; j < 16; ++j) o[j] = pack_half(__uint_as_float(v[2 * j]), __uint_as_float(v[2 * j + 1]));
            if (mirror && row < p.rows) {
#pragma unroll
              for (int j = 0; j < 32; ++j)
                if (c0 + j < p.cols)
                  reinterpret_cast<uint16_t*>(p.S)[mat + (int64_t)(c0 + j) * p.ld + row] =
                      (uint16_t)((j & 1) ? o[j >> 1] >> 16 : o[j >> 1] & 0xFFFFu);
            }
#pragma unroll
            for (int q = 0; q < 4; ++q) piece[4 * h + q] = make_uint4(o[4 * q], o[4 * q + 1], o[4 * q + 2], o[4 * q + 3]);
          }
          stage_put(stage, lane, piece);
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            int r, cc;
            const uint4 val = stage_get(stage, lane, i, r, cc);
            const int c = col0 + cc * 8;
            // the pitch is a multiple of 8, so a piece that begins inside the row may be stored whole
            if (row0 + r < p.rows && c < p.cols) *reinterpret_cast<uint4*>(p.S + mat + (int64_t)(row0 + r) * p.ld + c) = val;
          }
        }
      } else {
        const int64_t mat = (int64_t)tl.b * p.rows * p.ld, umat = (int64_t)tl.b * p.rows * p.cols;
        const bool vec = (p.cols & 3) == 0;
        const bool skip = p.bad != nullptr && p.bad[tl.b] != 0;
#pragma unroll 1
        for (int ch = 0; ch < BN / 2; ch += 32) {
          const int col0 = col_first + ch;
          if (col0 >= p.cols) break;
          uint2 xh[8], xl[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const int r = row0 + 4 * i + (lane >> 3), c = col0 + (lane & 7) * 4;
            xh[i] = xl[i] = make_uint2(0u, 0u);
            if (r < p.rows && c < p.cols) {
              xh[i] = *reinterpret_cast<const uint2*>(p.hi + mat + (int64_t)r * p.ld + c);
              xl[i] = *reinterpret_cast<const uint2*>(p.lo + mat + (int64_t)r * p.ld + c);
            }
          }
          uint32_t v[32];
          tmem_ld32(taddr + ch, v);
          uint4 piece[8];
#pragma unroll
          for (int q = 0; q < 8; ++q) piece[q] = make_uint4(v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]);
          stage_put(stage, lane, piece);
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            int rr, cc;
            const uint4 acc = stage_get(stage, lane, i, rr, cc);
            const int r = row0 + rr, c = col0 + cc * 4;
            if (r >= p.rows || c >= p.cols) continue;
            float x[4] = {__uint_as_float(acc.x), __uint_as_float(acc.y), __uint_as_float(acc.z), __uint_as_float(acc.w)};
            const float2 h0 = __half22float2(*reinterpret_cast<const __half2*>(&xh[i].x)),
                         h1 = __half22float2(*reinterpret_cast<const __half2*>(&xh[i].y)),
                         l0 = __half22float2(*reinterpret_cast<const __half2*>(&xl[i].x)),
                         l1 = __half22float2(*reinterpret_cast<const __half2*>(&xl[i].y));
            x[0] = fmaf(p.a, h0.x + l0.x, x[0]);
            x[1] = fmaf(p.a, h0.y + l0.y, x[1]);
            x[2] = fmaf(p.a, h1.x + l1.x, x[2]);
            x[3] = fmaf(p.a, h1.y + l1.y, x[3]);
            if (p.out_mode == OUT_PAIR) {
              // pitch a multiple of 8: whole pieces; columns past the end are never read as operands
              const uint2 hh = make_uint2(pack_half(x[0], x[1]), pack_half(x[2], x[3]));
              const float2 g0 = __half22float2(*reinterpret_cast<const __half2*>(&hh.x)),
                           g1 = __half22float2(*reinterpret_cast<const __half2*>(&hh.y));
              *reinterpret_cast<uint2*>(p.hi_out + mat + (int64_t)r * p.ld + c) = hh;
              *reinterpret_cast<uint2*>(p.lo + mat + (int64_t)r * p.ld + c) =
                  make_uint2(pack_half(x[0] - g0.x, x[1] - g0.y), pack_half(x[2] - g1.x, x[3] - g1.y));
              continue;
            }
            const int64_t at = umat + (int64_t)r * p.cols + c;
            if (p.out_mode == OUT_W_BF16 || p.out_mode == OUT_W_F32) {
              if (skip) continue;
              float w[4] = {0.0f, 0.0f, 0.0f, 0.0f};
              if (p.out_mode == OUT_W_F32) {
                float* W = reinterpret_cast<float*>(p.out) + at;
                if (vec) {
                  const float4 q = *reinterpret_cast<const float4*>(W);
                  w[0] = q.x; w[1] = q.y; w[2] = q.z; w[3] = q.w;
                } else {
                  for (int k = 0; k < 4 && c + k < p.cols; ++k) w[k] = W[k];
                }
              } else {
                const __nv_bfloat16* W = reinterpret_cast<const __nv_bfloat16*>(p.out) + at;
                if (vec) {
                  const uint2 q = *reinterpret_cast<const uint2*>(W);
                  w[0] = __uint_as_float(q.x << 16); w[1] = __uint_as_float(q.x & 0xFFFF0000u);
                  w[2] = __uint_as_float(q.y << 16); w[3] = __uint_as_float(q.y & 0xFFFF0000u);
                } else {
                  for (int k = 0; k < 4 && c + k < p.cols; ++k) w[k] = __bfloat162float(W[k]);
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
              if (vec) {
                *reinterpret_cast<float4*>(W) = make_float4(x[0], x[1], x[2], x[3]);
              } else {
                for (int k = 0; k < 4 && c + k < p.cols; ++k) W[k] = x[k];
              }
            } else {
              __nv_bfloat16* W = reinterpret_cast<__nv_bfloat16*>(p.out) + at;
              if (vec) {
                *reinterpret_cast<uint2*>(W) = make_uint2(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]));
              } else {
                for (int k = 0; k < 4 && c + k < p.cols; ++k) W[k] = __float2bfloat16_rn(x[k]);
              }
            }
          }
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive_cluster(map_to_cta(tempty0 + 8 * b, 0));
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
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(C::tmem_cols) : "memory");
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
  int64_t m, n, ld;                        // ld: pitch of hi / lo
  int blocks;                              // blocks (and norm partials) per matrix
  double* partials;                        // [batch][blocks]
  float eps, scale;
  __half *hi, *lo;
  int32_t *bad, *d_status;
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

// Momentum, and U / (|U|_F + eps) times the scale as the pair hi + lo.
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
  const float f = bad ? 0.0f : (float)((double)p.scale / (sqrt(tot) + (double)p.eps));
  if ((p.n & 3) == 0) {
    const int64_t q_row = p.n >> 2, quads = count >> 2;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < quads; i += (int64_t)gridDim.x * 256) {
      const int64_t r = i / q_row, c = (i - r * q_row) * 4;
      float g[4], u[4];
      ns_load4(p, mat + i * 4, g);
      if (p.momentum) {
        float4* mp = reinterpret_cast<float4*>(p.momentum + mat + i * 4);
        const float4 q = *mp;
        const float mo[4] = {q.x, q.y, q.z, q.w};
        float mn[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) u[k] = ns_momentum(p, g[k], mo[k], &mn[k]);
        if (!bad) *mp = make_float4(mn[0], mn[1], mn[2], mn[3]);
      } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) u[k] = g[k];
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) u[k] = bad ? 0.0f : u[k] * f;
      const uint2 hh = make_uint2(pack_half(u[0], u[1]), pack_half(u[2], u[3]));
      const float2 g0 = __half22float2(*reinterpret_cast<const __half2*>(&hh.x)),
                   g1 = __half22float2(*reinterpret_cast<const __half2*>(&hh.y));
      *reinterpret_cast<uint2*>(p.hi + xmat + r * p.ld + c) = hh;
      *reinterpret_cast<uint2*>(p.lo + xmat + r * p.ld + c) =
          make_uint2(pack_half(u[0] - g0.x, u[1] - g0.y), pack_half(u[2] - g1.x, u[3] - g1.y));
    }
  } else {
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < count; i += (int64_t)gridDim.x * 256) {
      const int64_t r = i / p.n, c = i - r * p.n;
      float u = ns_load(p, mat + i), mn;
      if (p.momentum) {
        u = ns_momentum(p, u, p.momentum[mat + i], &mn);
        if (!bad) p.momentum[mat + i] = mn;
      }
      u = bad ? 0.0f : u * f;
      const __half hh = __float2half_rn(u);
      p.hi[xmat + r * p.ld + c] = hh;
      p.lo[xmat + r * p.ld + c] = __float2half_rn(u - __half2float(hh));
    }
  }
}

// ---------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------
struct NsWs { size_t hi[2], lo, gram, poly, partials, bad, total; int64_t ld, mm, gld; int blocks; };

constexpr int kNormBlocks = 592;

NsWs ns_layout(int64_t m, int64_t n, int64_t batch) {
  NsWs L{};
  L.ld = (n + 7) / 8 * 8;
  L.mm = m < n ? m : n;
  L.gld = (L.mm + 7) / 8 * 8;
  const int64_t want = ceil_div(m * n, 4096);
  L.blocks = (int)(want < kNormBlocks ? want : kNormBlocks);
  const size_t x = (size_t)batch * m * L.ld * 2, g = (size_t)batch * L.mm * L.gld * 2;
  size_t off = 0;
  for (int i = 0; i < 2; ++i) { L.hi[i] = off; off = align_up(off + x, 256); }
  L.lo = off;       off = align_up(off + x, 256);
  L.gram = off;     off = align_up(off + g, 256);
  L.poly = off;     off = align_up(off + g, 256);
  L.partials = off; off = align_up(off + (size_t)batch * L.blocks * 8, 256);
  L.bad = off;      off = align_up(off + (size_t)batch * 4, 256);
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

struct NsOperand { const void* ptr; int64_t cols, rows, ld; };   // as stored

template <bool SYM, bool A_MN, bool B_MN, int BN>
cudaError_t launch_ns_t(const NsOperand& A, const NsOperand& B, NsParams p, cudaStream_t st) {
  using C = NsCfg<BN>;
  auto kern = ns_gemm_kernel<SYM, A_MN, B_MN, BN>;
  static std::atomic<int> ready[64];
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
  if (!ready[dev].load(std::memory_order_acquire)) {
    e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, C::smem);
    if (e != cudaSuccess) return e;
    ready[dev].store(1, std::memory_order_release);
  }
  CUtensorMap ma, mb;
  if (!make_map3(&ma, A.ptr, A.cols, A.rows, p.batch, A.ld, A_MN ? 64 : NS_BM) ||
      !make_map3(&mb, B.ptr, B.cols, B.rows, p.batch, B.ld, B_MN ? 64 : BN / 2))
    return cudaErrorInvalidValue;
  const int64_t mt = ceil_div(p.rows, 256), nt = ceil_div(p.cols, BN);
  int64_t tiles = mt * nt;
  if (SYM) tiles -= (256 / BN) * (mt * (mt - 1) / 2);
  if (tiles * p.batch > 0x7FFFFFFF) return cudaErrorInvalidValue;
  p.m_tiles = (int)mt;
  p.n_tiles = (int)nt;
  p.tiles = (int)tiles;
  const int64_t pairs = sm_count() / 2, total = tiles * p.batch;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(2 * (total < pairs ? total : pairs)), 1, 1);
  cfg.blockDim = dim3(NS_THREADS, 1, 1);
  cfg.dynamicSmemBytes = C::smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = 2;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kern, ma, mb, p);
}

template <bool SYM, bool A_MN, bool B_MN>
cudaError_t launch_ns(const NsOperand& A, const NsOperand& B, const NsParams& p, cudaStream_t st) {
  return launch_ns_t<SYM, A_MN, B_MN, 256>(A, B, p, st);
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
  in.lo = reinterpret_cast<__half*>(ws + L.lo);
  in.bad = reinterpret_cast<int32_t*>(ws + L.bad);
  in.d_status = a.d_status;
  const dim3 grid((unsigned)L.blocks, (unsigned)a.batch);
  ns_norm_kernel<<<grid, 256, 0, st>>>(in);
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  ns_split_kernel<<<grid, 256, 0, st>>>(in);
  if ((e = cudaGetLastError()) != cudaSuccess) return e;

  const bool tall = a.m > a.n;
  const int mm = (int)L.mm;
  __half* gram = reinterpret_cast<__half*>(ws + L.gram);
  __half* poly = reinterpret_cast<__half*>(ws + L.poly);
  const NsOperand og = {gram, mm, mm, L.gld}, op = {poly, mm, mm, L.gld};
  for (int k = 0; k < pr.steps; ++k) {
    const NsOperand ox = {ws + L.hi[k & 1], a.n, a.m, L.ld};
    NsParams p{};                                                // A = X X^T (X^T X)
    p.batch = a.batch; p.rows = mm; p.cols = mm;
    p.k_blocks = (int)ceil_div(longer, 64);
    p.S = gram; p.ld = L.gld; p.alpha = 1.0f / (s * s);
    p.d_status = a.d_status;
    e = tall ? launch_ns<true, true, true>(ox, ox, p, st) : launch_ns<true, false, false>(ox, ox, p, st);
    if (e != cudaSuccess) return e;
    p.k_blocks = (int)ceil_div(mm, 64);                          // b A + c A A
    p.S = poly; p.alpha = pr.coef_c; p.beta = pr.coef_b; p.Cin = gram;
    if ((e = launch_ns<true, false, false>(og, og, p, st)) != cudaSuccess) return e;
    NsParams q{};                                                // a X + (b A + c A A) X
    q.batch = a.batch; q.rows = (int)a.m; q.cols = (int)a.n;
    q.k_blocks = (int)ceil_div(mm, 64);
    q.ld = L.ld; q.a = pr.coef_a;
    q.hi = reinterpret_cast<const __half*>(ws + L.hi[k & 1]);
    q.lo = in.lo;
    q.hi_out = reinterpret_cast<__half*>(ws + L.hi[(k + 1) & 1]);
    q.out_mode = OUT_PAIR;
    q.d_status = a.d_status;
    if (k == pr.steps - 1) {
      q.out = a.out;
      if (a.update) {
        q.out_mode = a.out_dtype == SPO_DTYPE_BF16 ? OUT_W_BF16 : OUT_W_F32;
        q.out_scale = pr.lr * a.update_scale / s;
        q.decay = 1.0f - pr.lr * pr.weight_decay;
        q.bad = in.bad;
      } else {
        q.out_mode = a.out_dtype == SPO_DTYPE_BF16 ? OUT_BF16 : OUT_F32;
        q.out_scale = 1.0f / s;
      }
    }
    e = tall ? launch_ns<false, false, false>(ox, op, q, st) : launch_ns<false, false, true>(op, ox, q, st);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

}  // namespace spo
