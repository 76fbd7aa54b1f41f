// Log-probabilities of given tokens from hidden states, with entropy and the K most likely
// alternatives, and their gradients (spo_logprobs, spo_logprobs_bwd).
//
//   z = W h, lse = log sum_v exp(s z_v) with s = 1/temperature, logp = s z_y - lse,
//   entropy = lse - s sum_v p_v z_v, alternatives: the K largest z, equal ones by ascending id.
//
// Three ways to the logits, none of which stores [T x V] for a long batch:
//   many bf16 rows   the policy loss's contraction (spo_loss_tc.cu): online statistics per vocabulary
//                    split in registers, column groups of largest maximum listed on the way;
//                    lp_merge_kernel joins the splits.
//   few bf16 rows    (up to kLpStreamRows) lp_stream_kernel: bound by reading W once, so W is the operand
//                    with 128 rows a tile and the token rows are the narrow one; every CTA keeps statistics
//                    and a sorted list per token row under the stream, lp_merge_kernel joins the CTAs'.
//   fp32             sgemm_kernel into a chunk of scratch, lp_rows_kernel, lp_merge_kernel.
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

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.69314718055994531f;

__device__ __forceinline__ void flag(int32_t* d_status, int32_t bit) {
  if (d_status) atomicOr(d_status, bit);
}

// ---------------------------------------------------------------------------
// K largest values of a stream, kept by one warp: lane i holds the i-th largest (value descending,
// equal values by ascending id).  An insertion is a ballot, a population count and a few shuffles.
// ---------------------------------------------------------------------------
// AUX: entries carry one more integer.
template <bool AUX>
struct WarpTop {
  float v;
  int id, aux;
  float last_v;      // the K-th entry (what a candidate has to beat), uniform
  int last_id;
  __device__ __forceinline__ void init() { v = last_v = -CUDART_INF_F; id = last_id = 0x7FFFFFFF; aux = 0; }
  __device__ __forceinline__ bool beats(float x, int xi) const {
    return x > last_v || (x == last_v && xi < last_id && x > -CUDART_INF_F);
  }
  __device__ __forceinline__ void insert(float x, int xi, int xa, int K, int lane) {
    const unsigned before = __ballot_sync(0xffffffffu, lane < K && (v > x || (v == x && id < xi)));
    const int pos = __popc(before);
    const float uv = __shfl_up_sync(0xffffffffu, v, 1);
    const int ui = __shfl_up_sync(0xffffffffu, id, 1), ua = AUX ? __shfl_up_sync(0xffffffffu, aux, 1) : 0;
    if (lane == pos) { v = x; id = xi; aux = xa; }
    else if (lane > pos) { v = uv; id = ui; aux = ua; }
    last_v = __shfl_sync(0xffffffffu, v, K - 1);
    last_id = __shfl_sync(0xffffffffu, id, K - 1);
  }
  static __device__ __forceinline__ bool better(float x, int xi, float y, int yi) { return x > y || (x == y && xi < yi); }
  // Joins a list that is sorted over the lanes (descending, empty entries -inf): the larger of entries i and 31 - i are
  // the 32 largest of both and form a bitonic sequence, which five compare-exchanges sort.
  __device__ __forceinline__ void merge(float x, int xi, int xa, int K, int lane) {
    const float rx = __shfl_sync(0xffffffffu, x, 31 - lane);
    const int ri = __shfl_sync(0xffffffffu, xi, 31 - lane), ra = AUX ? __shfl_sync(0xffffffffu, xa, 31 - lane) : 0;
    if (better(rx, ri, v, id)) { v = rx; id = ri; aux = ra; }
#pragma unroll
    for (int s = 16; s > 0; s >>= 1) exchange(v, id, aux, s, (lane & s) == 0);
    if (lane >= K) { v = -CUDART_INF_F; id = 0x7FFFFFFF; }
    last_v = __shfl_sync(0xffffffffu, v, K - 1);
    last_id = __shfl_sync(0xffffffffu, id, K - 1);
  }
  static __device__ __forceinline__ void exchange(float& x, int& xi, int& xa, int s, bool keep_larger) {
    const float px = __shfl_xor_sync(0xffffffffu, x, s);
    const int pi = __shfl_xor_sync(0xffffffffu, xi, s), pa = AUX ? __shfl_xor_sync(0xffffffffu, xa, s) : 0;
    if (keep_larger ? better(px, pi, x, xi) : better(x, xi, px, pi)) { x = px; xi = pi; xa = pa; }
  }
  // One candidate per lane.  A few are inserted one after the other (some 70 clocks each); many are sorted
  // (15 compare-exchanges) and merged (6 steps), some 600 clocks whatever their number.
  __device__ __forceinline__ void offer(float x, int xi, int xa, int K, int lane) {
    const bool in = beats(x, xi);
    unsigned todo = __ballot_sync(0xffffffffu, in);
    if (__popc(todo) > 8) {
      if (!in) { x = -CUDART_INF_F; xi = 0x7FFFFFFF; }
#pragma unroll
      for (int k = 2; k <= 32; k <<= 1)
#pragma unroll
        for (int j = k >> 1; j > 0; j >>= 1) exchange(x, xi, xa, j, ((lane & j) == 0) == ((lane & k) == 0));
      merge(x, xi, xa, K, lane);
      return;
    }
    while (todo) {
      const int src = __ffs(todo) - 1;
      todo &= todo - 1;
      const float bx = __shfl_sync(0xffffffffu, x, src);
      const int bi = __shfl_sync(0xffffffffu, xi, src), ba = AUX ? __shfl_sync(0xffffffffu, xa, src) : 0;
      if (beats(bx, bi)) insert(bx, bi, ba, K, lane);
    }
  }
};

// The launch before this one in the stream may still be running (programmatic dependent launch): wait for it to
// have finished, and let the next launch come up behind this one.
__device__ __forceinline__ void pdl_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void pdl_trigger() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// (m2, l, ez) of two disjoint parts of a row, joined: m2 in log2 units, l = sum 2^(z sc2 - m2), ez = sum z 2^(...)
__device__ __forceinline__ void join_stats(float& m2, float& l, float& ez, float m2b, float lb, float ezb) {
  const float m = fmaxf(m2, m2b);
  const float wa = m2 == m ? 1.0f : exp2f(m2 - m), wb = m2b == m ? 1.0f : exp2f(m2b - m);
  l = l * wa + lb * wb;
  ez = ez * wa + ezb * wb;
  m2 = m;
}
__device__ __forceinline__ void warp_join_stats(float& m2, float& l, float& ez) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const float m2b = __shfl_xor_sync(0xffffffffu, m2, o), lb = __shfl_xor_sync(0xffffffffu, l, o),
                ezb = __shfl_xor_sync(0xffffffffu, ez, o);
    join_stats(m2, l, ez, m2b, lb, ezb);
  }
}

// What every path ends with.
struct LpOut {
  const int32_t* y;
  const uint8_t* mask;
  float *logp, *lse, *entropy;
  int32_t* top_ids;
  float* top_logp;
  float inv_t;
  int K;
  int32_t V;
  int32_t* d_status;
};

// Outputs of token t from its joined statistics; the whole warp calls it, lane i < K with the i-th alternative.
__device__ __forceinline__ void lp_finish(const LpOut& o, int64_t t, float m2, float l, float ez, float zt, bool odd, float top_v,
                                          int top_id, int lane) {
  float lse = (m2 + log2f(l)) * kLn2;
  if (odd) lse = CUDART_NAN_F;
  const bool on = o.mask == nullptr || o.mask[t] != 0;
  if (lane == 0) {
    if (on && !(fabsf(lse) < CUDART_INF_F)) flag(o.d_status, SPO_DEV_NONFINITE);
    if (o.logp) {
      const int32_t yt = o.y[t];
      float lp = fmaf(zt, o.inv_t, -lse);
      if (yt < 0 || yt >= o.V) {
        lp = -CUDART_INF_F;
        if (on) flag(o.d_status, SPO_DEV_ID_OUT_OF_RANGE);
      }
      o.logp[t] = on ? lp : 0.0f;
    }
    o.lse[t] = on ? lse : 0.0f;
    if (o.entropy) o.entropy[t] = on ? lse - o.inv_t * (ez / l) : 0.0f;
  }
  if (lane < o.K) {
    const bool found = top_v > -CUDART_INF_F;
    o.top_ids[t * o.K + lane] = on && found ? top_id : -1;
    o.top_logp[t * o.K + lane] = !on ? 0.0f : found ? fmaf(top_v, o.inv_t, -lse) : -CUDART_INF_F;
  }
}

// A float as an integer of the same order (and back: the mapping is its own inverse).
__device__ __forceinline__ int order_key(int b) { return b ^ ((b >> 31) & 0x7FFFFFFF); }

// The K largest entries of sorted lists in shared memory ([list][K] of (value, id), empty entries -inf), one per lane: K
// rounds over the lists' heads, of which a lane holds up to five.
constexpr int kMergeLists = 160;
__device__ __forceinline__ void merge_heads(const float2* s, int lists, int K, int lane, float* v_out, int* id_out) {
  constexpr int H = kMergeLists / 32;
  float hv[H];
  int hi[H], hp[H];
#pragma unroll
  for (int h = 0; h < H; ++h) {
    const int q = lane + 32 * h;
    hp[h] = 0;
    hv[h] = -CUDART_INF_F;
    hi[h] = 0x7FFFFFFF;
    if (q < lists) { const float2 c = s[q * K]; hv[h] = c.x; hi[h] = __float_as_int(c.y); }
  }
  float v = -CUDART_INF_F;
  int id = 0x7FFFFFFF;
  for (int k = 0; k < K; ++k) {
    float bv = hv[0];
    int bi = hi[0], bh = 0;
#pragma unroll
    for (int h = 1; h < H; ++h)
      if (hv[h] > bv || (hv[h] == bv && hi[h] < bi)) { bv = hv[h]; bi = hi[h]; bh = h; }
    const int key = order_key(__float_as_int(bv + 0.0f));            // (-0 counts as 0)
    const int best = __reduce_max_sync(0xffffffffu, key);
    const int best_id = __reduce_min_sync(0xffffffffu, key == best ? bi : 0x7FFFFFFF);
    if (best_id == 0x7FFFFFFF) break;                                // the lists are exhausted
    if (lane == k) { v = __int_as_float(order_key(best)); id = best_id; }
    if (key == best && bi == best_id) {                              // ids are distinct: one lane
#pragma unroll
      for (int h = 0; h < H; ++h)
        if (h == bh) {
          const int at = ++hp[h];
          hv[h] = -CUDART_INF_F;
          hi[h] = 0x7FFFFFFF;
          if (at < K) { const float2 c = s[(lane + 32 * h) * K + at]; hv[h] = c.x; hi[h] = __float_as_int(c.y); }
        }
    }
  }
  *v_out = v;
  *id_out = id;
}

// ---------------------------------------------------------------------------
// Statistics and alternatives of stored logit rows.  Block = (row, segment of the vocabulary); each
// warp takes a contiguous part of `part` columns, the block joins its warps and writes one partial and one
// sorted list, or, where it has the whole row, the outputs.  Reads every logit once; bound by L2 or HBM.
// ---------------------------------------------------------------------------
constexpr int kRowWarps = 8;

__global__ void __launch_bounds__(32 * kRowWarps)
lp_rows_kernel(const float* __restrict__ Z, int64_t ldz, int nseg, int part, int64_t t0, const LpOut o,
               FwdPartial* __restrict__ partials, float2* __restrict__ cand) {
  const int32_t V = o.V;
  const int K = o.K;
  const float sc2 = kLog2e * o.inv_t;
  pdl_trigger();
  pdl_wait();
  const int64_t row = blockIdx.x / nseg;
  const int seg = (int)(blockIdx.x - row * nseg);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const float* z = Z + row * ldz;
  const int64_t begin = ((int64_t)seg * kRowWarps + warp) * part;
  const int64_t end = begin + part < V ? begin + part : V;
  float m2 = -CUDART_INF_F, l = 0.0f, ez = 0.0f;
  WarpTop<false> top;
  top.init();
  for (int64_t c0 = begin; c0 < end; c0 += 256) {
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int64_t c = c0 + i * 32 + lane;
      x[i] = c < end ? z[c] : -1.0e30f;            // far below any logit: its exponential is zero, and zero times it too
    }
    float mx = x[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) mx = fmaxf(mx, x[i]);
    const float mn = fmaxf(fmaxf(m2, mx * sc2), -1.0e25f);   // a lane without columns: exponentials of -inf, not of rounding
    float s = 0.0f, t = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float e = fast_exp2(fmaf(x[i], sc2, -mn));
      s += e;
      t = fmaf(e, x[i], t);
    }
    const float down = fast_exp2(m2 - mn);
    l = fmaf(l, down, s);
    ez = fmaf(ez, down, t);
    m2 = mn;
    if (K > 0 && __any_sync(0xffffffffu, mx > top.last_v)) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int64_t c = c0 + i * 32 + lane;
        top.offer(c < end ? x[i] : -CUDART_INF_F, (int)c, 0, K, lane);
      }
    }
  }
  __shared__ float s_m[kRowWarps], s_l[kRowWarps], s_e[kRowWarps];
  __shared__ float2 s_top[kRowWarps * kMaxTopK];
  warp_join_stats(m2, l, ez);
  if (lane == 0) { s_m[warp] = m2; s_l[warp] = l; s_e[warp] = ez; }
  if (lane < K) s_top[warp * K + lane] = make_float2(top.v, __int_as_float(top.id));
  __syncthreads();
  if (warp != 0) return;
  m2 = lane < kRowWarps ? s_m[lane] : -CUDART_INF_F;
  l = lane < kRowWarps ? s_l[lane] : 0.0f;
  ez = lane < kRowWarps ? s_e[lane] : 0.0f;
  const bool odd = __any_sync(0xffffffffu, !(l >= 0.0f));            // a NaN, which fmaxf drops
  warp_join_stats(m2, l, ez);
  if (odd) l = CUDART_NAN_F;
  const int64_t lo = (int64_t)seg * kRowWarps * part, hi = lo + (int64_t)kRowWarps * part;
  const int32_t yt = o.y ? o.y[t0 + row] : -1;
  const float zt = yt >= lo && yt < hi && yt < V ? z[yt] : -CUDART_INF_F;
  float tv = -CUDART_INF_F;
  int ti = 0x7FFFFFFF;
  if (K > 0) merge_heads(s_top, kRowWarps, K, lane, &tv, &ti);
  if (nseg == 1) {
    lp_finish(o, t0 + row, m2, l, ez, zt, odd, tv, ti, lane);
    return;
  }
  if (lane == 0) {
    FwdPartial pt;
    pt.m2 = m2; pt.l = l; pt.pad = ez; pt.zt = zt;
    partials[row * nseg + seg] = pt;
  }
  if (lane < K) cand[(row * nseg + seg) * K + lane] = make_float2(tv, __int_as_float(ti));
}

// ---------------------------------------------------------------------------
// The end of every path: joins a token row's partials, finishes logp / lse / entropy, and finds the
// alternatives among the row's lists.  WARPS warps per row.  GROUPS: the lists hold column groups (maximum, group << 8 |
// slot) whose 32 logits are stored in `cand`; first the K groups of largest maximum, then the K largest logits
// in them.  Otherwise the lists hold the logits themselves, (value, id), sorted.
// ---------------------------------------------------------------------------
template <bool GROUPS, int WARPS>
__global__ void __launch_bounds__(WARPS == 1 ? 128 : 32 * WARPS)
lp_merge_kernel(const FwdPartial* __restrict__ partials, int lists, int64_t part_ld, const float2* __restrict__ tops,
                const float* __restrict__ cand, int list_len, int64_t rows, int64_t t0, const LpOut o) {
  static_assert((WARPS == 1) == GROUPS, "column groups are merged by one warp, plain lists by several");
  pdl_trigger();
  pdl_wait();
  const int lane = threadIdx.x & 31, warp = WARPS == 1 ? 0 : threadIdx.x >> 5;
  const int64_t row = WARPS == 1 ? (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5) : (int64_t)blockIdx.x;
  if (row >= rows) return;
  const int64_t t = t0 + row;
  const int K = o.K;
  __shared__ float2 s_lists[GROUPS ? 1 : kMergeLists * kMaxTopK];
  if (!GROUPS) {                                    // all lists into shared memory
    for (int i = threadIdx.x; i < lists * K; i += 32 * WARPS) s_lists[i] = tops[row * lists * K + i];
    __syncthreads();
    if (warp != 0) return;
  }
  // partial of list s: [s][part_ld] (GROUPS) or [row][lists]
  auto at = [&](int s) { return GROUPS ? (int64_t)s * part_ld + row : row * lists + s; };
  float m2 = -CUDART_INF_F, l = 0.0f, ez = 0.0f, zt = -CUDART_INF_F;
  bool odd = false;                                 // a partial that is NaN: fmaxf would drop it
#pragma unroll 4
  for (int s = lane; s < lists; s += 32) {
    const FwdPartial p = partials[at(s)];
    odd |= !(p.l >= 0.0f);
    zt = p.zt > -CUDART_INF_F || p.zt != p.zt ? p.zt : zt;   // at most one list has the target
    join_stats(m2, l, ez, p.m2, p.l, p.pad);
  }
  warp_join_stats(m2, l, ez);
  odd = __any_sync(0xffffffffu, odd);
  const unsigned has = __ballot_sync(0xffffffffu, zt > -CUDART_INF_F || zt != zt);
  zt = has ? __shfl_sync(0xffffffffu, zt, __ffs(has) - 1) : -CUDART_INF_F;
  float tv = -CUDART_INF_F;
  int ti = 0x7FFFFFFF;
  if (!GROUPS) {
    if (K > 0) merge_heads(s_lists, lists, K, lane, &tv, &ti);
  } else if (K > 0) {
    WarpTop<true> g;
    g.init();
    const int n = lists * list_len;
    for (int i0 = 0; i0 < n; i0 += 128) {           // four accesses in flight
      float2 c[4];
      int ax[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int i = i0 + 32 * u + lane;
        c[u] = make_float2(-CUDART_INF_F, __uint_as_float(0xFFFFFF00u));
        ax[u] = 0;
        if (i < n) {
          const int s = i / list_len, k = i - s * list_len;
          c[u] = tops[at(s) * list_len + k];
          ax[u] = s * list_len;
        }
      }
#pragma unroll
      for (int u = 0; u < 4; ++u)
        g.offer(c[u].x, (int)(__float_as_uint(c[u].y) >> 8), ax[u] + (int)(__float_as_uint(c[u].y) & 255u), K, lane);
    }
    WarpTop<false> top;
    top.init();
    for (int k = 0; k < K; ++k) {
      const float gm = __shfl_sync(0xffffffffu, g.v, k);
      const int gid = __shfl_sync(0xffffffffu, g.id, k), loc = __shfl_sync(0xffffffffu, g.aux, k);
      if (!(gm > -CUDART_INF_F)) break;             // fewer groups than K
      const int s = loc / list_len, slot = loc - s * list_len;
      const int id = gid * 32 + lane;
      const float x = cand[(at(s) * list_len + slot) * 32 + lane];
      top.offer(id < o.V ? x : -CUDART_INF_F, id, 0, K, lane);
    }
    tv = top.v;
    ti = top.id;
  }
  lp_finish(o, t, m2, l, ez, zt, odd, tv, ti, lane);
}

// ---------------------------------------------------------------------------
// Few bf16 token rows, with W streamed once.  One CTA per SM walks tiles of `tile_h` (at most 128) vocabulary
// rows; TMA brings 64-deep k-blocks of the tile and of all token rows, one MMA per 16 of k with M = 128 vocabulary rows
// and N = NT token rows accumulates in tensor memory (two buffers, so a tile is reduced while the next one
// streams).  W is read once, which is the floor (1.24 GB at d = 4096, V = 151936: 190 us at the measured copy rate); the token
// rows come from L2 once per tile, NT / tile_h of W's traffic.  tile_h is the smallest height that takes the same number of
// rounds over the SMs, so that the last round is full (V = 151936 on 148 SMs: 115 rows x 9 rounds reads 0.8 %
// more than an even share, 128-row tiles would leave the ninth round nearly empty).
// Reduction: eight warps turn the finished tile into [token][vocabulary row] in shared memory, then each takes
// the tokens w, w + 8, ..: a lane holds four logits, the row's maximum and sums are warp reductions, lane k keeps the
// running statistics of the warp's k-th token, and a tile whose maximum beats the token's K-th entry goes into its
// sorted list.  Storing the logits and reducing them in further launches took 254 us where this takes 196 (one token,
// K = 20): 80 us of launches that read 0.6 MB, most of it chains of list insertions in a few warps.
// ---------------------------------------------------------------------------
struct StreamParams {
  int tiles, tile_h, k_blocks;
  int T, K;
  int32_t V;
  float sc2;
  const int32_t* y;
  FwdPartial* partials;                      // [T][gridDim.x]
  float2* tops;                              // [T][gridDim.x][K]
  int32_t* d_status;
};

constexpr int kStreamWarps = 8;              // reducing warps
constexpr int kStreamThreads = 64 + 32 * kStreamWarps;
constexpr int kStreamA = 128 * 64 * 2;
template <int NT> struct StreamCfg {
  static constexpr int stage_bytes = kStreamA + NT * 128;
  static constexpr int tile_bytes = NT * 128 * 4;            // logits of a tile, [token][128]
  static constexpr int list_bytes = NT * 32 * 8;             // sorted lists, [token][32]
  static constexpr int stages = (226 * 1024 - tile_bytes - list_bytes - 2048) / stage_bytes;
  static constexpr int smem = stages * stage_bytes + tile_bytes + list_bytes + 1024 + 512;
  static constexpr int tmem_cols = 2 * NT < 32 ? 32 : 2 * NT;
};

// Barrier of the reducing warps; every one of them arrives, and all leave with the same answer.
__device__ __forceinline__ bool stream_barrier(bool good) {
  int all;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.s32 p, %1, 0;\n\t"
      "bar.red.and.pred q, 1, %2, p;\n\t"
      "selp.b32 %0, 1, 0, q;\n\t}"
      : "=r"(all)
      : "r"(good ? 1 : 0), "n"(32 * kStreamWarps)
      : "memory");
  return all != 0;
}

template <int NT>
__global__ void __launch_bounds__(kStreamThreads, 1)
lp_stream_kernel(const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmH, const StreamParams p) {
  using C = StreamCfg<NT>;
  constexpr int S = C::stages;
  static_assert(S >= 4 && 16 * S + 48 <= 512, "stages");
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t base = (raw + 1023u) & ~1023u;
  uint8_t* gen = smem_raw + (base - raw);
  float* tile_z = reinterpret_cast<float*>(gen + S * C::stage_bytes);
  float2* list = reinterpret_cast<float2*>(gen + S * C::stage_bytes + C::tile_bytes);
  constexpr int kBarAt = S * C::stage_bytes + C::tile_bytes + C::list_bytes;
  const uint32_t bars = base + kBarAt;
  const uint32_t full0 = bars, empty0 = bars + 8 * S, tfull0 = bars + 16 * S, tempty0 = tfull0 + 16;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(gen + kBarAt + 16 * S + 32);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  pdl_trigger();
  if (threadIdx.x == 0) {
    for (int s = 0; s < S; ++s) { mbar_init(full0 + 8 * s, 1); mbar_init(empty0 + 8 * s, 1); }
    for (int b = 0; b < 2; ++b) { mbar_init(tfull0 + 8 * b, 1); mbar_init(tempty0 + 8 * b, kStreamWarps); }
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 0) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(C::tmem_cols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;

  if (warp == 0) {
    if (lane == 0) {
      uint32_t it = 0;
      bool ok = true;
      const uint32_t bytes = (uint32_t)p.tile_h * 128u + NT * 128u;
      for (int tile = blockIdx.x; tile < p.tiles && ok; tile += gridDim.x) {
        for (int kb = 0; kb < p.k_blocks; ++kb, ++it) {
          const uint32_t s = it % S, ph = (it / S) & 1u;
          if (!mbar_wait(empty0 + 8 * s, ph ^ 1u, abort_flag, p.d_status)) { ok = false; break; }
          mbar_expect_tx(full0 + 8 * s, bytes);
          const uint32_t sa = base + s * C::stage_bytes;
          tma_load_2d_cta(sa, &tmW, kb * 64, tile * p.tile_h, full0 + 8 * s);
          tma_load_2d_cta(sa + kStreamA, &tmH, kb * 64, 0, full0 + 8 * s);
        }
      }
    }
  } else if (warp == 1) {
    if (lane == 0) {
      constexpr uint32_t idesc = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(NT >> 3) << 17) | (8u << 24);
      uint32_t it = 0, n = 0;
      bool ok = true;
      for (int tile = blockIdx.x; tile < p.tiles && ok; tile += gridDim.x, ++n) {
        const uint32_t b = n & 1u;
        if (!mbar_wait(tempty0 + 8 * b, ((n >> 1) & 1u) ^ 1u, abort_flag, p.d_status)) { ok = false; break; }
        tc_fence_after();
        for (int kb = 0; kb < p.k_blocks; ++kb, ++it) {
          const uint32_t s = it % S, ph = (it / S) & 1u;
          if (!mbar_wait(full0 + 8 * s, ph, abort_flag, p.d_status)) { ok = false; break; }
          tc_fence_after();
          const uint32_t sa = base + s * C::stage_bytes;
#pragma unroll
          for (int j = 0; j < 4; ++j)
            umma_f16_cta(tmem_base + b * NT, smem_desc(sa + j * 32, 16, 1024), smem_desc(sa + kStreamA + j * 32, 16, 1024),
                         idesc, (kb | j) != 0 ? 1u : 0u);
          umma_commit_cta(empty0 + 8 * s);
        }
        if (ok) umma_commit_cta(tfull0 + 8 * b);
      }
    }
  } else {
    const int quarter = warp & 3, half = (warp - 2) >> 2, w = warp - 2;
    constexpr int PER = NT / kStreamWarps;               // tokens w, w + 8, .. of this warp; lane k < PER keeps the k-th's state
    float m2 = -CUDART_INF_F, l = 0.0f, ez = 0.0f, zt = -CUDART_INF_F, thr = -CUDART_INF_F;
    const int my_t = w + kStreamWarps * lane;
    const int32_t my_y = lane < PER && my_t < p.T && p.y ? p.y[my_t] : -1;
    for (int k = 0; k < PER; ++k)
      list[(w + kStreamWarps * k) * 32 + lane] = make_float2(-CUDART_INF_F, __int_as_float(0x7FFFFFFF));
    __syncwarp();
    uint32_t n = 0;
    for (int tile = blockIdx.x; tile < p.tiles; tile += gridDim.x, ++n) {
      const uint32_t b = n & 1u;
      int good = 1;
      if (lane == 0) good = mbar_wait<32>(tfull0 + 8 * b, (n >> 1) & 1u, abort_flag, p.d_status) ? 1 : 0;
      good = __shfl_sync(0xffffffffu, good, 0);
      tc_fence_after();
      const uint32_t taddr = tmem_base + ((uint32_t)(quarter * 32) << 16) + b * NT;
      if (good) {
        constexpr int COLS = NT / 2 < 16 ? 16 : NT / 2;              // token columns per warp of a quarter
        if (half * COLS < NT) {
#pragma unroll 1
          for (int c = half * COLS; c < (half + 1) * COLS; c += 16) {
            uint32_t x[16];
            tmem_ld16(taddr + c, x);
#pragma unroll
            for (int j = 0; j < 16; ++j) tile_z[(c + j) * 128 + quarter * 32 + lane] = __uint_as_float(x[j]);
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_cta(tempty0 + 8 * b);
      }
      if (!stream_barrier(good != 0)) break;                          // the tile is in shared memory
      const int v0 = tile * p.tile_h;
      const int cols = p.V - v0 < p.tile_h ? p.V - v0 : p.tile_h;
#pragma unroll 1
      for (int k = 0; k < PER; ++k) {
        const int t = w + kStreamWarps * k;
        if (t >= p.T) break;
        const float* z = tile_z + t * 128;
        float x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = i * 32 + lane < cols ? z[i * 32 + lane] : -1.0e30f;
        const int b32 = __float_as_int(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])));
        const float mx = __int_as_float(order_key(__reduce_max_sync(0xffffffffu, order_key(b32))));
        const float mk = __shfl_sync(0xffffffffu, m2, k);
        const float mn = fmaxf(fmaxf(mk, mx * p.sc2), -1.0e25f);
        float s = 0.0f, u = 0.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float e = fast_exp2(fmaf(x[i], p.sc2, -mn));
          s += e;
          u = fmaf(e, x[i], u);
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
          s += __shfl_xor_sync(0xffffffffu, s, o);
          u += __shfl_xor_sync(0xffffffffu, u, o);
        }
        if (lane == k) {
          const float down = fast_exp2(mk - mn);
          l = fmaf(l, down, s);
          ez = fmaf(ez, down, u);
          m2 = mn;
          if (my_y >= v0 && my_y < v0 + cols) zt = z[my_y - v0];
        }
        if (p.K > 0 && mx > __shfl_sync(0xffffffffu, thr, k)) {
          float2* mine = list + t * 32 + lane;
          WarpTop<false> top;
          const float2 c = *mine;
          top.v = c.x; top.id = __float_as_int(c.y); top.aux = 0;
          top.last_v = __shfl_sync(0xffffffffu, top.v, p.K - 1);
          top.last_id = __shfl_sync(0xffffffffu, top.id, p.K - 1);
#pragma unroll
          for (int i = 0; i < 4; ++i)
            top.offer(i * 32 + lane < cols ? x[i] : -CUDART_INF_F, v0 + i * 32 + lane, 0, p.K, lane);
          *mine = make_float2(top.v, __int_as_float(top.id));
          if (lane == k) thr = top.last_v;
        }
      }
      if (!stream_barrier(true)) break;                               // the tile has been read
    }
    if (lane < PER && my_t < p.T) {
      FwdPartial pt;
      pt.m2 = m2; pt.l = l; pt.zt = zt; pt.pad = ez;
      p.partials[(int64_t)my_t * gridDim.x + blockIdx.x] = pt;
    }
    for (int k = 0; k < PER; ++k) {
      const int t = w + kStreamWarps * k;
      if (t < p.T && lane < p.K) p.tops[((int64_t)t * gridDim.x + blockIdx.x) * p.K + lane] = list[t * 32 + lane];
    }
  }

  __syncwarp();
  if (*abort_flag) {                       // let copies still in flight land before the CTA retires
    for (int i = 0; i < 200; ++i) __nanosleep(1000);
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 0)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(C::tmem_cols) : "memory");
}

// CTAs of lp_stream_kernel, and rows of its vocabulary tiles.
void stream_shape(int32_t V, int* grid, int* tile_h) {
  const int sms = sm_count() < kMergeLists ? sm_count() : kMergeLists;
  const int64_t rounds = ceil_div(V, (int64_t)128 * sms);
  int h = (int)ceil_div(V, rounds * sms);
  if (h < 8) h = 8;
  const int64_t tiles = ceil_div(V, h);
  *tile_h = h;
  *grid = (int)(tiles < sms ? tiles : sms);
}

template <int NT>
cudaError_t launch_stream_t(const LpFwd& a, FwdPartial* partials, float2* tops, cudaStream_t st) {
  using C = StreamCfg<NT>;
  static std::atomic<int> ready[64];
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
  if (!ready[dev].load(std::memory_order_acquire)) {
    e = cudaFuncSetAttribute(lp_stream_kernel<NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::smem);
    if (e != cudaSuccess) return e;
    ready[dev].store(1, std::memory_order_release);
  }
  StreamParams p{};
  int grid = 0;
  stream_shape(a.V, &grid, &p.tile_h);
  CUtensorMap mW, mH;
  if (!make_map(&mW, a.W, a.d, a.V, a.d, (uint32_t)p.tile_h) || !make_map(&mH, a.H, a.d, a.T, a.ldh, NT))
    return cudaErrorInvalidValue;
  p.tiles = (int)ceil_div(a.V, p.tile_h);
  p.k_blocks = (int)ceil_div(a.d, 64);
  p.T = (int)a.T;
  p.K = a.top_k;
  p.V = a.V;
  p.sc2 = kLog2e * a.inv_t;
  p.y = a.y;
  p.partials = partials;
  p.tops = tops;
  p.d_status = a.d_status;
  lp_stream_kernel<NT><<<grid, kStreamThreads, C::smem, st>>>(mW, mH, p);
  return cudaGetLastError();
}

cudaError_t launch_stream(const LpFwd& a, FwdPartial* partials, float2* tops, cudaStream_t st) {
  if (a.T <= 16) return launch_stream_t<16>(a, partials, tops, st);
  if (a.T <= 32) return launch_stream_t<32>(a, partials, tops, st);
  if (a.T <= 64) return launch_stream_t<64>(a, partials, tops, st);
  return launch_stream_t<128>(a, partials, tops, st);
}

// A launch whose kernel begins with pdl_wait(): it may come up while the launch before it still runs.
template <typename... P, typename... A>
cudaError_t launch_dependent(void (*kern)(P...), dim3 grid, dim3 block, cudaStream_t st, A... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kern, static_cast<P>(args)...);
}

// ---------------------------------------------------------------------------
// fp32 matrix product on the fp32 pipes: C[m][n] (+)= sum_k A(m,k) B(n,k).  A_K / B_K: the operand is
// contiguous along k, else along m / n.  Tiles of TILE x TILE x 16, 256 threads, TILE/16 squared results a
// thread; the next k-block is fetched into registers while this one is multiplied.  gridDim.z splits k:
// each split writes its own C (stride M * ldc) and sum_splits_kernel adds them in a fixed order.
// ---------------------------------------------------------------------------
struct SgemmParams {
  const float *A, *B;
  int64_t lda, ldb, ldc, M, N, K, k_per;
  float* C;
  int accumulate;
  const uint8_t* b_mask;            // k rows whose B is taken as zero where the mask is 0 (B contiguous along n)
};

template <int TILE, bool KC>
__device__ __forceinline__ float4 sg_fetch(const float* X, int64_t ld, int64_t row0, int64_t rows, int64_t k0, int64_t k_end,
                                           int idx, const uint8_t* kmask) {
  float4 r = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  if (KC) {
    const int64_t m = row0 + (idx >> 2), k = k0 + (idx & 3) * 4;
    if (m < rows && k < k_end) {
      const float* s = X + m * ld + k;
      if (k + 3 < k_end) return *reinterpret_cast<const float4*>(s);
      r.x = s[0];
      if (k + 1 < k_end) r.y = s[1];
      if (k + 2 < k_end) r.z = s[2];
    }
  } else {
    const int64_t k = k0 + idx / (TILE / 4), m = row0 + (idx % (TILE / 4)) * 4;
    if (k < k_end && m < rows && (kmask == nullptr || kmask[k] != 0)) {
      const float* s = X + k * ld + m;
      if (m + 3 < rows) return *reinterpret_cast<const float4*>(s);
      r.x = s[0];
      if (m + 1 < rows) r.y = s[1];
      if (m + 2 < rows) r.z = s[2];
    }
  }
  return r;
}
template <int TILE, bool KC>
__device__ __forceinline__ void sg_store(float (*s)[TILE + 4], int idx, float4 v) {
  if (KC) {
    const int m = idx >> 2, k = (idx & 3) * 4;
    s[k][m] = v.x; s[k + 1][m] = v.y; s[k + 2][m] = v.z; s[k + 3][m] = v.w;
  } else {
    *reinterpret_cast<float4*>(&s[idx / (TILE / 4)][(idx % (TILE / 4)) * 4]) = v;
  }
}

template <int TILE, bool A_K, bool B_K>
__global__ void __launch_bounds__(256)
sgemm_kernel(const SgemmParams p) {
  constexpr int R = TILE / 64;                       // groups of four rows (columns) per thread, 64 apart
  constexpr int LOADS = TILE * 16 / 4 / 256;
  __shared__ __align__(16) float As[2][16][TILE + 4], Bs[2][16][TILE + 4];
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  const int64_t m0 = (int64_t)blockIdx.x * TILE, n0 = (int64_t)blockIdx.y * TILE;
  const int64_t k_begin = (int64_t)blockIdx.z * p.k_per;
  const int64_t k_end = k_begin + p.k_per < p.K ? k_begin + p.k_per : p.K;
  float acc[4 * R][4 * R] = {};
  pdl_trigger();
  float4 ra[LOADS], rb[LOADS];
#pragma unroll
  for (int i = 0; i < LOADS; ++i) {
    ra[i] = sg_fetch<TILE, A_K>(p.A, p.lda, m0, p.M, k_begin, k_end, threadIdx.x + i * 256, nullptr);
    rb[i] = sg_fetch<TILE, B_K>(p.B, p.ldb, n0, p.N, k_begin, k_end, threadIdx.x + i * 256, p.b_mask);
  }
  int buf = 0;
  for (int64_t k0 = k_begin; k0 < k_end; k0 += 16, buf ^= 1) {
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      sg_store<TILE, A_K>(As[buf], threadIdx.x + i * 256, ra[i]);
      sg_store<TILE, B_K>(Bs[buf], threadIdx.x + i * 256, rb[i]);
    }
    __syncthreads();
    if (k0 + 16 < k_end) {
#pragma unroll
      for (int i = 0; i < LOADS; ++i) {
        ra[i] = sg_fetch<TILE, A_K>(p.A, p.lda, m0, p.M, k0 + 16, k_end, threadIdx.x + i * 256, nullptr);
        rb[i] = sg_fetch<TILE, B_K>(p.B, p.ldb, n0, p.N, k0 + 16, k_end, threadIdx.x + i * 256, p.b_mask);
      }
    }
#pragma unroll
    for (int k = 0; k < 16; ++k) {
      float a[4 * R], b[4 * R];
#pragma unroll
      for (int r = 0; r < R; ++r) {
        *reinterpret_cast<float4*>(a + 4 * r) = *reinterpret_cast<const float4*>(&As[buf][k][ty * 4 + 64 * r]);
        *reinterpret_cast<float4*>(b + 4 * r) = *reinterpret_cast<const float4*>(&Bs[buf][k][tx * 4 + 64 * r]);
      }
#pragma unroll
      for (int i = 0; i < 4 * R; ++i)
#pragma unroll
        for (int j = 0; j < 4 * R; ++j) acc[i][j] = fmaf(a[i], b[j], acc[i][j]);
    }
  }
  float* C = p.C + (int64_t)blockIdx.z * p.M * p.ldc;
#pragma unroll
  for (int i = 0; i < 4 * R; ++i) {
    const int64_t m = m0 + ty * 4 + (i & 3) + 64 * (i >> 2);
    if (m >= p.M) continue;
#pragma unroll
    for (int j = 0; j < 4 * R; ++j) {
      const int64_t n = n0 + tx * 4 + (j & 3) + 64 * (j >> 2);
      if (n >= p.N) continue;
      float* dst = C + m * p.ldc + n;
      *dst = p.accumulate ? *dst + acc[i][j] : acc[i][j];
    }
  }
}

__global__ void __launch_bounds__(256)
sum_splits_kernel(const float* __restrict__ parts, int splits, int64_t n, float* __restrict__ out, int accumulate) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    float s = accumulate ? out[i] : 0.0f;
    for (int z = 0; z < splits; ++z) s += parts[(int64_t)z * n + i];
    out[i] = s;
  }
}

constexpr int kSplitBlocks = 444;                              // blocks that a split of k fills the GPU with
constexpr size_t kSplitBytes = (size_t)kSplitBlocks * 128 * 128 * 4;   // room for all splits' results together

template <bool A_K, bool B_K>
cudaError_t launch_sgemm(SgemmParams p, float* split_ws, cudaStream_t st) {
  const int64_t big = ceil_div(p.M, 128) * ceil_div(p.N, 128);
  const int tile = big >= sm_count() ? 128 : 64;               // 64: four times the blocks where 128 leaves SMs idle
  const int64_t bm = ceil_div(p.M, tile), bn = ceil_div(p.N, tile);
  int64_t splits = 1;
  if (split_ws && p.ldc == p.N && bm * bn < 2 * sm_count()) {
    splits = kSplitBlocks / (bm * bn);
    const int64_t most = ceil_div(p.K, 128);                   // at least 8 k-blocks a split
    if (splits > most) splits = most;
    while (splits > 1 && (size_t)splits * p.M * p.N * 4 > kSplitBytes) --splits;
    if (splits < 1) splits = 1;
  }
  p.k_per = ceil_div(ceil_div(p.K, 16), splits) * 16;
  splits = ceil_div(p.K, p.k_per);
  if (bn > 65535 || splits > 65535) return cudaErrorInvalidConfiguration;
  float* out = p.C;
  const int accumulate = p.accumulate;
  if (splits > 1) { p.C = split_ws; p.accumulate = 0; }
  const dim3 grid((unsigned)bm, (unsigned)bn, (unsigned)splits);
  if (tile == 128) sgemm_kernel<128, A_K, B_K><<<grid, 256, 0, st>>>(p);
  else sgemm_kernel<64, A_K, B_K><<<grid, 256, 0, st>>>(p);
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess || splits == 1) return e;
  const int64_t n = p.M * p.N;
  int64_t blocks = ceil_div(n, 256);
  if (blocks > (int64_t)sm_count() * 8) blocks = (int64_t)sm_count() * 8;
  sum_splits_kernel<<<(unsigned)blocks, 256, 0, st>>>(split_ws, (int)splits, n, out, accumulate);
  return cudaGetLastError();
}

// fp32 logits to their gradient, in place (the formula of g_values_lp, with log p in nats).
__global__ void __launch_bounds__(256)
lp_g_f32_kernel(float* __restrict__ Z, int64_t ldz, int nseg, int32_t V, int64_t t0, const int32_t* __restrict__ y,
                const uint8_t* __restrict__ mask, const float* __restrict__ lse, const float* __restrict__ ent,
                const float* __restrict__ g_logp, const float* __restrict__ g_lse, const float* __restrict__ g_ent,
                float inv_t, int32_t* d_status) {
  const int64_t row = blockIdx.x / nseg;
  const int seg = (int)(blockIdx.x - row * nseg);
  const int64_t t = t0 + row;
  float* z = Z + row * ldz;
  const bool live = mask == nullptr || mask[t] != 0;
  float gl = g_logp ? g_logp[t] : 0.0f;
  const int32_t yt = y ? y[t] : -1;
  if (g_logp && (yt < 0 || yt >= V)) {
    if (live && seg == 0 && threadIdx.x == 0) flag(d_status, SPO_DEV_ID_OUT_OF_RANGE);
    gl = 0.0f;
  }
  const float ge = g_ent ? g_ent[t] : 0.0f, gs = g_lse ? g_lse[t] : 0.0f;
  const float a = inv_t * (gs - gl - (g_ent ? ge * ent[t] : 0.0f)), b = -inv_t * ge, tgt = inv_t * gl, ls = lse[t];
  const int64_t lo = (int64_t)seg * 4096, hi = lo + 4096 < V ? lo + 4096 : V;
  for (int64_t v = lo + threadIdx.x; v < hi; v += 256) {
    float g = 0.0f;
    if (live) {
      const float u = fmaf(z[v], inv_t, -ls);
      g = expf(u) * fmaf(b, u, a);
      if (v == yt) g += tgt;
    }
    z[v] = g;
  }
}

__global__ void __launch_bounds__(256)
clean_rows_kernel(const uint4* __restrict__ H, int64_t ld_vec, const uint8_t* __restrict__ mask, int64_t t0, int64_t rows,
                  int row_vec, uint4* __restrict__ out) {
  const int lane = threadIdx.x & 31;
  for (int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) >> 5; i < rows; i += ((int64_t)gridDim.x * 256) >> 5) {
    const bool on = mask[t0 + i] != 0;
    for (int k = lane; k < row_vec; k += 32)
      out[i * row_vec + k] = on ? __ldg(H + (t0 + i) * ld_vec + k) : make_uint4(0u, 0u, 0u, 0u);
  }
}

// ---------------------------------------------------------------------------
// scratch
// ---------------------------------------------------------------------------
constexpr int64_t kLpChunkRows = 18944;              // bf16 token rows per contraction launch: bounds the lists' scratch
constexpr size_t kLpLogitBytes = (size_t)512 << 20;  // stored fp32 logits of one chunk of rows (fp32 path)

int64_t pad4(int64_t v) { return (v + 3) / 4 * 4; }

// fp32: rows whose logits are held at a time
int64_t f32_chunk_rows(int64_t T, int32_t V) {
  int64_t rows = (int64_t)(kLpLogitBytes / ((size_t)pad4(V) * 4)) / 64 * 64;
  if (rows < 64) rows = 64;
  return rows < T ? rows : (T > 0 ? T : 1);
}

// Segments of the vocabulary a stored row is reduced in: enough blocks to fill the GPU when the rows are few, at most as
// many as one block merges; a warp's part is a multiple of 32 columns.
void row_segments(int64_t rows, int32_t V, int* nseg, int* part) {
  int64_t want = ceil_div((int64_t)sm_count() * 4, rows);            // segments per row
  if (want > kMergeLists) want = kMergeLists;
  int64_t pt = ceil_div(ceil_div(V, kRowWarps * want), 32) * 32;
  if (want > 1 && pt < 256) pt = 256;                                // no shorter than one step of the loop
  if (pt > 4096 && ceil_div(V, kRowWarps * 4096) <= kMergeLists) pt = 4096;
  *part = (int)pt;
  *nseg = (int)ceil_div(V, kRowWarps * pt);
}

enum : int { LP_STREAM = 0, LP_TILES = 1, LP_F32 = 2 };
struct LpFwdWs { size_t z, partials, tops, cand, progress, total; int64_t chunk, ldz; int path; };

LpFwdWs lp_fwd_layout(int64_t T, int32_t d, int32_t V, int top_k, int32_t dtype) {
  LpFwdWs L{};
  L.path = dtype == SPO_DTYPE_F32 ? LP_F32 : T <= kLpStreamRows ? LP_STREAM : LP_TILES;
  size_t off = 0;
  if (L.path == LP_STREAM) {
    L.chunk = T > 0 ? T : 1;
    int grid, h;
    stream_shape(V, &grid, &h);
    L.partials = off; off = align_up(off + sizeof(FwdPartial) * (size_t)L.chunk * grid, 256);
    L.tops = off;     off = align_up(off + sizeof(float2) * (size_t)L.chunk * grid * (top_k > 0 ? top_k : 1), 256);
  } else if (L.path == LP_F32) {
    L.chunk = f32_chunk_rows(T, V);
    L.ldz = pad4(V);
    // rows x segments: `want` segments a row come to at most 4 SMs' worth + rows, longer rows to one per 32 k columns
    const int64_t segs = (int64_t)sm_count() * 4 + L.chunk * (1 + ceil_div(V, kRowWarps * 4096));
    L.z = off;        off = align_up(off + (size_t)L.chunk * L.ldz * 4, 256);
    L.partials = off; off = align_up(off + sizeof(FwdPartial) * (size_t)segs, 256);
    L.tops = off;     off = align_up(off + sizeof(float2) * (size_t)segs * (top_k > 0 ? top_k : 1), 256);
  } else {
    const int64_t n = ceil_div(T, kLpChunkRows);
    L.chunk = ceil_div(ceil_div(T, n), 256) * 256;               // chunks of like size
    size_t rl = 0;                                               // rows x lists, the largest of a full and of the last chunk
    const int64_t first = T < L.chunk ? T : L.chunk, last = T - (ceil_div(T, L.chunk) - 1) * L.chunk;
    for (int64_t rows : {first, last}) {
      const size_t x = (size_t)rows * lp_fwd_lists(rows, d, V);
      if (x > rl) rl = x;
    }
    const int len = lp_list_len(top_k);
    L.progress = off; off = align_up(off + kProgressBytes, 256);
    L.partials = off; off = align_up(off + sizeof(FwdPartial) * rl, 256);
    L.tops = off;     off = align_up(off + sizeof(float2) * rl * len, 256);
    L.cand = off;     off = align_up(off + (size_t)128 * rl * len, 256);
  }
  L.total = off;
  return L;
}

struct LpBwdWs { size_t g, h_clean, partial, progress, split, total; int64_t chunk, ldg; };

LpBwdWs lp_bwd_layout(int64_t T, int32_t d, int32_t V, int32_t dtype) {
  LpBwdWs L{};
  size_t off = 0;
  if (dtype == SPO_DTYPE_F32) {
    L.chunk = f32_chunk_rows(T, V);
    L.ldg = pad4(V);
    L.g = off;     off = align_up(off + (size_t)L.chunk * L.ldg * 4, 256);
    L.split = off; off = align_up(off + kSplitBytes, 256);
  } else {
    const BwdWs b = bwd_ws_layout(T, d, V);
    L.chunk = b.chunk_rows;
    L.ldg = b.ldg;
    L.g = off;        off = align_up(off + (size_t)L.chunk * L.ldg * 2, 256);
    L.h_clean = off;  off = align_up(off + (size_t)L.chunk * d * 2, 256);
    L.progress = off; off = align_up(off + kProgressBytes, 256);
    L.partial = off;
    if (T > L.chunk) off = align_up(off + (size_t)V * d * 4, 256);
  }
  L.total = off;
  return L;
}

LpOut out_of(const LpFwd& a) {
  LpOut o;
  o.y = a.y; o.mask = a.mask; o.logp = a.logp; o.lse = a.lse; o.entropy = a.entropy;
  o.top_ids = a.top_ids; o.top_logp = a.top_logp;
  o.inv_t = a.inv_t; o.K = a.top_k; o.V = a.V; o.d_status = a.d_status;
  return o;
}

}  // namespace

size_t lp_fwd_ws_bytes(int64_t T, int32_t d, int32_t V, int top_k, int32_t dtype) {
  return lp_fwd_layout(T, d, V, top_k, dtype).total;
}
size_t lp_bwd_ws_bytes(int64_t T, int32_t d, int32_t V, int32_t dtype) { return lp_bwd_layout(T, d, V, dtype).total; }

cudaError_t launch_clean_rows(const void* H, int64_t ldh, const uint8_t* mask, int64_t t0, int64_t rows, int32_t d,
                              void* out, cudaStream_t st) {
  int64_t blocks = ceil_div(rows * 32, 256);
  if (blocks > (int64_t)sm_count() * 16) blocks = (int64_t)sm_count() * 16;
  clean_rows_kernel<<<(unsigned)blocks, 256, 0, st>>>(reinterpret_cast<const uint4*>(H), ldh / 8, mask, t0, rows, d / 8,
                                                      reinterpret_cast<uint4*>(out));
  return cudaGetLastError();
}

cudaError_t lp_forward(const LpFwd& a, char* ws, cudaStream_t st) {
  if (a.T == 0) return cudaSuccess;
  const LpFwdWs L = lp_fwd_layout(a.T, a.d, a.V, a.top_k, a.dtype);
  FwdPartial* partials = reinterpret_cast<FwdPartial*>(ws + L.partials);
  float2* tops = reinterpret_cast<float2*>(ws + L.tops);
  const LpOut o = out_of(a);
  cudaError_t e;
  for (int64_t t0 = 0; t0 < a.T; t0 += L.chunk) {
    const int64_t rows = a.T - t0 < L.chunk ? a.T - t0 : L.chunk;
    if (L.path == LP_TILES) {
      float* cand = reinterpret_cast<float*>(ws + L.cand);
      e = launch_lp_fwd_bf16(a, t0, rows, partials, cand, tops, reinterpret_cast<uint32_t*>(ws + L.progress), st);
      if (e == cudaSuccess)
        e = launch_dependent(lp_merge_kernel<true, 1>, dim3((unsigned)ceil_div(rows, 4)), dim3(128), st, partials,
                             lp_fwd_lists(rows, a.d, a.V), rows, tops, cand, lp_list_len(a.top_k), rows, t0, o);
      if (e != cudaSuccess) return e;
      continue;
    }
    int lists;
    if (L.path == LP_STREAM) {
      int h;
      stream_shape(a.V, &lists, &h);
      e = launch_stream(a, partials, tops, st);
    } else {
      float* Z = reinterpret_cast<float*>(ws + L.z);
      SgemmParams p{};
      p.A = (const float*)a.H + t0 * a.ldh; p.lda = a.ldh; p.M = rows;
      p.B = (const float*)a.W; p.ldb = a.d; p.N = a.V;
      p.K = a.d;
      p.C = Z; p.ldc = L.ldz;
      if ((e = launch_sgemm<true, true>(p, nullptr, st)) != cudaSuccess) return e;
      int part;
      row_segments(rows, a.V, &lists, &part);
      e = launch_dependent(lp_rows_kernel, dim3((unsigned)(rows * lists)), dim3(32 * kRowWarps), st, Z, L.ldz, lists, part, t0, o,
                           partials, tops);
      if (e == cudaSuccess && lists == 1) continue;
    }
    if (e != cudaSuccess) return e;
    e = launch_dependent(lp_merge_kernel<false, 8>, dim3((unsigned)rows), dim3(256), st, partials, lists, (int64_t)0, tops, nullptr,
                         a.top_k, rows, t0, o);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

cudaError_t lp_backward(const LpBwd& a, char* ws, cudaStream_t st) {
  const size_t dw_bytes = (size_t)a.V * a.d * (a.dW_dtype == SPO_DTYPE_BF16 ? 2 : 4);
  if (a.T == 0) return a.accumulate ? cudaSuccess : cudaMemsetAsync(a.dW, 0, dw_bytes, st);
  const LpBwdWs L = lp_bwd_layout(a.T, a.d, a.V, a.dtype);
  if (a.dtype == SPO_DTYPE_BF16)
    return launch_lp_bwd_bf16(a, reinterpret_cast<__nv_bfloat16*>(ws + L.g), L.chunk, L.ldg,
                              reinterpret_cast<float*>(ws + L.partial), ws + L.h_clean,
                              reinterpret_cast<uint32_t*>(ws + L.progress), st);
  float* Z = reinterpret_cast<float*>(ws + L.g);
  float* split = reinterpret_cast<float*>(ws + L.split);
  cudaError_t e;
  for (int64_t t0 = 0; t0 < a.T; t0 += L.chunk) {
    const int64_t rows = a.T - t0 < L.chunk ? a.T - t0 : L.chunk;
    const float* H = (const float*)a.H + t0 * a.ldh;
    SgemmParams p{};
    p.A = H; p.lda = a.ldh; p.M = rows;
    p.B = (const float*)a.W; p.ldb = a.d; p.N = a.V;
    p.K = a.d;
    p.C = Z; p.ldc = L.ldg;
    if ((e = launch_sgemm<true, true>(p, nullptr, st)) != cudaSuccess) return e;
    const int nseg = (int)ceil_div(a.V, 4096);
    lp_g_f32_kernel<<<(unsigned)(rows * nseg), 256, 0, st>>>(Z, L.ldg, nseg, a.V, t0, a.y, a.mask, a.lse, a.ent, a.g_logp,
                                                             a.g_lse, a.g_ent, a.inv_t, a.d_status);
    if ((e = cudaGetLastError()) != cudaSuccess) return e;
    SgemmParams q{};                                           // dH = G W
    q.A = Z; q.lda = L.ldg; q.M = rows;
    q.B = (const float*)a.W; q.ldb = a.d; q.N = a.d;
    q.K = a.V;
    q.C = (float*)a.dH + t0 * a.d; q.ldc = a.d;
    if ((e = launch_sgemm<true, false>(q, split, st)) != cudaSuccess) return e;
    SgemmParams r{};                                           // dW (+)= G^T H
    r.A = Z; r.lda = L.ldg; r.M = a.V;
    r.B = H; r.ldb = a.ldh; r.N = a.d;
    r.K = rows;
    r.C = (float*)a.dW; r.ldc = a.d; r.accumulate = (a.accumulate || t0 > 0) ? 1 : 0;
    r.b_mask = a.mask ? a.mask + t0 : nullptr;
    if ((e = launch_sgemm<false, false>(r, split, st)) != cudaSuccess) return e;
  }
  return cudaSuccess;
}

}  // namespace spo
