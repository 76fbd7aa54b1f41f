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
//                    with 128 rows a tile and the token rows are the narrow one; every CTA keeps the token
//                    rows' statistics under the stream, and where alternatives are wanted the logits of these few
//                    rows go to scratch with the maximum of every 64; lp_pick_kernel finishes.
//   fp32             sgemm_kernel into a chunk of scratch, lp_rows_kernel, and lp_pick_kernel where a row has more
//                    than one block.
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
constexpr int kMaxSegments = 160;                    // parts of the vocabulary that a row's statistics come in

__device__ __forceinline__ void flag(int32_t* d_status, int32_t bit) {
  if (d_status) atomicOr(d_status, bit);
}

// ---------------------------------------------------------------------------
// The K largest of n candidates (value descending, equal values by ascending id), found by a block of TH threads.
// Every TH / 32 threads take the maximum of their share; the K-th largest of these 32 distinct candidates bounds the K-th
// largest of all from below, and usually little more than K candidates reach it (31 for K = 20).  They are collected and
// each counts how many precede it.  No step is a chain of dependent comparisons: for one row of 5000 group maxima the kernel around it
// takes 9 us (two selections and the finish); with sorted lists kept by insertion it took 42.  When more than 256 reach the bound (many equal values, or one thread's
// share holds most of the large ones) the exact bound is found by bisection, first on the value, then on the id.
// ---------------------------------------------------------------------------
constexpr int kTopThreads = 256;
constexpr int kTopKept = 12;
constexpr int kTopFew = 48;
constexpr int kTopRoom = 256;             // candidates that are ranked
static_assert(SPO_MAX_TOP_K <= 32, "the bound is one of 32 maxima");
constexpr int kNoKey = -0x7FFFFFFF - 1;
template <int TH>
struct __align__(16) TopSmem {
  int key[kTopRoom], id[kTopRoom], at[kTopRoom];
  int count[2][TH / 32];
  int n;
  int out_key[kMaxTopK], out_id[kMaxTopK], out_at[kMaxTopK];     // out_key kNoKey: fewer than that many candidates
};

// A float as an integer of the same order (and back: the mapping is its own inverse on the ordered values).
__device__ __forceinline__ int order_key(int b) { return b ^ ((b >> 31) & 0x7FFFFFFF); }
// The same for a logit that may be listed: -0 counts as 0; NaN and -inf are no candidates.
__device__ __forceinline__ int top_key(float x) { return x > -CUDART_INF_F ? order_key(__float_as_int(x + 0.0f)) : kNoKey; }

template <int TH, class Pred>
__device__ __forceinline__ int block_count(int n, Pred pred, TopSmem<TH>& sh, int& buf) {
  int c = 0;
  for (int i = threadIdx.x; i < n; i += TH) c += pred(i) ? 1 : 0;
  c = __reduce_add_sync(0xffffffffu, c);
  if ((threadIdx.x & 31) == 0) sh.count[buf][threadIdx.x >> 5] = c;
  __syncthreads();
  int total = 0;
#pragma unroll
  for (int w = 0; w < TH / 32; ++w) total += sh.count[buf][w];
  buf ^= 1;
  return total;
}

// How many of the first n entries of sh.key / sh.id precede (k, d).
template <int TH>
__device__ __forceinline__ int rank_of(int k, int d, int n, const TopSmem<TH>& sh) {
  int before = 0;
#pragma unroll 4
  for (int q = 0; q < (n + 3) / 4; ++q) {
    const int4 kk = reinterpret_cast<const int4*>(sh.key)[q], dd = reinterpret_cast<const int4*>(sh.id)[q];
    before += (kk.x > k || (kk.x == k && dd.x < d)) + (kk.y > k || (kk.y == k && dd.y < d)) +
              (kk.z > k || (kk.z == k && dd.z < d)) + (kk.w > k || (kk.w == k && dd.w < d));
  }
  return before;
}

// key(i) is candidate i's top_key, id(i) its id (distinct).  Results in sh.out_*, after a barrier; every thread calls it.
template <int TH, class Key, class Id>
__device__ __forceinline__ void block_top(int n, int K, Key key, Id id, TopSmem<TH>& sh) {
  const int tid = threadIdx.x;
  __syncthreads();                                  // the caller is done with what sh held
  if (tid == 0) sh.n = 0;
  if (tid < kMaxTopK) sh.out_key[tid] = kNoKey;
  int bound = kNoKey;
  int kept[kTopKept];                               // the first candidates of this thread, fetched together
  kept[0] = key(min(tid, n - 1));
  if (tid >= n) kept[0] = kNoKey;
  if (n > kTopFew) {
    int m = kept[0];
    if (n > TH) {
#pragma unroll
      for (int u = 1; u < kTopKept; ++u) kept[u] = key(min(tid + u * TH, n - 1));
#pragma unroll
      for (int u = 1; u < kTopKept; ++u) {
        if (tid + u * TH >= n) kept[u] = kNoKey;
        m = max(m, kept[u]);
      }
#pragma unroll 4
      for (int i = tid + kTopKept * TH; i < n; i += TH) m = max(m, key(i));
    }
    sh.key[tid] = m;
    __syncthreads();
    const int lane = tid & 31;
#pragma unroll
    for (int w = 0; w < TH / 32; ++w) m = max(m, sh.key[w * 32 + lane]);     // of the threads of this lane
    int before = 0;
#pragma unroll
    for (int q = 0; q < 32; ++q) {
      const int other = __shfl_sync(0xffffffffu, m, q);
      before += other > m || (other == m && q < lane);
    }
    bound = __shfl_sync(0xffffffffu, m, __ffs(__ballot_sync(0xffffffffu, before == K - 1)) - 1);
    __syncthreads();
  }
  int last_id = 0x7FFFFFFF;                         // of the candidates at the bound, those up to this id count
  auto take = [&](int i, int k) {
    if (k < bound || k == kNoKey) return;
    const int d = id(i);
    if (k == bound && d > last_id) return;
    const int at = atomicAdd(&sh.n, 1);
    if (at < kTopRoom) { sh.key[at] = k; sh.id[at] = d; sh.at[at] = i; }
  };
  auto collect = [&]() {
    take(tid, kept[0]);
    if (n > TH) {
#pragma unroll
      for (int u = 1; u < kTopKept; ++u) take(tid + u * TH, kept[u]);
    }
    for (int i = tid + kTopKept * TH; i < n; i += TH) take(i, key(i));
    __syncthreads();
  };
  if (n > kTopFew) {
    collect();
  } else {                                          // so few that ranking all is less than looking for a bound
    sh.key[tid] = kept[0];
    sh.id[tid] = tid < n ? id(tid) : 0;
    sh.at[tid] = tid;
    if (tid == 0) sh.n = n;
    __syncthreads();
  }
  if (sh.n > kTopRoom) {
    int buf = 0;
    long long lo = bound, hi = 0x7FFFFFFF;          // the largest bound that K candidates reach
    while (lo < hi) {
      const long long mid = lo + (hi - lo + 1) / 2;
      if (block_count(n, [&](int i) { return key(i) >= mid; }, sh, buf) >= K) lo = mid; else hi = mid - 1;
    }
    bound = (int)lo;
    const int want = K - block_count(n, [&](int i) { return key(i) > bound; }, sh, buf);
    lo = 0; hi = 0x7FFFFFFF;
    while (lo < hi) {
      const long long mid = (lo + hi) / 2;
      if (block_count(n, [&](int i) { return key(i) == bound && id(i) <= mid; }, sh, buf) >= want) hi = mid; else lo = mid + 1;
    }
    last_id = (int)lo;
    if (tid == 0) sh.n = 0;
    __syncthreads();
    collect();
  }
  const int total = sh.n;
  if (tid < 4 && total + tid < ((total + 3) & ~3)) sh.key[total + tid] = kNoKey;      // rank_of takes four at a time
  __syncthreads();
  for (int c = tid; c < total; c += TH) {
    const int k = sh.key[c], d = sh.id[c];
    if (k == kNoKey) continue;
    const int before = rank_of(k, d, total, sh);
    if (before < K) { sh.out_key[before] = k; sh.out_id[before] = d; sh.out_at[before] = sh.at[c]; }
  }
  __syncthreads();
}

// The launch before this one in the stream may still be running (programmatic dependent launch): wait for it to
// have finished, and let the next launch come up behind this one.
__device__ __forceinline__ void pdl_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void pdl_trigger() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// (m2, l, ez) of two disjoint parts of a row, joined: m2 in log2 units, l = sum 2^(z sc2 - m2), ez = sum z 2^(...)
__device__ __forceinline__ void join_stats(float& m2, float& l, float& ez, float m2b, float lb, float ezb) {
  const float m = fmaxf(m2, m2b);
  const float wa = m2 == m ? 1.0f : fast_exp2(m2 - m), wb = m2b == m ? 1.0f : fast_exp2(m2b - m);
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

// A token's target and mask, fetched before the work that ends in lp_finish.
struct LpRow {
  int32_t y;
  bool on;
  __device__ __forceinline__ LpRow(const LpOut& o, int64_t t) : y(o.y ? o.y[t] : -1), on(o.mask == nullptr || o.mask[t] != 0) {}
};

// Outputs of token t from its joined statistics and the selected alternatives; one whole warp calls it.
template <int TH>
__device__ __forceinline__ void lp_finish(const LpOut& o, int64_t t, const LpRow& r, float m2, float l, float ez, float zt, bool odd,
                                          const TopSmem<TH>& top, int lane) {
  float lse = (m2 + log2f(l)) * kLn2;
  if (odd) lse = CUDART_NAN_F;
  const bool on = r.on;
  if (lane == 0) {
    if (on && !(fabsf(lse) < CUDART_INF_F)) flag(o.d_status, SPO_DEV_NONFINITE);
    if (o.logp) {
      const int32_t yt = r.y;
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
    const int key = top.out_key[lane];
    const bool found = key != kNoKey;
    o.top_ids[t * o.K + lane] = on && found ? top.out_id[lane] : -1;
    o.top_logp[t * o.K + lane] = !on ? 0.0f : found ? fmaf(__int_as_float(order_key(key)), o.inv_t, -lse) : -CUDART_INF_F;
  }
}

// The K largest logits of a row, from its groups of kGroup columns: the K groups of largest maximum hold them.  Group g covers
// columns (g >> h) tile_h + (g & h) kGroup .., stored from z[(g >> h) pitch + (g & h) kGroup] on, where h = 1 for tiles of
// more than kGroup columns (two groups a tile) and 0 for others; gmax(g) is its maximum as a float (NaN and -inf: nothing in it counts).
constexpr int kGroup = 64;
template <class Gmax>
__device__ __forceinline__ void block_pick(const float* z, int64_t pitch, int groups, int tile_h, int32_t V, int K, Gmax gmax, TopSmem<kTopThreads>& sh,
                                           int* s_key, int* s_id) {
  block_top(groups, K, [&](int g) { return top_key(gmax(g)); }, [](int g) { return g; }, sh);
  constexpr int kSteps = kMaxTopK * kGroup / kTopThreads;
  const int h = tile_h > kGroup ? 1 : 0;
  float x[kSteps];
  int id[kSteps];
#pragma unroll
  for (int u = 0; u < kSteps; ++u) {                // fetched together
    int64_t at = 0;
    const int i = threadIdx.x + u * kTopThreads, q = i / kGroup;
    id[u] = -1;
    if (q < K && sh.out_key[q] != kNoKey) {
      const int g = sh.out_id[q], c = (g & h) * kGroup + i % kGroup;
      if (c < tile_h && (g >> h) * tile_h + c < V) {
        id[u] = (g >> h) * tile_h + c;
        at = (int64_t)(g >> h) * pitch + c;
      }
    }
    x[u] = z[at];
  }
#pragma unroll
  for (int u = 0; u < kSteps; ++u) {
    const int i = threadIdx.x + u * kTopThreads;
    const int to = (i % kGroup) * K + i / kGroup;   // the groups' first columns, then their second ones, .. (shares alike)
    if (i < K * kGroup) { s_key[to] = id[u] < 0 ? kNoKey : top_key(x[u]); s_id[to] = id[u]; }
  }
  block_top(K * kGroup, K, [&](int i) { return s_key[i]; }, [&](int i) { return s_id[i]; }, sh);
}

// ---------------------------------------------------------------------------
// Statistics of stored logit rows and the maxima of their groups of kGroup columns.  Block = (row, segment of the vocabulary);
// each warp takes a contiguous part of `part` columns (a multiple of kGroup).  A block that has the whole row finishes it,
// otherwise it leaves its partial and its groups' maxima to lp_pick_kernel.  Reads every logit once; bound by L2 or HBM.
// ---------------------------------------------------------------------------
constexpr int kRowWarps = kTopThreads / 32;
constexpr int kRowGroups = kRowWarps * 4096 / kGroup;      // groups of a row that one block takes whole

__global__ void __launch_bounds__(32 * kRowWarps)
lp_rows_kernel(const float* __restrict__ Z, int64_t ldz, int nseg, int part, int64_t t0, const LpOut o,
               FwdPartial* __restrict__ partials, float* __restrict__ gmax, int groups) {
  __shared__ TopSmem<kTopThreads> sh;
  __shared__ int s_key[kMaxTopK * kGroup], s_id[kMaxTopK * kGroup];
  __shared__ float s_gmax[kRowGroups];
  __shared__ float s_m[kRowWarps], s_l[kRowWarps], s_e[kRowWarps];
  pdl_trigger();
  pdl_wait();
  const int32_t V = o.V;
  const int K = o.K;
  const float sc2 = kLog2e * o.inv_t;
  const int64_t row = blockIdx.x / nseg;
  const LpRow tr(o, t0 + row);
  const int seg = (int)(blockIdx.x - row * nseg);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const float* z = Z + row * ldz;
  float* gm = nseg == 1 ? s_gmax : gmax + row * groups;
  const int64_t begin = ((int64_t)seg * kRowWarps + warp) * part;
  const int64_t end = begin + part < V ? begin + part : V;
  float m2 = -CUDART_INF_F, l = 0.0f, ez = 0.0f;
  for (int64_t c0 = begin; c0 < end; c0 += 256) {
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int64_t c = c0 + i * 32 + lane;
      x[i] = c < end ? z[c] : -CUDART_INF_F;
    }
    float mx = x[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) mx = fmaxf(mx, x[i]);
    if (K > 0) {
      float mine = 0.0f;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int key = __reduce_max_sync(0xffffffffu, max(top_key(x[2 * i]), top_key(x[2 * i + 1])));
        if (lane == i) mine = key == kNoKey ? -CUDART_INF_F : __int_as_float(order_key(key));
      }
      if (lane < 4 && c0 + lane * kGroup < end) gm[c0 / kGroup + lane] = mine;
    }
    const float mn = fmaxf(fmaxf(m2, mx * sc2), kMaxFloor);  // a lane without columns: exponentials of -inf, not of rounding
    float s = 0.0f, t = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float e = fast_exp2(fmaf(x[i], sc2, -mn));
      s += e;
      t = fmaf(e, fmaxf(x[i], kFarBelow), t);
    }
    const float down = fast_exp2(m2 - mn);
    l = fmaf(l, down, s);
    ez = fmaf(ez, down, t);
    m2 = mn;
  }
  warp_join_stats(m2, l, ez);
  if (lane == 0) { s_m[warp] = m2; s_l[warp] = l; s_e[warp] = ez; }
  __syncthreads();
  if (nseg == 1 && K > 0) block_pick(z, 128, groups, 128, V, K, [&](int g) { return s_gmax[g]; }, sh, s_key, s_id);
  if (warp != 0) return;
  m2 = lane < kRowWarps ? s_m[lane] : -CUDART_INF_F;
  l = lane < kRowWarps ? s_l[lane] : 0.0f;
  ez = lane < kRowWarps ? s_e[lane] : 0.0f;
  const bool odd = __any_sync(0xffffffffu, !(l >= 0.0f));            // a NaN, which fmaxf drops
  warp_join_stats(m2, l, ez);
  if (odd) l = CUDART_NAN_F;
  const int64_t lo = (int64_t)seg * kRowWarps * part, hi = lo + (int64_t)kRowWarps * part;
  const int32_t yt = tr.y;
  const float zt = yt >= lo && yt < hi && yt < V ? z[yt] : -CUDART_INF_F;
  if (nseg == 1) {
    lp_finish(o, t0 + row, tr, m2, l, ez, zt, odd, sh, lane);
  } else if (lane == 0) {
    FwdPartial pt;
    pt.m2 = m2; pt.l = l; pt.pad = ez; pt.zt = zt;
    partials[row * nseg + seg] = pt;
  }
}

// A row's partials, fetched by one warp (at(s) is the place of the s-th) and joined later: the fetch is in flight meanwhile.
struct RowParts {
  float4 p[kMaxSegments / 32];
  template <class At>
  __device__ __forceinline__ void fetch(const FwdPartial* partials, int lists, At at, int lane) {
#pragma unroll
    for (int u = 0; u < kMaxSegments / 32; ++u)
      p[u] = lane + 32 * u < lists ? *reinterpret_cast<const float4*>(partials + at(lane + 32 * u))
                                   : make_float4(-CUDART_INF_F, 0.0f, -CUDART_INF_F, 0.0f);
  }
  __device__ __forceinline__ void join(float& m2, float& l, float& ez, float& zt, bool& odd) const {
    m2 = -CUDART_INF_F; l = 0.0f; ez = 0.0f; zt = -CUDART_INF_F;
    odd = false;                                    // a partial that is NaN: fmaxf would drop it
#pragma unroll
    for (int u = 0; u < kMaxSegments / 32; ++u) {
      odd |= !(p[u].y >= 0.0f);
      zt = p[u].z > -CUDART_INF_F || p[u].z != p[u].z ? p[u].z : zt;   // at most one part has the target
      join_stats(m2, l, ez, p[u].x, p[u].y, p[u].w);
    }
    warp_join_stats(m2, l, ez);
    odd = __any_sync(0xffffffffu, odd);
    const unsigned has = __ballot_sync(0xffffffffu, zt > -CUDART_INF_F || zt != zt);
    zt = has ? __shfl_sync(0xffffffffu, zt, __ffs(has) - 1) : -CUDART_INF_F;
  }
};

// ---------------------------------------------------------------------------
// The end of the tiled path, a block per token row: joins the row's partials ([list][rows]) and picks the alternatives from
// its lists of column groups (maximum, group << 8 | slot), whose 32 logits each are stored in `cand`.
// ---------------------------------------------------------------------------
constexpr int kMergeThreads = 128;        // half of what the others use: many rows with a hundred or two entries each
template <int LIST>
__global__ void __launch_bounds__(kMergeThreads)
lp_merge_kernel(const FwdPartial* __restrict__ partials, int lists, const float2* __restrict__ tops, const float* __restrict__ cand,
                int slots, int64_t rows, int64_t t0, const LpOut o) {
  __shared__ TopSmem<kMergeThreads> sh;
  __shared__ int s_key[kMaxTopK * 32], s_id[kMaxTopK * 32];
  pdl_trigger();
  pdl_wait();
  const int64_t row = blockIdx.x;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, K = o.K;
  const LpRow tr(o, t0 + row);
  RowParts parts;
  if (warp == 0) parts.fetch(partials, lists, [&](int s) { return (int64_t)s * rows + row; }, lane);
  {
    // All lists' first entries, then their second ones, ..: the shares that give the bound are alike that way (list by list,
    // a share would hold the same few places of every list).
    auto entry = [&](int i) {
      const int k = i / lists;
      return tops[((int64_t)(i - k * lists) * rows + row) * LIST + k];
    };
    block_top(lists * LIST, K, [&](int i) { return top_key(entry(i).x); },
              [&](int i) { return (int)(__float_as_uint(entry(i).y) >> 8); }, sh);
    for (int i = threadIdx.x; i < K * 32; i += kMergeThreads) {
      int key = kNoKey, id = 0;
      if (sh.out_key[i >> 5] != kNoKey) {
        const int at = sh.out_at[i >> 5], s = at % lists, slot = (int)(__float_as_uint(entry(at).y) & 255u);
        id = sh.out_id[i >> 5] * 32 + (i & 31);
        if (id < o.V) key = top_key(cand[(((int64_t)s * rows + row) * slots + slot) * 32 + (i & 31)]);
      }
      s_key[(i & 31) * K + (i >> 5)] = key;
      s_id[(i & 31) * K + (i >> 5)] = id;
    }
    block_top(K * 32, K, [&](int i) { return s_key[i]; }, [&](int i) { return s_id[i]; }, sh);
  }
  if (warp != 0) return;
  float m2, l, ez, zt;
  bool odd;
  parts.join(m2, l, ez, zt, odd);
  lp_finish(o, t0 + row, tr, m2, l, ez, zt, odd, sh, lane);
}

// The same for rows of which one warp joins the partials and no alternatives are wanted.
__global__ void __launch_bounds__(128)
lp_join_kernel(const FwdPartial* __restrict__ partials, int lists, int64_t rows, int64_t t0, const LpOut o) {
  __shared__ TopSmem<32> none;                          // not read: K = 0
  pdl_trigger();
  pdl_wait();
  const int lane = threadIdx.x & 31;
  const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5);
  if (row >= rows) return;
  const LpRow tr(o, t0 + row);
  RowParts parts;
  parts.fetch(partials, lists, [&](int s) { return (int64_t)s * rows + row; }, lane);
  float m2, l, ez, zt;
  bool odd;
  parts.join(m2, l, ez, zt, odd);
  lp_finish(o, t0 + row, tr, m2, l, ez, zt, odd, none, lane);
}

// The end of the paths whose logits are stored, a block per token row: joins the row's partials ([row][lists]) and picks the
// alternatives from the maxima of its groups.
__global__ void __launch_bounds__(kTopThreads)
lp_pick_kernel(const FwdPartial* __restrict__ partials, int lists, const float* __restrict__ gmax, int groups, int tile_h,
               const float* __restrict__ Z, int64_t ldz, int64_t pitch, int64_t t0, const LpOut o) {
  __shared__ TopSmem<kTopThreads> sh;
  __shared__ int s_key[kMaxTopK * kGroup], s_id[kMaxTopK * kGroup];
  pdl_trigger();
  pdl_wait();
  const int64_t row = blockIdx.x;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const LpRow tr(o, t0 + row);
  RowParts parts;
  if (warp == 0) parts.fetch(partials, lists, [&](int s) { return row * lists + s; }, lane);
  if (o.K > 0) {
    const float* gm = gmax + row * groups;
    block_pick(Z + row * ldz, pitch, groups, tile_h, o.V, o.K, [&](int g) { return gm[g]; }, sh, s_key, s_id);
  }
  if (warp != 0) return;
  float m2, l, ez, zt;
  bool odd;
  parts.join(m2, l, ez, zt, odd);
  lp_finish(o, t0 + row, tr, m2, l, ez, zt, odd, sh, lane);
}

// ---------------------------------------------------------------------------
// Few bf16 token rows, with W streamed once.  One CTA per SM walks tiles of `tile_h` (at most 128) vocabulary
// rows; TMA brings 64-deep k-blocks of the tile and of all token rows, one MMA per 16 of k with M = 128 vocabulary rows
// and N = NT token rows accumulates in tensor memory (two buffers, so a tile is reduced while the next one
// streams).  W is read once, which is the floor (1.24 GB at d = 4096, V = 151936: 190 us at the measured copy rate); the token
// rows come from L2 once per tile, NT / tile_h of W's traffic.  tile_h is the smallest height that takes the same number of
// rounds over the SMs, so that the last round is full (V = 151936 on 148 SMs: 115 rows x 9 rounds reads 0.8 %
// more than an even share, 128-row tiles would leave the ninth round nearly empty).  Pairs of CTAs on one 256-row tile
// (half the traffic of token rows each) are slower, 207 against 197 us for one row, 217 against 207 for 48.
// Reduction: eight warps turn the finished tile into [token][vocabulary row] in shared memory, then each takes
// the tokens w, w + 8, .., two at a time: a lane holds four logits, the row's maximum and sums are warp reductions, lane k
// keeps the running statistics of the warp's k-th token.  For the alternatives the tile's logits are stored ([tile][token][128]
// fp32, 4 T / (2 d) of W's bytes) with the maxima of their groups of 64; the K largest of a row lie in its K groups of largest
// maximum, which lp_pick_kernel looks up.  (Keeping a sorted list per token row and CTA instead costs a chain of dependent
// shuffles per tile: 128 rows with K = 20 took 438 us that way.)
// ---------------------------------------------------------------------------
struct StreamParams {
  int tiles, tile_h, k_blocks;
  int T;
  int32_t V;
  float sc2;
  const int32_t* y;
  FwdPartial* partials;                      // [T][gridDim.x]
  float* Z;                                  // logits [tiles][T][128] and maxima of their groups [T][tiles x 1 or 2]; NULL: not wanted
  float* gmax;
  int32_t* d_status;
};

constexpr int kStreamWarps = 8;              // reducing warps
constexpr int kStreamThreads = 64 + 32 * kStreamWarps;
constexpr int kStreamA = 128 * 64 * 2;
template <int NT> struct StreamCfg {
  static constexpr int stage_bytes = kStreamA + NT * 128;
  static constexpr int round = NT % 32 != 0 ? 16 : 32;       // tokens reduced at a time
  static constexpr int tile_bytes = round * 128 * 4;         // their logits, [token][128]
  static constexpr int stages = (226 * 1024 - tile_bytes - 2048) / stage_bytes;
  static constexpr int smem = stages * stage_bytes + tile_bytes + 1024 + 512;
  static constexpr int tmem_cols = NT <= 16 ? 32 : NT <= 32 ? 64 : NT <= 64 ? 128 : 256;
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
  constexpr int kBarAt = S * C::stage_bytes + C::tile_bytes;
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
    const int per_tile = p.tile_h > kGroup ? 2 : 1;      // groups of columns
    constexpr int PER = NT / kStreamWarps;               // tokens w, w + 8, .. of this warp; lane k < PER keeps the k-th's state
    float m2 = -CUDART_INF_F, l = 0.0f, ez = 0.0f, zt = -CUDART_INF_F;
    const int my_t = w + kStreamWarps * lane;
    const int32_t my_y = lane < PER && my_t < p.T && p.y ? p.y[my_t] : -1;
    uint32_t n = 0;
    for (int tile = blockIdx.x; tile < p.tiles; tile += gridDim.x, ++n) {
      const uint32_t b = n & 1u;
      int good = 1;
      if (lane == 0) good = mbar_wait<32>(tfull0 + 8 * b, (n >> 1) & 1u, abort_flag, p.d_status) ? 1 : 0;
      good = __shfl_sync(0xffffffffu, good, 0);
      tc_fence_after();
      const uint32_t taddr = tmem_base + ((uint32_t)(quarter * 32) << 16) + b * NT;
      const int v0 = tile * p.tile_h;
      const int cols = p.V - v0 < p.tile_h ? p.V - v0 : p.tile_h;
      bool on = true;
#pragma unroll 1
      for (int r = 0; r < NT / C::round; ++r) {
        if (good) {
#pragma unroll 1
          for (int c = half * 16; c < C::round; c += 32) {               // 16 token columns at a time
            uint32_t x[16];
            tmem_ld16(taddr + r * C::round + c, x);
#pragma unroll
            for (int j = 0; j < 16; ++j) tile_z[(c + j) * 128 + quarter * 32 + lane] = __uint_as_float(x[j]);
            if (p.Z) {                                                    // whole lines, past the tile's last row too
              float* dst = p.Z + ((int64_t)tile * p.T + r * C::round + c) * 128 + quarter * 32 + lane;
#pragma unroll
              for (int j = 0; j < 16; ++j)
                if (r * C::round + c + j < p.T) dst[j * 128] = __uint_as_float(x[j]);
            }
          }
          if (r == NT / C::round - 1) {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_cta(tempty0 + 8 * b);
          }
        }
        on = stream_barrier(good != 0);                                   // the logits are in shared memory
        if (!on) break;
        constexpr int KR = C::round / kStreamWarps;                       // this warp's tokens of the round: 2 or 4
#pragma unroll 1
        for (int k0 = r * KR; k0 < (r + 1) * KR; k0 += 2) {
          if (w + kStreamWarps * k0 >= p.T) break;
          float s[2], u[2], mx[2], mk[2], mn[2];
#pragma unroll
          for (int e = 0; e < 2; ++e) {                                   // (a second token past T has logits of zero rows)
            const float* z = tile_z + (w + kStreamWarps * (k0 + e) - r * C::round) * 128;
            float x[4];
            int key[2];
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = i * 32 + lane < cols ? z[i * 32 + lane] : -CUDART_INF_F;
            if (p.Z) {
#pragma unroll
              for (int i = 0; i < 2; ++i) key[i] = __reduce_max_sync(0xffffffffu, max(top_key(x[2 * i]), top_key(x[2 * i + 1])));
              const int mine = lane == 0 ? key[0] : key[1];
              const int t = w + kStreamWarps * (k0 + e);
              if (lane < per_tile && t < p.T)
                p.gmax[((int64_t)t * p.tiles + tile) * per_tile + lane] = mine == kNoKey ? -CUDART_INF_F : __int_as_float(order_key(mine));
              const int top = max(key[0], key[1]);
              mx[e] = top == kNoKey ? -CUDART_INF_F : __int_as_float(order_key(top));
            } else {
              const float lm = fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3]));
              mx[e] = __int_as_float(order_key(__reduce_max_sync(0xffffffffu, order_key(__float_as_int(lm)))));
            }
            mk[e] = __shfl_sync(0xffffffffu, m2, k0 + e);
            mn[e] = fmaxf(fmaxf(mk[e], mx[e] * p.sc2), kMaxFloor);
            s[e] = u[e] = 0.0f;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const float ex = fast_exp2(fmaf(x[i], p.sc2, -mn[e]));
              s[e] += ex;
              u[e] = fmaf(ex, fmaxf(x[i], kFarBelow), u[e]);
            }
          }
#pragma unroll
          for (int o = 16; o > 0; o >>= 1) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              s[e] += __shfl_xor_sync(0xffffffffu, s[e], o);
              u[e] += __shfl_xor_sync(0xffffffffu, u[e], o);
            }
          }
#pragma unroll
          for (int e = 0; e < 2; ++e)
            if (lane == k0 + e) {
              const float down = fast_exp2(mk[e] - mn[e]);
              l = fmaf(l, down, s[e]);
              ez = fmaf(ez, down, u[e]);
              m2 = mn[e];
              if (my_y >= v0 && my_y < v0 + cols) zt = tile_z[(my_t - r * C::round) * 128 + my_y - v0];
            }
        }
        stream_barrier(true);                                             // they have been read
      }
      if (!on) break;
    }
    if (lane < PER && my_t < p.T) {
      FwdPartial pt;
      pt.m2 = m2; pt.l = l; pt.zt = zt; pt.pad = ez;
      p.partials[(int64_t)my_t * gridDim.x + blockIdx.x] = pt;
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
  const int sms = sm_count() < kMaxSegments ? sm_count() : kMaxSegments;
  const int64_t rounds = ceil_div(V, (int64_t)128 * sms);
  int h = (int)ceil_div(V, rounds * sms);
  if (h < 8) h = 8;
  const int64_t tiles = ceil_div(V, h);
  *tile_h = h;
  *grid = (int)(tiles < sms ? tiles : sms);
}

template <int NT>
cudaError_t launch_stream_t(const LpFwd& a, FwdPartial* partials, float* Z, float* gmax, cudaStream_t st) {
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
  p.V = a.V;
  p.sc2 = kLog2e * a.inv_t;
  p.y = a.y;
  p.partials = partials;
  p.Z = Z;
  p.gmax = gmax;
  p.d_status = a.d_status;
  lp_stream_kernel<NT><<<grid, kStreamThreads, C::smem, st>>>(mW, mH, p);
  return cudaGetLastError();
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

// Z and gmax may be NULL when no alternatives are wanted.
cudaError_t launch_stream(const LpFwd& a, const LpOut& o, FwdPartial* partials, float* Z, float* gmax, cudaStream_t st) {
  if (a.top_k == 0) Z = nullptr;
  cudaError_t e = a.T <= 16   ? launch_stream_t<16>(a, partials, Z, gmax, st)
                  : a.T <= 32 ? launch_stream_t<32>(a, partials, Z, gmax, st)
                  : a.T <= 48 ? launch_stream_t<48>(a, partials, Z, gmax, st)
                  : a.T <= 64 ? launch_stream_t<64>(a, partials, Z, gmax, st)
                  : a.T <= 96 ? launch_stream_t<96>(a, partials, Z, gmax, st)
                              : launch_stream_t<128>(a, partials, Z, gmax, st);
  if (e != cudaSuccess) return e;
  int grid, h;
  stream_shape(a.V, &grid, &h);
  return launch_dependent(lp_pick_kernel, dim3((unsigned)a.T), dim3(kTopThreads), st, partials, grid, gmax, (h > kGroup ? 2 : 1) * (int)ceil_div(a.V, h),
                          h, Z, (int64_t)128, a.T * 128, (int64_t)0, o);
}

// ---------------------------------------------------------------------------
// fp32 matrix product on the fp32 pipes: C[m][n] (+)= sum_k A(m,k) B(n,k).  A_K / B_K: the operand is
// contiguous along k, else along m / n.  Tiles of TILE x TILE x 16, PT x PT results a thread; the next k-block is fetched into registers while this one is multiplied.  gridDim.z splits k:
// each split writes its own C (stride M * ldc) and sum_splits_kernel adds them in a fixed order.  GRAD: the results are
// logits, and their gradient is stored in their place (the formula of g_values_lp, with log p in nats).
// ---------------------------------------------------------------------------
struct GradParams {
  const int32_t* y;                 // all by row of C
  const uint8_t* mask;
  const float *lse, *ent, *g_logp, *g_lse, *g_ent;
  float inv_t;
  int32_t V;
  int32_t* d_status;
};
struct SgemmParams {
  const float *A, *B;
  int64_t lda, ldb, ldc, M, N, K, k_per;
  float* C;
  int accumulate;
  const uint8_t* b_mask;            // k rows whose B is taken as zero where the mask is 0 (B contiguous along n)
  GradParams grad;
};

// One thread's share of an operand's k-blocks: where its float4s come from, advanced block by block.
template <int TILE, bool KC, int LOADS, int THREADS>
struct SgOperand {
  const float* at[LOADS];
  int k[LOADS], live[LOADS];        // k within a block; KC: whether the row exists, else how many of the four columns do
  int64_t step, ld;
  __device__ __forceinline__ void init(const float* X, int64_t ld_, int64_t row0, int64_t rows, int64_t k0) {
    ld = ld_;
    step = KC ? 16 : 16 * ld;
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int idx = threadIdx.x + i * THREADS;
      const int64_t m = row0 + (KC ? idx >> 2 : (idx % (TILE / 4)) * 4);
      k[i] = KC ? (idx & 3) * 4 : idx / (TILE / 4);
      live[i] = KC ? (m < rows ? 1 : 0) : m + 3 < rows ? 4 : m < rows ? (int)(rows - m) : 0;
      at[i] = live[i] ? (KC ? X + m * ld + k0 + k[i] : X + (k0 + k[i]) * ld + m) : X;
    }
  }
  // The block whose first k is k0 (left = k_end - k0 > 0), then on to the next.
  __device__ __forceinline__ void fetch(float4 (&r)[LOADS], int64_t k0, int64_t left, const uint8_t* kmask) {
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      r[i] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      const int n = KC ? (live[i] == 0 || left <= k[i] ? 0 : left - k[i] >= 4 ? 4 : (int)(left - k[i]))
                       : (left <= k[i] || (kmask != nullptr && kmask[k0 + k[i]] == 0) ? 0 : live[i]);
      if (n == 4) {
        r[i] = *reinterpret_cast<const float4*>(at[i]);
      } else if (n > 0) {
        r[i].x = at[i][0];
        if (n > 1) r[i].y = at[i][1];
        if (n > 2) r[i].z = at[i][2];
      }
      at[i] += step;
    }
  }
  __device__ __forceinline__ void store(float (*s)[TILE + 4], const float4 (&r)[LOADS]) const {
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int idx = threadIdx.x + i * THREADS;
      if (KC) {
        const int m = idx >> 2, kk = (idx & 3) * 4;
        s[kk][m] = r[i].x; s[kk + 1][m] = r[i].y; s[kk + 2][m] = r[i].z; s[kk + 3][m] = r[i].w;
      } else {
        *reinterpret_cast<float4*>(&s[idx / (TILE / 4)][(idx % (TILE / 4)) * 4]) = r[i];
      }
    }
  }
};
// Two fused multiply-adds in one instruction: (x0, x1) += a (b0, b1), each rounded like fmaf.
__device__ __forceinline__ void ffma2(uint64_t& acc, uint64_t a, uint64_t b) {
  asm("fma.rn.f32x2 %0, %1, %2, %0;" : "+l"(acc) : "l"(a), "l"(b));
}
__device__ __forceinline__ uint64_t pair(float lo, float hi) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}

template <int TILE, int PT, bool A_K, bool B_K, bool GRAD>
__global__ void __launch_bounds__((TILE / PT) * (TILE / PT), TILE == 128 ? 2 : 4)
sgemm_kernel(const SgemmParams p) {
  constexpr int R = PT / 4;                          // groups of four rows (columns) per thread, APART apart
  constexpr int APART = TILE / R;
  constexpr int SIDE = TILE / PT, THREADS = SIDE * SIDE;
  constexpr int LOADS = TILE * 16 / 4 / THREADS;
  __shared__ __align__(16) float As[2][16][TILE + 4], Bs[2][16][TILE + 4];
  const int tx = threadIdx.x % SIDE, ty = threadIdx.x / SIDE;
  const int64_t m0 = (int64_t)blockIdx.x * TILE, n0 = (int64_t)blockIdx.y * TILE;
  const int64_t k_begin = (int64_t)blockIdx.z * p.k_per;
  const int64_t k_end = k_begin + p.k_per < p.K ? k_begin + p.k_per : p.K;
  uint64_t acc2[4 * R][2 * R] = {};                  // pairs of neighbouring columns
  pdl_trigger();
  pdl_wait();
  SgOperand<TILE, A_K, LOADS, THREADS> oa;
  SgOperand<TILE, B_K, LOADS, THREADS> ob;
  oa.init(p.A, p.lda, m0, p.M, k_begin);
  ob.init(p.B, p.ldb, n0, p.N, k_begin);
  float4 ra[LOADS], rb[LOADS];
  oa.fetch(ra, k_begin, k_end - k_begin, nullptr);
  ob.fetch(rb, k_begin, k_end - k_begin, p.b_mask);
  int buf = 0;
  for (int64_t k0 = k_begin; k0 < k_end; k0 += 16, buf ^= 1) {
    oa.store(As[buf], ra);
    ob.store(Bs[buf], rb);
    __syncthreads();
    if (k0 + 16 < k_end) {
      oa.fetch(ra, k0 + 16, k_end - k0 - 16, nullptr);
      ob.fetch(rb, k0 + 16, k_end - k0 - 16, p.b_mask);
    }
#pragma unroll
    for (int k = 0; k < 16; ++k) {
      float a[4 * R];
      uint64_t b[2 * R];
#pragma unroll
      for (int r = 0; r < R; ++r) {
        *reinterpret_cast<float4*>(a + 4 * r) = *reinterpret_cast<const float4*>(&As[buf][k][ty * 4 + APART * r]);
        const ulonglong2 bb = *reinterpret_cast<const ulonglong2*>(&Bs[buf][k][tx * 4 + APART * r]);
        b[2 * r] = bb.x;
        b[2 * r + 1] = bb.y;
      }
#pragma unroll
      for (int i = 0; i < 4 * R; ++i) {
        const uint64_t aa = pair(a[i], a[i]);
#pragma unroll
        for (int j = 0; j < 2 * R; ++j) ffma2(acc2[i][j], aa, b[j]);
      }
    }
  }
  float acc[4 * R][4 * R];
#pragma unroll
  for (int i = 0; i < 4 * R; ++i)
#pragma unroll
    for (int j = 0; j < 2 * R; ++j)
      asm("mov.b64 {%0, %1}, %2;" : "=f"(acc[i][2 * j]), "=f"(acc[i][2 * j + 1]) : "l"(acc2[i][j]));
  float* C = p.C + (int64_t)blockIdx.z * p.M * p.ldc;
#pragma unroll
  for (int i = 0; i < 4 * R; ++i) {
    const int64_t m = m0 + ty * 4 + (i & 3) + APART * (i >> 2);
    if (m >= p.M) continue;
    bool live = true;
    float a = 0.0f, b = 0.0f, tgt = 0.0f, ls = 0.0f;
    int32_t yt = -1;
    if (GRAD) {
      const GradParams& g = p.grad;
      live = g.mask == nullptr || g.mask[m] != 0;
      float gl = g.g_logp ? g.g_logp[m] : 0.0f;
      yt = g.y ? g.y[m] : -1;
      if (g.g_logp && (yt < 0 || yt >= g.V)) {               // no such target: its log-prob is the constant -inf
        if (live && blockIdx.y == 0 && tx == 0) flag(g.d_status, SPO_DEV_ID_OUT_OF_RANGE);
        gl = 0.0f;
      }
      const float ge = g.g_ent ? g.g_ent[m] : 0.0f, gs = g.g_lse ? g.g_lse[m] : 0.0f;
      a = g.inv_t * (gs - gl - (g.g_ent ? ge * g.ent[m] : 0.0f));
      b = -g.inv_t * ge;
      tgt = g.inv_t * gl;
      ls = g.lse[m];
    }
#pragma unroll
    for (int j = 0; j < 4 * R; ++j) {
      const int64_t n = n0 + tx * 4 + (j & 3) + APART * (j >> 2);
      if (n >= p.N) continue;
      float* dst = C + m * p.ldc + n;
      if (GRAD) {
        float v = 0.0f;
        if (live) {
          const float u = fmaf(acc[i][j], p.grad.inv_t, -ls);
          v = expf(u) * fmaf(b, fmaxf(u, kNoChance), a);
          if (n == yt) v += tgt;
        }
        *dst = v;
      } else {
        *dst = p.accumulate ? *dst + acc[i][j] : acc[i][j];
      }
    }
  }
}

// out[i] (+)= sum of the splits' results, in order; blockIdx.y selects one of two sums.
struct SplitSum { const float* parts; int splits; int64_t n; float* out; int accumulate; };
__global__ void __launch_bounds__(256)
sum_splits_kernel(const SplitSum s0, const SplitSum s1) {
  pdl_trigger();
  pdl_wait();
  const SplitSum& s = blockIdx.y == 0 ? s0 : s1;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < s.n; i += (int64_t)gridDim.x * 256) {
    float x = s.accumulate ? s.out[i] : 0.0f;
#pragma unroll 4
    for (int z = 0; z < s.splits; ++z) x += s.parts[(int64_t)z * s.n + i];
    s.out[i] = x;
  }
}

constexpr int kSplitBlocks = 444;                              // blocks that a split of k fills the GPU with
constexpr size_t kSplitBytes = (size_t)kSplitBlocks * 128 * 128 * 4;   // room for all splits' results together

// `sum` (NULL: k is not split): receives what is left to be summed, n = 0 for nothing.  `first`: the first launch of a call.
template <bool A_K, bool B_K, bool GRAD = false>
cudaError_t launch_sgemm(SgemmParams p, bool first, float* split_ws, SplitSum* sum, cudaStream_t st) {
  const int64_t big = ceil_div(p.M, 128) * ceil_div(p.N, 128);
  const int tile = big >= sm_count() ? 128 : 64;               // 64: four times the blocks where 128 leaves SMs idle
  const int64_t bm = ceil_div(p.M, tile), bn = ceil_div(p.N, tile);
  int64_t splits = 1;
  if (sum && p.ldc == p.N && bm * bn < 2 * sm_count()) {
    splits = kSplitBlocks / (bm * bn);
    const int64_t most = ceil_div(p.K, 128);                   // at least 8 k-blocks a split
    if (splits > most) splits = most;
    while (splits > 1 && (size_t)splits * p.M * p.N * 4 > kSplitBytes) --splits;
    if (splits < 1) splits = 1;
  }
  p.k_per = ceil_div(ceil_div(p.K, 16), splits) * 16;
  splits = ceil_div(p.K, p.k_per);
  if (bn > 65535 || splits > 65535) return cudaErrorInvalidConfiguration;
  if (sum) *sum = SplitSum{split_ws, (int)splits, splits > 1 ? p.M * p.N : 0, p.C, p.accumulate};
  if (splits > 1) { p.C = split_ws; p.accumulate = 0; }
  const dim3 grid((unsigned)bm, (unsigned)bn, (unsigned)splits);
  // 64-wide tiles: 8 x 8 results a thread (half the shared-memory reads per product) when the blocks fill the GPU,
  // 4 x 4 and four times the threads when they do not and a block's own latency counts
  const bool fat = tile == 128 || bm * bn * splits >= sm_count();
  auto kern = tile == 128 ? sgemm_kernel<128, 8, A_K, B_K, GRAD>
              : fat       ? sgemm_kernel<64, 8, A_K, B_K, GRAD>
                          : sgemm_kernel<64, 4, A_K, B_K, GRAD>;
  const dim3 block(tile == 64 && fat ? 64 : 256);
  if (first) {
    kern<<<grid, block, 0, st>>>(p);
    return cudaGetLastError();
  }
  return launch_dependent(kern, grid, block, st, p);
}

// What follows the logit gradient of a chunk in bf16 (see TargetRest).  The first `sum_blocks` blocks add the parts of dH and
// the tokens' rests; each of the others has a token, and if no earlier token has its target, sums rest H over all that do,
// in their order.  Finding them is a scan of the chunk's targets by every block: 9472 tokens, the most there are, take 5 rounds of
// 2048, and nothing has to be sorted or counted first.  A target's tokens follow one another in its block, so common targets cost: with
// uniform ones, Zipf's and one for all the backward takes 86, 92 and 190 us for 203 rows (d = 1024, V = 32000), 25.9, 27.1 and 34.0 ms
// for 9472 (d = 4096, V = 151936).  The last `clean_blocks` blocks copy H with zeros in the masked rows: their
// gradient is zero, but zero times a NaN is not.  203 rows, d = 1024: 8.5 us, 13 as two launches.
struct RestParams {
  const float4* src;
  int parts, sum_blocks, token_blocks, clean_blocks;
  uint32_t quads, row_quads;               // float4s of dH, and of a row
  void* dh;
  const uint2* W;
  const __nv_bfloat16* H;
  int64_t ldh;
  int32_t rows, d, V;
  TargetRest r;
  float* dw;
  const uint8_t* mask;
  uint4* clean;
};
__device__ __forceinline__ int32_t rest_target(const RestParams& p, int32_t t) {
  const int32_t y = p.r.y[t];
  return y >= 0 && y < p.V && (p.r.mask == nullptr || p.r.mask[t] != 0) ? y : -1;
}

template <bool BF16>
__global__ void __launch_bounds__(256)
lp_rest_kernel(const RestParams p) {
  if ((int)blockIdx.x < p.sum_blocks) {
    for (uint32_t i = blockIdx.x * 256u + threadIdx.x; i < p.quads; i += (uint32_t)p.sum_blocks * 256u) {
      float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 4
      for (int z = 0; z < p.parts; ++z) {
        const float4 x = p.src[(int64_t)z * p.quads + i];
        s.x += x.x; s.y += x.y; s.z += x.z; s.w += x.w;
      }
      if (p.r.rest) {
        const uint32_t t = i / p.row_quads;
        const int32_t y = rest_target(p, (int32_t)t);
        const float r = y >= 0 ? p.r.rest[t] : 0.0f;
        if (r != 0.0f) {
          const uint2 w = __ldg(p.W + (int64_t)y * p.row_quads + (i - t * p.row_quads));
          s.x = fmaf(r, __uint_as_float(w.x << 16), s.x);
          s.y = fmaf(r, __uint_as_float(w.x & 0xFFFF0000u), s.y);
          s.z = fmaf(r, __uint_as_float(w.y << 16), s.z);
          s.w = fmaf(r, __uint_as_float(w.y & 0xFFFF0000u), s.w);
        }
      }
      if (BF16) reinterpret_cast<uint2*>(p.dh)[i] = make_uint2(pack_bf16(s.x, s.y), pack_bf16(s.z, s.w));
      else reinterpret_cast<float4*>(p.dh)[i] = s;
    }
    return;
  }
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int32_t t = (int32_t)blockIdx.x - p.sum_blocks;
  if (t >= p.token_blocks) {
    const int32_t row_vec = p.d / 8;
    for (int64_t i = (int64_t)(t - p.token_blocks) * 8 + warp; i < p.rows; i += (int64_t)p.clean_blocks * 8) {
      const bool on = p.mask[i] != 0;
      const uint4* src = reinterpret_cast<const uint4*>(p.H + i * p.ldh);
#pragma unroll 4
      for (int32_t k = lane; k < row_vec; k += 32) p.clean[i * row_vec + k] = on ? __ldg(src + k) : make_uint4(0u, 0u, 0u, 0u);
    }
    return;
  }
  __shared__ uint32_t found[64];
  const int32_t y = rest_target(p, t);
  if (y < 0) return;
  for (int32_t c0 = 0; c0 < p.d; c0 += 2048) {
    const int32_t c = c0 + (int32_t)threadIdx.x * 8;
    float acc[8] = {};
    for (int32_t t0 = 0; t0 < p.rows; t0 += 2048) {
      int32_t ys[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const int32_t i = t0 + k * 256 + (int32_t)threadIdx.x;
        ys[k] = i < p.rows ? __ldg(p.r.y + i) : -1;
      }
      bool any = false, earlier = false;
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const int32_t i = t0 + k * 256 + (int32_t)threadIdx.x;
        const bool hit = ys[k] == y && (p.r.mask == nullptr || p.r.mask[i] != 0);
        earlier = earlier || (hit && i < t);
        any = any || hit;
        const uint32_t b = __ballot_sync(0xffffffffu, hit);
        if (lane == 0) found[k * 8 + warp] = b;
      }
      if (__syncthreads_or(earlier)) return;
      if (__syncthreads_or(any)) {
        const uint32_t lo = __ballot_sync(0xffffffffu, found[lane] != 0), hi = __ballot_sync(0xffffffffu, found[32 + lane] != 0);
        for (uint64_t words = (uint64_t)hi << 32 | lo; words != 0; words &= words - 1) {
          const int q = __ffsll((long long)words) - 1;
          for (uint32_t b = found[q]; b != 0; b &= b - 1) {
            const int32_t i = t0 + q * 32 + __ffs(b) - 1;
            const float r = p.r.rest[i];
            if (r == 0.0f || c >= p.d) continue;
            const uint4 h = __ldg(reinterpret_cast<const uint4*>(p.H + (int64_t)i * p.ldh + c));
            const uint32_t x[4] = {h.x, h.y, h.z, h.w};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              acc[2 * k] = fmaf(r, __uint_as_float(x[k] << 16), acc[2 * k]);
              acc[2 * k + 1] = fmaf(r, __uint_as_float(x[k] & 0xFFFF0000u), acc[2 * k + 1]);
            }
          }
        }
        __syncthreads();
      }
    }
    if (c < p.d) {
      if (p.dw) {
        float4* dst = reinterpret_cast<float4*>(p.dw + (int64_t)y * p.d + c);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          float4 v = dst[h];
          v.x += acc[4 * h]; v.y += acc[4 * h + 1]; v.z += acc[4 * h + 2]; v.w += acc[4 * h + 3];
          dst[h] = v;
        }
      } else {
        *reinterpret_cast<uint4*>(p.r.rows + (int64_t)t * p.d + c) =
            make_uint4(pack_bf16(acc[0], acc[1]), pack_bf16(acc[2], acc[3]), pack_bf16(acc[4], acc[5]), pack_bf16(acc[6], acc[7]));
      }
    }
  }
  if (p.dw == nullptr && threadIdx.x == 0) p.r.slot[y] = t;
}

// ---------------------------------------------------------------------------
// scratch
// ---------------------------------------------------------------------------
constexpr int64_t kLpChunkRows = 18944;              // bf16 token rows per contraction launch: bounds the lists' scratch
constexpr size_t kLpLogitBytes = (size_t)256 << 20;  // stored fp32 logits of one chunk of rows (fp32 path)

int64_t pad4(int64_t v) { return (v + 3) / 4 * 4; }

// fp32: rows whose logits are held at a time
int64_t f32_chunk_rows(int64_t T, int32_t V) {
  int64_t rows = (int64_t)(kLpLogitBytes / ((size_t)pad4(V) * 4)) / 64 * 64;
  if (rows < 64) rows = 64;
  return rows < T ? rows : (T > 0 ? T : 1);
}

// Segments of the vocabulary a stored row is reduced in: enough blocks to fill the GPU when the rows are few; a warp's part is
// a multiple of kGroup columns.
void row_segments(int64_t rows, int32_t V, int* nseg, int* part) {
  int64_t want = ceil_div((int64_t)sm_count() * 4, rows);            // segments per row
  if (want > kMaxSegments) want = kMaxSegments;
  int64_t pt = ceil_div(ceil_div(V, kRowWarps * want), kGroup) * kGroup;
  if (want > 1 && pt < 256) pt = 256;                                // no shorter than one step of the loop
  if (pt > 4096 && ceil_div(V, kRowWarps * 4096) <= kMaxSegments) pt = 4096;
  *part = (int)pt;
  *nseg = (int)ceil_div(V, kRowWarps * pt);
}

enum : int { LP_STREAM = 0, LP_TILES = 1, LP_F32 = 2 };
struct LpFwdWs { size_t z, partials, tops, cand, progress, total; int64_t chunk, ldz; int path; };

struct LpLists { size_t rl, rs; };        // rows x lists, rows x lists x slots of one launch of the tiled path
LpLists lp_lists(int64_t rows, int32_t d, int32_t V, int top_k) {
  const int lists = lp_fwd_lists(rows, d, V);
  return {(size_t)rows * lists, (size_t)rows * lists * lp_fwd_slots(lists, d, V, top_k)};
}
void lp_lists_layout(LpFwdWs& L, size_t rl, size_t rs, int top_k) {
  size_t off = 0;
  L.progress = off; off = align_up(off + kProgressBytes, 256);
  L.partials = off; off = align_up(off + sizeof(FwdPartial) * rl, 256);
  L.tops = off;     off = align_up(off + sizeof(float2) * rl * lp_list_len(top_k), 256);
  L.cand = off;     off = align_up(off + (size_t)128 * rs, 256);
  L.total = off;
}

LpFwdWs lp_fwd_layout(int64_t T, int32_t d, int32_t V, int top_k, int32_t dtype) {
  LpFwdWs L{};
  L.path = dtype == SPO_DTYPE_F32 ? LP_F32 : T <= kLpStreamRows ? LP_STREAM : LP_TILES;
  size_t off = 0;
  if (L.path == LP_STREAM) {
    L.chunk = T > 0 ? T : 1;
    int grid, h;
    stream_shape(V, &grid, &h);
    L.partials = off; off = align_up(off + sizeof(FwdPartial) * (size_t)L.chunk * grid, 256);
    L.ldz = ceil_div(V, h) * 128;                                // a tile's logits on whole lines, behind one another
    L.z = L.tops = off;
    if (top_k > 0) {
      off = align_up(off + (size_t)L.chunk * L.ldz * 4, 256);
      L.tops = off;   off = align_up(off + (size_t)L.chunk * ceil_div(V, h) * 8, 256);
    }
  } else if (L.path == LP_F32) {
    L.chunk = f32_chunk_rows(T, V);
    L.ldz = pad4(V);
    // rows x segments: `want` segments a row come to at most 4 SMs' worth + rows, longer rows to one per 32 k columns
    const int64_t segs = (int64_t)sm_count() * 4 + L.chunk * (1 + ceil_div(V, kRowWarps * 4096));
    L.z = off;        off = align_up(off + (size_t)L.chunk * L.ldz * 4, 256);
    L.partials = off; off = align_up(off + sizeof(FwdPartial) * (size_t)segs, 256);
    L.tops = off;
    if (top_k > 0) off = align_up(off + (size_t)L.chunk * ceil_div(V, kGroup) * 4, 256);      // maxima of the groups
  } else {
    const int64_t n = ceil_div(T, kLpChunkRows);
    L.chunk = ceil_div(ceil_div(T, n), 256) * 256;               // chunks of like size
    size_t rl = 0, rs = 0;                                       // rows x lists, and x slots: the largest of a full and of the last chunk
    const int64_t first = T < L.chunk ? T : L.chunk, last = T - (ceil_div(T, L.chunk) - 1) * L.chunk;
    for (int64_t rows : {first, last}) {
      const LpLists x = lp_lists(rows, d, V, top_k);
      if (x.rl > rl) rl = x.rl;
      if (x.rs > rs) rs = x.rs;
    }
    lp_lists_layout(L, rl, rs, top_k);
    return L;
  }
  L.total = off;
  return L;
}

struct LpBwdWs { size_t g, h_clean, partial, progress, split, rest, slot, rest_rows, total; int64_t chunk, ldg; };

LpBwdWs lp_bwd_layout(int64_t T, int32_t d, int32_t V, int32_t dtype) {
  LpBwdWs L{};
  size_t off = 0;
  if (dtype == SPO_DTYPE_F32) {
    L.chunk = f32_chunk_rows(T, V);
    L.ldg = pad4(V);
    L.g = off;     off = align_up(off + (size_t)L.chunk * L.ldg * 4, 256);
    L.split = off; off = align_up(off + 2 * kSplitBytes, 256);           // of dH and of dW
  } else {
    const BwdWs b = bwd_ws_layout(T, d, V);
    L.chunk = b.chunk_rows;
    L.ldg = b.ldg;
    L.g = off;        off = align_up(off + (size_t)L.chunk * L.ldg * 2, 256);
    L.h_clean = off;  off = align_up(off + (size_t)L.chunk * d * 2, 256);
    L.progress = off; off = align_up(off + kProgressBytes, 256);
    L.partial = off;
    if (T > L.chunk) off = align_up(off + (size_t)V * d * 4, 256);
    const int64_t t_eff = T > 0 ? T : 1, first = t_eff < L.chunk ? t_eff : L.chunk;
    L.split = off; off = align_up(off + lp_dh_split_bytes(first, d), 256);
    L.rest = off;      off = align_up(off + (size_t)first * 4, 256);
    L.slot = off;      off = align_up(off + (size_t)V * 4, 256);
    L.rest_rows = off; off = align_up(off + (size_t)first * d * 2, 256);
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
// The tiled path's lists are not monotone in the rows (d = 4096, V = 151936, K = 20: 3840 rows take 693 MB, 8192 take 403: the
// fewer the row tiles, the finer the vocabulary is split), so the bound takes every number of row tiles that a launch can have.
size_t lp_fwd_ws_bound(int64_t T, int32_t d, int32_t V, int top_k, int32_t dtype) {
  if (dtype == SPO_DTYPE_F32 || T <= kLpStreamRows) return lp_fwd_layout(T, d, V, top_k, dtype).total;   // these grow with the rows
  size_t rl = 0, rs = 0;
  for (int64_t rows = 256; rows < kLpChunkRows + 256; rows += 256) {
    const LpLists x = lp_lists(rows < T ? rows : T, d, V, top_k);    // (full row tiles: the splits depend on their number alone)
    if (x.rl > rl) rl = x.rl;
    if (x.rs > rs) rs = x.rs;
    if (rows >= T) break;
  }
  LpFwdWs L{};
  lp_lists_layout(L, rl, rs, top_k);
  const size_t few = lp_fwd_layout(kLpStreamRows, d, V, top_k, dtype).total;
  return L.total > few ? L.total : few;
}
size_t lp_bwd_ws_bytes(int64_t T, int32_t d, int32_t V, int32_t dtype) { return lp_bwd_layout(T, d, V, dtype).total; }

cudaError_t launch_lp_rest(const float* src, int parts, int64_t rows, int32_t d, int32_t V, void* dh, int32_t dh_dtype,
                           const void* W, const void* H, int64_t ldh, const TargetRest& rest, bool targets, float* dw,
                           const uint8_t* mask, void* clean, cudaStream_t st) {
  RestParams p{};
  p.src = reinterpret_cast<const float4*>(src);
  p.parts = parts;
  if (parts > 0) {
    p.quads = (uint32_t)(rows * d / 4);
    const int64_t blocks = ceil_div(p.quads, 256), most = (int64_t)sm_count() * 8;
    p.sum_blocks = (int)(blocks < most ? blocks : most);
  }
  p.row_quads = (uint32_t)d / 4;
  p.dh = dh;
  p.W = reinterpret_cast<const uint2*>(W);
  p.H = reinterpret_cast<const __nv_bfloat16*>(H); p.ldh = ldh;
  p.rows = (int32_t)rows; p.d = d; p.V = V;
  p.r = rest;
  p.dw = dw;
  p.token_blocks = targets && rest.rest ? (int)rows : 0;
  p.mask = mask;
  p.clean = reinterpret_cast<uint4*>(clean);
  if (clean) {
    const int64_t want = ceil_div(rows, 8), most = (int64_t)sm_count() * 16;
    p.clean_blocks = (int)(want < most ? want : most);
  }
  const int blocks = p.sum_blocks + p.token_blocks + p.clean_blocks;
  if (blocks == 0) return cudaSuccess;
  if (dh_dtype == SPO_DTYPE_BF16) lp_rest_kernel<true><<<(unsigned)blocks, 256, 0, st>>>(p);
  else lp_rest_kernel<false><<<(unsigned)blocks, 256, 0, st>>>(p);
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
      const int lists = lp_fwd_lists(rows, a.d, a.V);
      if (e == cudaSuccess && a.top_k == 0)
        e = launch_dependent(lp_join_kernel, dim3((unsigned)ceil_div(rows, 4)), dim3(128), st, partials, lists, rows, t0, o);
      else if (e == cudaSuccess)
        e = launch_dependent(lp_list_len(a.top_k) == 8 ? lp_merge_kernel<8> : lp_merge_kernel<kMaxTopK>, dim3((unsigned)rows),
                             dim3(kMergeThreads), st, partials, lists, tops, cand, lp_fwd_slots(lists, a.d, a.V, a.top_k), rows, t0, o);
      if (e != cudaSuccess) return e;
      continue;
    }
    if (L.path == LP_STREAM)
      return launch_stream(a, o, partials, reinterpret_cast<float*>(ws + L.z), reinterpret_cast<float*>(ws + L.tops), st);
    float* Z = reinterpret_cast<float*>(ws + L.z);
    SgemmParams p{};
    p.A = (const float*)a.H + t0 * a.ldh; p.lda = a.ldh; p.M = rows;
    p.B = (const float*)a.W; p.ldb = a.d; p.N = a.V;
    p.K = a.d;
    p.C = Z; p.ldc = L.ldz;
    if ((e = launch_sgemm<true, true>(p, t0 == 0, nullptr, nullptr, st)) != cudaSuccess) return e;
    int lists, part;
    row_segments(rows, a.V, &lists, &part);
    float* gmax = reinterpret_cast<float*>(ws + L.tops);
    const int groups = (int)ceil_div(a.V, kGroup);
    e = launch_dependent(lp_rows_kernel, dim3((unsigned)(rows * lists)), dim3(32 * kRowWarps), st, Z, L.ldz, lists, part, t0, o,
                         partials, gmax, groups);
    if (e == cudaSuccess && lists > 1)
      e = launch_dependent(lp_pick_kernel, dim3((unsigned)rows), dim3(kTopThreads), st, partials, lists, gmax, groups, 128, Z, L.ldz,
                           (int64_t)128, t0, o);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

cudaError_t lp_backward(const LpBwd& a, char* ws, cudaStream_t st) {
  const size_t dw_bytes = (size_t)a.V * a.d * (a.dW_dtype == SPO_DTYPE_BF16 ? 2 : 4);
  if (a.T == 0) return a.accumulate ? cudaSuccess : cudaMemsetAsync(a.dW, 0, dw_bytes, st);
  const LpBwdWs L = lp_bwd_layout(a.T, a.d, a.V, a.dtype);
  if (a.dtype == SPO_DTYPE_BF16) {
    LpBwdScratch w{};
    w.g = reinterpret_cast<__nv_bfloat16*>(ws + L.g);
    w.chunk = L.chunk; w.ldg = L.ldg;
    w.partial = reinterpret_cast<float*>(ws + L.partial);
    w.h_clean = ws + L.h_clean;
    w.split = reinterpret_cast<float*>(ws + L.split);
    w.rest = reinterpret_cast<float*>(ws + L.rest);
    w.slot = reinterpret_cast<int32_t*>(ws + L.slot);
    w.rest_rows = reinterpret_cast<__nv_bfloat16*>(ws + L.rest_rows);
    w.progress = reinterpret_cast<uint32_t*>(ws + L.progress);
    return launch_lp_bwd_bf16(a, w, st);
  }
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
    GradParams& g = p.grad;
    g.y = a.y ? a.y + t0 : nullptr;
    g.mask = a.mask ? a.mask + t0 : nullptr;
    g.lse = a.lse + t0;
    g.ent = a.ent ? a.ent + t0 : nullptr;
    g.g_logp = a.g_logp ? a.g_logp + t0 : nullptr;
    g.g_lse = a.g_lse ? a.g_lse + t0 : nullptr;
    g.g_ent = a.g_ent ? a.g_ent + t0 : nullptr;
    g.inv_t = a.inv_t;
    g.V = a.V;
    g.d_status = a.d_status;
    if ((e = launch_sgemm<true, true, true>(p, t0 == 0, nullptr, nullptr, st)) != cudaSuccess) return e;
    SplitSum sums[2];
    SgemmParams q{};                                           // dH = G W
    q.A = Z; q.lda = L.ldg; q.M = rows;
    q.B = (const float*)a.W; q.ldb = a.d; q.N = a.d;
    q.K = a.V;
    q.C = (float*)a.dH + t0 * a.d; q.ldc = a.d;
    if ((e = launch_sgemm<true, false>(q, false, split, &sums[0], st)) != cudaSuccess) return e;
    SgemmParams r{};                                           // dW (+)= G^T H
    r.A = Z; r.lda = L.ldg; r.M = a.V;
    r.B = H; r.ldb = a.ldh; r.N = a.d;
    r.K = rows;
    r.C = (float*)a.dW; r.ldc = a.d; r.accumulate = (a.accumulate || t0 > 0) ? 1 : 0;
    r.b_mask = a.mask ? a.mask + t0 : nullptr;
    if ((e = launch_sgemm<false, false>(r, false, split + kSplitBytes / 4, &sums[1], st)) != cudaSuccess) return e;
    const int64_t n = sums[0].n > sums[1].n ? sums[0].n : sums[1].n;
    if (n > 0) {
      int64_t blocks = ceil_div(n, 256);
      if (blocks > (int64_t)sm_count() * 8) blocks = (int64_t)sm_count() * 8;
      if ((e = launch_dependent(sum_splits_kernel, dim3((unsigned)blocks, 2), dim3(256), st, sums[0], sums[1])) != cudaSuccess) return e;
    }
  }
  return cudaSuccess;
}

}  // namespace spo
