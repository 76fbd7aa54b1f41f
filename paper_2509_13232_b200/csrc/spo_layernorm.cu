// Layer norm and RMS norm over the rows of hidden states, forward and backward (spo_layernorm_fwd, spo_layernorm_bwd).
//
//   h = x (+ residual, rounded to the type of x),  mu = mean h (layer norm; 0 for RMS norm),  rstd = (mean (h - mu)^2 + eps)^-1/2,
//   y = (h - mu) rstd w + b;
//   backward, with xh = (h - mu) rstd and a = w dy:  dx = rstd (a - mean a [layer norm] - xh mean(a xh)) + dh,
//   dw = sum_t dy xh,  db = sum_t dy.
//
// Both directions are bound by HBM: each input is read once and each output written once.  A row belongs to a group of threads that
// keeps it in registers between the reduction over it and its output.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "spo_internal.h"
#include "spo_vec.cuh"

namespace spo {
namespace {

// ---------------------------------------------------------------------------
// V consecutive elements of type T, as loaded
// ---------------------------------------------------------------------------
template <typename T, int V>
struct Pack {
  static constexpr int kBytes = (int)sizeof(T) * V;
  uint32_t w[(kBytes + 3) / 4];
};

template <typename T, int V>
__device__ __forceinline__ Pack<T, V> load_pack(const T* p) {
  Pack<T, V> r;
  constexpr int kBytes = Pack<T, V>::kBytes;
  if constexpr (kBytes >= 16) {
#pragma unroll
    for (int i = 0; i < kBytes / 16; ++i) {
      const uint4 q = reinterpret_cast<const uint4*>(p)[i];
      r.w[4 * i] = q.x; r.w[4 * i + 1] = q.y; r.w[4 * i + 2] = q.z; r.w[4 * i + 3] = q.w;
    }
  } else if constexpr (kBytes == 8) {
    const uint2 q = *reinterpret_cast<const uint2*>(p);
    r.w[0] = q.x; r.w[1] = q.y;
  } else if constexpr (kBytes == 4) {
    r.w[0] = *reinterpret_cast<const uint32_t*>(p);
  } else {
    r.w[0] = *reinterpret_cast<const uint16_t*>(p);
  }
  return r;
}

// The same for rows that are read once: they leave the L1 cache to the weights, which every row wants again (24 000 rows of 4096 with a
// residual: 155 and 12X us).
template <typename T, int V>
__device__ __forceinline__ Pack<T, V> stream_pack(const T* p) {
  Pack<T, V> r;
  constexpr int kBytes = Pack<T, V>::kBytes;
  if constexpr (kBytes >= 16) {
#pragma unroll
    for (int i = 0; i < kBytes / 16; ++i)
      asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
                   : "=r"(r.w[4 * i]), "=r"(r.w[4 * i + 1]), "=r"(r.w[4 * i + 2]), "=r"(r.w[4 * i + 3])
                   : "l"(reinterpret_cast<const char*>(p) + 16 * i));
  } else if constexpr (kBytes == 8) {
    asm volatile("ld.global.L1::no_allocate.v2.u32 {%0, %1}, [%2];" : "=r"(r.w[0]), "=r"(r.w[1]) : "l"(p));
  } else {
    r = load_pack<T, V>(p);
  }
  return r;
}

template <typename T, int V>
__device__ __forceinline__ void zero_pack(Pack<T, V>& r) {
#pragma unroll
  for (int i = 0; i < (int)(sizeof(r.w) / 4); ++i) r.w[i] = 0u;
}

// Element k from its bits (for 16-bit types in the low half); the element was 0.
template <typename T, int V>
__device__ __forceinline__ void put_element(Pack<T, V>& r, int k, uint32_t bits) {
  if constexpr (sizeof(T) == 4) r.w[k] = bits;
  else r.w[k >> 1] |= bits << (16 * (k & 1));
}

template <typename T, int V>
__device__ __forceinline__ float element(const Pack<T, V>& r, int k) {
  if constexpr (sizeof(T) == 4) return __uint_as_float(r.w[k]);
  return (k & 1) ? high_bf16(r.w[k >> 1]) : low_bf16(r.w[k >> 1]);
}
template <typename T, int V>
__device__ __forceinline__ float2 pair_of(const Pack<T, V>& r, int p) { return make_float2(element(r, 2 * p), element(r, 2 * p + 1)); }

template <typename T, int V>
__device__ __forceinline__ Pack<T, V> round_pack(const float* f) {
  Pack<T, V> r;
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int k = 0; k < V; ++k) r.w[k] = __float_as_uint(f[k]);
  } else if constexpr (V == 1) {
    r.w[0] = __bfloat16_as_ushort(__float2bfloat16_rn(f[0]));
  } else {
#pragma unroll
    for (int k = 0; k < V / 2; ++k) {
      const __nv_bfloat162 q = __floats2bfloat162_rn(f[2 * k], f[2 * k + 1]);
      r.w[k] = *reinterpret_cast<const uint32_t*>(&q);
    }
  }
  return r;
}

template <typename T, int V>
__device__ __forceinline__ void store_pack(T* p, const Pack<T, V>& r) {
  constexpr int kBytes = Pack<T, V>::kBytes;
  if constexpr (kBytes >= 16) {
#pragma unroll
    for (int i = 0; i < kBytes / 16; ++i)
      reinterpret_cast<uint4*>(p)[i] = make_uint4(r.w[4 * i], r.w[4 * i + 1], r.w[4 * i + 2], r.w[4 * i + 3]);
  } else if constexpr (kBytes == 8) {
    *reinterpret_cast<uint2*>(p) = make_uint2(r.w[0], r.w[1]);
  } else if constexpr (kBytes == 4) {
    *reinterpret_cast<uint32_t*>(p) = r.w[0];
  } else {
    *reinterpret_cast<uint16_t*>(p) = (uint16_t)r.w[0];
  }
}

// V weights (or biases) from column c on; `none` where there are no weights
template <int V>
__device__ __forceinline__ void load_weights(const void* p, int bf16, int64_t c, float none, float* f) {
  if (!p) {
#pragma unroll
    for (int k = 0; k < V; ++k) f[k] = none;
  } else if (bf16) {
    const Pack<__nv_bfloat16, V> r = load_pack<__nv_bfloat16, V>(static_cast<const __nv_bfloat16*>(p) + c);
#pragma unroll
    for (int k = 0; k < V; ++k) f[k] = element(r, k);
  } else {
    const Pack<float, V> r = load_pack<float, V>(static_cast<const float*>(p) + c);
#pragma unroll
    for (int k = 0; k < V; ++k) f[k] = element(r, k);
  }
}

__host__ __device__ __forceinline__ constexpr int align16(int n) { return (n + 15) & ~15; }

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

__device__ __forceinline__ void flag(int32_t* d_status, int bit) {
  if (d_status) atomicOr(d_status, bit);
}

__device__ __forceinline__ void pdl_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void pdl_release() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// ---------------------------------------------------------------------------
// forward
// ---------------------------------------------------------------------------
struct FwdParams {
  const void *x, *residual, *weight, *bias;
  const uint8_t* mask;
  int64_t ldx, T;
  int32_t d, w_bf16, y_bf16;
  float eps;
  void *y, *h;
  float *mean, *rstd;
  int32_t* d_status;
};

// Chunks.  A thread holds NV chunks of V elements (16 bytes) of a row: chunk i * threads + thread, so that a warp's accesses are
// contiguous.  Where rows do not begin on 16 bytes (SHIFT), chunk c has the columns V c - shift + (0 .. V - 1), shift = (t d) mod V: in the
// tensors without a pitch it then lies on 16 bytes again, but for the columns that the first and last chunk do not have, which are
// moved one by one.
template <typename T, int V, bool SHIFT>
__device__ __forceinline__ Pack<T, V> load_chunk(const T* row, int j, int d) {            // columns j .. of a row
  if constexpr (SHIFT) {
    if (j < 0 || j + V > d) {
      Pack<T, V> r;
      zero_pack(r);
#pragma unroll
      for (int k = 0; k < V; ++k)
        if (j + k >= 0 && j + k < d) put_element<T, V>(r, k, load_pack<T, 1>(row + j + k).w[0]);
      return r;
    }
  }
  return stream_pack<T, V>(row + j);
}
template <typename T, int V, bool SHIFT>
__device__ __forceinline__ void store_chunk(T* row, int j, int d, const Pack<T, V>& r) {
  if constexpr (SHIFT) {
    if (j < 0 || j + V > d) {
#pragma unroll
      for (int k = 0; k < V; ++k)
        if (j + k >= 0 && j + k < d) {
          Pack<T, 1> one;
          if constexpr (sizeof(T) == 4) one.w[0] = r.w[k];
          else one.w[0] = (k & 1) ? r.w[k >> 1] >> 16 : r.w[k >> 1];
          store_pack(row + j + k, one);
        }
      return;
    }
  }
  store_pack(row + j, r);
}
// Whether all of a chunk's columns are in the row; otherwise which.
template <int V, bool SHIFT>
__device__ __forceinline__ bool is_whole(int j, int d) { return !SHIFT || (j >= 0 && j + V <= d); }
__device__ __forceinline__ bool has_column(int j, int k, int d) { return j + k >= 0 && j + k < d; }

// Rows with another shift than the tensors without a pitch: through shared memory, as they are in memory, and out again by column.
// Called by all threads of the row's group; the barrier is the caller's.
template <typename T, int V, int NV>
__device__ __forceinline__ void stage_row(const T* row, int shift, int d, T* s_row, int tid, int threads) {
#pragma unroll
  for (int i = 0; i <= NV; ++i) {                     // (another shift may have one chunk more)
    const int j = (i * threads + tid) * V - shift;
    if (j < d) store_pack(s_row + j + shift, load_chunk<T, V, true>(row, j, d));
  }
}
template <typename T, int V>
__device__ __forceinline__ Pack<T, V> staged_chunk(const T* s_row, int shift, int j, int d) {
  Pack<T, V> r;
  zero_pack(r);
  if (is_whole<V, true>(j, d)) {
#pragma unroll
    for (int k = 0; k < V; ++k) put_element<T, V>(r, k, load_pack<T, 1>(s_row + j + k + shift).w[0]);
  } else {
#pragma unroll
    for (int k = 0; k < V; ++k)
      if (has_column(j, k, d)) put_element<T, V>(r, k, load_pack<T, 1>(s_row + j + k + shift).w[0]);
  }
  return r;
}

// V values to fp32 or bf16 rows.
template <int V, bool SHIFT>
__device__ __forceinline__ void store_values(void* base, bool bf16, int64_t row, int j, int d, const float* f) {
  if (bf16) store_chunk<__nv_bfloat16, V, SHIFT>(static_cast<__nv_bfloat16*>(base) + row, j, d, round_pack<__nv_bfloat16, V>(f));
  else store_chunk<float, V, SHIFT>(static_cast<float*>(base) + row, j, d, round_pack<float, V>(f));
}

// Weight and bias by column in shared memory (SHIFT, where a chunk's columns are not aligned in them): one place in V + 1 is left out, so
// that threads V columns apart do not meet on a bank.
template <int V>
__device__ __forceinline__ int spread(int j) { return j + j / V; }

// Mean and squared deviations of a row from those of its warps, each about a point near its own mean: M2 = sum M2_w + n_w (near_w - mu)^2,
// up to the square of what a point is off its warp's mean by, some 2^-23 of it.  The accuracy of two passes, with one barrier.
struct WarpStats { float sum, m2, near, count; };

constexpr int kFwdBlocks = 6;
constexpr int kSpreadMost = 8192;         // longest row whose weights are kept in shared memory

template <typename X, int NV, int MOST, bool SHIFT, bool CENTER, bool RES>
__global__ void __launch_bounds__(MOST, MOST == 128 ? (RES ? 5 : kFwdBlocks) : 1) ln_fwd_kernel(FwdParams a, int span) {
  constexpr int V = 16 / (int)sizeof(X), P = V / 2;
  // The row stays in registers as fp32 values, or as it is in memory: with both inputs of the next row on their way there is no room for
  // the values (their loads would be put off; 24 000 rows of 4096 with a residual: 155 and 12X us).
  constexpr bool PACKED = RES && sizeof(X) == 2;
  __shared__ WarpStats s_stats[2][32];
  extern __shared__ __align__(16) char s_raw[];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, threads = blockDim.x, warps = threads >> 5;
  const int d = a.d;
  const float inv_d = 1.0f / (float)d;
  const int64_t t0 = (int64_t)blockIdx.x * span;
  const int rows = (int)(a.T - t0 < span ? a.T - t0 : span);
  const uint32_t live_rows = __ballot_sync(0xffffffffu, lane < rows && (!a.mask || a.mask[t0 + (lane < rows ? lane : 0)] != 0));
  const bool staged = SHIFT && a.ldx % V != d % V && a.T > 1;
  const bool spread_out = SHIFT && d <= kSpreadMost;
  float2* const s_wb = reinterpret_cast<float2*>(s_raw);
  X* const s_row = reinterpret_cast<X*>(s_raw + (spread_out ? align16(8 * (spread<V>(d) + 1)) : 0));

  Pack<X, V> next[NV], pr[RES ? NV : 1];
  auto shift_of = [&](int64_t t) { return SHIFT ? (int)((t * d) % V) : 0; };
  auto column = [&](int shift, int i) { return (i * threads + tid) * V - shift; };
  auto fetch = [&](int r) {                            // the row's inputs, in flight while another one is worked on
    if (!(live_rows >> r & 1)) return;
    const int64_t t = t0 + r;
    const int shift = shift_of(t);
    const X *const x = static_cast<const X*>(a.x) + t * a.ldx, *const res = static_cast<const X*>(a.residual) + t * d;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int j = column(shift, i);
      if (j >= d) continue;
      if (!staged) next[i] = load_chunk<X, V, SHIFT>(x, j, d);
      if (RES) pr[i] = load_chunk<X, V, SHIFT>(res, j, d);
    }
  };
  fetch(0);
  int count = 0;                                       // columns of this warp; where rows are shifted it is counted in each
  if (CENTER && !SHIFT) {
#pragma unroll
    for (int i = 0; i < NV; ++i) count += column(0, i) < d ? V : 0;
    count = __reduce_add_sync(0xffffffffu, count);
  }
  if (spread_out) {
    for (int j = tid * V; j < d; j += threads * V) {
      float w[V], b[V];
      if (j + V <= d) {
        load_weights<V>(a.weight, a.w_bf16, j, 1.0f, w);
        load_weights<V>(a.bias, a.w_bf16, j, 0.0f, b);
#pragma unroll
        for (int k = 0; k < V; ++k) s_wb[spread<V>(j) + k] = make_float2(w[k], b[k]);
      } else {
        for (int k = 0; j + k < d; ++k) {
          load_weights<1>(a.weight, a.w_bf16, j + k, 1.0f, w);
          load_weights<1>(a.bias, a.w_bf16, j + k, 0.0f, b);
          s_wb[spread<V>(j) + k] = make_float2(w[0], b[0]);
        }
      }
    }
    __syncthreads();
  }
#pragma unroll 1
  for (int r = 0; r < rows; ++r) {
    const int64_t t = t0 + r;
    const int shift = shift_of(t);
    X* const h = static_cast<X*>(a.h) + t * d;
    if (!(live_rows >> r & 1)) {                       // (all threads of the block: the bits are the same in every warp)
      float zero[V];
#pragma unroll
      for (int k = 0; k < V; ++k) zero[k] = 0.0f;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int j = column(shift, i);
        if (j >= d) continue;
        store_values<V, SHIFT>(a.y, a.y_bf16, t * d, j, d, zero);
        if (RES) store_chunk<X, V, SHIFT>(h, j, d, round_pack<X, V>(zero));
      }
      if (tid == 0) {
        if (CENTER && a.mean) a.mean[t] = 0.0f;
        if (a.rstd) a.rstd[t] = 0.0f;
      }
      if (r + 1 < rows) fetch(r + 1);
      continue;
    }
    if (staged) {
      const int own = (int)((t * a.ldx) % V);
      stage_row<X, V, NV>(static_cast<const X*>(a.x) + t * a.ldx, own, d, s_row, tid, threads);
      __syncthreads();
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int j = column(shift, i);
        if (j < d) next[i] = staged_chunk<X, V>(s_row, own, j, d);
      }
    }
    float2 f[PACKED ? 1 : NV * P] = {}, part = both(0.0f);
    Pack<X, V> now[PACKED ? NV : 1] = {};
    auto value = [&](int i, int p) {
      if constexpr (PACKED) return pair_of(now[i], p);
      else return f[i * P + p];
    };
    if (CENTER && SHIFT) count = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int j = column(shift, i);
      if (j < d) {
        if (RES) {
          float2 both_in[P];
#pragma unroll
          for (int p = 0; p < P; ++p) both_in[p] = add2(pair_of(next[i], p), pair_of(pr[i], p));
          next[i] = round_pack<X, V>(&both_in[0].x);
          store_chunk<X, V, SHIFT>(h, j, d, next[i]);
        }
        if constexpr (PACKED) now[i] = next[i];
#pragma unroll
        for (int p = 0; p < P; ++p) {
          if constexpr (!PACKED) f[i * P + p] = pair_of(next[i], p);
          if (CENTER) part = add2(part, value(i, p));                                   // (0 where there is no column)
        }
        if (CENTER && SHIFT) count += min(j + V, d) - max(j, 0);
      } else {
        if constexpr (PACKED) zero_pack(now[i]);
#pragma unroll
        for (int p = 0; p < P; ++p)
          if constexpr (!PACKED) f[i * P + p] = both(0.0f);
      }
    }
    if (r + 1 < rows) fetch(r + 1);
    float sum = 0.0f, mu = 0.0f;
    if (CENTER) {
      sum = warp_sum(part.x + part.y);
      if (SHIFT) count = __reduce_add_sync(0xffffffffu, count);
      mu = count ? __fdividef(sum, (float)count) : 0.0f;      // any point near the mean serves to measure the deviations from
    }
    part = both(0.0f);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int j = column(shift, i);
      if (CENTER && j >= d) continue;
#pragma unroll
      for (int p = 0; p < P; ++p) {
        float2 c = CENTER ? add2(value(i, p), both(-mu)) : value(i, p);
        if (CENTER && !is_whole<V, SHIFT>(j, d)) {
          if (!has_column(j, 2 * p, d)) c.x = 0.0f;
          if (!has_column(j, 2 * p + 1, d)) c.y = 0.0f;
        }
        part = fma2(c, c, part);
      }
    }
    float m2 = warp_sum(part.x + part.y);
    if (warps > 1) {
      WarpStats* const st = s_stats[r & 1];
      if (lane == 0) st[warp] = WarpStats{sum, m2, mu, (float)count};
      __syncthreads();
      m2 = 0.0f;
      if (CENTER) {
        sum = 0.0f;
        for (int w = 0; w < warps; ++w) sum += st[w].sum;
        mu = sum * inv_d;
        for (int w = 0; w < warps; ++w) {
          const float c = st[w].near - mu;
          m2 += fmaf(st[w].count * c, c, st[w].m2);
        }
      } else {
        for (int w = 0; w < warps; ++w) m2 += st[w].m2;
      }
    } else {
      if (CENTER) {
        const float c = sum * inv_d - mu;
        mu = sum * inv_d;
        m2 = fmaf((float)count * c, c, m2);
      }
      if (staged) __syncwarp();
    }
    const float var = m2 * inv_d, rstd = rsqrtf(var + a.eps), drop = -mu * rstd;
    if (tid == 0) {
      if (CENTER && a.mean) a.mean[t] = mu;
      if (a.rstd) a.rstd[t] = rstd;
      if (!(var < INFINITY)) flag(a.d_status, SPO_DEV_NONFINITE);
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int j = column(shift, i);
      if (j >= d) continue;
      float2 w[P], b[P];
      if (!SHIFT) {
        load_weights<V>(a.weight, a.w_bf16, j, 1.0f, &w[0].x);
        load_weights<V>(a.bias, a.w_bf16, j, 0.0f, &b[0].x);
      } else if (spread_out && is_whole<V, SHIFT>(j, d)) {
        const int at = spread<V>(j), first = V - j % V;  // V columns from j on: a place is skipped behind the first multiple of V
#pragma unroll
        for (int p = 0; p < P; ++p) {
          const float2 q0 = s_wb[at + 2 * p + (2 * p >= first)], q1 = s_wb[at + 2 * p + 1 + (2 * p + 1 >= first)];
          w[p] = make_float2(q0.x, q1.x);
          b[p] = make_float2(q0.y, q1.y);
        }
      } else {
#pragma unroll
        for (int k = 0; k < V; ++k) {
          const int c = has_column(j, k, d) ? j + k : 0;
          load_weights<1>(a.weight, a.w_bf16, c, 1.0f, &w[0].x + k);
          load_weights<1>(a.bias, a.w_bf16, c, 0.0f, &b[0].x + k);
        }
      }
#pragma unroll
      for (int p = 0; p < P; ++p) {
        const float2 xh = CENTER ? fma2(value(i, p), both(rstd), both(drop)) : mul2(value(i, p), both(rstd));
        w[p] = fma2(xh, w[p], b[p]);
      }
      store_values<V, SHIFT>(a.y, a.y_bf16, t * d, j, d, &w[0].x);
    }
  }
}

// Rows longer than a block's registers hold: the row is read again for each of the three passes.
template <typename X, bool CENTER>
__global__ void __launch_bounds__(1024) ln_fwd_long_kernel(FwdParams a) {
  __shared__ float s_part[32];
  const int64_t t = blockIdx.x;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, nw = blockDim.x >> 5;
  const bool live = !a.mask || a.mask[t] != 0;
  const X* row = static_cast<const X*>(a.x) + t * a.ldx;
  if (a.residual) {
    const X* r = static_cast<const X*>(a.residual) + t * a.d;
    X* h = static_cast<X*>(a.h) + t * a.d;
    for (int64_t c = threadIdx.x; c < a.d; c += blockDim.x) {
      const float v = live ? element(load_pack<X, 1>(row + c), 0) + element(load_pack<X, 1>(r + c), 0) : 0.0f;
      store_pack(h + c, round_pack<X, 1>(&v));
    }
    row = h;                                   // every thread reads back what it wrote itself
  }
  auto total = [&](float v) {
    v = warp_sum(v);
    __syncthreads();
    if (lane == 0) s_part[warp] = v;
    __syncthreads();
    v = 0.0f;
    for (int w = 0; w < nw; ++w) v += s_part[w];
    return v;
  };
  float mu = 0.0f, m2 = 0.0f;
  if (live) {
    if (CENTER) {
      float sum = 0.0f;
      for (int64_t c = threadIdx.x; c < a.d; c += blockDim.x) sum += element(load_pack<X, 1>(row + c), 0);
      mu = total(sum) / (float)a.d;
    }
    for (int64_t c = threadIdx.x; c < a.d; c += blockDim.x) {
      const float v = element(load_pack<X, 1>(row + c), 0) - mu;
      m2 = fmaf(v, v, m2);
    }
    m2 = total(m2);
  }
  const float var = m2 / (float)a.d;
  const float rstd = live ? 1.0f / sqrtf(var + a.eps) : 0.0f;
  if (threadIdx.x == 0) {
    if (CENTER && a.mean) a.mean[t] = mu;
    if (a.rstd) a.rstd[t] = rstd;
    if (live && !(var < INFINITY)) flag(a.d_status, SPO_DEV_NONFINITE);
  }
  for (int64_t c = threadIdx.x; c < a.d; c += blockDim.x) {
    float v = 0.0f;
    if (live) {
      float w, b;
      load_weights<1>(a.weight, a.w_bf16, c, 1.0f, &w);
      load_weights<1>(a.bias, a.w_bf16, c, 0.0f, &b);
      v = fmaf((element(load_pack<X, 1>(row + c), 0) - mu) * rstd, w, b);
    }
    store_values<1, false>(a.y, a.y_bf16, t * a.d, c, a.d, &v);
  }
}

// Threads per row: chunks of V elements, NV a thread.
int group_of(int64_t chunks, int nv) {
  int64_t g = 32;
  while (g * nv < chunks) g *= 2;
  return (int)(g > 2048 ? 2048 : g);
}

constexpr int kFwdThreadsPerSm = 640;     // that fit with their registers
constexpr int kFwdSpanMost = 4, kFwdSpanShift = 12, kFwdRounds = 3;

template <typename X, int NV, int MOST, bool SHIFT, bool CENTER, bool RES>
cudaError_t run_fwd(const FwdParams& a, int64_t chunks, cudaStream_t st) {
  constexpr int V = 16 / (int)sizeof(X);
  const auto kernel = ln_fwd_kernel<X, NV, MOST, SHIFT, CENTER, RES>;
  const int threads = (int)align_up((size_t)ceil_div(chunks, NV), 32);
  const int64_t at_once = (int64_t)sm_count() * (threads >= kFwdThreadsPerSm ? 1 : kFwdThreadsPerSm / threads);
  int64_t span = a.T / (at_once * kFwdRounds);
  const int64_t most = SHIFT ? kFwdSpanShift : kFwdSpanMost;
  span = span < 1 ? 1 : span > most ? most : span;
  int smem = 0;
  if (SHIFT) {
    if (a.d <= kSpreadMost) smem += align16(8 * (a.d + a.d / V + 1));
    if (a.T > 1 && a.ldx % V != a.d % V) smem += align16((int)sizeof(X) * (a.d + 2 * V));
    if (smem > 32 * 1024) {
      const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
      if (e != cudaSuccess) return e;
    }
  }
  kernel<<<(unsigned)ceil_div(a.T, span), threads, smem, st>>>(a, (int)span);
  return cudaGetLastError();
}

template <typename X, bool CENTER, bool RES>
cudaError_t pick_fwd(const FwdParams& a, cudaStream_t st) {
  constexpr int V = 16 / (int)sizeof(X);
  const bool shift = !(a.d % V == 0 && (a.T == 1 || a.ldx % V == 0));
  const int64_t chunks = shift ? ceil_div(a.d + V - 1, V) : a.d / V;
  if (chunks > 4 * 1024) {
    ln_fwd_long_kernel<X, CENTER><<<(unsigned)a.T, 1024, 0, st>>>(a);
    return cudaGetLastError();
  }
  // One warp with one chunk a thread for short rows; up to 128 threads with four chunks, whose registers leave room for five blocks an SM;
  // then as many threads as two chunks (at last four) a thread need.  Where there are fewer rows than SMs, as many threads as there
  // are chunks: one row of 4096 takes 2.9 us so and 3.4 on 128 threads.
  auto form = [&](auto sh) {
    constexpr bool S = decltype(sh)::value;
    if (chunks <= 32) return run_fwd<X, 1, 128, S, CENTER, RES>(a, chunks, st);
    if (chunks <= 1024 && a.T <= sm_count()) return run_fwd<X, 1, 1024, S, CENTER, RES>(a, chunks, st);
    if (chunks <= 4 * 128) return run_fwd<X, 4, 128, S, CENTER, RES>(a, chunks, st);
    if (chunks <= 2 * 1024) return run_fwd<X, 2, 1024, S, CENTER, RES>(a, chunks, st);
    return run_fwd<X, 4, 1024, S, CENTER, RES>(a, chunks, st);
  };
  return shift ? form(std::true_type{}) : form(std::false_type{});
}

// ---------------------------------------------------------------------------
// backward
// ---------------------------------------------------------------------------
struct BwdParams {
  const void *dy, *x, *weight, *dh;
  const uint8_t* mask;
  const float *mean, *rstd;
  int64_t ldx, T;
  int32_t d, w_bf16;
  void* dx;
  float* partial;                // [blocks][want][d]: dw, then db
  int want_dw, want_db;
};

// A group of threads per row as in the forward pass, and a thread keeps its columns for all rows that its group walks through
// (rows g, g + groups of the grid, ...): weights and the sums of dw and db stay in registers.  The next row is loaded before the
// current one is reduced.  Both row means take one barrier.  At the end the groups of a block add up in shared memory, in order,
// and each block leaves one partial row of dw and db.
template <typename X, typename DY, int V, int NV, bool CENTER>
__global__ void __launch_bounds__(1024) ln_bwd_kernel(BwdParams a, int group) {
  constexpr int E = V * NV;
  __shared__ float2 s_sum[2][32];
  extern __shared__ float s_cols[];                     // [groups - 1][2][d], where a block has several groups
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = threadIdx.x / group, tid = threadIdx.x - g * group;
  const int groups = blockDim.x / group;
  const int64_t step = (int64_t)gridDim.x * groups;
  float w[E], dw[E], db[E];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int64_t c = (int64_t)(i * group + tid) * V;
    if (c < a.d) {
      load_weights<V>(a.weight, a.w_bf16, c, 1.0f, w + i * V);
    } else {
#pragma unroll
      for (int k = 0; k < V; ++k) w[i * V + k] = 0.0f;
    }
  }
#pragma unroll
  for (int e = 0; e < E; ++e) dw[e] = db[e] = 0.0f;

  Pack<X, V> px[NV], ph[NV];
  Pack<DY, V> py[NV];
  float mu = 0.0f, rstd = 0.0f;
  bool live = false;
  auto fetch = [&](int64_t t) {
    live = t < a.T && (!a.mask || a.mask[t] != 0);
    rstd = live ? a.rstd[t] : 0.0f;
    mu = CENTER && live ? a.mean[t] : 0.0f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int64_t c = (int64_t)(i * group + tid) * V;
      zero_pack(px[i]);
      zero_pack(py[i]);
      zero_pack(ph[i]);
      if (live && c < a.d) {
        px[i] = load_pack<X, V>(static_cast<const X*>(a.x) + t * a.ldx + c);
        py[i] = load_pack<DY, V>(static_cast<const DY*>(a.dy) + t * a.d + c);
        if (a.dh) ph[i] = load_pack<X, V>(static_cast<const X*>(a.dh) + t * a.d + c);
      }
    }
  };
  const float inv_d = 1.0f / (float)a.d;
  int buf = 0;
  int64_t t = (int64_t)blockIdx.x * groups + g;
  fetch(t);
  for (int64_t first = (int64_t)blockIdx.x * groups; first < a.T; first += step, t += step, buf ^= 1) {
    float xh[E], dy[E];
    Pack<X, V> h[NV];
    const float r = rstd;
    float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      h[i] = ph[i];
#pragma unroll
      for (int k = 0; k < V; ++k) {
        const int e = i * V + k;
        xh[e] = (element(px[i], k) - mu) * r;
        dy[e] = element(py[i], k);
      }
    }
#pragma unroll
    for (int e = 0; e < E; ++e) {
      dw[e] = fmaf(dy[e], xh[e], dw[e]);
      db[e] += dy[e];
      dy[e] *= w[e];
      s1 = fmaf(dy[e], xh[e], s1);
      if (CENTER) s2 += dy[e];
    }
    fetch(t + step);
    s1 = warp_sum(s1);
    if (CENTER) s2 = warp_sum(s2);
    if (group > 32) {
      if (lane == 0) s_sum[buf][warp] = make_float2(s1, s2);
      __syncthreads();
      s1 = s2 = 0.0f;
      const int w0 = g * (group >> 5);
      for (int q = 0; q < (group >> 5); ++q) {
        const float2 v = s_sum[buf][w0 + q];
        s1 += v.x;
        if (CENTER) s2 += v.y;
      }
    }
    s1 *= inv_d;
    s2 *= inv_d;
    if (t < a.T) {
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int64_t c = (int64_t)(i * group + tid) * V;
        if (c < a.d) {
          float o[V];
#pragma unroll
          for (int k = 0; k < V; ++k) {
            const int e = i * V + k;
            o[k] = fmaf(r, CENTER ? fmaf(-xh[e], s1, dy[e] - s2) : fmaf(-xh[e], s1, dy[e]), element(h[i], k));
          }
          store_pack(static_cast<X*>(a.dx) + t * a.d + c, round_pack<X, V>(o));
        }
      }
    }
  }
  if (!a.partial) return;
  pdl_release();
  if (g > 0) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int64_t c = (int64_t)(i * group + tid) * V;
      if (c < a.d) {
#pragma unroll
        for (int k = 0; k < V; ++k) {
          s_cols[(int64_t)(2 * (g - 1)) * a.d + c + k] = dw[i * V + k];
          s_cols[(int64_t)(2 * (g - 1) + 1) * a.d + c + k] = db[i * V + k];
        }
      }
    }
  }
  if (groups > 1) __syncthreads();
  if (g == 0) {
    const int want = a.want_dw + a.want_db;
    float* row = a.partial + (int64_t)blockIdx.x * want * a.d;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int64_t c = (int64_t)(i * group + tid) * V;
      if (c < a.d) {
        for (int q = 0; q < groups - 1; ++q) {
#pragma unroll
          for (int k = 0; k < V; ++k) {
            dw[i * V + k] += s_cols[(int64_t)(2 * q) * a.d + c + k];
            db[i * V + k] += s_cols[(int64_t)(2 * q + 1) * a.d + c + k];
          }
        }
        if (a.want_dw) store_pack(row + c, round_pack<float, V>(dw + i * V));
        if (a.want_db) store_pack(row + (int64_t)a.want_dw * a.d + c, round_pack<float, V>(db + i * V));
      }
    }
  }
}

// Rows longer than a block's registers hold: one block per row finds the two means and writes dx ...
template <typename X, typename DY, bool CENTER>
__global__ void __launch_bounds__(1024) ln_bwd_long_rows_kernel(BwdParams a) {
  __shared__ float2 s_sum[32];
  const int64_t t = blockIdx.x;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, nw = blockDim.x >> 5;
  const bool live = !a.mask || a.mask[t] != 0;
  const X* x = static_cast<const X*>(a.x) + t * a.ldx;
  const X* dh = a.dh ? static_cast<const X*>(a.dh) + t * a.d : nullptr;
  const DY* dy = static_cast<const DY*>(a.dy) + t * a.d;
  X* dx = static_cast<X*>(a.dx) + t * a.d;
  const float r = live ? a.rstd[t] : 0.0f, mu = CENTER && live ? a.mean[t] : 0.0f;
  float s1 = 0.0f, s2 = 0.0f;
  if (live)
    for (int64_t c = threadIdx.x; c < a.d; c += blockDim.x) {
      float w;
      load_weights<1>(a.weight, a.w_bf16, c, 1.0f, &w);
      const float up = w * element(load_pack<DY, 1>(dy + c), 0);
      s1 = fmaf(up, (element(load_pack<X, 1>(x + c), 0) - mu) * r, s1);
      s2 += up;
    }
  s1 = warp_sum(s1);
  s2 = warp_sum(s2);
  if (lane == 0) s_sum[warp] = make_float2(s1, s2);
  __syncthreads();
  s1 = s2 = 0.0f;
  for (int q = 0; q < nw; ++q) {
    s1 += s_sum[q].x;
    s2 += s_sum[q].y;
  }
  s1 /= (float)a.d;
  s2 = CENTER ? s2 / (float)a.d : 0.0f;
  for (int64_t c = threadIdx.x; c < a.d; c += blockDim.x) {
    float o = 0.0f;
    if (live) {
      float w;
      load_weights<1>(a.weight, a.w_bf16, c, 1.0f, &w);
      const float xh = (element(load_pack<X, 1>(x + c), 0) - mu) * r;
      o = r * fmaf(-xh, s1, w * element(load_pack<DY, 1>(dy + c), 0) - s2);
      if (dh) o += element(load_pack<X, 1>(dh + c), 0);
    }
    store_pack(dx + c, round_pack<X, 1>(&o));
  }
}

// ... and before that (dx may take dy's place) blocks of 256 columns by a share of the rows sum dw and db.
template <typename X, typename DY, bool CENTER>
__global__ void __launch_bounds__(256) ln_bwd_long_cols_kernel(BwdParams a) {
  const int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (c >= a.d) return;
  float dw = 0.0f, db = 0.0f;
  for (int64_t t = blockIdx.y; t < a.T; t += gridDim.y) {
    if (a.mask && a.mask[t] == 0) continue;
    const float dy = element(load_pack<DY, 1>(static_cast<const DY*>(a.dy) + t * a.d + c), 0);
    const float x = element(load_pack<X, 1>(static_cast<const X*>(a.x) + t * a.ldx + c), 0);
    dw = fmaf(dy, (x - (CENTER ? a.mean[t] : 0.0f)) * a.rstd[t], dw);
    db += dy;
  }
  float* row = a.partial + (int64_t)blockIdx.y * (a.want_dw + a.want_db) * a.d;
  if (a.want_dw) row[c] = dw;
  if (a.want_db) row[(int64_t)a.want_dw * a.d + c] = db;
}

// dw and db from the blocks' partial rows, in their order: 32 columns a block, eight warps that take every eighth partial row each.
__global__ void __launch_bounds__(256) ln_bwd_columns_kernel(const float* __restrict__ partial, int parts, int64_t width, int32_t d,
                                                             void* dw, void* db, int bf16, int accumulate) {
  __shared__ float s_sum[8][32];
  pdl_wait();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t j = (int64_t)blockIdx.x * 32 + lane;
  float sum = 0.0f;
  if (j < width) {
#pragma unroll 8
    for (int p = warp; p < parts; p += 8) sum += partial[(int64_t)p * width + j];
  }
  s_sum[warp][lane] = sum;
  __syncthreads();
  if (warp != 0 || j >= width) return;
#pragma unroll
  for (int q = 1; q < 8; ++q) sum += s_sum[q][lane];
  void* out = dw && j < d ? dw : db;
  const int64_t at = j < d ? j : j - d;
  if (bf16) {
    __nv_bfloat16* o = static_cast<__nv_bfloat16*>(out) + at;
    if (accumulate) sum += __bfloat162float(*o);
    *o = __float2bfloat16_rn(sum);
  } else {
    float* o = static_cast<float*>(out) + at;
    *o = accumulate ? *o + sum : sum;
  }
}

// The launch of a backward pass; a function of d and T alone, so that the scratch can be sized by it.
constexpr int kLongRows = 16384;           // elements of a row that a block's registers hold
struct BwdPlan {
  int v, nv, group, threads, blocks;       // v = 0: the long form; blocks then is the number of row shares
};
BwdPlan bwd_plan(int64_t T, int32_t d, int v) {
  BwdPlan p{};
  if (d > kLongRows) {
    p.blocks = (int)(T < 64 ? T : 64);
    return p;
  }
  p.v = v;
  p.nv = (d <= 8192 ? 8 : 16) / v;
  p.group = group_of(ceil_div(d, v), p.nv);
  p.threads = p.group > 256 ? p.group : 256;
  const int64_t most = (int64_t)sm_count() * (1024 / p.threads), need = ceil_div(T, p.threads / p.group);
  p.blocks = (int)(need < most ? need : most);
  return p;
}

template <typename X, typename DY, int V, int NV, bool CENTER>
cudaError_t run_bwd(const BwdParams& a, const BwdPlan& p, cudaStream_t st) {
  const int smem = a.partial ? (p.threads / p.group - 1) * 2 * a.d * (int)sizeof(float) : 0;      // below 16 KB: groups are as long as rows
  ln_bwd_kernel<X, DY, V, NV, CENTER><<<p.blocks, p.threads, smem, st>>>(a, p.group);
  return cudaGetLastError();
}

template <typename X, typename DY, bool CENTER>
cudaError_t pick_bwd(const BwdParams& a, const BwdPlan& p, cudaStream_t st) {
  if (p.v == 0) {
    cudaError_t e = cudaSuccess;
    if (a.partial) {
      ln_bwd_long_cols_kernel<X, DY, CENTER><<<dim3((unsigned)ceil_div(a.d, 256), p.blocks), 256, 0, st>>>(a);
      if ((e = cudaGetLastError()) != cudaSuccess) return e;
    }
    ln_bwd_long_rows_kernel<X, DY, CENTER><<<(unsigned)a.T, 1024, 0, st>>>(a);
    return cudaGetLastError();
  }
  constexpr int V = 16 / (int)sizeof(X);
  const bool two = p.nv * p.v > 8;
  if (p.v == 1) return two ? run_bwd<X, DY, 1, 16, CENTER>(a, p, st) : run_bwd<X, DY, 1, 8, CENTER>(a, p, st);
  return two ? run_bwd<X, DY, V, 16 / V, CENTER>(a, p, st) : run_bwd<X, DY, V, 8 / V, CENTER>(a, p, st);
}

}  // namespace

size_t layernorm_bwd_ws_bytes(int64_t T, int32_t d) {
  if (T < 1) return 256;
  size_t most = 0;
  for (int v : {8, 4, 1}) {                // aligned bf16, aligned fp32, any other rows
    const BwdPlan p = bwd_plan(T, d, v);
    const size_t n = (size_t)p.blocks * 2 * (size_t)d * sizeof(float);
    if (n > most) most = n;
  }
  return align_up(most, 256);
}

cudaError_t launch_layernorm_fwd(const LayerNormFwd& q, cudaStream_t st) {
  if (q.T == 0) return cudaSuccess;
  FwdParams a{};
  a.x = q.x; a.residual = q.residual; a.weight = q.weight; a.bias = q.bias; a.mask = q.mask; a.ldx = q.ldx; a.T = q.T; a.d = q.d;
  a.w_bf16 = q.w_dtype == SPO_DTYPE_BF16; a.eps = q.eps; a.y = q.y; a.h = q.h; a.mean = q.mean; a.rstd = q.rstd; a.d_status = q.d_status;
  a.y_bf16 = q.y_dtype == SPO_DTYPE_BF16;
  auto typed = [&](auto center, auto res) {
    constexpr bool C = decltype(center)::value, R = decltype(res)::value;
    return q.dtype == SPO_DTYPE_BF16 ? pick_fwd<__nv_bfloat16, C, R>(a, st) : pick_fwd<float, C, R>(a, st);
  };
  using yes = std::true_type;
  using no = std::false_type;
  if (q.kind == SPO_NORM_LAYER) return q.residual ? typed(yes{}, yes{}) : typed(yes{}, no{});
  return q.residual ? typed(no{}, yes{}) : typed(no{}, no{});
}

cudaError_t launch_layernorm_bwd(const LayerNormBwd& q, char* ws, cudaStream_t st) {
  const int size = q.dw_dtype == SPO_DTYPE_BF16 ? 2 : 4;
  cudaError_t e = cudaSuccess;
  if (q.T == 0) {
    for (void* o : {q.dw, q.db})
      if (o && !q.dw_accumulate && (e = cudaMemsetAsync(o, 0, (size_t)q.d * size, st)) != cudaSuccess) return e;
    return e;
  }
  const int v = 16 / (q.dtype == SPO_DTYPE_BF16 ? 2 : 4);
  const bool aligned = q.d % v == 0 && (q.T == 1 || q.ldx % v == 0);
  const BwdPlan p = bwd_plan(q.T, q.d, aligned ? v : 1);
  BwdParams a{};
  a.dy = q.dy; a.x = q.x; a.weight = q.weight; a.dh = q.dh; a.mask = q.mask; a.mean = q.mean; a.rstd = q.rstd; a.ldx = q.ldx;
  a.T = q.T; a.d = q.d; a.w_bf16 = q.w_dtype == SPO_DTYPE_BF16; a.dx = q.dx;
  a.want_dw = q.dw != nullptr; a.want_db = q.db != nullptr;
  a.partial = a.want_dw || a.want_db ? reinterpret_cast<float*>(ws) : nullptr;
  using bf = __nv_bfloat16;
  const bool x16 = q.dtype == SPO_DTYPE_BF16, y16 = q.dy_dtype == SPO_DTYPE_BF16;
  if (q.kind == SPO_NORM_LAYER) {
    if (x16) e = y16 ? pick_bwd<bf, bf, true>(a, p, st) : pick_bwd<bf, float, true>(a, p, st);
    else e = y16 ? pick_bwd<float, bf, true>(a, p, st) : pick_bwd<float, float, true>(a, p, st);
  } else {
    if (x16) e = y16 ? pick_bwd<bf, bf, false>(a, p, st) : pick_bwd<bf, float, false>(a, p, st);
    else e = y16 ? pick_bwd<float, bf, false>(a, p, st) : pick_bwd<float, float, false>(a, p, st);
  }
  if (e != cudaSuccess || !a.partial) return e;
  const int64_t width = (int64_t)(a.want_dw + a.want_db) * q.d;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)ceil_div(width, 32));
  cfg.blockDim = dim3(256);
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = p.v ? 1 : 0;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, ln_bwd_columns_kernel, (const float*)a.partial, p.blocks, width, q.d, q.dw, q.db,
                            (int)(q.dw_dtype == SPO_DTYPE_BF16), (int)q.dw_accumulate);
}

}  // namespace spo
