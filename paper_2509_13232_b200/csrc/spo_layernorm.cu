// Layer norm and RMS norm over the rows of hidden states, forward and backward (spo_layernorm_fwd, spo_layernorm_bwd).
//
//   h = x (+ residual, rounded to the type of x),  mu = mean h (layer norm; 0 for RMS norm),  rstd = (mean (h - mu)^2 + eps)^-1/2,
//   y = (h - mu) rstd w + b;
//   backward, with xh = (h - mu) rstd and a = w dy:  dx = rstd (a - mean a [layer norm] - xh mean(a xh)) + dh,
//   dw = sum_t dy xh,  db = sum_t dy.
//
// Both directions are bound by HBM, as far as their instructions let them: each input is read once and each output written once.  A row
// belongs to a block, which keeps it in registers (forward) or shared memory (backward) between the reduction over it and its output.
// At 6550 GB/s of a copy: forward, 24 000 bf16 rows of 4096 with a residual 126 us (6250 GB/s), without 71 us (5540; 14 instructions an element
// are in the way), layer norm with a bias 90 (4370; 20 instructions); backward, the same rows with fp32 dy, dh and a mask 155 us (6340), layer norm
// with dw and db 132 (4460; 31 instructions).
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>
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

// The same for rows that are read once: issued where it is written, and past the L1 cache.
template <typename T, int V>
__device__ __forceinline__ Pack<T, V> stream_pack(const T* p) {
  static_assert(Pack<T, V>::kBytes == 16, "rows are read by 16 bytes");
  Pack<T, V> r;
  asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
               : "=r"(r.w[0]), "=r"(r.w[1]), "=r"(r.w[2]), "=r"(r.w[3]) : "l"(p));
  return r;
}

template <typename T, int V>
__device__ __forceinline__ void zero_pack(Pack<T, V>& r) {
#pragma unroll
  for (int i = 0; i < (int)(sizeof(r.w) / 4); ++i) r.w[i] = 0u;
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

// Chunks.  A thread holds NV chunks of V elements (16 bytes) of a row: chunk c = i * threads + thread, so that a warp's accesses are
// contiguous.  Where rows do not begin on 16 bytes (SHIFT), chunk c has the columns V c - shift + (0 .. V - 1), shift = (t d) mod V: in the
// tensors without a pitch it then lies on 16 bytes again.  The first and the last chunk of such a row have columns that are the
// neighbouring rows': they are read along (not behind the end of the last row), count as zeros, and are not written.  A block takes
// rows of one shift only, so that its threads' columns stay the same.
template <int V, bool SHIFT>
__device__ __forceinline__ bool is_whole(int j, int d) { return !SHIFT || (j >= 0 && j + V <= d); }
__device__ __forceinline__ bool has_column(int j, int k, int d) { return j + k >= 0 && j + k < d; }

template <typename T, int V, bool SHIFT>
__device__ __forceinline__ void store_chunk(T* row, int j, int d, const Pack<T, V>& r) {
  if constexpr (SHIFT) {
    if (!is_whole<V, SHIFT>(j, d)) {
#pragma unroll
      for (int k = 0; k < V; ++k)
        if (has_column(j, k, d)) {
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
// V values to fp32 or bf16 rows.
template <int V, bool SHIFT>
__device__ __forceinline__ void store_values(void* base, bool bf16, int64_t row, int j, int d, const float* f) {
  if (bf16) store_chunk<__nv_bfloat16, V, SHIFT>(static_cast<__nv_bfloat16*>(base) + row, j, d, round_pack<__nv_bfloat16, V>(f));
  else store_chunk<float, V, SHIFT>(static_cast<float*>(base) + row, j, d, round_pack<float, V>(f));
}

// Rows come through a ring in shared memory: a thread copies its own chunks there, one or two rows ahead, and reads them itself, so that
// rows on their way take no registers and no barrier.
// The first `bytes` come from memory, the rest are zeros.
__device__ __forceinline__ void copy16(void* s, const void* g, int bytes = 16) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(s)), "l"(g), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy8(void* s, const void* g, int bytes = 8) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(s)), "l"(g), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copies_issued() { asm volatile("cp.async.commit_group;" ::: "memory"); }
// All but the newest `newer` groups of this thread's copies have arrived.
__device__ __forceinline__ void copies_arrived(int newer) {
  if (newer >= 2) asm volatile("cp.async.wait_group 2;" ::: "memory");
  else if (newer == 1) asm volatile("cp.async.wait_group 1;" ::: "memory");
  else asm volatile("cp.async.wait_group 0;" ::: "memory");
}
template <typename T, int V, bool SHIFT>
__device__ __forceinline__ void copy_chunk(char* s, const T* row, int j, int end) {
  constexpr int kSize = V * (int)sizeof(T);
  const int there = SHIFT ? min(end - j, V) * (int)sizeof(T) : kSize;           // bytes up to the end of the tensor
  if constexpr (kSize == 8) {
    copy8(s, row + j, there);
  } else {
#pragma unroll
    for (int o = 0; o < kSize; o += 16) {
      const int left = max(min(there - o, 16), 0);
      copy16(s + o, reinterpret_cast<const char*>(row + j) + (left > 0 ? o : 0), left);
    }
  }
}
// Elements from the beginning of row t to the end of the tensor, behind which nothing is read.
__device__ __forceinline__ int end_of(int64_t T, int64_t t, int64_t ld, int d) {
  const int64_t n = (T - 1 - t) * ld + d;
  return n < (1 << 30) ? (int)n : 1 << 30;
}
// The first and the last chunk of a row, as far as they are this thread's and have columns of a neighbouring row; otherwise -1.
template <int V>
__device__ __forceinline__ int2 edge_chunks(int shift, int d, int tid, int threads) {
  const int last = (d + shift - 1) / V;
  return make_int2(tid == 0 && shift > 0 ? 0 : -1, last % threads == tid && (d + shift) % V != 0 && (last > 0 || shift == 0) ? last : -1);
}
// Zeros for the columns of a copied chunk that are not the row's.
template <typename T, int V>
__device__ __forceinline__ void blank(char* s, int j, int d) {
#pragma unroll 1
  for (int k = 0; k < V; ++k) {
    Pack<T, 1> zero;
    zero.w[0] = 0;
    if (!has_column(j, k, d)) store_pack(reinterpret_cast<T*>(s) + k, zero);
  }
}
// Columns j .. of a row that lies in shared memory with its own shift, from the two aligned chunks that hold them: up to a chunk in front
// of the row and one behind it are read, and count as zeros.
template <typename T, int V>
__device__ __forceinline__ Pack<T, V> staged_chunk(const char* s, int own, int j, int d) {
  const int at = (own + j) * (int)sizeof(T), words = at >> 2 & 3, bits = 8 * (at & 3);          // (the same for all of a row)
  const uint4* const p = reinterpret_cast<const uint4*>(s) + (at >> 4);
  const uint4 lo = p[0], hi = p[1];
  uint32_t w[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
  if (words & 2) {
#pragma unroll
    for (int i = 0; i < 6; ++i) w[i] = w[i + 2];
  }
  if (words & 1) {
#pragma unroll
    for (int i = 0; i < 5; ++i) w[i] = w[i + 1];
  }
  Pack<T, V> r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r.w[i] = __funnelshift_r(w[i], w[i + 1], bits);
  if (!is_whole<V, true>(j, d)) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      constexpr int kEach = 4 / (int)sizeof(T);
      if (!has_column(j, i * kEach, d)) r.w[i] &= kEach == 2 ? 0xffff0000u : 0u;
      if (kEach == 2 && !has_column(j, 2 * i + 1, d)) r.w[i] &= 0x0000ffffu;
    }
  }
  return r;
}

// A vector of weights (or biases) in shared memory as fp32, by chunk: quarter q of chunk c at q held + c.
template <int V>
__device__ __forceinline__ void spread_quarters(float4* s, int held, int c, const float* w) {
#pragma unroll
  for (int q = 0; q < V / 4; ++q) s[q * held + c] = make_float4(w[4 * q], w[4 * q + 1], w[4 * q + 2], w[4 * q + 3]);
}
template <int V>
__device__ __forceinline__ void spread_weights(float4* s, const void* p, int bf16, int held, int c, int d) {
  float w[V];
#pragma unroll
  for (int k = 0; k < V; ++k) w[k] = 0.0f;
  if (c * V < d) load_weights<V>(p, bf16, c * V, 1.0f, w);
  spread_quarters<V>(s, held, c, w);
}
// The same for all chunks of a thread of a shifted row: every load is on its way before the first one is waited for
// (2003 rows of 2730 with a bias: 14.8 us so and 16.4 chunk by chunk).
template <typename W, int V, int NV>
__device__ __forceinline__ void spread_shifted(float4* s, const W* p, int held, int shift, int d, int tid, int threads) {
  Pack<W, 1> q[NV * V];
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int k = 0; k < V; ++k) q[i * V + k] = load_pack<W, 1>(p + min(max((i * threads + tid) * V - shift + k, 0), d - 1));
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = i * threads + tid, j = c * V - shift;
    float w[V];
#pragma unroll
    for (int k = 0; k < V; ++k) w[k] = has_column(j, k, d) ? element(q[i * V + k], 0) : 0.0f;
    spread_quarters<V>(s, held, c, w);
  }
}
template <int V, int NV>
__device__ __forceinline__ void spread_shifted(float4* s, const void* p, int bf16, int held, int shift, int d, int tid, int threads) {
  if (!p) {                                            // no weight: 1
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = i * threads + tid;
      float w[V];
#pragma unroll
      for (int k = 0; k < V; ++k) w[k] = has_column(c * V - shift, k, d) ? 1.0f : 0.0f;
      spread_quarters<V>(s, held, c, w);
    }
  } else if (bf16) {
    spread_shifted<__nv_bfloat16, V, NV>(s, static_cast<const __nv_bfloat16*>(p), held, shift, d, tid, threads);
  } else {
    spread_shifted<float, V, NV>(s, static_cast<const float*>(p), held, shift, d, tid, threads);
  }
}
template <int V>
__device__ __forceinline__ void chunk_weights(const float4* s, int held, int c, float2* w) {
#pragma unroll
  for (int q = 0; q < V / 4; ++q) {
    const float4 v = s[q * held + c];
    w[2 * q] = make_float2(v.x, v.y);
    w[2 * q + 1] = make_float2(v.z, v.w);
  }
}

constexpr int kRowMost = 16384;           // elements of a row that a block's registers hold
constexpr int kSharedMost = 228 * 1024;   // of an SM, for the blocks that run on it,
constexpr int kSharedOwn = 2304;          // with what each of them has besides its ring and weights

int shifts_of(int32_t d, int v) {         // shifts that rows of d elements have
  int n = 1;
  while (n < v && (int64_t)n * d % v != 0) n *= 2;
  return n;
}
// Chunks a thread holds in the backward pass: one in a single warp, otherwise 16 elements; of shifted bf16 rows on up to 128 threads 32
// (24 000 rows: of 2730 164 us so and 190 with 16, of 4096 with residual and fp32 gradients 187 and 154).
int row_form(int64_t chunks, int v, bool shift) { return chunks <= 32 ? 1 : shift && v == 8 && chunks * v <= 32 * 128 ? 32 / v : 16 / v; }
int row_threads(int64_t chunks, int nv) { return (int)align_up((size_t)ceil_div(chunks, nv), 32); }
// Blocks on an SM and rows in the ring: three rows where as many blocks still fit as the registers allow, two otherwise, and for the longest
// rows one.
struct RowPlan { int per_sm, stages; };
RowPlan plan_rows(int per_sm, int fixed, int stage) {
  RowPlan p{per_sm, 3};
  auto fits = [&] { return p.per_sm * (fixed + p.stages * stage + kSharedOwn) <= kSharedMost; };
  while (p.stages > 2 && !fits()) --p.stages;
  while (p.per_sm > 1 && !fits()) --p.per_sm;
  while (p.stages > 1 && !fits()) --p.stages;
  if (p.stages == 2 && p.per_sm * (fixed + 3 * stage + kSharedOwn) <= kSharedMost) p.stages = 3;
  return p;
}
// What a kernel may ask for belongs to the kernel, not to the call: the most that any plan asks for, once on each device, so that a call with
// less does not lower it between another thread's permission and its launch.
template <class Kernel>
cudaError_t allow_shared(Kernel kernel, std::atomic<int> (&ready)[64]) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
  if (ready[dev].load(std::memory_order_acquire)) return cudaSuccess;
  e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSharedMost - kSharedOwn);
  if (e == cudaSuccess) ready[dev].store(1, std::memory_order_release);
  return e;
}

// Mean and squared deviations of a row from sums over its warps, each about a point of its own:  with S_w = sum (x - near_w)^2 and
// E_w = sum (x - near_w),  mu = sum (n_w near_w + E_w) / d,  and with c = near_w - mu  M2 = sum S_w + c (2 E_w + n_w c),  exactly, whatever the points.
// near_w is the mean of the threads' first chunks, one of NV equal parts of the warp's columns and so at most sqrt(NV - 1) deviations off its mean:
// S_w is at most NV times the squares about that, and the differences lose two bits at the worst, as two passes with two barriers would not.
// (Without E_w what near_w is rounded by counts where the columns of different warps have different means: fp32 rows with a mean of 1000
// deviations had the variance off by 1e-4.)  A point that is not finite gives way to zero, so that the mean is that of the formula.
struct __align__(16) WarpStats { float near, count, squares, off; };
// ONE: a single warp of one chunk a thread, whose point is the row's mean.
template <bool ONE>
__device__ __forceinline__ float point_near(float mean) { return ONE || fabsf(mean) < INFINITY ? mean : 0.0f; }

// The sums of a and of b over a warp, by as many exchanges as of one: a's in lanes 0 to 15, b's in lanes 16 to 31.
__device__ __forceinline__ float warp_sums(float a, float b, int lane) {
  const bool high = lane & 16;
  float v = high ? b : a;
  v += __shfl_xor_sync(0xffffffffu, high ? a : b, 16);
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// From each warp's to the row's: mu, the point of this warp, becomes the mean (of CENTER), and the squared deviations from it are returned.
// squares, off: the thread's own shares of S_w and E_w;  the counts are in st.  A lane takes a warp (10 000 rows of 8192 of layer norm: 92 us
// so, 132 where every thread goes through all warps);  EACH: every thread all of them (24 000 aligned rows of 4096 of RMS norm, four warps each:
// 71 us so, 75 by lanes).  (Also the barrier between the row's reads of the ring and the copies that follow.)
template <bool CENTER, int MOST, bool EACH>
__device__ __forceinline__ float merge_warps(WarpStats* st, int lane, int warp, int warps, int d, float squares, float off, float& mu, float inv_d) {
  static_assert(!CENTER || !EACH, "the mean is summed by lanes");
  auto about = [&](const WarpStats& q) {
    const float c = q.near - mu;
    return fmaf(c, fmaf(q.count, c, 2.0f * q.off), q.squares);
  };
  if (warps == 1) {
    __syncwarp();
    if (!CENTER || MOST == 32) return warp_sum(squares);  // (about the mean already)
    const float v = warp_sums(squares, off, lane);
    const WarpStats q{mu, (float)d, __shfl_sync(0xffffffffu, v, 0), __shfl_sync(0xffffffffu, v, 16)};
    mu = fmaf(q.near, q.count, q.off) * inv_d;
    return about(q);
  }
  if (CENTER) {
    const float v = warp_sums(squares, off, lane);
    if (lane == 0) {
      st[warp].near = mu;
      st[warp].squares = v;
    }
    if (lane == 16) st[warp].off = v;
  } else {
    const float v = warp_sum(squares);
    if (lane == 0) st[warp].squares = v;
  }
  __syncthreads();
  float m2 = 0.0f;
  if (EACH) {
#pragma unroll 4
    for (int w = 0; w < warps; ++w) m2 += st[w].squares;
    return m2;
  }
  constexpr int kLanes = MOST <= 128 ? 4 : 32;         // (warps are fewer or as many)
  const int w = lane & (kLanes - 1);
  if (CENTER) {
    WarpStats q{0.0f, 0.0f, 0.0f, 0.0f};
    if (w < warps) q = st[w];
    float sum = fmaf(q.near, q.count, q.off);
#pragma unroll
    for (int o = 1; o < kLanes; o <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    mu = sum * inv_d;
    m2 = about(q);                                     // (of a lane without a warp zero, but where mu is not finite)
  } else if (w < warps) {
    m2 = st[w].squares;
  }
#pragma unroll
  for (int o = 1; o < kLanes; o <<= 1) m2 += __shfl_xor_sync(0xffffffffu, m2, o);
  return m2;
}

// Rows that begin on 16 bytes.  A block takes `span` rows in a row; the next row's inputs are on their way to registers while one is worked
// on.  (Through the ring 5 to 15 % slower: 24 000 rows of 4096 with a residual 125 and 132 us, without 72 and 77.)
template <typename X, int NV, int MOST, int LEAST, bool CENTER, bool RES>
__global__ void __launch_bounds__(MOST, LEAST) ln_fwd_kernel(FwdParams a, int span) {
  constexpr int V = 16 / (int)sizeof(X), P = V / 2;
  // The row stays in registers as fp32 values, or as it is in memory: with both inputs of the next row on their way there is no room for
  // the values (their loads would be put off; 24 000 rows of 4096 with a residual: 155 and 125 us).
  constexpr bool PACKED = RES && sizeof(X) == 2;
  // fp32 rows with a residual take up the registers of four blocks of 256 threads: one sum at a time (12 000 rows of 4096: 159 us so, 172 in
  // pairs).
  constexpr bool TIGHT = RES && CENTER && sizeof(X) == 4;
  __shared__ WarpStats s_stats[2][32];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, threads = blockDim.x, warps = threads >> 5;
  const int d = a.d;
  const float inv_d = 1.0f / (float)d;
  const int64_t t0 = (int64_t)blockIdx.x * span;
  const int rows = (int)(a.T - t0 < span ? a.T - t0 : span);
  const uint32_t live_rows = __ballot_sync(0xffffffffu, lane < rows && (!a.mask || a.mask[t0 + (lane < rows ? lane : 0)] != 0));
  Pack<X, V> next[NV], pr[RES ? NV : 1];
  auto column = [&](int i) { return (i * threads + tid) * V; };
  auto fetch = [&](int r) {
    if (!(live_rows >> r & 1)) return;
    const int64_t t = t0 + r;
    const X *const x = static_cast<const X*>(a.x) + t * a.ldx, *const res = static_cast<const X*>(a.residual) + t * d;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int j = column(i);
      if (j >= d) continue;
      next[i] = stream_pack<X, V>(x + j);
      if (RES) pr[i] = stream_pack<X, V>(res + j);
    }
  };
  fetch(0);
  int columns = 0, firsts = 0;                         // columns of this warp, and those in its threads' first chunks
  if (CENTER) {
#pragma unroll
    for (int i = 0; i < NV; ++i) columns += column(i) < d ? V : 0;
    columns = __reduce_add_sync(0xffffffffu, columns);
    firsts = __reduce_add_sync(0xffffffffu, column(0) < d ? V : 0);
  }
  if (CENTER && lane == 0) s_stats[0][warp].count = s_stats[1][warp].count = (float)columns;
  const float inv_firsts = firsts ? 1.0f / (float)firsts : 0.0f;
  int buf = 0;
#pragma unroll 1
  for (int r = 0; r < rows; ++r) {
    const int64_t t = t0 + r;
    X* const h = static_cast<X*>(a.h) + t * d;
    if (!(live_rows >> r & 1)) {                       // (all threads of the block: the bits are the same in every warp)
      float zero[V];
#pragma unroll
      for (int k = 0; k < V; ++k) zero[k] = 0.0f;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int j = column(i);
        if (j >= d) continue;
        store_values<V, false>(a.y, a.y_bf16, t * d, j, d, zero);
        if (RES) store_pack(h + j, round_pack<X, V>(zero));
      }
      if (tid == 0) {
        if (CENTER && a.mean) a.mean[t] = 0.0f;
        if (a.rstd) a.rstd[t] = 0.0f;
      }
      if (r + 1 < rows) fetch(r + 1);
      continue;
    }
    float2 f[PACKED ? 1 : NV * P] = {}, part = both(0.0f);
    Pack<X, V> now[PACKED ? NV : 1] = {};
    auto value = [&](int i, int p) {
      if constexpr (PACKED) return pair_of(now[i], p);
      else return f[i * P + p];
    };
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int j = column(i);
      if (j < d) {
        if (RES) {
          float2 sums[P];
#pragma unroll
          for (int p = 0; p < P; ++p) sums[p] = add2(pair_of(next[i], p), pair_of(pr[i], p));
          next[i] = round_pack<X, V>(&sums[0].x);
          store_pack(h + j, next[i]);
        }
        if constexpr (PACKED) now[i] = next[i];
#pragma unroll
        for (int p = 0; p < P; ++p) {
          if constexpr (!PACKED) f[i * P + p] = pair_of(next[i], p);
          if (CENTER && i == 0) part = add2(part, value(i, p));
        }
      } else {
        if constexpr (PACKED) zero_pack(now[i]);
#pragma unroll
        for (int p = 0; p < P; ++p)
          if constexpr (!PACKED) f[i * P + p] = both(0.0f);
      }
    }
    if (r + 1 < rows) fetch(r + 1);
    float mu = CENTER ? point_near<MOST == 32>(warp_sum(part.x + part.y) * inv_firsts) : 0.0f;
    part = both(0.0f);
    float2 off = both(0.0f);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      if (CENTER && column(i) >= d) continue;
#pragma unroll
      for (int p = 0; p < P; ++p) {
        const float2 c = CENTER ? add2(value(i, p), both(-mu)) : value(i, p);
        if constexpr (TIGHT) {
          part.x = fmaf(c.x, c.x, fmaf(c.y, c.y, part.x));
          off.x += c.x + c.y;
        } else {
          part = fma2(c, c, part);
          if (CENTER) off = add2(off, c);
        }
      }
    }
    const float m2 = merge_warps<CENTER, MOST, !CENTER && MOST <= 128>(s_stats[buf], lane, warp, warps, d, part.x + part.y, off.x + off.y, mu, inv_d);
    buf ^= 1;                                          // (of rows that are not masked: two barriers lie between two uses of a buffer)
    const float var = m2 * inv_d, rstd = rsqrtf(var + a.eps);
    if (tid == 0) {
      if (CENTER && a.mean) a.mean[t] = mu;
      if (a.rstd) a.rstd[t] = rstd;
      if (!(var < INFINITY)) flag(a.d_status, SPO_DEV_NONFINITE);
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int j = column(i);
      if (j >= d) continue;
      float2 w[P], b[P];
      load_weights<V>(a.weight, a.w_bf16, j, 1.0f, &w[0].x);
      if (a.bias) load_weights<V>(a.bias, a.w_bf16, j, 0.0f, &b[0].x);
#pragma unroll
      for (int p = 0; p < P; ++p) {
        const float2 xh = mul2(CENTER ? add2(value(i, p), both(-mu)) : value(i, p), both(rstd));
        w[p] = a.bias ? fma2(xh, w[p], b[p]) : mul2(xh, w[p]);
      }
      store_values<V, false>(a.y, a.y_bf16, t * d, j, d, &w[0].x);
    }
  }
}

// Rows that do not begin on 16 bytes, through the ring.  A block takes `span` rows of one shift; x rows of another shift than y's (`staged`)
// are copied by their own chunks and read by column after a barrier.
template <typename X, int NV, int MOST, int LEAST, bool CENTER, bool RES>
__global__ void __launch_bounds__(MOST, LEAST) ln_fwd_shift_kernel(FwdParams a, int span, int stages, int shifts) {
  constexpr int V = 16 / (int)sizeof(X), P = V / 2;
  constexpr bool SHIFT = true;
  __shared__ WarpStats s_stats[2][32];
  extern __shared__ __align__(16) char s_raw[];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, threads = blockDim.x, warps = threads >> 5;
  const int d = a.d, held = threads * NV;
  const float inv_d = 1.0f / (float)d;
  // rows first + k step, k < rows
  const int64_t first = blockIdx.x % shifts + (int64_t)shifts * span * (blockIdx.x / shifts);
  const int step = shifts;
  const int64_t reach = (a.T - first + step - 1) / step;
  const int rows = reach < 0 ? 0 : (int)(reach < span ? reach : span);
  const uint32_t live_rows = __ballot_sync(0xffffffffu, lane < rows && (!a.mask || a.mask[first + (int64_t)(lane < rows ? lane : 0) * step] != 0));
  const int shift = (int)((first * d) % V);
  const bool staged = a.ldx % V != d % V && a.T > 1;
  const int2 edges = edge_chunks<V>(shift, d, tid, threads);
  float4* const s_w = reinterpret_cast<float4*>(s_raw);
  float4* const s_b = s_w + V / 4 * held;
  const int fixed = held * V * 4 * (a.bias ? 2 : 1), x_bytes = held * 16 + 16;
  const int stage = x_bytes + (RES ? held * 16 : 0);
  auto column = [&](int i) { return (i * threads + tid) * V - shift; };
  auto fetch = [&](int r, int slot) {
    if (r < rows && (live_rows >> r & 1)) {
      const int64_t t = first + (int64_t)r * step;
      char* const s = s_raw + fixed + slot * stage;
      const X *const x = static_cast<const X*>(a.x) + t * a.ldx, *const res = static_cast<const X*>(a.residual) + t * d;
      const int own = staged ? (int)((t * a.ldx) % V) : shift;
      const int end_x = end_of(a.T, t, a.ldx, d), end = end_of(a.T, t, d, d);
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int c = i * threads + tid, j = c * V - shift, jx = c * V - own;
        if (jx < d) copy_chunk<X, V, SHIFT>(s + c * 16, x, jx, end_x);
        if (RES && j < d) copy_chunk<X, V, SHIFT>(s + x_bytes + c * 16, res, j, end);
      }
    }
    copies_issued();
  };
  for (int k = 0; k < stages - 1; ++k) fetch(k, k);
  spread_shifted<V, NV>(s_w, a.weight, a.w_bf16, held, shift, d, tid, threads);
  if (a.bias) spread_shifted<V, NV>(s_b, a.bias, a.w_bf16, held, shift, d, tid, threads);
  int columns = 0, firsts = 0;                         // columns of this warp, and those in its threads' first chunks
  if (CENTER) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      if (column(i) < d) columns += min(column(i) + V, d) - max(column(i), 0);
      if (i == 0) firsts = columns;
    }
    columns = __reduce_add_sync(0xffffffffu, columns);
    firsts = __reduce_add_sync(0xffffffffu, firsts);
  }
  if (CENTER && lane == 0) s_stats[0][warp].count = s_stats[1][warp].count = (float)columns;
  const float inv_firsts = firsts ? 1.0f / (float)firsts : 0.0f;
  int slot = 0, buf = 0;
#pragma unroll 1
  for (int k = 0; k < rows; ++k) {
    const int64_t t = first + (int64_t)k * step;
    char* const s = s_raw + fixed + slot * stage;
    fetch(k + stages - 1, slot == 0 ? stages - 1 : slot - 1);
    slot = slot + 1 == stages ? 0 : slot + 1;
    X* const h = static_cast<X*>(a.h) + t * d;
    copies_arrived(stages - 1);
    if (!(live_rows >> k & 1)) {                       // (all threads of the block: the bits are the same in every warp)
      float zero[V];
#pragma unroll
      for (int e = 0; e < V; ++e) zero[e] = 0.0f;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int j = column(i);
        if (j >= d) continue;
        store_values<V, SHIFT>(a.y, a.y_bf16, t * d, j, d, zero);
        if (RES) store_chunk<X, V, SHIFT>(h, j, d, round_pack<X, V>(zero));
      }
      if (tid == 0) {
        if (CENTER && a.mean) a.mean[t] = 0.0f;
        if (a.rstd) a.rstd[t] = 0.0f;
      }
      continue;
    }
    if (staged) __syncthreads();
    for (int e = 0; e < 2; ++e) {
      const int c = e == 0 ? edges.x : edges.y;
      if (c < 0) continue;
      if (!staged) blank<X, V>(s + c * 16, c * V - shift, d);
      if (RES) blank<X, V>(s + x_bytes + c * 16, c * V - shift, d);
    }
    const int own = staged ? (int)((t * a.ldx) % V) : 0;
    float2 f[NV * P], part = both(0.0f);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = i * threads + tid, j = column(i);
      if (j < d) {
        Pack<X, V> q;
        if (staged) q = staged_chunk<X, V>(s, own, j, d);
        else q = load_pack<X, V>(reinterpret_cast<const X*>(s + c * 16));
        if (RES) {
          const Pack<X, V> pr = load_pack<X, V>(reinterpret_cast<const X*>(s + x_bytes + c * 16));
          float2 sums[P];
#pragma unroll
          for (int p = 0; p < P; ++p) sums[p] = add2(pair_of(q, p), pair_of(pr, p));
          q = round_pack<X, V>(&sums[0].x);
          store_chunk<X, V, SHIFT>(h, j, d, q);
        }
#pragma unroll
        for (int p = 0; p < P; ++p) {
          f[i * P + p] = pair_of(q, p);
          if (CENTER && i == 0) part = add2(part, f[i * P + p]);
        }
      } else {
#pragma unroll
        for (int p = 0; p < P; ++p) f[i * P + p] = both(0.0f);
      }
    }
    float mu = CENTER ? point_near<MOST == 32>(warp_sum(part.x + part.y) * inv_firsts) : 0.0f;
    part = both(0.0f);
    float2 off = both(0.0f);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int j = column(i);
      if (CENTER && j >= d) continue;
#pragma unroll
      for (int p = 0; p < P; ++p) {
        float2 c = CENTER ? add2(f[i * P + p], both(-mu)) : f[i * P + p];
        if (CENTER && !is_whole<V, SHIFT>(j, d)) {
          if (!has_column(j, 2 * p, d)) c.x = 0.0f;
          if (!has_column(j, 2 * p + 1, d)) c.y = 0.0f;
        }
        part = fma2(c, c, part);
        if (CENTER) off = add2(off, c);
      }
    }
    const float m2 = merge_warps<CENTER, MOST, false>(s_stats[buf], lane, warp, warps, d, part.x + part.y, off.x + off.y, mu, inv_d);
    buf ^= 1;
    const float var = m2 * inv_d, rstd = rsqrtf(var + a.eps);
    if (tid == 0) {
      if (CENTER && a.mean) a.mean[t] = mu;
      if (a.rstd) a.rstd[t] = rstd;
      if (!(var < INFINITY)) flag(a.d_status, SPO_DEV_NONFINITE);
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int j = column(i);
      if (j >= d) continue;
      float2 w[P], b[P];
      chunk_weights<V>(s_w, held, i * threads + tid, w);
      if (a.bias) chunk_weights<V>(s_b, held, i * threads + tid, b);
#pragma unroll
      for (int p = 0; p < P; ++p) {
        const float2 xh = mul2(CENTER ? add2(f[i * P + p], both(-mu)) : f[i * P + p], both(rstd));
        w[p] = a.bias ? fma2(xh, w[p], b[p]) : mul2(xh, w[p]);
      }
      store_values<V, SHIFT>(a.y, a.y_bf16, t * d, j, d, &w[0].x);
    }
  }
  copies_arrived(0);
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

constexpr int kFwdSpan = 4, kFwdSpanShift = 16, kFwdRounds = 3;
// Rows of a block: as many as leave so many rounds of blocks over the GPU, or one round of a short batch.
int fwd_span(int64_t T, int per_sm, int rounds, int most) {
  const int64_t at_once = (int64_t)sm_count() * per_sm, span = T <= rounds * at_once ? ceil_div(T, at_once) : T / (rounds * at_once);
  return (int)(span < 1 ? 1 : span > most ? most : span);
}

template <typename X, int NV, int MOST, int LEAST, bool CENTER, bool RES>
cudaError_t run_fwd(const FwdParams& a, int64_t chunks, bool shift, cudaStream_t st) {
  constexpr int V = 16 / (int)sizeof(X);
  const int threads = row_threads(chunks, NV), held = threads * NV;
  const int by_registers = LEAST * MOST / threads > 32 ? 32 : LEAST * MOST / threads > 1 ? LEAST * MOST / threads : 1;
  if (!shift) {
    const int span = fwd_span(a.T, by_registers, kFwdRounds, kFwdSpan);
    ln_fwd_kernel<X, NV, MOST, LEAST, CENTER, RES><<<(unsigned)ceil_div(a.T, span), threads, 0, st>>>(a, span);
    return cudaGetLastError();
  }
  const auto kernel = ln_fwd_shift_kernel<X, NV, MOST, LEAST, CENTER, RES>;
  const int fixed = held * V * 4 * (a.bias ? 2 : 1), stage = held * 16 + 16 + (RES ? held * 16 : 0);
  const RowPlan p = plan_rows(by_registers, fixed, stage);
  const int shifts = shifts_of(a.d, V), span = fwd_span(a.T, p.per_sm, kFwdRounds, kFwdSpanShift), smem = fixed + p.stages * stage;
  static std::atomic<int> ready[64];
  const cudaError_t e = allow_shared(kernel, ready);
  if (e != cudaSuccess) return e;
  kernel<<<(unsigned)(ceil_div(a.T, (int64_t)span * shifts) * shifts), threads, smem, st>>>(a, span, p.stages, shifts);
  return cudaGetLastError();
}

template <typename X, bool CENTER, bool RES>
cudaError_t pick_fwd(const FwdParams& a, cudaStream_t st) {
  constexpr int V = 16 / (int)sizeof(X);
  const bool shift = !(a.d % V == 0 && (a.T == 1 || a.ldx % V == 0));
  const int64_t chunks = ceil_div(shift ? a.d + V - 1 : a.d, V);
  const int nv = chunks <= 32 ? 1 : chunks <= 4 * 128 ? 4 : 16 / V, threads = row_threads(chunks, nv), held = threads * nv;
  if (a.d > kRowMost || threads > 1024 || (shift && held * (V * 8 + 32) + 16 + kSharedOwn > kSharedMost)) {
    ln_fwd_long_kernel<X, CENTER><<<(unsigned)a.T, 1024, 0, st>>>(a);
    return cudaGetLastError();
  }
  // Where there are fewer rows than SMs, as many threads as there are chunks: one row of 4096 takes 2.7 us so and 3.4 on 128 threads.
  if (chunks <= 32) return run_fwd<X, 1, 32, 20, CENTER, RES>(a, chunks, shift, st);
  if (chunks <= 1024 && a.T <= sm_count()) return run_fwd<X, 1, 1024, 1, CENTER, RES>(a, chunks, shift, st);
  if (chunks <= 4 * 128) return run_fwd<X, 4, 128, 5, CENTER, RES>(a, chunks, shift, st);
  return run_fwd<X, 16 / V, 1024, 1, CENTER, RES>(a, chunks, shift, st);
}

// ---------------------------------------------------------------------------
// backward
// ---------------------------------------------------------------------------
struct BwdParams {
  const void *dy, *x, *weight, *dh;
  const uint8_t* mask;
  const float *mean, *rstd;
  int64_t ldx, T;
  int32_t d, w_bf16, dy_bf16;
  void* dx;
  float* partial;                // [blocks][want][d]: dw, then db
  int want_dw, want_db;
};

// V sums to a partial row of d of them, which begins on 16 bytes only where d is a multiple of 4.
template <int V, bool SHIFT>
__device__ __forceinline__ void store_partial(float* row, int j, int d, const float* f) {
  if constexpr (SHIFT) {
#pragma unroll
    for (int k = 0; k < V; ++k)
      if (has_column(j, k, d)) row[j + k] = f[k];
  } else {
    store_pack(row + j, round_pack<float, V>(f));
  }
}

// A block walks through rows b, b + blocks, ... (shifted ones: the number of blocks is a multiple of that of shifts); its threads keep
// their columns for all of them, so the sums of dw and db stay in registers, and each block leaves one partial row of both.  A row is
// read twice from shared memory, for the two row means and for dx.  Columns that are not a shifted row's are zeros of x, dy and w, which
// add nothing.
// Bytes of the ring and the weights of a block: `held` chunks.
struct BwdShared {
  int weights, x, dy, dh, stage;
};
__host__ __device__ __forceinline__ BwdShared bwd_shared(int held, int v, int dy_size, bool dh, bool shift) {
  BwdShared b;
  b.weights = held * v * 4;
  b.x = held * 16 + (shift ? 16 : 0);
  b.dy = align16(held * v * dy_size);
  b.dh = dh ? held * 16 : 0;
  b.stage = b.x + b.dy + b.dh;
  return b;
}

template <typename X, int NV, int MOST, int LEAST, bool SHIFT, bool CENTER, bool DB>
__global__ void __launch_bounds__(MOST, LEAST) ln_bwd_kernel(BwdParams a, int stages) {
  constexpr int V = 16 / (int)sizeof(X), P = V / 2;
  __shared__ float2 s_sum[2][32];
  extern __shared__ __align__(16) char s_raw[];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, threads = blockDim.x, warps = threads >> 5;
  const int d = a.d, held = threads * NV, dy_size = a.dy_bf16 ? 2 : 4;
  const BwdShared at = bwd_shared(held, V, dy_size, a.dh != nullptr, SHIFT);
  float4* const s_w = reinterpret_cast<float4*>(s_raw);
  char* const s_ring = s_raw + at.weights;
  const int64_t first = blockIdx.x, step = gridDim.x;
  const int shift = SHIFT ? (int)((first * d) % V) : 0;
  const bool staged = SHIFT && a.ldx % V != d % V && a.T > 1;
  const int2 edges = edge_chunks<V>(shift, d, tid, threads);
  auto column = [&](int i) { return (i * threads + tid) * V - shift; };

  // a row's mask byte (0 behind the last row), looked at a row later: a comparison here would wait for it
  auto mask_of = [&](int64_t t) -> uint32_t {
    uint32_t m = t < a.T;
    if (a.mask && t < a.T) asm volatile("ld.global.u8 %0, [%1];" : "=r"(m) : "l"(a.mask + t));
    return m;
  };
  auto fetch = [&](int64_t t, bool live, int slot) {
    if (live) {
      char* const s = s_ring + slot * at.stage;
      const X *const x = static_cast<const X*>(a.x) + t * a.ldx, *const dh = static_cast<const X*>(a.dh) + t * d;
      const int own = staged ? (int)((t * a.ldx) % V) : shift;
      const int end_x = SHIFT ? end_of(a.T, t, a.ldx, d) : 0, end = SHIFT ? end_of(a.T, t, d, d) : 0;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int c = i * threads + tid, j = c * V - shift, jx = c * V - own;
        if (jx < d) copy_chunk<X, V, SHIFT>(s + c * 16, x, jx, end_x);
        if (j >= d) continue;
        if (a.dy_bf16) copy_chunk<__nv_bfloat16, V, SHIFT>(s + at.x + c * V * 2, static_cast<const __nv_bfloat16*>(a.dy) + t * d, j, end);
        else copy_chunk<float, V, SHIFT>(s + at.x + c * V * 4, static_cast<const float*>(a.dy) + t * d, j, end);
        if (a.dh) copy_chunk<X, V, SHIFT>(s + at.x + at.dy + c * 16, dh, j, end);
      }
    }
    copies_issued();
  };
  // the first rows on their way, then the weights
  uint32_t live_bits = 0;                               // bit i: row i from the current one on
  for (int k = 0; k < stages - 1; ++k) {
    const bool live = mask_of(first + k * step) != 0;
    live_bits |= (uint32_t)live << k;
    fetch(first + k * step, live, k);
  }
  uint32_t mask_next = mask_of(first + (stages - 1) * step);
  float r_next = first < a.T ? a.rstd[first] : 0.0f, mu_next = CENTER && first < a.T ? a.mean[first] : 0.0f;
  if constexpr (SHIFT) {
    spread_shifted<V, NV>(s_w, a.weight, a.w_bf16, held, shift, d, tid, threads);
  } else {
#pragma unroll
    for (int i = 0; i < NV; ++i) spread_weights<V>(s_w, a.weight, a.w_bf16, held, i * threads + tid, d);
  }
  float2 dw[NV * P], db[DB ? NV * P : 1];
#pragma unroll
  for (int e = 0; e < NV * P; ++e) {
    dw[e] = both(0.0f);
    if constexpr (DB) db[e] = both(0.0f);
  }
  const float inv_d = 1.0f / (float)d;
  int slot = 0, buf = 0;
#pragma unroll 1
  for (int64_t t = first; t < a.T; t += step) {
    const int64_t ahead = t + (stages - 1) * step;
    const bool live_ahead = mask_next != 0;
    live_bits |= (uint32_t)live_ahead << (stages - 1);
    fetch(ahead, live_ahead, slot == 0 ? stages - 1 : slot - 1);
    mask_next = mask_of(ahead + step);
    const float r = r_next, mu = mu_next;
    if (t + step < a.T) {
      r_next = a.rstd[t + step];
      if (CENTER) mu_next = a.mean[t + step];
    }
    const bool live = live_bits & 1;
    live_bits >>= 1;
    char* const s = s_ring + slot * at.stage;
    slot = slot + 1 == stages ? 0 : slot + 1;
    X* const out = static_cast<X*>(a.dx) + t * d;
    copies_arrived(stages - 1);
    if (!live) {                                        // (the same for all threads of the block)
      Pack<X, V> zero;
      zero_pack(zero);
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if (column(i) < d) store_chunk<X, V, SHIFT>(out, column(i), d, zero);
      continue;
    }
    if (SHIFT) {
      if (staged) __syncthreads();
      for (int e = 0; e < 2; ++e) {
        const int c = e == 0 ? edges.x : edges.y, j = c * V - shift;
        if (c < 0) continue;
        if (!staged) blank<X, V>(s + c * 16, j, d);
        if (a.dy_bf16) blank<__nv_bfloat16, V>(s + at.x + c * V * 2, j, d);
        else blank<float, V>(s + at.x + c * V * 4, j, d);
      }
    }
    const int own = staged ? (int)((t * a.ldx) % V) : 0;
    auto normalised = [&](int i, float2* xh) {          // of chunk i
      const int c = i * threads + tid;
      Pack<X, V> px;
      if (SHIFT && staged) px = staged_chunk<X, V>(s, own, column(i), d);
      else px = load_pack<X, V>(reinterpret_cast<const X*>(s + c * 16));
#pragma unroll
      for (int p = 0; p < P; ++p) xh[p] = mul2(CENTER ? add2(pair_of(px, p), both(-mu)) : pair_of(px, p), both(r));
    };
    auto gradient = [&](int i, float2* g) {
      const int c = i * threads + tid;
      if (a.dy_bf16) {
        const Pack<__nv_bfloat16, V> q = load_pack<__nv_bfloat16, V>(reinterpret_cast<const __nv_bfloat16*>(s + at.x) + c * V);
#pragma unroll
        for (int p = 0; p < P; ++p) g[p] = pair_of(q, p);
      } else {
        const Pack<float, V> q = load_pack<float, V>(reinterpret_cast<const float*>(s + at.x) + c * V);
#pragma unroll
        for (int p = 0; p < P; ++p) g[p] = pair_of(q, p);
      }
    };
    auto weights = [&](int i, float2* w) { chunk_weights<V>(s_w, held, i * threads + tid, w); };
    float2 p1 = both(0.0f), p2 = both(0.0f);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      if (column(i) >= d) continue;
      float2 xh[P], g[P], w[P];
      normalised(i, xh);
      gradient(i, g);
      weights(i, w);
#pragma unroll
      for (int p = 0; p < P; ++p) {
        dw[i * P + p] = fma2(g[p], xh[p], dw[i * P + p]);
        if constexpr (DB) db[i * P + p] = add2(db[i * P + p], g[p]);
        const float2 up = mul2(g[p], w[p]);
        p1 = fma2(up, xh[p], p1);
        if (CENTER) p2 = add2(p2, up);
      }
    }
    float s1 = p1.x + p1.y, s2 = p2.x + p2.y;
    if (CENTER) {
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) {
        const float2 v = add2(make_float2(s1, s2), make_float2(__shfl_xor_sync(0xffffffffu, s1, o), __shfl_xor_sync(0xffffffffu, s2, o)));
        s1 = v.x;
        s2 = v.y;
      }
    } else {
      s1 = warp_sum(s1);
    }
    if (warps > 1) {
      if (lane == 0) s_sum[buf][warp] = make_float2(s1, s2);
      __syncthreads();
      s1 = s2 = 0.0f;
#pragma unroll 4
      for (int q = 0; q < warps; ++q) {
        const float2 v = s_sum[buf][q];
        s1 += v.x;
        if (CENTER) s2 += v.y;
      }
      buf ^= 1;                                         // (of rows that are not masked: two barriers lie between two uses of a buffer)
    }
    // dx = r (up - mean up - xh mean(up xh)) + dh
    const float c1 = -inv_d * s1, c2 = -inv_d * s2;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = i * threads + tid, j = column(i);
      if (j >= d) continue;
      float2 xh[P], g[P], w[P];
      normalised(i, xh);
      gradient(i, g);
      weights(i, w);
#pragma unroll
      for (int p = 0; p < P; ++p) w[p] = fma2(xh[p], both(c1), CENTER ? fma2(g[p], w[p], both(c2)) : mul2(g[p], w[p]));
      if (a.dh) {
        const Pack<X, V> ph = load_pack<X, V>(reinterpret_cast<const X*>(s + at.x + at.dy) + c * V);
#pragma unroll
        for (int p = 0; p < P; ++p) w[p] = fma2(w[p], both(r), pair_of(ph, p));
      } else {
#pragma unroll
        for (int p = 0; p < P; ++p) w[p] = mul2(w[p], both(r));
      }
      store_chunk<X, V, SHIFT>(out, j, d, round_pack<X, V>(&w[0].x));
    }
    if (staged) __syncthreads();                        // others read these chunks of x: they are overwritten in the next round
  }
  copies_arrived(0);
  if (!a.partial) return;
  pdl_release();
  float* const row = a.partial + (int64_t)blockIdx.x * (a.want_dw + a.want_db) * d;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int j = column(i);
    if (j >= d) continue;
    float* const both_rows[2] = {a.want_dw ? row : nullptr, a.want_db ? row + (int64_t)a.want_dw * d : nullptr};
    if (both_rows[0]) store_partial<V, SHIFT>(both_rows[0], j, d, &dw[i * P].x);
    if constexpr (DB) {
      if (both_rows[1]) store_partial<V, SHIFT>(both_rows[1], j, d, &db[i * P].x);
    }
  }
}

// Rows longer than a block's registers hold: one block per row finds the two means and writes dx ...
__device__ __forceinline__ float one_gradient(const BwdParams& a, int64_t at) {
  return a.dy_bf16 ? element(load_pack<__nv_bfloat16, 1>(static_cast<const __nv_bfloat16*>(a.dy) + at), 0) : static_cast<const float*>(a.dy)[at];
}
template <typename X, bool CENTER>
__global__ void __launch_bounds__(1024) ln_bwd_long_rows_kernel(BwdParams a) {
  __shared__ float2 s_sum[32];
  const int64_t t = blockIdx.x;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, nw = blockDim.x >> 5;
  const bool live = !a.mask || a.mask[t] != 0;
  const X* x = static_cast<const X*>(a.x) + t * a.ldx;
  const X* dh = a.dh ? static_cast<const X*>(a.dh) + t * a.d : nullptr;
  X* dx = static_cast<X*>(a.dx) + t * a.d;
  const float r = live ? a.rstd[t] : 0.0f, mu = CENTER && live ? a.mean[t] : 0.0f;
  float s1 = 0.0f, s2 = 0.0f;
  if (live)
    for (int64_t c = threadIdx.x; c < a.d; c += blockDim.x) {
      float w;
      load_weights<1>(a.weight, a.w_bf16, c, 1.0f, &w);
      const float up = w * one_gradient(a, t * a.d + c);
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
      o = r * fmaf(-xh, s1, w * one_gradient(a, t * a.d + c) - s2);
      if (dh) o += element(load_pack<X, 1>(dh + c), 0);
    }
    store_pack(dx + c, round_pack<X, 1>(&o));
  }
}

// ... and before that (dx may take dy's place) blocks of 256 columns by a share of the rows sum dw and db.
template <typename X, bool CENTER>
__global__ void __launch_bounds__(256) ln_bwd_long_cols_kernel(BwdParams a) {
  const int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (c >= a.d) return;
  float dw = 0.0f, db = 0.0f;
  for (int64_t t = blockIdx.y; t < a.T; t += gridDim.y) {
    if (a.mask && a.mask[t] == 0) continue;
    const float dy = one_gradient(a, t * a.d + c);
    const float x = element(load_pack<X, 1>(static_cast<const X*>(a.x) + t * a.ldx + c), 0);
    dw = fmaf(dy, (x - (CENTER ? a.mean[t] : 0.0f)) * a.rstd[t], dw);
    db += dy;
  }
  float* row = a.partial + (int64_t)blockIdx.y * (a.want_dw + a.want_db) * a.d;
  if (a.want_dw) row[c] = dw;
  if (a.want_db) row[(int64_t)a.want_dw * a.d + c] = db;
}

// dw and db from the blocks' partial rows, in their order: 32 columns a block, and as many warps as leave each some four rows.
__global__ void __launch_bounds__(1024) ln_bwd_columns_kernel(const float* __restrict__ partial, int parts, int64_t width, int32_t d, void* dw,
                                                              void* db, int bf16, int accumulate) {
  __shared__ float s_sum[32][32];
  pdl_wait();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  const int64_t j = (int64_t)blockIdx.x * 32 + lane;
  float sum = 0.0f;
  if (j < width) {
#pragma unroll 8
    for (int p = warp; p < parts; p += warps) sum += partial[(int64_t)p * width + j];
  }
  s_sum[warp][lane] = sum;
  __syncthreads();
  if (warp != 0 || j >= width) return;
  for (int q = 1; q < warps; ++q) sum += s_sum[q][lane];
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

// The launch of a backward pass.  The number of blocks is at most bwd_blocks_most(), so that the scratch can be sized by d and T alone.
int bwd_per_sm(int threads) { return threads <= 512 ? 512 / threads : 1; }
int64_t bwd_blocks_most(int64_t T, int32_t d) {
  int64_t most = T < 64 ? T : 64;          // of rows that take the long form
  if (d > kRowMost) return most;
  for (int v : {4, 8}) {                   // rows of fp32 and of bf16; shifted rows may have a chunk more
    for (bool shift : {false, true}) {
      const int64_t chunks = ceil_div(shift ? d + v - 1 : d, v);
      const int64_t n = (int64_t)sm_count() * bwd_per_sm(row_threads(chunks, row_form(chunks, v, shift)));
      most = n > most ? n : most;
    }
  }
  const int64_t rows = (T + 7) / 8 * 8;    // shifted rows: blocks are a multiple of the shifts, up to eight
  return rows < most ? rows : most;
}

template <typename X, int NV, int MOST, int LEAST, bool SHIFT, bool CENTER, bool DB>
cudaError_t run_bwd(const BwdParams& a, int64_t chunks, int* blocks, cudaStream_t st) {
  constexpr int V = 16 / (int)sizeof(X);
  const auto kernel = ln_bwd_kernel<X, NV, MOST, LEAST, SHIFT, CENTER, DB>;
  const int threads = row_threads(chunks, NV);
  const BwdShared at = bwd_shared(threads * NV, V, a.dy_bf16 ? 2 : 4, a.dh != nullptr, SHIFT);
  const RowPlan p = plan_rows(bwd_per_sm(threads), at.weights, at.stage);
  const int shifts = SHIFT ? shifts_of(a.d, V) : 1;
  const int64_t most = (int64_t)sm_count() * p.per_sm / shifts * shifts, rows = (a.T + shifts - 1) / shifts * shifts;
  *blocks = (int)(rows < most ? rows : most);
  const int smem = at.weights + p.stages * at.stage;
  static std::atomic<int> ready[64];
  const cudaError_t e = allow_shared(kernel, ready);
  if (e != cudaSuccess) return e;
  kernel<<<*blocks, threads, smem, st>>>(a, p.stages);
  return cudaGetLastError();
}

template <typename X, bool CENTER, bool DB>
cudaError_t pick_bwd(const BwdParams& a, int* blocks, cudaStream_t st) {
  constexpr int V = 16 / (int)sizeof(X);
  const bool shift = !(a.d % V == 0 && (a.T == 1 || a.ldx % V == 0));
  const int64_t chunks = ceil_div(shift ? a.d + V - 1 : a.d, V);
  const int nv = row_form(chunks, V, shift), threads = row_threads(chunks, nv);
  const BwdShared at = bwd_shared(threads * nv, V, a.dy_bf16 ? 2 : 4, a.dh != nullptr, shift);
  if (a.d > kRowMost || threads > 1024 || at.weights + at.stage + kSharedOwn > kSharedMost) {
    *blocks = (int)(a.T < 64 ? a.T : 64);
    cudaError_t e = cudaSuccess;
    if (a.partial) {
      ln_bwd_long_cols_kernel<X, CENTER><<<dim3((unsigned)ceil_div(a.d, 256), *blocks), 256, 0, st>>>(a);
      if ((e = cudaGetLastError()) != cudaSuccess) return e;
    }
    ln_bwd_long_rows_kernel<X, CENTER><<<(unsigned)a.T, 1024, 0, st>>>(a);
    return cudaGetLastError();
  }
  auto form = [&](auto sh) {
    constexpr bool S = decltype(sh)::value;
    if (chunks <= 32) return run_bwd<X, 1, 32, 16, S, CENTER, DB>(a, chunks, blocks, st);
    if constexpr (S && V == 8) {
      if (nv == 32 / V) return run_bwd<X, 32 / V, 128, 4, S, CENTER, DB>(a, chunks, blocks, st);
    }
    if (threads <= 256) return run_bwd<X, 16 / V, 256, 2, S, CENTER, DB>(a, chunks, blocks, st);
    if (threads <= 512) return run_bwd<X, 16 / V, 512, 1, S, CENTER, DB>(a, chunks, blocks, st);
    return run_bwd<X, 16 / V, 1024, 1, S, CENTER, DB>(a, chunks, blocks, st);
  };
  return shift ? form(std::true_type{}) : form(std::false_type{});
}

}  // namespace

size_t layernorm_bwd_ws_bytes(int64_t T, int32_t d) {
  if (T < 1) return 256;
  return align_up((size_t)bwd_blocks_most(T, d) * 2 * (size_t)d * sizeof(float), 256);
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
  BwdParams a{};
  a.dy = q.dy; a.x = q.x; a.weight = q.weight; a.dh = q.dh; a.mask = q.mask; a.mean = q.mean; a.rstd = q.rstd; a.ldx = q.ldx;
  a.T = q.T; a.d = q.d; a.w_bf16 = q.w_dtype == SPO_DTYPE_BF16; a.dy_bf16 = q.dy_dtype == SPO_DTYPE_BF16; a.dx = q.dx;
  a.want_dw = q.dw != nullptr; a.want_db = q.db != nullptr;
  a.partial = a.want_dw || a.want_db ? reinterpret_cast<float*>(ws) : nullptr;
  int blocks = 0;
  auto typed = [&](auto center, auto bias) {
    constexpr bool C = decltype(center)::value, D = decltype(bias)::value;
    return q.dtype == SPO_DTYPE_BF16 ? pick_bwd<__nv_bfloat16, C, D>(a, &blocks, st) : pick_bwd<float, C, D>(a, &blocks, st);
  };
  using yes = std::true_type;
  using no = std::false_type;
  if (q.kind == SPO_NORM_LAYER) e = q.db ? typed(yes{}, yes{}) : typed(yes{}, no{});
  else e = q.db ? typed(no{}, yes{}) : typed(no{}, no{});
  if (e != cudaSuccess || !a.partial) return e;
  const int64_t width = (int64_t)(a.want_dw + a.want_db) * q.d;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)ceil_div(width, 32));
  cfg.blockDim = dim3(32u * (unsigned)(blocks >= 128 ? 32 : ceil_div(blocks, 4)));
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, ln_bwd_columns_kernel, (const float*)a.partial, blocks, width, q.d, q.dw, q.db,
                            (int)(q.dw_dtype == SPO_DTYPE_BF16), (int)q.dw_accumulate);
}

}  // namespace spo
