// What follows the gradients: their global norm with the clip factor (spo_grad_norm) and the AdamW step (spo_adamw_update), each over
// many tensors in one launch, with the optimiser's states in 32 or in 8 bits (spo_adamw_decode: the values of 8-bit states).
//
//   g~ = f g;  m' = b1 m + (1 - b1) g~;  v' = b2 v + (1 - b2) g~^2;
//   w' = w - ( lr/(1 - b1^t) m' / (sqrt(v') / sqrt(1 - b2^t) + eps) + lr decay w ).
//
// Everything here is bound by HBM.  The table of tensors travels in the kernel's parameters: no copy to the device, nothing kept
// between calls, and a captured launch carries its own.
//
// 8-bit states: blocks of 256 consecutive elements share an fp32 scale s, the largest magnitude of the block (or a floor);
//   m = s sgn(c) (c/127)^2,  v = s (c/255)^4,
// so that neighbouring codes are 1.6 % of the value apart at the top and cover 1.6e-5 (m) and 4e-10 (v) of it at the bottom.  A code is
// the number of borders (j - 1/2)^2 or (j - 1/2)^4 at or below the magnitude in units of the first code; every operation up to that
// comparison is rounded by itself (nothing fused), so the codes are fixed bit for bit.  v > 0 never takes code 0: the step's
// denominator does not vanish beside a momentum that is not zero.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include "spo_internal.h"

namespace spo {
namespace {

__device__ __forceinline__ void flag(int32_t* d_status, int bit) {
  if (d_status) atomicOr(d_status, bit);
}
__device__ __forceinline__ void pdl_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void pdl_release() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

__device__ __forceinline__ float low_bf16(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float high_bf16(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// ---------------------------------------------------------------------------
// gradient norm
// ---------------------------------------------------------------------------
constexpr int kNormThreads = 256;
constexpr int kNormChunk = 8192;                    // elements that a block takes at a time
constexpr int kNormBlocksPerSm = 8;
constexpr int kGradsMost = 1200;                    // tensors per launch: 24 bytes each, of the 32764 bytes that parameters may have
constexpr int kGradsFew = 40;

struct Grad {
  const void* g;
  uint64_t n_type;                                  // 2 n + (1 for bf16)
  uint64_t first;                                   // chunk of the launch that is its first
};
template <int N>
struct GradTable {
  Grad t[N];
  int32_t count;
  uint64_t chunks;
};

// The last index whose first chunk is at or below `chunk`.
template <class Table>
__device__ __forceinline__ int find_tensor(const Table& tab, uint64_t chunk) {
  int lo = 0, hi = tab.count - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (tab.t[mid].first <= chunk) lo = mid; else hi = mid - 1;
  }
  return lo;
}

// Squares of one thread's share are summed in fp32; where that sum leaves the range in which this loses nothing it is formed again
// in fp64.
template <int N>
__device__ __forceinline__ double sum_squares(const float (&f)[N]) {
  float s = 0.0f;
#pragma unroll
  for (int k = 0; k < N; ++k) s = fmaf(f[k], f[k], s);
  if (s > 0x1p-80f && s < INFINITY) return (double)s;
  float any = 0.0f;
#pragma unroll
  for (int k = 0; k < N; ++k) any = fmaxf(any, fabsf(f[k]));
  if (s == 0.0f && any == 0.0f) return 0.0;         // (a NaN is in s)
  double d = 0.0;
#pragma unroll
  for (int k = 0; k < N; ++k) d = fma((double)f[k], (double)f[k], d);
  return d;
}

__device__ __forceinline__ double block_sum(double v, double* s_part) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  if ((threadIdx.x & 31) == 0) s_part[threadIdx.x >> 5] = v;
  __syncthreads();
  v = 0.0;
  for (int w = 0; w < (int)(blockDim.x >> 5); ++w) v += s_part[w];
  return v;
}

__device__ __forceinline__ void finish_norm(double sum, float max_norm, float scale, float* out, int32_t* d_status) {
  const double norm = sqrt(sum) * fabs((double)scale);
  const float n = (float)norm;
  const bool fine = n < INFINITY;
  out[0] = n;
  out[1] = fine ? (float)((double)scale * (max_norm > 0.0f && norm > (double)max_norm ? (double)max_norm / norm : 1.0)) : NAN;
  out[2] = fine ? 1.0f : 0.0f;
  out[3] = 0.0f;
  if (!fine) flag(d_status, SPO_DEV_NONFINITE);
}

// Block b leaves its sum in partial[b] (adds to it for b < have: an earlier launch of the same call left one there).  A call of one block
// finishes by itself.
template <int N>
__global__ void __launch_bounds__(kNormThreads) grad_norm_kernel(const __grid_constant__ GradTable<N> tab, double* partial, int have,
                                                                 int last, float max_norm, float scale, float* out,
                                                                 int32_t* d_status) {
  __shared__ double s_part[kNormThreads / 32];
  pdl_release();
  double sum = 0.0;
  if (blockIdx.x < tab.chunks) {
    int i = find_tensor(tab, blockIdx.x);
    for (uint64_t chunk = blockIdx.x; chunk < tab.chunks; chunk += gridDim.x) {
      while (i + 1 < tab.count && tab.t[i + 1].first <= chunk) ++i;
      const bool bf16 = tab.t[i].n_type & 1;
      const int64_t n = (int64_t)(tab.t[i].n_type >> 1), base = (int64_t)(chunk - tab.t[i].first) * kNormChunk;
      const void* g = tab.t[i].g;
      const bool whole = n - base >= kNormChunk && (reinterpret_cast<uintptr_t>(g) & 15) == 0;
      if (whole && bf16) {
        const uint4* p = reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(g) + base) + threadIdx.x;
        uint4 q[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) q[k] = __ldcs(p + k * kNormThreads);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float f[8] = {low_bf16(q[k].x), high_bf16(q[k].x), low_bf16(q[k].y), high_bf16(q[k].y),
                              low_bf16(q[k].z), high_bf16(q[k].z), low_bf16(q[k].w), high_bf16(q[k].w)};
          sum += sum_squares(f);
        }
      } else if (whole) {
        const float4* p = reinterpret_cast<const float4*>(static_cast<const float*>(g) + base) + threadIdx.x;
        float4 q[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) q[k] = __ldcs(p + k * kNormThreads);
#pragma unroll
        for (int k = 0; k < 8; k += 2) {
          const float f[8] = {q[k].x, q[k].y, q[k].z, q[k].w, q[k + 1].x, q[k + 1].y, q[k + 1].z, q[k + 1].w};
          sum += sum_squares(f);
        }
      } else {
        const int64_t end = n - base < kNormChunk ? n : base + kNormChunk;
        for (int64_t e = base + threadIdx.x; e < end; e += kNormThreads) {
          const float f[1] = {bf16 ? low_bf16(static_cast<const uint16_t*>(g)[e]) : static_cast<const float*>(g)[e]};
          sum += sum_squares(f);
        }
      }
    }
  }
  sum = block_sum(sum, s_part);
  if (threadIdx.x == 0) {
    if ((int)blockIdx.x < have) sum += partial[blockIdx.x];
    if (last && gridDim.x == 1 && have <= 1) {
      finish_norm(sum, max_norm, scale, out, d_status);
    } else {
      partial[blockIdx.x] = sum;
    }
  }
}

__global__ void __launch_bounds__(kNormThreads) grad_norm_finish_kernel(const double* partial, int parts, float max_norm, float scale,
                                                                        float* out, int32_t* d_status) {
  __shared__ double s_part[kNormThreads / 32];
  pdl_wait();
  double sum = 0.0;
#pragma unroll 4
  for (int p = threadIdx.x; p < parts; p += kNormThreads) sum += partial[p];
  sum = block_sum(sum, s_part);
  if (threadIdx.x == 0) finish_norm(sum, max_norm, scale, out, d_status);
}

template <int N>
cudaError_t norm_launch(const spo_grad_tensor* grads, int from, int to, double* partial, int* have, bool last, float max_norm, float scale,
                        float* out, int32_t* d_status, cudaStream_t st) {
  GradTable<N> tab;
  tab.count = 0;
  tab.chunks = 0;
  for (int i = from; i < to; ++i) {
    if (grads[i].n == 0) continue;
    tab.t[tab.count++] = Grad{grads[i].g, (uint64_t)grads[i].n * 2 + (grads[i].dtype == SPO_DTYPE_BF16), tab.chunks};
    tab.chunks += (uint64_t)ceil_div(grads[i].n, kNormChunk);
  }
  const int64_t most = (int64_t)sm_count() * kNormBlocksPerSm;
  const int blocks = (int)(tab.chunks < 1 ? 1 : (int64_t)tab.chunks < most ? (int64_t)tab.chunks : most);
  grad_norm_kernel<N><<<blocks, kNormThreads, 0, st>>>(tab, partial, *have, last, max_norm, scale, out, d_status);
  if (*have < blocks) *have = blocks;
  return cudaGetLastError();
}

// ---------------------------------------------------------------------------
// AdamW
// ---------------------------------------------------------------------------
constexpr int kStepThreads = 256;
constexpr int kStepChunk = 2048;                    // elements that a block takes at a time: a warp takes one block of an 8-bit state
constexpr int kStepBlocksPerSm = 4;
constexpr int kTensorsMost = 400;                   // tensors per launch, 80 bytes each
constexpr int kTensorsFew = 12;

constexpr float kMFloor = 0x1p-100f, kVFloor = 0x1p-90f;     // least scales: 1 / scale and scale / 255^4 are normal numbers
constexpr float kSquareMost = 0x1p120f;                      // of a scaled gradient: beyond it (or NaN) the element is left out

enum : uint32_t { kW16 = 1, kG16 = 2, kEight = 4, kAligned = 8 };

struct Tensor {
  void* w;
  const void* g;
  void *m, *v;
  float *m_scale, *v_scale;
  __nv_bfloat16* copy;
  int64_t n;
  float lr_scale, decay;
  uint32_t first, kind;
};
static_assert(sizeof(Tensor) == 80, "two tables have to fit the parameters of a kernel");

struct StepScalars {
  const float *d_scale, *d_lr;
  int32_t* d_step;
  double log_b1, log_b2;
  float lr, b1, b1c, b2, b2c, eps;
  float rate, root;                                 // lr-free 1/(1 - b1^t) and 1/sqrt(1 - b2^t), where the host knows t
  int32_t advance;                                  // the last launch of a call counts the step
  int32_t* d_status;
};

template <int N>
struct StepTable {
  Tensor t[N];
  int32_t count;
  uint32_t chunks;
};

struct Rates {                                      // of one launch, in shared memory
  float f, lr, rate, root;
};

// One element: m and v become the new moments; returns the new weight.  A gradient that is not usable changes nothing.
__device__ __forceinline__ float step_element(float w, float g, float& m, float& v, const StepScalars& a, float step, float root,
                                              float pull, bool& bad) {
  const float g2 = __fmul_rn(g, g);
  if (!(g2 <= kSquareMost)) {
    bad = true;
    return w;
  }
  m = __fadd_rn(__fmul_rn(m, a.b1), __fmul_rn(g, a.b1c));
  v = __fadd_rn(__fmul_rn(v, a.b2), __fmul_rn(g2, a.b2c));
  float s;
  asm("sqrt.approx.f32 %0, %1;" : "=f"(s) : "f"(v));
  const float u = __fdividef(m, fmaf(s, root, a.eps));
  return w - fmaf(step, u, pull * w);
}

__device__ __forceinline__ float warp_max(float v) {          // of magnitudes: their bit patterns are in order
  return __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(v)));
}

__device__ __forceinline__ float decode_m(int c, float unit) { return __fmul_rn((float)(c * abs(c)), unit); }
__device__ __forceinline__ float decode_v(uint32_t c, float unit) {
  const float q = (float)(c * c);
  return __fmul_rn(__fmul_rn(q, q), unit);
}
__device__ __forceinline__ float unit_m(float scale) { return __fmul_rn(scale, (float)(1.0 / 16129.0)); }
__device__ __forceinline__ float unit_v(float scale) { return __fmul_rn(scale, (float)(1.0 / 4228250625.0)); }

// Codes: the estimate from the approximate root is the count of borders or one beside it, and the comparison with the borders next
// to it says which.
__device__ __forceinline__ int encode_m(float m, float to_unit) {
  const float y = __fmul_rn(fabsf(m), to_unit);
  float r;
  asm("sqrt.approx.f32 %0, %1;" : "=f"(r) : "f"(y));
  float c = rintf(r);
  const float below = fmaf(c, c, 0.25f) - c, above = fmaf(c, c, 0.25f) + c;      // (c - 1/2)^2 and (c + 1/2)^2, exact
  if (c > 0.0f && y < below) c -= 1.0f;
  if (y >= above) c += 1.0f;
  return (int)copysignf(c, m);
}
__device__ __forceinline__ uint32_t encode_v(float v, float to_unit) {
  const float y = __fmul_rn(v, to_unit);
  float r;
  asm("sqrt.approx.f32 %0, %1;" : "=f"(r) : "f"(y));
  asm("sqrt.approx.f32 %0, %0;" : "+f"(r));
  float c = rintf(r);
  const float below = fmaf(c, c, 0.25f) - c, above = fmaf(c, c, 0.25f) + c;      // their squares are rounded once, as the borders are
  if (c > 0.0f && y < __fmul_rn(below, below)) c -= 1.0f;
  if (y >= __fmul_rn(above, above)) c += 1.0f;
  if (v > 0.0f) c = fmaxf(c, 1.0f);
  return (uint32_t)c;
}

// Four consecutive elements, of which `left` exist (4 or more: all); `vec`: they are aligned.
__device__ __forceinline__ void load4(const void* p, bool is16, int64_t e, int64_t left, bool vec, float* f) {
  if (vec && left >= 4) {
    if (is16) {
      const uint2 q = *reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(p) + e);
      f[0] = low_bf16(q.x); f[1] = high_bf16(q.x); f[2] = low_bf16(q.y); f[3] = high_bf16(q.y);
    } else {
      const float4 q = *reinterpret_cast<const float4*>(static_cast<const float*>(p) + e);
      f[0] = q.x; f[1] = q.y; f[2] = q.z; f[3] = q.w;
    }
    return;
  }
#pragma unroll
  for (int k = 0; k < 4; ++k)
    f[k] = k < left ? (is16 ? low_bf16(static_cast<const uint16_t*>(p)[e + k]) : static_cast<const float*>(p)[e + k]) : 0.0f;
}
__device__ __forceinline__ void store4(void* p, bool is16, int64_t e, int64_t left, bool vec, const float* f) {
  if (vec && left >= 4) {
    if (is16) {
      const __nv_bfloat162 a = __floats2bfloat162_rn(f[0], f[1]), b = __floats2bfloat162_rn(f[2], f[3]);
      *reinterpret_cast<uint2*>(static_cast<uint16_t*>(p) + e) =
          make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
    } else {
      *reinterpret_cast<float4*>(static_cast<float*>(p) + e) = make_float4(f[0], f[1], f[2], f[3]);
    }
    return;
  }
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if (k < left) {
      if (is16) static_cast<__nv_bfloat16*>(p)[e + k] = __float2bfloat16_rn(f[k]);
      else static_cast<float*>(p)[e + k] = f[k];
    }
}
__device__ __forceinline__ uint32_t load4_codes(const void* p, int64_t e, int64_t left, bool vec) {
  const uint8_t* c = static_cast<const uint8_t*>(p) + e;
  if (vec && left >= 4) return *reinterpret_cast<const uint32_t*>(c);
  uint32_t q = 0;
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if (k < left) q |= (uint32_t)c[k] << (8 * k);
  return q;
}
__device__ __forceinline__ void store4_codes(void* p, int64_t e, int64_t left, bool vec, uint32_t q) {
  uint8_t* c = static_cast<uint8_t*>(p) + e;
  if (vec && left >= 4) {
    *reinterpret_cast<uint32_t*>(c) = q;
    return;
  }
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if (k < left) c[k] = (uint8_t)(q >> (8 * k));
}

// A warp's 256 elements from `base` on: a lane has elements 4 lane .. + 3 and 128 + 4 lane .. + 3.
template <bool W16, bool G16, bool EIGHT>
__device__ __forceinline__ void step_warp(const Tensor& t, int64_t base, const StepScalars& a, const Rates& s, bool& bad) {
  const int lane = threadIdx.x & 31;
  const bool vec = t.kind & kAligned;
  float w[8], g[8], m[8], v[8];
  uint32_t cm[2], cv[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int64_t e = base + 128 * h + 4 * lane, left = t.n - e;
    load4(t.g, G16, e, left, vec, g + 4 * h);
    load4(t.w, W16, e, left, vec, w + 4 * h);
    if (EIGHT) {
      cm[h] = load4_codes(t.m, e, left, vec);
      cv[h] = load4_codes(t.v, e, left, vec);
    } else {
      load4(t.m, false, e, left, vec, m + 4 * h);
      load4(t.v, false, e, left, vec, v + 4 * h);
    }
  }
  if (EIGHT) {
    const float um = unit_m(t.m_scale[base >> 8]), uv = unit_v(t.v_scale[base >> 8]);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      m[k] = decode_m((int)(int8_t)(cm[k >> 2] >> (8 * (k & 3))), um);
      v[k] = decode_v((cv[k >> 2] >> (8 * (k & 3))) & 0xffu, uv);
    }
  }
  const float lr = s.lr * t.lr_scale, step = lr * s.rate, pull = lr * t.decay;
#pragma unroll
  for (int k = 0; k < 8; ++k) w[k] = step_element(w[k], __fmul_rn(g[k], s.f), m[k], v[k], a, step, s.root, pull, bad);
  if (EIGHT) {
    float top_m = kMFloor, top_v = kVFloor;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      top_m = fmaxf(top_m, fabsf(m[k]));
      top_v = fmaxf(top_v, v[k]);
    }
    top_m = warp_max(top_m);
    top_v = warp_max(top_v);
    const float to_m = __fdiv_rn(16129.0f, top_m), to_v = __fdiv_rn(4228250625.0f, top_v);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      cm[h] = cv[h] = 0u;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        cm[h] |= ((uint32_t)encode_m(m[4 * h + k], to_m) & 0xffu) << (8 * k);
        cv[h] |= encode_v(v[4 * h + k], to_v) << (8 * k);
      }
    }
    if (lane == 0) {
      t.m_scale[base >> 8] = top_m;
      t.v_scale[base >> 8] = top_v;
    }
  }
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int64_t e = base + 128 * h + 4 * lane, left = t.n - e;
    store4(t.w, W16, e, left, vec, w + 4 * h);
    if (t.copy) store4(t.copy, true, e, left, vec, w + 4 * h);
    if (EIGHT) {
      store4_codes(t.m, e, left, vec, cm[h]);
      store4_codes(t.v, e, left, vec, cv[h]);
    } else {
      store4(t.m, false, e, left, vec, m + 4 * h);
      store4(t.v, false, e, left, vec, v + 4 * h);
    }
  }
}

template <int N>
__global__ void __launch_bounds__(kStepThreads, kStepBlocksPerSm) adamw_kernel(const __grid_constant__ StepTable<N> tab,
                                                                              const __grid_constant__ StepScalars a) {
  __shared__ Rates s_rates;
  if (threadIdx.x == 0) {
    Rates r;
    r.f = a.d_scale ? *a.d_scale : 1.0f;
    r.lr = a.d_lr ? *a.d_lr : a.lr;
    r.rate = a.rate;
    r.root = a.root;
    if (a.d_step) {
      const int32_t taken = *a.d_step;
      const double t = (double)(taken < 0 ? 0 : taken) + 1.0;
      r.rate = (float)(-1.0 / expm1(t * a.log_b1));
      r.root = (float)rsqrt(-expm1(t * a.log_b2));
    }
    s_rates = r;
  }
  __syncthreads();
  const Rates s = s_rates;
  if (!(fabsf(s.f) < INFINITY) || !(fabsf(s.lr) < INFINITY)) {       // the step is not taken, and not counted
    if (blockIdx.x == 0 && threadIdx.x == 0) flag(a.d_status, SPO_DEV_NONFINITE);
    return;
  }
  bool bad = false;
  int i = find_tensor(tab, blockIdx.x);
  for (uint64_t chunk = blockIdx.x; chunk < tab.chunks; chunk += gridDim.x) {
    while (i + 1 < tab.count && tab.t[i + 1].first <= chunk) ++i;
    const Tensor& t = tab.t[i];
    const int64_t base = (int64_t)(chunk - t.first) * kStepChunk + (threadIdx.x >> 5) * 256;
    if (base >= t.n) continue;
    switch (t.kind & (kW16 | kG16 | kEight)) {
      case 0: step_warp<false, false, false>(t, base, a, s, bad); break;
      case kW16: step_warp<true, false, false>(t, base, a, s, bad); break;
      case kG16: step_warp<false, true, false>(t, base, a, s, bad); break;
      case kW16 | kG16: step_warp<true, true, false>(t, base, a, s, bad); break;
      case kEight: step_warp<false, false, true>(t, base, a, s, bad); break;
      case kEight | kW16: step_warp<true, false, true>(t, base, a, s, bad); break;
      case kEight | kG16: step_warp<false, true, true>(t, base, a, s, bad); break;
      default: step_warp<true, true, true>(t, base, a, s, bad); break;
    }
  }
  if (bad) flag(a.d_status, SPO_DEV_NONFINITE);
  if (a.d_step && a.advance && threadIdx.x == 0) {
    // every block has read the counter before it arrives here; the last one to arrive moves it
    const int arrived = atomicAdd(a.d_step + 1, 1);
    if (arrived == (int)gridDim.x - 1) {
      a.d_step[1] = 0;
      if (a.d_step[0] < 0x7fffffff) a.d_step[0] = (a.d_step[0] < 0 ? 0 : a.d_step[0]) + 1;
    }
  }
}

template <int N>
cudaError_t step_launch(const spo_adamw_tensor* tensors, int from, int to, StepScalars a, const spo_adamw_params& p, cudaStream_t st) {
  StepTable<N> tab;
  tab.count = 0;
  uint64_t chunks = 0;
  for (int i = from; i < to; ++i) {
    const spo_adamw_tensor& q = tensors[i];
    if (q.n == 0) continue;
    Tensor& t = tab.t[tab.count++];
    t = Tensor{q.w, q.g, q.m, q.v, q.m_scale, q.v_scale, static_cast<__nv_bfloat16*>(q.copy), q.n, q.lr_scale,
               q.decay_scale * p.weight_decay, (uint32_t)chunks, 0};
    uintptr_t at = 0;
    for (const void* x : {(const void*)q.w, q.g, (const void*)q.m, (const void*)q.v, (const void*)q.copy}) at |= reinterpret_cast<uintptr_t>(x);
    t.kind = (q.w_dtype == SPO_DTYPE_BF16 ? kW16 : 0) | (q.g_dtype == SPO_DTYPE_BF16 ? kG16 : 0) |
             (q.state_bits == 8 ? kEight : 0) | ((at & 15) == 0 ? kAligned : 0);
    chunks += (uint64_t)ceil_div(q.n, kStepChunk);
  }
  tab.chunks = (uint32_t)chunks;
  if (chunks == 0) return cudaSuccess;
  const int64_t most = (int64_t)sm_count() * kStepBlocksPerSm;
  adamw_kernel<N><<<(unsigned)((int64_t)chunks < most ? (int64_t)chunks : most), kStepThreads, 0, st>>>(tab, a);
  return cudaGetLastError();
}

// Values of 8-bit states: four of each a thread.
__global__ void __launch_bounds__(256) adamw_decode_kernel(const int8_t* __restrict__ m, const float* __restrict__ m_scale,
                                                           const uint8_t* __restrict__ v, const float* __restrict__ v_scale, int64_t n,
                                                           bool vec, float* __restrict__ m_out, float* __restrict__ v_out) {
  for (int64_t e = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4; e < n; e += (int64_t)gridDim.x * 1024) {
    const int64_t left = n - e;
    float f[4];
    if (m) {
      const uint32_t c = load4_codes(m, e, left, vec);
      const float unit = unit_m(m_scale[e >> 8]);
#pragma unroll
      for (int k = 0; k < 4; ++k) f[k] = decode_m((int)(int8_t)(c >> (8 * k)), unit);
      store4(m_out, false, e, left, vec, f);
    }
    if (v) {
      const uint32_t c = load4_codes(v, e, left, vec);
      const float unit = unit_v(v_scale[e >> 8]);
#pragma unroll
      for (int k = 0; k < 4; ++k) f[k] = decode_v((c >> (8 * k)) & 0xffu, unit);
      store4(v_out, false, e, left, vec, f);
    }
  }
}

}  // namespace

size_t grad_norm_ws_bytes() { return align_up(sizeof(double) * (size_t)sm_count() * kNormBlocksPerSm, 256); }

cudaError_t launch_grad_norm(const spo_grad_tensor* grads, int count, float max_norm, float scale, float* out, char* ws,
                             int32_t* d_status, cudaStream_t st) {
  double* partial = reinterpret_cast<double*>(ws);
  int have = 0, from = 0;
  bool one = true;
  do {
    const int left = count - from, take = left < kGradsMost ? left : kGradsMost;
    const bool last = take == left;
    const cudaError_t e = take <= kGradsFew ? norm_launch<kGradsFew>(grads, from, from + take, partial, &have, last, max_norm, scale, out, d_status, st)
                                            : norm_launch<kGradsMost>(grads, from, from + take, partial, &have, last, max_norm, scale, out, d_status, st);
    if (e != cudaSuccess) return e;
    one = one && last;
    from += take;
  } while (from < count);
  if (have == 1) return cudaSuccess;               // the one block has written the results
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(1);
  cfg.blockDim = dim3(kNormThreads);
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = one ? 1 : 0;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, grad_norm_finish_kernel, (const double*)partial, have, max_norm, scale, out, d_status);
}

cudaError_t launch_adamw(const spo_adamw_tensor* tensors, int count, const float* d_scale, const float* d_lr, int32_t* d_step,
                         const spo_adamw_params& p, int32_t* d_status, cudaStream_t st) {
  StepScalars a{};
  a.d_scale = d_scale; a.d_lr = d_lr; a.d_step = d_step; a.d_status = d_status;
  const double b1 = p.beta1, b2 = p.beta2, t = p.step;
  a.log_b1 = log(b1);                               // -inf for 0, whose powers are then 0
  a.log_b2 = log(b2);
  a.lr = p.lr; a.eps = p.eps;
  a.b1 = p.beta1; a.b1c = (float)(1.0 - b1); a.b2 = p.beta2; a.b2c = (float)(1.0 - b2);
  a.rate = (float)(-1.0 / expm1(t * a.log_b1));
  a.root = (float)(1.0 / sqrt(-expm1(t * a.log_b2)));
  // the launches of a call, the last of which counts the step: those that hold an element
  int end = count;
  while (end > 0 && tensors[end - 1].n == 0) --end;
  for (int from = 0; from < end;) {
    const int left = end - from, take = left < kTensorsMost ? left : kTensorsMost;
    a.advance = take == left;
    const cudaError_t e = take <= kTensorsFew ? step_launch<kTensorsFew>(tensors, from, from + take, a, p, st)
                                              : step_launch<kTensorsMost>(tensors, from, from + take, a, p, st);
    if (e != cudaSuccess) return e;
    from += take;
  }
  return cudaSuccess;
}

cudaError_t launch_adamw_decode(const int8_t* m, const float* m_scale, const uint8_t* v, const float* v_scale, int64_t n, float* m_out,
                                float* v_out, cudaStream_t st) {
  if (n == 0 || (!m && !v)) return cudaSuccess;
  uintptr_t at = 0;
  for (const void* x : {(const void*)m, (const void*)v, (const void*)m_out, (const void*)v_out}) at |= reinterpret_cast<uintptr_t>(x);
  const int64_t need = ceil_div(n, 1024), most = (int64_t)sm_count() * 8 * 4;
  adamw_decode_kernel<<<(unsigned)(need < most ? need : most), 256, 0, st>>>(m, m_scale, v, v_scale, n, (at & 15) == 0, m_out, v_out);
  return cudaGetLastError();
}

}  // namespace spo
