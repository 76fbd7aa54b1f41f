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
#include <float.h>
#include <math.h>
#include <stdint.h>

#include "spo_internal.h"
#include "spo_vec.cuh"

namespace spo {
namespace {

__device__ __forceinline__ void flag(int32_t* d_status, int bit) {
  if (d_status) atomicOr(d_status, bit);
}
__device__ __forceinline__ void pdl_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void pdl_release() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// ---------------------------------------------------------------------------
// gradient norm
// ---------------------------------------------------------------------------
constexpr int kNormThreads = 128, kFinishThreads = 512;
constexpr int kNormChunk = 4096;                    // elements that a block takes at a time
constexpr int kNormBlocksPerSm = 32;                // more than fit at once: the SMs do not run at one pace
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

// The sum of the squares of a few values in fp64, whose products of fp32 values are exact, so that the norm and the factor do not depend on
// the order of the terms once they are rounded to fp32.  The conversion instructions would be the bound of the whole: |x| 2^-128 is put
// together from the bits instead, as if x were a normal number.  A zero then counts as 2^-127 and an infinity as 2^128; a sum that this
// could change, or that holds one, is formed again from converted values.
__device__ __forceinline__ double wide_normal(uint32_t w) { return __hiloint2double((int)((w >> 3 & 0x0fffffffu) | 0x30000000u), (int)(w << 29)); }
__device__ __forceinline__ double wide_low(uint32_t w) { return __hiloint2double((int)((w << 13 & 0x0fffe000u) | 0x30000000u), 0); }
__device__ __forceinline__ double wide_high(uint32_t w) { return __hiloint2double((int)((w >> 3 & 0x0fffe000u) | 0x30000000u), 0); }
template <bool BF16, int N>
__device__ __forceinline__ double sum_squares(const uint32_t (&w)[N]) {
  double s[2] = {0.0, 0.0};
#pragma unroll
  for (int k = 0; k < N; ++k) {
    const double x = BF16 ? wide_low(w[k]) : wide_normal(w[k]);
    s[k & 1] = fma(x, x, s[k & 1]);
    if (BF16) s[k & 1] = fma(wide_high(w[k]), wide_high(w[k]), s[k & 1]);
  }
  const double sum = s[0] + s[1];
  if (sum > 0x1p-446 && sum < 1.0) return sum * 0x1p256;
  uint32_t any = 0;
#pragma unroll
  for (int k = 0; k < N; ++k) any |= w[k];
  if ((any & (BF16 ? 0x7fff7fffu : 0x7fffffffu)) == 0) return 0.0;
  double d = 0.0;
#pragma unroll
  for (int k = 0; k < N; ++k) {
    const double x = BF16 ? low_bf16(w[k]) : __uint_as_float(w[k]);
    d = fma(x, x, d);
    if (BF16) d = fma((double)high_bf16(w[k]), (double)high_bf16(w[k]), d);
  }
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
        uint32_t w[16];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          w[4 * k] = q[k].x; w[4 * k + 1] = q[k].y; w[4 * k + 2] = q[k].z; w[4 * k + 3] = q[k].w;
        }
        sum += sum_squares<true>(w);
      } else if (whole) {
        const uint4* p = reinterpret_cast<const uint4*>(static_cast<const float*>(g) + base) + threadIdx.x;
        uint4 q[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) q[k] = __ldcs(p + k * kNormThreads);
        uint32_t w[32];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          w[4 * k] = q[k].x; w[4 * k + 1] = q[k].y; w[4 * k + 2] = q[k].z; w[4 * k + 3] = q[k].w;
        }
        sum += sum_squares<false>(w);
      } else {
        const int64_t end = n - base < kNormChunk ? n : base + kNormChunk;
        for (int64_t e = base + threadIdx.x; e < end; e += kNormThreads) {
          const uint32_t w[1] = {bf16 ? (uint32_t)static_cast<const uint16_t*>(g)[e] << 16 : static_cast<const uint32_t*>(g)[e]};
          sum += sum_squares<false>(w);
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

__global__ void __launch_bounds__(kFinishThreads) grad_norm_finish_kernel(const double* partial, int parts, float max_norm, float scale,
                                                                        float* out, int32_t* d_status) {
  __shared__ double s_part[kFinishThreads / 32];
  pdl_wait();
  double sum = 0.0;
#pragma unroll 4
  for (int p = threadIdx.x; p < parts; p += kFinishThreads) sum += partial[p];
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
// A block is one warp: it shares nothing with others, and an SM starts the next one as soon as one is done.
constexpr int kStepChunk = 256;                     // elements that a warp takes at a time, a block of an 8-bit state
constexpr int kStepBlocksPerSm = 24;
// Chunks in a row that a warp takes: enough for its start to be paid (the constants, the first inputs) and, in 8 bits, for the inputs that
// are fetched ahead; few enough for kRounds rounds of warps over the GPU.  155 million elements: 8 bits 479 us (bf16 weights 323) with
// up to 16 and 516 (369) with up to 6, 32 bits 694 us and 682; 11 million in 8 bits: 37 us with one round, 30 with three.
constexpr int kSpanMost8 = 16, kSpanMost32 = 6, kRounds = 3;
constexpr int kTensorsMost = 400;                   // tensors per launch, 80 bytes each
constexpr int kTensorsSome = 136, kTensorsFew = 12;  // smaller tables for shorter lists: what a launch costs the host grows with them

constexpr float kMFloor = 0x1p-100f, kVFloor = 0x1p-90f;     // least scales: 1 / scale and scale / 255^4 are normal numbers
constexpr double kRateMost = 0x1p100;                         // of a tensor's rate, and that times its decay: 1 / (1 - b1^t) is up to 2^24
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
static_assert(sizeof(Tensor) == 80, "kTensorsMost of them have to fit the parameters of a kernel");

struct StepScalars {
  const float *d_scale, *d_lr;
  int32_t* d_step;
  float log_b1, log_b2;                             // -inf for 0, whose powers are then 0
  float lr, b1, b1c, b2, b2c, eps;
  float one;                                        // 1: a product and a sum that must not become one multiply-add go through it
  float lr_most;                                    // beyond it (or NaN) no step is taken: the same for all tensors of a call
  float rate, root;                                 // lr-free 1/(1 - b1^t) and 1/sqrt(1 - b2^t), where the host knows t
  uint32_t span;
  int32_t advance;                                  // the last launch of a call counts the step
  int32_t* d_status;
};

template <int N>
struct StepTable {
  Tensor t[N];
  int32_t count;
  uint32_t chunks;
};

// What a launch reads from the device, as issued, and the constants that come of it.
struct Rates {
  float f, lr;
  int32_t taken;
  float rate;
  bool ready, fine;
};

// Approximate root and reciprocal (relative error below 2^-22); arguments and results below 2^-126 count as zero, but for full_sqrt.
__device__ __forceinline__ float near_sqrt(float x) {
  float r;
  asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float full_sqrt(float x) {
  float r;
  asm("sqrt.approx.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float near_inverse(float x) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float2 near_sqrt2(float2 x) { return make_float2(near_sqrt(x.x), near_sqrt(x.y)); }

__device__ __forceinline__ float warp_max(float v) {          // of magnitudes: their bit patterns are in order
  return __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(v)));
}

// Constants of the packed operations, as pairs in shared memory: each is read where it is used (two at a time), because as many pairs as
// there are would take half of the registers.
enum { kCb1, kCb1c, kCb2, kCb2c, kCone, kCf, kCbyte, kCbyte128, kCwhole, kCminus, kCeps, kCroot, kConstants };
__device__ __forceinline__ void pair_of(const float2* c, float2& a, float2& b) {       // c[0] and c[1], 16 bytes aligned
  asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];"
               : "=f"(a.x), "=f"(a.y), "=f"(b.x), "=f"(b.y) : "r"((uint32_t)__cvta_generic_to_shared(c)));
}

// The four bytes of a word as floats: a byte is the low end of the mantissa of 2^23.
constexpr float kByteBase = 8388608.0f;
__device__ __forceinline__ float byte_float(uint32_t w, int k) { return __uint_as_float(__byte_perm(w, 0x4B000000u, 0x7540 + k)); }
__device__ __forceinline__ float2 decode_m2(uint32_t w, int k, float unit, float2 byte128 = both(-(kByteBase + 128.0f))) {
  const float2 c = add2(make_float2(byte_float(w ^ 0x80808080u, k), byte_float(w ^ 0x80808080u, k + 1)), byte128);   // codes k and k + 1
  return mul2(make_float2(c.x * fabsf(c.x), c.y * fabsf(c.y)), both(unit));            // (c |c| is exact)
}
__device__ __forceinline__ float2 decode_v2(uint32_t w, int k, float unit, float2 byte = both(-kByteBase)) {
  float2 c = add2(make_float2(byte_float(w, k), byte_float(w, k + 1)), byte);
  c = mul2(c, c);
  return mul2(mul2(c, c), both(unit));
}
__device__ __forceinline__ float unit_m(float scale) { return __fmul_rn(scale, (float)(1.0 / 16129.0)); }
__device__ __forceinline__ float unit_v(float scale) { return __fmul_rn(scale, (float)(1.0 / 4228250625.0)); }

// Codes.  Adding 1.5 x 2^23 to the root of a scaled magnitude rounds it to a whole number and leaves that, in two's complement, in the low
// bits.  The approximate root does for a code unless it lies within kNear of a border (its error is below 2^-22 of it, 6e-5 at 255)
// or belongs to a v that might take code 0; one warp in thirty has such an element, and forms its codes by the comparison with the
// borders: the root, enlarged by more than its error, rounds to the count of borders or one more, and the border below,
// (c - 1/2)^2 (exact) or that squared (rounded once, as the borders are), says which.
constexpr float kWhole = 12582912.0f, kEnlarge = 1.0f + 0x1p-20f, kNear = 0x1p-13f;
__device__ __forceinline__ uint32_t low_bytes(float2 a, float2 b) {
  const uint32_t lo = __byte_perm(__float_as_uint(a.x), __float_as_uint(a.y), 0x0040);
  const uint32_t hi = __byte_perm(__float_as_uint(b.x), __float_as_uint(b.y), 0x0040);
  return __byte_perm(lo, hi, 0x5410);
}
__device__ __forceinline__ float encode_m(float m, float to_unit) {                     // in the low bits
  const float y = __fmul_rn(fabsf(m), to_unit);
  float c = rintf(near_sqrt(y) * kEnlarge);
  const float h = c - 0.5f;                                                             // (-1/2 where c is 0: its square counts as negative)
  if (y < h * fabsf(h)) c -= 1.0f;
  return copysignf(c, m) + kWhole;
}
__device__ __forceinline__ float encode_v(float v, float to_unit) {
  const float y = __fmul_rn(v, to_unit);
  float c = fmaxf(rintf(near_sqrt(near_sqrt(y)) * kEnlarge), 1.0f);
  const float h = c - 0.5f, b = h * h;
  if (y < __fmul_rn(b, b)) c -= 1.0f;
  if (v > 0.0f) c = fmaxf(c, 1.0f);
  return c + kWhole;
}
__device__ __forceinline__ float2 encode_m2(float2 m, float to_unit) { return make_float2(encode_m(m.x, to_unit), encode_m(m.y, to_unit)); }
__device__ __forceinline__ float2 encode_v2(float2 v, float to_unit) { return make_float2(encode_v(v.x, to_unit), encode_v(v.y, to_unit)); }

// Four consecutive elements, aligned, as they are in memory.  The loads of a chunk are issued where they are written, all of them before the
// first one is waited for, and past the L1 cache: nothing is read twice.
template <bool IS16>
struct Raw4 {
  uint32_t x[IS16 ? 2 : 4];
};
__device__ __forceinline__ void issue(const void* p, Raw4<true>& r) {
  asm volatile("ld.global.L1::no_allocate.v2.u32 {%0, %1}, [%2];" : "=r"(r.x[0]), "=r"(r.x[1]) : "l"(p));
}
__device__ __forceinline__ void issue(const void* p, Raw4<false>& r) {
  asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(r.x[0]), "=r"(r.x[1]), "=r"(r.x[2]), "=r"(r.x[3]) : "l"(p));
}
__device__ __forceinline__ void issue(const void* p, uint32_t& x) { asm volatile("ld.global.L1::no_allocate.u32 %0, [%1];" : "=r"(x) : "l"(p)); }
__device__ __forceinline__ void issue(const int32_t* p, int32_t& x) { asm volatile("ld.global.s32 %0, [%1];" : "=r"(x) : "l"(p)); }
__device__ __forceinline__ void issue(const float* p, float& x) { asm volatile("ld.global.f32 %0, [%1];" : "=f"(x) : "l"(p)); }
template <bool IS16>
__device__ __forceinline__ float2 pair_in(const Raw4<IS16>& r, int p) {                // elements 2 p and 2 p + 1
  if constexpr (IS16) return make_float2(low_bf16(r.x[p]), high_bf16(r.x[p]));
  else return make_float2(__uint_as_float(r.x[2 * p]), __uint_as_float(r.x[2 * p + 1]));
}
__device__ __forceinline__ void store4(void* p, bool is16, const float* f) {
  if (is16) {
    const __nv_bfloat162 a = __floats2bfloat162_rn(f[0], f[1]), b = __floats2bfloat162_rn(f[2], f[3]);
    *static_cast<uint2*>(p) = make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
  } else {
    *static_cast<float4*>(p) = make_float4(f[0], f[1], f[2], f[3]);
  }
}

// Element e of an array whose elements have `bytes` bytes.
__device__ __forceinline__ char* at_element(const void* p, int bytes, int64_t e) {
  return const_cast<char*>(static_cast<const char*>(p)) + e * bytes;
}

// What a lane reads of 256 elements: 4 lane .. + 3 and 128 + 4 lane .. + 3.
template <bool W16, bool G16, bool EIGHT>
struct Inputs {
  Raw4<G16> g[2];
  Raw4<W16> w[2];
  Raw4<false> m[EIGHT ? 1 : 2], v[EIGHT ? 1 : 2];
  uint32_t cm[2], cv[2];
  float m_scale, v_scale;
  __device__ __forceinline__ void fetch(const Tensor& t, int64_t base) {
    constexpr int kW = W16 ? 2 : 4, kG = G16 ? 2 : 4;
    const int64_t e = base + 4 * (threadIdx.x & 31);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      issue(at_element(t.g, kG, e) + 128 * h * kG, g[h]);
      if constexpr (EIGHT) {
        issue(at_element(t.m, 1, e) + 128 * h, cm[h]);
        issue(at_element(t.v, 1, e) + 128 * h, cv[h]);
      } else {
        issue(at_element(t.m, 4, e) + 512 * h, m[h]);
        issue(at_element(t.v, 4, e) + 512 * h, v[h]);
      }
    }
    if constexpr (EIGHT) {
      issue(t.m_scale + (base >> 8), m_scale);
      issue(t.v_scale + (base >> 8), v_scale);
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) issue(at_element(t.w, kW, e) + 128 * h * kW, w[h]);
  }
};

// A warp's 256 elements from `base` on, whole and aligned, as four pairs a lane.
// Returns false, with nothing written, where a gradient may not be usable: v stays below 2^96 where all are, because (1 - b2) g~^2 is at
// least 2^-24 times g~^2.
template <bool W16, bool G16, bool EIGHT>
__device__ __forceinline__ bool step_warp(const Tensor& t, int64_t base, const Inputs<W16, G16, EIGHT>& in, const float2* consts, float step,
                                          float pull) {
  const int lane = threadIdx.x & 31;
  const int64_t e = base + 4 * lane;
  constexpr int kW = W16 ? 2 : 4, kS = EIGHT ? 1 : 4;
  float2 m[4], v[4];
  uint32_t cm[2], cv[2];
  if constexpr (EIGHT) {
    const float um = unit_m(in.m_scale), uv = unit_v(in.v_scale);
    float2 byte, byte128;
    pair_of(consts + kCbyte, byte, byte128);
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      m[p] = decode_m2(in.cm[p >> 1], 2 * (p & 1), um, byte128);
      v[p] = decode_v2(in.cv[p >> 1], 2 * (p & 1), uv, byte);
    }
  } else {
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      m[p] = pair_in(in.m[p >> 1], p & 1);
      v[p] = pair_in(in.v[p >> 1], p & 1);
    }
  }
  float top_m = kMFloor;
  uint32_t top_v = __float_as_uint(kVFloor);                  // as bits: a NaN is above all numbers
  {
    float2 one, f, b1, b1c, b2, b2c;
    pair_of(consts + kCone, one, f);
    pair_of(consts + kCb1, b1, b1c);
    pair_of(consts + kCb2, b2, b2c);
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      const float2 gs = mul2(pair_in(in.g[p >> 1], p & 1), f);
      m[p] = fma2(mul2(m[p], b1), one, mul2(gs, b1c));
      v[p] = fma2(mul2(v[p], b2), one, mul2(mul2(gs, gs), b2c));
      if (EIGHT) top_m = fmaxf(top_m, fmaxf(fabsf(m[p].x), fabsf(m[p].y)));
      top_v = max(top_v, max(__float_as_uint(v[p].x), __float_as_uint(v[p].y)));
    }
  }
  if (EIGHT) {
    top_m = warp_max(top_m);
    top_v = __reduce_max_sync(0xffffffffu, top_v);
    if (top_v >= __float_as_uint(0x1p96f)) return false;
  } else {
    if (__any_sync(0xffffffffu, top_v >= __float_as_uint(0x1p96f))) return false;
  }
  float2 w[4], eps, root_unit;
  pair_of(consts + kCeps, eps, root_unit);
  if (EIGHT) {
    const float scale_v = __uint_as_float(top_v);
    const float to_m = __fdiv_rn(16129.0f, top_m), to_v = __fdiv_rn(4228250625.0f, scale_v);
    root_unit = both(root_unit.x * (near_sqrt(scale_v) * (1.0f / 65025.0f)));       // of the root of the scaled v
    float2 whole, minus;
    pair_of(consts + kCwhole, whole, minus);
    float far = 0.0f, low = 1.0f;                             // the largest distance from a whole number, the lowest root of a v
    float2 tm[2], tv[2];
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      const float2 y = mul2(v[p], both(to_v)), root = near_sqrt2(y);
      const float2 d = fma2(root, root_unit, eps);
      const float2 u = mul2(m[p], make_float2(near_inverse(d.x), near_inverse(d.y)));
      const float2 w0 = pair_in(in.w[p >> 1], p & 1);
      w[p] = add2(w0, fma2(both(step), u, mul2(both(pull), w0)));
      const float2 z = mul2(m[p], both(to_m)), rv = near_sqrt2(root);
      const float2 rm = make_float2(copysignf(near_sqrt(fabsf(z.x)), z.x), copysignf(near_sqrt(fabsf(z.y)), z.y));
      tm[p & 1] = add2(rm, whole);
      tv[p & 1] = add2(rv, whole);
      const float2 fm = sub2(rm, add2(tm[p & 1], minus)), fv = sub2(rv, add2(tv[p & 1], minus));
      far = fmaxf(fmaxf(far, fabsf(fm.x)), fabsf(fm.y));
      far = fmaxf(fmaxf(far, fabsf(fv.x)), fabsf(fv.y));
      low = fminf(fminf(low, rv.x), rv.y);
      if (p & 1) {
        cm[p >> 1] = low_bytes(tm[0], tm[1]);
        cv[p >> 1] = low_bytes(tv[0], tv[1]);
      }
    }
    if (__any_sync(0xffffffffu, far > 0.5f - kNear || low < 0.5f + kNear)) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        cm[h] = low_bytes(encode_m2(m[2 * h], to_m), encode_m2(m[2 * h + 1], to_m));
        cv[h] = low_bytes(encode_v2(v[2 * h], to_v), encode_v2(v[2 * h + 1], to_v));
      }
    }
    if (lane == 0) {
      t.m_scale[base >> 8] = top_m;
      t.v_scale[base >> 8] = scale_v;
    }
  } else {
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      const float2 d = fma2(make_float2(full_sqrt(v[p].x), full_sqrt(v[p].y)), root_unit, eps);
      const float2 u = mul2(m[p], make_float2(near_inverse(d.x), near_inverse(d.y)));
      const float2 w0 = pair_in(in.w[p >> 1], p & 1);
      w[p] = add2(w0, fma2(both(step), u, mul2(both(pull), w0)));
    }
  }
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    store4(at_element(t.w, kW, e) + 128 * h * kW, W16, &w[2 * h].x);
    if (t.copy) store4(t.copy + e + 128 * h, true, &w[2 * h].x);
    if (EIGHT) {
      *reinterpret_cast<uint32_t*>(at_element(t.m, 1, e) + 128 * h) = cm[h];
      *reinterpret_cast<uint32_t*>(at_element(t.v, 1, e) + 128 * h) = cv[h];
    } else {
      store4(at_element(t.m, kS, e) + 128 * h * kS, false, &m[2 * h].x);
      store4(at_element(t.v, kS, e) + 128 * h * kS, false, &v[2 * h].x);
    }
  }
  return true;
}

// The same for any 256 elements or the rest of a tensor, element by element (lane, lane + 32, ...): unaligned tensors, ends, and gradients
// that are not usable, whose elements keep their moments and weight.  Returns whether there was one.  Nothing is held from one
// element to the next, and the moments are formed twice where their largest has to be known first: a call, or arrays, would cost the
// loop above its registers.
__device__ __forceinline__ bool step_warp_any(const Tensor& t, int64_t base, const float2* consts, float step, float pull) {
  const int lane = threadIdx.x & 31;
  const bool w16 = t.kind & kW16, g16 = t.kind & kG16, eight = t.kind & kEight;
  const int64_t end = t.n - base < 256 ? t.n : base + 256;
  float um = 0.0f, uv = 0.0f, to_m = 0.0f, to_v = 0.0f;
  bool kept = false;
  auto moments = [&](int64_t e, float& m, float& v) {           // whether the gradient was usable
    const float g = __fmul_rn(g16 ? low_bf16(static_cast<const uint16_t*>(t.g)[e]) : static_cast<const float*>(t.g)[e], consts[kCf].x);
    m = eight ? decode_m2(static_cast<const uint8_t*>(t.m)[e], 0, um).x : static_cast<const float*>(t.m)[e];
    v = eight ? decode_v2(static_cast<const uint8_t*>(t.v)[e], 0, uv).x : static_cast<const float*>(t.v)[e];
    const float g2 = __fmul_rn(g, g);
    if (!(g2 <= kSquareMost)) return false;
    m = __fadd_rn(__fmul_rn(m, consts[kCb1].x), __fmul_rn(g, consts[kCb1c].x));
    v = __fadd_rn(__fmul_rn(v, consts[kCb2].x), __fmul_rn(g2, consts[kCb2c].x));
    return true;
  };
  if (eight) {
    um = unit_m(t.m_scale[base >> 8]);
    uv = unit_v(t.v_scale[base >> 8]);
    float top_m = kMFloor, top_v = kVFloor, m, v;
#pragma unroll 1
    for (int64_t e = base + lane; e < end; e += 32) {
      moments(e, m, v);
      top_m = fmaxf(top_m, fabsf(m));
      top_v = fmaxf(top_v, v);
    }
    __syncwarp();
    top_m = warp_max(top_m);
    top_v = warp_max(top_v);
    to_m = __fdiv_rn(16129.0f, top_m);
    to_v = __fdiv_rn(4228250625.0f, top_v);
    if (lane == 0) {
      t.m_scale[base >> 8] = top_m;
      t.v_scale[base >> 8] = top_v;
    }
  }
#pragma unroll 1
  for (int64_t e = base + lane; e < end; e += 32) {
    float m, v;
    const bool usable = moments(e, m, v);
    const float w0 = w16 ? low_bf16(static_cast<const uint16_t*>(t.w)[e]) : static_cast<const float*>(t.w)[e];
    const float u = m * near_inverse(fmaf(full_sqrt(v), consts[kCroot].x, consts[kCeps].x));
    const float w = usable ? w0 + fmaf(step, u, pull * w0) : w0;
    kept |= !usable;
    if (eight) {
      static_cast<uint8_t*>(t.m)[e] = (uint8_t)__float_as_uint(encode_m(m, to_m));
      static_cast<uint8_t*>(t.v)[e] = (uint8_t)__float_as_uint(encode_v(v, to_v));
    } else {
      static_cast<float*>(t.m)[e] = m;
      static_cast<float*>(t.v)[e] = v;
    }
    if (w16) static_cast<__nv_bfloat16*>(t.w)[e] = __float2bfloat16_rn(w);
    else static_cast<float*>(t.w)[e] = w;
    if (t.copy) t.copy[e] = __float2bfloat16_rn(w);
  }
  __syncwarp();
  return kept;
}

// The constants of a launch, in shared memory; whether the step is taken at all.
__device__ __forceinline__ void make_constants(float2* consts, const StepScalars& a, Rates& s) {
  float root = a.root;
  s.rate = a.rate;
  if (a.d_step) {
    const float t = (float)max(s.taken, 0) + 1.0f;
    s.rate = -1.0f / expm1f(t * a.log_b1);
    root = rsqrtf(-expm1f(t * a.log_b2));
  }
  if (threadIdx.x == 0) {
    consts[kCf] = both(s.f); consts[kCroot] = both(root);
    consts[kCb1] = both(a.b1); consts[kCb1c] = both(a.b1c); consts[kCb2] = both(a.b2); consts[kCb2c] = both(a.b2c);
    consts[kCone] = both(a.one); consts[kCeps] = both(a.eps);
    consts[kCbyte] = both(-kByteBase); consts[kCbyte128] = both(-(kByteBase + 128.0f));
    consts[kCwhole] = both(kWhole); consts[kCminus] = both(-kWhole);
  }
  __syncwarp();
  s.ready = true;
  s.fine = fabsf(s.f) < INFINITY && fabsf(s.lr) <= a.lr_most;
}

// A warp's share, `chunks` chunks from `base` on, as far as they are whole.  Returns the chunks (a bit each) that are left
// for step_warp_any: it is kept out of this loop, whose registers its call would cost.
template <bool W16, bool G16, bool EIGHT>
__device__ __forceinline__ uint32_t step_span(const Tensor& t, int64_t base, int chunks, float2* consts, const StepScalars& a, Rates& s) {
  const int64_t whole = t.n - base >= 256 ? (t.n - base - 256) / kStepChunk + 1 : 0;
  const int n = whole < chunks ? (int)whole : chunks;
  const uint32_t left = ((1u << chunks) - 1) & ~((1u << n) - 1);
  if (n == 0) return left;
  Inputs<W16, G16, EIGHT> in;
  in.fetch(t, base);
  if (!s.ready) make_constants(consts, a, s);
  if (!s.fine) return 0;
  const float lr = s.lr * t.lr_scale, step = -lr * s.rate, pull = -lr * t.decay;
  uint32_t again = 0;
#pragma unroll 1
  for (int c = 0; c < n; ++c, base += kStepChunk) {
    if (EIGHT) {                             // the next chunk's inputs are on their way while this one is worked on
      Inputs<W16, G16, EIGHT> next = in;
      if (c + 1 < n) next.fetch(t, base + kStepChunk);
      if (!step_warp<W16, G16, EIGHT>(t, base, in, consts, step, pull)) again |= 1u << c;
      in = next;
    } else {
      if (!step_warp<W16, G16, EIGHT>(t, base, in, consts, step, pull)) again |= 1u << c;
      if (c + 1 < n) in.fetch(t, base + kStepChunk);
    }
  }
  return left | again;
}

// Many more blocks than fit at once, each with a few chunks in a row, come out ahead of as many as fit that walk through all of it: the SMs
// do not run at one pace (32-bit states, 155 million elements: 644 us and 732 us).
template <int N>
__global__ void __launch_bounds__(32, kStepBlocksPerSm) adamw_kernel(const __grid_constant__ StepTable<N> tab,
                                                                     const __grid_constant__ StepScalars a) {
  __shared__ __align__(16) float2 s_const[kConstants];
  Rates s;
  s.f = 1.0f;
  s.lr = a.lr;
  s.taken = 0;
  if (a.d_scale) issue(a.d_scale, s.f);
  if (a.d_lr) issue(a.d_lr, s.lr);
  if (a.d_step) issue(a.d_step, s.taken);
  s.ready = false;
  bool bad = false;
  uint32_t chunk = blockIdx.x * a.span;
  const uint32_t end = min(chunk + a.span, tab.chunks);
  for (int i = find_tensor(tab, chunk); chunk < end; ++i) {
    const Tensor& t = tab.t[i];
    const uint32_t stop = min(end, i + 1 < tab.count ? tab.t[i + 1].first : tab.chunks);
    const int64_t base = (int64_t)(chunk - t.first) * kStepChunk;
    const int here = (int)(stop - chunk);
    uint32_t left = (1u << here) - 1;
    switch (t.kind) {
      case kAligned: left = step_span<false, false, false>(t, base, here, s_const, a, s); break;
      case kAligned | kW16: left = step_span<true, false, false>(t, base, here, s_const, a, s); break;
      case kAligned | kG16: left = step_span<false, true, false>(t, base, here, s_const, a, s); break;
      case kAligned | kW16 | kG16: left = step_span<true, true, false>(t, base, here, s_const, a, s); break;
      case kAligned | kEight: left = step_span<false, false, true>(t, base, here, s_const, a, s); break;
      case kAligned | kEight | kW16: left = step_span<true, false, true>(t, base, here, s_const, a, s); break;
      case kAligned | kEight | kG16: left = step_span<false, true, true>(t, base, here, s_const, a, s); break;
      case kAligned | kEight | kW16 | kG16: left = step_span<true, true, true>(t, base, here, s_const, a, s); break;
      default: break;                                         // unaligned: all of them are left
    }
    if (!s.ready) make_constants(s_const, a, s);
    if (!s.fine) break;
    const float lr = s.lr * t.lr_scale;
    for (; left; left &= left - 1)
      bad |= step_warp_any(t, base + (int64_t)(__ffs(left) - 1) * kStepChunk, s_const, -lr * s.rate, -lr * t.decay);
    chunk = stop;
  }
  if (!s.fine) {                                              // the step is not taken, and not counted
    if (blockIdx.x == 0 && threadIdx.x == 0) flag(a.d_status, SPO_DEV_NONFINITE);
    return;
  }
  if (bad) flag(a.d_status, SPO_DEV_NONFINITE);
  // every block has read the counter before it arrives here; the last one to arrive moves it
  if (a.d_step && a.advance && threadIdx.x == 0 && atomicAdd(a.d_step + 1, 1) == (int)gridDim.x - 1) {
    a.d_step[1] = 0;
    if (s.taken < 0x7fffffff) a.d_step[0] = (s.taken < 0 ? 0 : s.taken) + 1;
  }
}

template <int N>
cudaError_t step_launch(const spo_adamw_tensor* tensors, int from, int to, StepScalars a, const spo_adamw_params& p, cudaStream_t st) {
  StepTable<N> tab;
  tab.count = 0;
  uint64_t chunks = 0, eight = 0;
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
    if (q.state_bits == 8) eight += (uint64_t)ceil_div(q.n, kStepChunk);
  }
  tab.chunks = (uint32_t)chunks;
  if (chunks == 0) return cudaSuccess;
  const uint64_t at_once = (uint64_t)sm_count() * kStepBlocksPerSm, span = chunks / (at_once * kRounds);
  const uint64_t most = 2 * eight > chunks ? kSpanMost8 : kSpanMost32;
  a.span = (uint32_t)(chunks <= at_once ? 1 : span < 2 ? 2 : span > most ? most : span);
  adamw_kernel<N><<<(unsigned)ceil_div((int64_t)chunks, a.span), 32, 0, st>>>(tab, a);
  return cudaGetLastError();
}

// Values of 8-bit states: a warp takes the 256 elements of a block, a lane elements 4 lane .. + 3 and 128 + 4 lane .. + 3 (or, where they are
// not aligned or end, every 32nd).
__global__ void __launch_bounds__(256) adamw_decode_kernel(const uint8_t* __restrict__ m, const float* __restrict__ m_scale,
                                                           const uint8_t* __restrict__ v, const float* __restrict__ v_scale, int64_t n,
                                                           bool aligned, float* __restrict__ m_out, float* __restrict__ v_out) {
  const int lane = threadIdx.x & 31;
  for (int64_t base = ((int64_t)blockIdx.x * 8 + (threadIdx.x >> 5)) * 256; base < n; base += (int64_t)gridDim.x * 2048) {
    const float um = m ? unit_m(m_scale[base >> 8]) : 0.0f, uv = v ? unit_v(v_scale[base >> 8]) : 0.0f;
    if (aligned && n - base >= 256) {
      const int64_t e = base + 4 * lane;
      uint32_t cm[2] = {0, 0}, cv[2] = {0, 0};
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        if (m) cm[h] = *reinterpret_cast<const uint32_t*>(m + e + 128 * h);
        if (v) cv[h] = *reinterpret_cast<const uint32_t*>(v + e + 128 * h);
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        if (m) {
          const float2 f[2] = {decode_m2(cm[h], 0, um), decode_m2(cm[h], 2, um)};
          store4(m_out + e + 128 * h, false, &f[0].x);
        }
        if (v) {
          const float2 f[2] = {decode_v2(cv[h], 0, uv), decode_v2(cv[h], 2, uv)};
          store4(v_out + e + 128 * h, false, &f[0].x);
        }
      }
    } else {
      for (int64_t e = base + lane; e < n && e < base + 256; e += 32) {
        if (m) m_out[e] = decode_m2(m[e], 0, um).x;
        if (v) v_out[e] = decode_v2(v[e], 0, uv).x;
      }
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
  cfg.blockDim = dim3(kFinishThreads);
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
  a.log_b1 = (float)log(b1);
  a.log_b2 = (float)log(b2);
  a.lr = p.lr; a.eps = p.eps; a.one = 1.0f;
  a.b1 = p.beta1; a.b1c = (float)(1.0 - b1); a.b2 = p.beta2; a.b2c = (float)(1.0 - b2);
  a.rate = (float)(-1.0 / expm1(t * log(b1)));
  a.root = (float)(1.0 / sqrt(-expm1(t * log(b2))));
  // the launches of a call, the last of which counts the step: those that hold an element
  int end = count;
  while (end > 0 && tensors[end - 1].n == 0) --end;
  float scale = 1e-30f, decay = 1.0f;
  for (int i = 0; i < end; ++i) {
    const float one = tensors[i].n ? fabsf(tensors[i].lr_scale) : 0.0f, other = tensors[i].n ? fabsf(tensors[i].decay_scale * p.weight_decay) : 0.0f;
    scale = one > scale ? one : scale;
    decay = other > decay ? other : decay;
  }
  const double most = kRateMost / ((double)scale * decay);
  a.lr_most = decay < INFINITY ? most < FLT_MAX ? (float)most : FLT_MAX : -1.0f;
  for (int from = 0; from < end;) {
    const int left = end - from, take = left < kTensorsMost ? left : kTensorsMost;
    a.advance = take == left;
    const cudaError_t e = take <= kTensorsFew    ? step_launch<kTensorsFew>(tensors, from, from + take, a, p, st)
                          : take <= kTensorsSome ? step_launch<kTensorsSome>(tensors, from, from + take, a, p, st)
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
  const int64_t need = ceil_div(n, 2048), most = 0x7fffffff;
  adamw_decode_kernel<<<(unsigned)(need < most ? need : most), 256, 0, st>>>(reinterpret_cast<const uint8_t*>(m), m_scale, v, v_scale, n, (at & 15) == 0,
                                                                             m_out, v_out);
  return cudaGetLastError();
}

}  // namespace spo
