// Linear layers: what the kernels of strads_linear_forward / strads_linear_backward share.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <type_traits>

#include "strads_internal.cuh"

namespace strads {

// Every product is D[a][b] = sum_k A[a][k] B[b][k], written through Finish.  a is the side whose neighbours lie side by side in
// D's memory wherever one of D's strides is 1: lanes run along a, so that every store, and every load of a residual laid out
// alike, is one run of memory whatever the alignment.
struct Operand { const void* p; long long rs, ks; };                 // element (row, k) at p + row rs + k ks
struct Side { const void* p; long long sa, sb; };                     // element (a, b) at p + a sa + b sb
struct Finish {
  Side out, residual, preact;                                         // residual, preact: p null = none
  const void* bias;                                                   // element a bias_a + b bias_b (one of the two is 0); null = none
  long long bias_a, bias_b;
  int act;
  float scale;
  int plain;                                                          // no bias, activation, residual, preact
  const float* factor;                                                // plain results of binary16: element a factor_a + b factor_b; null = none
  long long factor_a, factor_b;
};

__device__ __forceinline__ float load_f32(const float* p) { return *p; }
__device__ __forceinline__ float load_f32(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ float load_f32(const __half* p) { return __half2float(*p); }
__device__ __forceinline__ void store_f32(float* p, float v) { *p = v; }
__device__ __forceinline__ void store_f32(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }
__device__ __forceinline__ void store_f32(__half* p, float v) { *p = __float2half_rn(v); }

// For binary32 results (kExact) CUDA's exponential and quotient, for 16-bit ones the hardware's, good to 2^-20 for
// arguments up to 16 and, by the rounding of x log2(e), to 2^-18 at 80 (16-bit results are rounded by 2^-12 at least).  Phi(-z), z >= 0, is exp(-z^2/2)
// t P(t), t = 1 / (1 + 0.285 z): P is fitted to erfcx, weighted so that the relative error is even (1.6e-7; 4.7e-7 as evaluated here).  Nothing
// cancels for negative z in any of them.
__device__ __forceinline__ float fast_inverse(float x) { float r; asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x)); return r; }
__device__ __forceinline__ float fast_exp(float x) { float r; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x * 1.4426950408889634f)); return r; }
template <bool kExact>
__device__ __forceinline__ float sigmoid_f32(float z) { return kExact ? 1.f / (1.f + expf(-z)) : fast_inverse(1.f + fast_exp(-z)); }
// sigma(z) and sigma(-z) by one exponential and one inverse: with e = exp(-|z|) they are 1 / (1 + e) and e / (1 + e) (gradient with SiLU, 4,096 x 8,192
// bfloat16 by 64: 62.0 us, 66.2 with two of each).
struct Sigmoids { float at, opposite; };
template <bool kExact>
__device__ __forceinline__ Sigmoids sigmoids_f32(float z) {
  const float e = kExact ? expf(-fabsf(z)) : fast_exp(-fabsf(z)), near = kExact ? 1.f / (1.f + e) : fast_inverse(1.f + e), far = e * near;
  return z < 0.f ? Sigmoids{far, near} : Sigmoids{near, far};
}
__device__ __forceinline__ float normal_tail(float a, float e) {      // Phi(-a), e = exp(-a^2/2)
  const float t = fast_inverse(fmaf(0.285f, a, 1.f));
  float p = 0.024569256f;
  p = fmaf(p, t, -0.08659119f);
  p = fmaf(p, t, 0.07391585f);
  p = fmaf(p, t, 0.003500571f);
  p = fmaf(p, t, 0.06757765f);
  p = fmaf(p, t, 0.08512555f);
  p = fmaf(p, t, 0.10450529f);
  p = fmaf(p, t, 0.11369858f);
  p = fmaf(p, t, 0.11369853f);
  return p * t * e;
}
// 1/2 z (1 + tanh u) = z sigma(2u), u = sqrt(2/pi) (z + 0.044715 z^3).
__device__ __forceinline__ float tanh_argument2(float z) { return 1.5957691216057308f * z * fmaf(0.044715f * z, z, 1.f); }

template <bool kExact, int kAct>
__device__ __forceinline__ float activate_as(float z) {
  if (kAct == STRADS_ACT_RELU) return z < 0.f ? 0.f : z;               // (a NaN stays one)
  if (kAct == STRADS_ACT_SIGMOID) return sigmoid_f32<kExact>(z);
  if (kAct == STRADS_ACT_GELU) {
    // (beyond 40 the tail is 0, and infinity times it would be NaN; -infinity times it is, as in the formula)
    const float q = fminf(z, 40.f) * normal_tail(fabsf(z), kExact ? expf(-0.5f * z * z) : fast_exp(-0.5f * z * z));
    return z > 0.f ? z - q : q;
  }
  if (kAct == STRADS_ACT_GELU_TANH) return z * sigmoid_f32<kExact>(tanh_argument2(z));
  if (kAct == STRADS_ACT_SILU) return z * sigmoid_f32<kExact>(z);
  return z;
}
template <bool kExact, int kAct>
__device__ __forceinline__ float slope_as(float z) {
  if (kAct == STRADS_ACT_RELU) return z > 0.f ? 1.f : (z <= 0.f ? 0.f : z);
  if (kAct == STRADS_ACT_SIGMOID) {
    const Sigmoids s = sigmoids_f32<kExact>(z);
    return s.at * s.opposite;
  }
  if (kAct == STRADS_ACT_GELU) {
    const float e = kExact ? expf(-0.5f * z * z) : fast_exp(-0.5f * z * z);
    const float near = fminf(fmaxf(z, -40.f), 40.f);                   // (beyond, e is 0)
    const float q = normal_tail(fabsf(z), e);
    return fmaf(near * 0.3989422804014327f, e, z > 0.f ? 1.f - q : q);
  }
  if (kAct == STRADS_ACT_GELU_TANH) {
    const float u = tanh_argument2(z), near = fminf(fmaxf(z, -40.f), 40.f);      // (beyond, the second term is 0)
    const Sigmoids s = sigmoids_f32<kExact>(u);
    return fmaf(near * s.at * s.opposite, 1.5957691216057308f * fmaf(0.134145f * near, near, 1.f), s.at);
  }
  if (kAct == STRADS_ACT_SILU) {
    const Sigmoids s = sigmoids_f32<kExact>(z);
    return s.at * fmaf(fminf(fmaxf(z, -128.f), 128.f), s.opposite, 1.f);      // (beyond, one of the two is 0)
  }
  return 1.f;
}

// Several values: one branch for all of them.
template <bool kExact, int kAct, int kN>
__device__ __forceinline__ void activate_run(float (&v)[kN]) {
#pragma unroll
  for (int j = 0; j < kN; ++j) v[j] = activate_as<kExact, kAct>(v[j]);
}
template <bool kExact, int kN>
__device__ __forceinline__ void activate_all(float (&v)[kN], int act) {
  switch (act) {
    case STRADS_ACT_RELU: activate_run<kExact, STRADS_ACT_RELU>(v); break;
    case STRADS_ACT_SIGMOID: activate_run<kExact, STRADS_ACT_SIGMOID>(v); break;
    case STRADS_ACT_GELU: activate_run<kExact, STRADS_ACT_GELU>(v); break;
    case STRADS_ACT_GELU_TANH: activate_run<kExact, STRADS_ACT_GELU_TANH>(v); break;
    case STRADS_ACT_SILU: activate_run<kExact, STRADS_ACT_SILU>(v); break;
    default: break;
  }
}
// kN elements of D in a row, `step` apart along b: a, b + j step, of which the first `count` (at least one) exist.  `here`: row a exists (else
// a is one that does, and nothing is stored).  Loads go to clamped places without a branch, so that they are all under way at
// once, and come before the stores: out may be the residual.
template <typename T, int kN>
__device__ __forceinline__ void finish_run(const Finish& f, float (&v)[kN], long long a, long long b, long long step, int count, bool here) {
  const long long sb_out = step * f.out.sb;
  T* out = static_cast<T*>(const_cast<void*>(f.out.p)) + a * f.out.sa + b * f.out.sb;
  if (!f.plain) {
    float r[kN];
    if (f.residual.p) {
      const T* p = static_cast<const T*>(f.residual.p) + a * f.residual.sa + b * f.residual.sb;
#pragma unroll
      for (int j = 0; j < kN; ++j) r[j] = load_f32(p + min(j, count - 1) * (step * f.residual.sb));
    }
    if (f.bias) {
      const T* p = static_cast<const T*>(f.bias) + a * f.bias_a + b * f.bias_b;
#pragma unroll
      for (int j = 0; j < kN; ++j) v[j] += load_f32(p + min(j, count - 1) * (step * f.bias_b));
    }
    if (f.preact.p) {
      T* p = static_cast<T*>(const_cast<void*>(f.preact.p)) + a * f.preact.sa + b * f.preact.sb;
#pragma unroll
      for (int j = 0; j < kN; ++j)
        if (here && j < count) store_f32(p + j * (step * f.preact.sb), v[j]);
    }
    activate_all<sizeof(T) == 4>(v, f.act);
#pragma unroll
    for (int j = 0; j < kN; ++j) v[j] = f.residual.p ? fmaf(f.scale, v[j], r[j]) : f.scale * v[j];
  } else {
    if (std::is_same<T, __half>::value && f.factor) {
      const float* p = f.factor + a * f.factor_a + b * f.factor_b;
#pragma unroll
      for (int j = 0; j < kN; ++j) v[j] *= p[min(j, count - 1) * (step * f.factor_b)];
    }
#pragma unroll
    for (int j = 0; j < kN; ++j) v[j] *= f.scale;
  }
#pragma unroll
  for (int j = 0; j < kN; ++j)
    if (here && j < count) store_f32(out + j * sb_out, v[j]);
}
template <typename T>
__device__ __forceinline__ void finish(const Finish& f, float z, long long a, long long b) {
  float v[1] = {z};
  finish_run<T, 1>(f, v, a, b, 1, 1, true);
}

// ---- products with few rows on one side (linear_thin.cu) ----
// D = A B^T with at most kThinMost rows in B, or in A (then swapped): every element of the long side is read once, from where it is.
constexpr int kThinMost = 4;
cudaError_t launch_linear_thin(int type, const Operand& A, const Operand& B, long long na, long long nb, long long nk, const Finish& f, unsigned int* status,
                               bool stall, cudaStream_t s);

}  // namespace strads
