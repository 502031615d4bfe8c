// Linear layers: what the kernels of strads_linear_forward / strads_linear_backward share.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

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
};

__device__ __forceinline__ float load_f32(const float* p) { return *p; }
__device__ __forceinline__ float load_f32(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ float load_f32(const __half* p) { return __half2float(*p); }
__device__ __forceinline__ void store_f32(float* p, float v) { *p = v; }
__device__ __forceinline__ void store_f32(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }
__device__ __forceinline__ void store_f32(__half* p, float v) { *p = __float2half_rn(v); }

// 1/2 z (1 + tanh u) = z sigma(2u), u = sqrt(2/pi) (z + 0.044715 z^3): in this form nothing cancels for negative z.
__device__ __forceinline__ float tanh_argument2(float z) { return 1.5957691216057308f * (z + 0.044715f * z * z * z); }
__device__ __forceinline__ float sigmoid_f32(float z) { return 1.f / (1.f + expf(-z)); }
__device__ __forceinline__ float activate(float z, int act) {
  switch (act) {
    case STRADS_ACT_RELU: return z < 0.f ? 0.f : z;                    // (a NaN stays one)
    case STRADS_ACT_SIGMOID: return sigmoid_f32(z);
    case STRADS_ACT_GELU: return z * normcdff(z);
    case STRADS_ACT_GELU_TANH: return z * sigmoid_f32(tanh_argument2(z));
    case STRADS_ACT_SILU: return z * sigmoid_f32(z);
    default: return z;
  }
}
__device__ __forceinline__ float slope(float z, int act) {
  switch (act) {
    case STRADS_ACT_RELU: return z > 0.f ? 1.f : (z <= 0.f ? 0.f : z);
    case STRADS_ACT_SIGMOID: { const float s = sigmoid_f32(z); return s * sigmoid_f32(-z); }
    case STRADS_ACT_GELU: return normcdff(z) + z * expf(-0.5f * z * z) * 0.3989422804014327f;
    case STRADS_ACT_GELU_TANH: {
      const float u = tanh_argument2(z), s = sigmoid_f32(u), near = fminf(fmaxf(z, -40.f), 40.f);      // (beyond, the second term is 0)
      return s + z * s * sigmoid_f32(-u) * 1.5957691216057308f * (1.f + 0.134145f * near * near);
    }
    case STRADS_ACT_SILU: { const float s = sigmoid_f32(z); return s * (1.f + z * sigmoid_f32(-z)); }
    default: return 1.f;
  }
}

// The same for several values: one branch for all of them.
template <int kN>
__device__ __forceinline__ void activate_all(float (&v)[kN], int act) {
  if (act == STRADS_ACT_IDENTITY) return;
  if (act == STRADS_ACT_RELU) {
#pragma unroll
    for (int j = 0; j < kN; ++j) v[j] = activate(v[j], STRADS_ACT_RELU);
  } else if (act == STRADS_ACT_SIGMOID) {
#pragma unroll
    for (int j = 0; j < kN; ++j) v[j] = activate(v[j], STRADS_ACT_SIGMOID);
  } else if (act == STRADS_ACT_GELU) {
#pragma unroll
    for (int j = 0; j < kN; ++j) v[j] = activate(v[j], STRADS_ACT_GELU);
  } else if (act == STRADS_ACT_GELU_TANH) {
#pragma unroll
    for (int j = 0; j < kN; ++j) v[j] = activate(v[j], STRADS_ACT_GELU_TANH);
  } else {
#pragma unroll
    for (int j = 0; j < kN; ++j) v[j] = activate(v[j], STRADS_ACT_SILU);
  }
}

// One element of D.
template <typename T>
__device__ __forceinline__ void finish(const Finish& f, float z, long long a, long long b) {
  if (f.plain) {
    z *= f.scale;
  } else {
    if (f.bias) z += load_f32(static_cast<const T*>(f.bias) + a * f.bias_a + b * f.bias_b);
    if (f.preact.p) store_f32(static_cast<T*>(const_cast<void*>(f.preact.p)) + a * f.preact.sa + b * f.preact.sb, z);
    z = f.scale * activate(z, f.act);
    if (f.residual.p) z += load_f32(static_cast<const T*>(f.residual.p) + a * f.residual.sa + b * f.residual.sb);
  }
  store_f32(static_cast<T*>(const_cast<void*>(f.out.p)) + a * f.out.sa + b * f.out.sb, z);
}

// ---- products with few rows on one side (linear_thin.cu) ----
// D = A B^T with nb <= kThinMost rows in B, or in A (then swapped): every element of the long side is read once, from where it is.
constexpr int kThinMost = 8;
cudaError_t launch_linear_thin(int type, const Operand& A, const Operand& B, long long na, long long nb, long long nk, const Finish& f, cudaStream_t s);

}  // namespace strads
