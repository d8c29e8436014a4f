// Shared by the kernels of linear layers: activations and their derivatives, launch parameters.
#pragma once

#include "row_vectors.cuh"

namespace surgeon {

constexpr int kActNone = 0, kActRelu = 1, kActGelu = 2;

// Phi(z) = erfc(-z / sqrt 2) / 2 and e^(-z^2/2), the two parts of GELU(z) = z Phi(z) and of its derivative
// Phi(z) + z e^(-z^2/2) / sqrt(2 pi).  erfc by Abramowitz and Stegun, "Handbook of Mathematical Functions", 7.1.26
// (error below 1.5e-7 of erf): t = 1 / (1 + 0.3275911 |x|), erfc(|x|) = (a1 t + ... + a5 t^5) e^(-x^2).  Some 14 instructions,
// two of them approximate ones of the special function unit, and no branch.
__device__ __forceinline__ void normal_parts(float z, float& phi, float& e) {
  const float t = __fdividef(1.0f, fmaf(0.3275911f * 0.70710678f, fabsf(z), 1.0f));
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(-0.72134752f * z * z));      // e^(-z^2/2)
  float p = fmaf(1.061405429f, t, -1.453152027f);
  p = fmaf(p, t, 1.421413741f);
  p = fmaf(p, t, -0.284496736f);
  p = fmaf(p, t, 0.254829592f);
  const float tail = 0.5f * (p * t) * e;              // Phi(-|z|)
  phi = z < 0.0f ? tail : 1.0f - tail;
}

// ReLU and GELU let a NaN through.  GELU(-inf): -inf * 0 would be NaN, and is 0.
template <int ACT>
__device__ __forceinline__ float activate(float z) {
  if (ACT == kActRelu) return z < 0.0f ? 0.0f : z;
  if (ACT == kActGelu) {
    float phi, e;
    normal_parts(z, phi, e);
    return z < -14.0f ? 0.0f : z * phi;
  }
  return z;
}
__device__ __forceinline__ float activate(float z, int act) {
  return act == kActRelu ? activate<kActRelu>(z) : act == kActGelu ? activate<kActGelu>(z) : z;
}
// The derivative; 0 at 0 for ReLU.  NaN for a NaN.
__device__ __forceinline__ float slope(float z, int act) {
  if (act == kActRelu) return z > 0.0f ? 1.0f : (z <= 0.0f ? 0.0f : z);
  if (act == kActGelu) {
    float phi, e;
    normal_parts(z, phi, e);
    return fabsf(z) > 14.0f ? (z > 0.0f ? 1.0f : 0.0f) : fmaf(z * 0.39894228f, e, phi);
  }
  return 1.0f;
}

// y = act(a b^T + bias) + residual, z = a b^T + bias.  a: bf16 [m, k], rows `lda` elements apart.  b: bf16, element (n, k)
// at n * ldb + k, or (b_mn) at k * ldb + n.  y, residual: [m, n] of type dt; pre (z, bf16): [m, n].
struct Product {
  const void* a;
  const void* b;
  int m, n, k, lda, ldb, b_mn;
  const float* bias;
  const void* residual;
  void* y;
  void* pre;
  int act, dt;
};

cudaError_t launch_product(const Product& p, uint32_t* status, cudaStream_t stream);

}  // namespace surgeon
