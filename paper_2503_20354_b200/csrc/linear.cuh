// Shared by the kernels of linear layers: activations and their derivatives, launch parameters.
#pragma once

#include "row_vectors.cuh"

namespace surgeon {

constexpr int kActNone = 0, kActRelu = 1, kActGelu = 2;

// Phi(-a) and e^(-a^2/2) for a >= 0, the parts of GELU and of its derivative.  Phi(-a) = erfc(a / sqrt 2) / 2; erfc by Abramowitz
// and Stegun, "Handbook of Mathematical Functions", 7.1.26 (error below 1.5e-7 of erf): t = 1 / (1 + 0.3275911 x),
// erfc(x) = (a1 t + ... + a5 t^5) e^(-x^2); the coefficients below are halved.  Ten instructions of the FMA pipe and two
// approximate ones of the special function unit, no branch.
__device__ __forceinline__ void normal_tail(float a, float& tail, float& e) {
  float t;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(t) : "f"(fmaf(0.3275911f * 0.70710678f, a, 1.0f)));
  const float u = 0.84932180f * a;                    // sqrt(log2(e) / 2) a
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(-u * u));
  float p = fmaf(0.5307027145f, t, -0.7265760135f);
  p = fmaf(p, t, 0.7107068705f);
  p = fmaf(p, t, -0.142248368f);
  p = fmaf(p, t, 0.127414796f);
  tail = p * t * e;
}
// max(z, 0), NaN for NaN; min(|z|, 16), where Phi(-16) is 0 in fp32
__device__ __forceinline__ float positive(float z) {
  float m;
  asm("max.NaN.f32 %0, %1, 0f00000000;" : "=f"(m) : "f"(z));
  return m;
}

// GELU(z) = z Phi(z) = max(z, 0) - |z| Phi(-|z|).  ReLU and GELU let a NaN through; GELU(-inf) is 0 (not -inf * 0).
template <int ACT>
__device__ __forceinline__ float activate(float z) {
  if (ACT == kActRelu) return positive(z);
  if (ACT == kActGelu) {
    const float a = fminf(fabsf(z), 16.0f);
    float tail, e;
    normal_tail(a, tail, e);
    return fmaf(-a, tail, positive(z));
  }
  return z;
}
__device__ __forceinline__ float activate(float z, int act) {
  return act == kActRelu ? activate<kActRelu>(z) : act == kActGelu ? activate<kActGelu>(z) : z;
}
// The derivative: ReLU 1 above 0, else 0; GELU Phi(z) + z e^(-z^2/2) / sqrt(2 pi).  NaN for a NaN.
template <int ACT>
__device__ __forceinline__ float slope(float z) {
  if (ACT == kActRelu) return z > 0.0f ? 1.0f : (z <= 0.0f ? 0.0f : z);
  if (ACT == kActGelu) {
    const float a = fminf(fabsf(z), 16.0f);
    float tail, e;
    normal_tail(a, tail, e);
    const float half = fmaf(-0.39894228f * a, e, tail);         // the derivative at -|z|
    return z > 0.0f ? 1.0f - half : (z <= 0.0f ? half : z);
  }
  return 1.0f;
}

// Column sums that a kernel before left in `slabs` rows of partial sums, to be added in order into `out` (null: none).
struct ColumnSums {
  const float* partial;
  float* out;
  int slabs, cols, accumulate;
};
constexpr int kSumSlices = 32;
// Every ctas-th group of 32 columns, by WARPS warps of CTA `cta`: 32 slices of the slabs, then the slices, in order.
template <int WARPS>
__device__ __forceinline__ void add_columns(const ColumnSums& s, int cta, int ctas, int warp, float (&buf)[kSumSlices][32]) {
  const int lane = static_cast<int>(lane_id());
  for (int g = cta; g * 32 < s.cols; g += ctas) {
    const int c = g * 32 + lane;
#pragma unroll 4
    for (int slice = warp; slice < kSumSlices; slice += WARPS) {
      float t = 0.0f;
      if (c < s.cols) {
#pragma unroll 4
        for (int i = slice; i < s.slabs; i += kSumSlices) t += s.partial[static_cast<long long>(i) * s.cols + c];
      }
      buf[slice][lane] = t;
    }
    named_barrier(1, 32 * WARPS);
    if (warp == 0 && c < s.cols) {
      float t = 0.0f;
#pragma unroll
      for (int i = 0; i < kSumSlices; ++i) t += buf[i][lane];
      s.out[c] = s.accumulate ? s.out[c] + t : t;
    }
    named_barrier(1, 32 * WARPS);
  }
}

// a itself in fp32 to `out` [m, k] (where wanted) and its column sums, 128 rows a slab, to `partial` [slabs][k] (or, one slab, to
// `sums`, added to what is there with `accumulate`): taken from the tiles that the product has in shared memory anyway.
struct CopyOut {
  float* out;
  float* partial;
  float* sums;
  int accumulate;
};

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
  ColumnSums sums;                               // taken along by the first warps that are free
  int copy_a;                                    // (an N-major b)
  CopyOut copy;
};

cudaError_t launch_product(const Product& p, uint32_t* status, cudaStream_t stream);

}  // namespace surgeon
