// Loads and stores of short vectors of fp32 or bf16 elements as fp32 numbers (layer norm, linear layers, gradient lists).
#pragma once

#include "surgeon_internal.cuh"

namespace surgeon {

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
// Two fp32 numbers as bf16 in one word, each rounded to nearest even once.
__device__ __forceinline__ uint32_t to_bf16x2(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

// E consecutive elements of type DT at element `at` of `base` (aligned to the vector's size, 16 bytes at most).
template <int DT, int E>
__device__ __forceinline__ void load_elems(const void* __restrict__ base, long long at, float (&f)[E]) {
  if constexpr (DT == 0) {
    const float* p = static_cast<const float*>(base) + at;
    if constexpr (E % 4 == 0) {
#pragma unroll
      for (int i = 0; i < E / 4; ++i) {
        const float4 v = reinterpret_cast<const float4*>(p)[i];
        f[4 * i] = v.x; f[4 * i + 1] = v.y; f[4 * i + 2] = v.z; f[4 * i + 3] = v.w;
      }
    } else {
#pragma unroll
      for (int i = 0; i < E; ++i) f[i] = p[i];
    }
  } else {
    const unsigned short* p = static_cast<const unsigned short*>(base) + at;
    if constexpr (E == 8) {
      const uint4 v = *reinterpret_cast<const uint4*>(p);
      f[0] = bf16_lo(v.x); f[1] = bf16_hi(v.x); f[2] = bf16_lo(v.y); f[3] = bf16_hi(v.y);
      f[4] = bf16_lo(v.z); f[5] = bf16_hi(v.z); f[6] = bf16_lo(v.w); f[7] = bf16_hi(v.w);
    } else if constexpr (E == 4) {
      const uint2 v = *reinterpret_cast<const uint2*>(p);
      f[0] = bf16_lo(v.x); f[1] = bf16_hi(v.x); f[2] = bf16_lo(v.y); f[3] = bf16_hi(v.y);
    } else {
#pragma unroll
      for (int i = 0; i < E; ++i) f[i] = __uint_as_float(static_cast<uint32_t>(p[i]) << 16);
    }
  }
}

template <int DT, int E>
__device__ __forceinline__ void store_elems(void* __restrict__ base, long long at, const float (&f)[E]) {
  if constexpr (DT == 0) {
    float* p = static_cast<float*>(base) + at;
    if constexpr (E % 4 == 0) {
#pragma unroll
      for (int i = 0; i < E / 4; ++i)
        reinterpret_cast<float4*>(p)[i] = make_float4(f[4 * i], f[4 * i + 1], f[4 * i + 2], f[4 * i + 3]);
    } else {
#pragma unroll
      for (int i = 0; i < E; ++i) p[i] = f[i];
    }
  } else {
    unsigned short* p = static_cast<unsigned short*>(base) + at;
    if constexpr (E == 8) {
      *reinterpret_cast<uint4*>(p) = make_uint4(to_bf16x2(f[0], f[1]), to_bf16x2(f[2], f[3]), to_bf16x2(f[4], f[5]),
                                                to_bf16x2(f[6], f[7]));
    } else if constexpr (E == 4) {
      *reinterpret_cast<uint2*>(p) = make_uint2(to_bf16x2(f[0], f[1]), to_bf16x2(f[2], f[3]));
    } else {
#pragma unroll
      for (int i = 0; i < E; ++i) p[i] = static_cast<unsigned short>(to_bf16x2(f[i], 0.0f) & 0xFFFFu);
    }
  }
}

// A 16-byte vector as numbers.
template <int DT>
__device__ __forceinline__ void vector_elems(uint4 v, float (&f)[DT == 0 ? 4 : 8]) {
  if constexpr (DT == 0) {
    f[0] = __uint_as_float(v.x); f[1] = __uint_as_float(v.y); f[2] = __uint_as_float(v.z); f[3] = __uint_as_float(v.w);
  } else {
    f[0] = bf16_lo(v.x); f[1] = bf16_hi(v.x); f[2] = bf16_lo(v.y); f[3] = bf16_hi(v.y);
    f[4] = bf16_lo(v.z); f[5] = bf16_hi(v.z); f[6] = bf16_lo(v.w); f[7] = bf16_hi(v.w);
  }
}

// Barrier `id` for `threads` threads, whole warps.  The instruction takes a warp's lanes together: they come together first, since
// the code before may have sent them different ways.
__device__ __forceinline__ void named_barrier(int id, int threads) {
  __syncwarp();
  asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory");
}

// Sum over groups of W lanes (W a power of two up to 32), the same bits in every lane of the group.
template <int W, typename T>
__device__ __forceinline__ T lanes_sum(T v) {
#pragma unroll
  for (int o = W / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
  return v;
}

}  // namespace surgeon
