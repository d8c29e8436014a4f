// Dropout whose mask is never stored: the random bits are a function of an element's index, made again in the backward pass.
//
//   y_i = (u_i >= t ? x_i * 65536 / (65536 - t) : 0) + residual_i,   t = round(65536 p),   u_i: 16 random bits
//
// Bits: Philox 4x32 with ten rounds (Salmon, Moraes, Dror and Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011), one counter
// for eight elements: (i / 8, offset), the key is the seed.  16 bits an element: with 32 the generator's products are 10 an element,
// more than the integer pipe gives at the memory's rate.
// A thread takes eight elements, so that a counter serves one thread.
#include "row_vectors.cuh"

namespace surgeon {

namespace {

constexpr int kThreads = 256;
constexpr int kPer = 8;                          // elements of a counter, and of a thread

__device__ __forceinline__ uint4 philox(uint4 c, uint32_t k0, uint32_t k1) {
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t p = static_cast<uint64_t>(c.x) * 0xD2511F53u, q = static_cast<uint64_t>(c.z) * 0xCD9E8D57u;
    c = make_uint4(static_cast<uint32_t>(q >> 32) ^ c.y ^ k0, static_cast<uint32_t>(q), static_cast<uint32_t>(p >> 32) ^ c.w ^ k1,
                   static_cast<uint32_t>(p));
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return c;
}

template <int DT, bool RES>
__global__ void __launch_bounds__(kThreads)
dropout_kernel(const void* x, const void* residual, void* y, uint32_t n, uint32_t dropped, float scale, uint64_t seed, uint64_t offset,
               const uint64_t* device_offset) {
  pdl_trigger();
  pdl_wait();
  const uint32_t group = blockIdx.x * kThreads + threadIdx.x, at = group * kPer;
  if (at >= n) return;
  const bool whole = at + kPer <= n;
  float f[kPer], r[kPer];
  if (whole) {                                   // (loads first: the generator's chain hides their latency)
    load_elems<DT, 8>(x, at, f);
    if (RES) load_elems<DT, 8>(residual, at, r);
  }
  if (device_offset) offset += *device_offset;
  const uint4 w = philox(make_uint4(group, 0u, static_cast<uint32_t>(offset), static_cast<uint32_t>(offset >> 32)),
                         static_cast<uint32_t>(seed), static_cast<uint32_t>(seed >> 32));
  const uint32_t words[4] = {w.x, w.y, w.z, w.w};
  const auto one = [&](int i, float v) {
    const uint32_t u = i & 1 ? words[i >> 1] >> 16 : words[i >> 1] & 0xFFFFu;
    return u >= dropped ? v * scale : 0.0f;
  };
  if (whole) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) f[i] = RES ? one(i, f[i]) + r[i] : one(i, f[i]);
    store_elems<DT, 8>(y, at, f);
    return;
  }
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    if (at + i >= n) break;
    float v[1], s[1];
    load_elems<DT, 1>(x, at + i, v);
    v[0] = one(i, v[0]);
    if (RES) {
      load_elems<DT, 1>(residual, at + i, s);
      v[0] += s[0];
    }
    store_elems<DT, 1>(y, at + i, v);
  }
}

}  // namespace

cudaError_t launch_dropout(const void* x, long long n, int dt, uint32_t dropped, uint64_t seed, uint64_t offset,
                           const uint64_t* device_offset, const void* residual, void* y, cudaStream_t stream) {
  if (n == 0) return cudaSuccess;
  const float scale = dropped < 65536u ? static_cast<float>(65536.0 / (65536u - dropped)) : 0.0f;
  const uint32_t grid = static_cast<uint32_t>((n + kThreads * kPer - 1) / (kThreads * kPer));
  const auto kernel = dt ? (residual ? dropout_kernel<1, true> : dropout_kernel<1, false>)
                         : (residual ? dropout_kernel<0, true> : dropout_kernel<0, false>);
  const cudaError_t e = launch_kernel(kernel, dim3(grid), dim3(kThreads), 0, stream, true, x, residual, y, static_cast<uint32_t>(n),
                                      dropped, scale, seed, offset, device_offset);
  note_launches(1);
  return e;
}

}  // namespace surgeon
