// Layer norm over the channels of [rows, channels], and its backward pass.
//
//   mean = sum_c x / C;  r = 1 / sqrt(sum_c (x - mean)^2 / C + eps);  xh = (x - mean) r;  y = xh gamma + beta
//   g = dy gamma;  dx = r (g - sum_c g / C - xh sum_c (g xh) / C) (+ residual_grad)
//   dgamma = sum_t dy xh;  dbeta = sum_t dy
//
// A row is held in the registers of the threads that share it, so it is read once; the variance is the mean of
// centred squares (of E[x^2] - mean^2 nothing is left where the mean is large).  All sums are fp32, in a fixed order.
// Forward and backward are bound by HBM: 2 and 3 (4 with the residual's gradient) passes over the row.
#include "row_vectors.cuh"
#include "tc_common.cuh"

namespace surgeon {

namespace {

constexpr int kLnThreads = 256;
constexpr int kLnPartials = 296;     // CTAs that keep column sums: two per SM; rows of the partial sums' scratch

// Sum over the TPR threads that share a row; a row of more than 32 threads is the whole CTA.
// `buf`: one word per warp; two calls in a row use different ones.
template <int TPR>
__device__ __forceinline__ float row_sum(float v, float* buf) {
  v = lanes_sum<(TPR < 32 ? TPR : 32)>(v);
  if constexpr (TPR > 32) {
    if ((threadIdx.x & 31) == 0) buf[threadIdx.x >> 5] = v;
    __syncthreads();
    v = 0.0f;
#pragma unroll
    for (int w = 0; w < TPR / 32; ++w) v += buf[w];
  }
  return v;
}

template <int DT, int E, int V, int TPR>
__global__ void __launch_bounds__(TPR > 32 ? TPR : kLnThreads)
ln_forward_kernel(const void* __restrict__ x, long long rows, int channels, const float* __restrict__ gamma,
                  const float* __restrict__ beta, float eps, void* __restrict__ y, float* __restrict__ stats) {
  constexpr int kRows = TPR > 32 ? 1 : kLnThreads / TPR;       // rows per CTA at a time
  __shared__ float buf[2][TPR > 32 ? TPR / 32 : 1];
  pdl_wait();
  pdl_trigger();
  const int l = static_cast<int>(threadIdx.x) % TPR;
  const float inv_c = 1.0f / static_cast<float>(channels);
  const long long row = static_cast<long long>(blockIdx.x) * kRows + static_cast<int>(threadIdx.x) / TPR;
  const bool on = row < rows;
  float f[V][E];
  float s = 0.0f;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int c = (v * TPR + l) * E;
    if (on && c < channels) load_elems<DT, E>(x, row * channels + c, f[v]);
    else {
#pragma unroll
      for (int e = 0; e < E; ++e) f[v][e] = 0.0f;
    }
#pragma unroll
    for (int e = 0; e < E; ++e) s += f[v][e];
  }
  const float mean = row_sum<TPR>(s, buf[0]) * inv_c;
  float q = 0.0f;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    if ((v * TPR + l) * E < channels) {
#pragma unroll
      for (int e = 0; e < E; ++e) {
        f[v][e] -= mean;
        q += f[v][e] * f[v][e];
      }
    }
  }
  const float r = rsqrtf(row_sum<TPR>(q, buf[1]) * inv_c + eps);
  if (!on) return;
  if (stats && l == 0) {
    stats[row] = mean;
    stats[rows + row] = r;
  }
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int c = (v * TPR + l) * E;
    if (c < channels) {
#pragma unroll
      for (int e = 0; e < E; ++e) f[v][e] *= r;
      if (gamma) {
        float w[E];
        load_elems<0, E>(gamma, c, w);
#pragma unroll
        for (int e = 0; e < E; ++e) f[v][e] *= w[e];
      }
      if (beta) {
        float w[E];
        load_elems<0, E>(beta, c, w);
#pragma unroll
        for (int e = 0; e < E; ++e) f[v][e] += w[e];
      }
      store_elems<DT, E>(y, row * channels + c, f[v]);
    }
  }
}

// Parameters in shared memory, in the order in which the lanes read them: four at a time, without bank conflicts.
template <int E, int TPR>
__device__ __forceinline__ void fill_params(int threads, float* to, const float* __restrict__ from, float none, int channels) {
  if constexpr (E == 1) {
#pragma unroll 8
    for (int c = threadIdx.x; c < channels; c += threads) to[c] = from ? __ldg(from + c) : none;
  } else {
#pragma unroll 4
    for (int q = threadIdx.x; q < channels / 4; q += threads) {
      const int vec = q / (E / 4), h = q % (E / 4), v = vec / TPR, l = vec % TPR;
      reinterpret_cast<float4*>(to)[(v * (E / 4) + h) * TPR + l] =
          from ? __ldg(reinterpret_cast<const float4*>(from) + q) : make_float4(none, none, none, none);
    }
  }
}
template <int E, int TPR>
__device__ __forceinline__ void load_params(const float* from, int v, int l, float (&w)[E]) {
  if constexpr (E == 1) {
    w[0] = from[v * TPR + l];
  } else {
#pragma unroll
    for (int h = 0; h < E / 4; ++h) {
      const float4 q = *reinterpret_cast<const float4*>(from + ((v * (E / 4) + h) * TPR + l) * 4);
      w[4 * h] = q.x; w[4 * h + 1] = q.y; w[4 * h + 2] = q.z; w[4 * h + 3] = q.w;
    }
  }
}
// More rows than the SMs hold at once: CTAs that stay, each warp's (or part of a warp's) next row on its way while it works on
// one, the parameters in shared memory.  12608 x 768 bf16: 8.2 us, 4.7 TB/s, by four CTAs an SM (three 8.4, five 10.9); one row
// per warp and CTAs that go 10.3.
template <int DT, int V, int TPR>
constexpr int rows_ctas() { return DT == 1 && V <= 3 ? 4 : 3; }

template <int DT, int V, int TPR>
__global__ void __launch_bounds__(kLnThreads, rows_ctas<DT, V, TPR>())
ln_forward_rows_kernel(const void* __restrict__ x, long long rows, int channels, const float* __restrict__ gamma,
                       const float* __restrict__ beta, float eps, void* __restrict__ y, float* __restrict__ stats) {
  constexpr int E = DT ? 8 : 4, kRows = kLnThreads / TPR, kSize = DT ? 2 : 4;
  __shared__ __align__(16) float s_gamma[V * TPR * E], s_beta[V * TPR * E];
  pdl_wait();
  pdl_trigger();
  const int l = static_cast<int>(threadIdx.x) % TPR, sub = static_cast<int>(threadIdx.x) / TPR;
  const float inv_c = 1.0f / static_cast<float>(channels);
  const unsigned char* from = static_cast<const unsigned char*>(x);
  uint4 raw[V];
  const auto fetch = [&](long long row) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int c = (v * TPR + l) * E;
      if (row < rows && c < channels) raw[v] = *reinterpret_cast<const uint4*>(from + (row * channels + c) * kSize);
    }
  };
#pragma unroll
  for (int v = 0; v < V; ++v) raw[v] = make_uint4(0, 0, 0, 0);                // (columns behind the last stay zero)
  const long long step = static_cast<long long>(gridDim.x) * kRows;
  fetch(static_cast<long long>(blockIdx.x) * kRows + sub);
  fill_params<E, TPR>(kLnThreads, s_gamma, gamma, 1.0f, channels);
  fill_params<E, TPR>(kLnThreads, s_beta, beta, 0.0f, channels);
  __syncthreads();
  for (long long first = static_cast<long long>(blockIdx.x) * kRows; first < rows; first += step) {
    const long long row = first + sub;
    float f[V][E], s = 0.0f, q = 0.0f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      vector_elems<DT>(raw[v], f[v]);
#pragma unroll
      for (int e = 0; e < E; ++e) s += f[v][e];
    }
    fetch(row + step);
    const float mean = lanes_sum<TPR>(s) * inv_c;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      if ((v * TPR + l) * E < channels) {
#pragma unroll
        for (int e = 0; e < E; ++e) {
          f[v][e] -= mean;
          q += f[v][e] * f[v][e];
        }
      }
    }
    const float r = rsqrtf(lanes_sum<TPR>(q) * inv_c + eps);
    if (row >= rows) continue;
    if (stats && l == 0) {
      stats[row] = mean;
      stats[rows + row] = r;
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int c = (v * TPR + l) * E;
      if (c < channels) {
        float w[E], b[E];
        load_params<E, TPR>(s_gamma, v, l, w);
        load_params<E, TPR>(s_beta, v, l, b);
#pragma unroll
        for (int e = 0; e < E; ++e) f[v][e] = fmaf(f[v][e] * r, w[e], b[e]);
        store_elems<DT, E>(y, row * channels + c, f[v]);
      }
    }
  }
}

// Rows too long for registers: one CTA per row, which is read three times (from L1 or L2 but for the first).
template <int DT>
__global__ void __launch_bounds__(1024)
ln_forward_long_kernel(const void* __restrict__ x, long long rows, int channels, const float* __restrict__ gamma,
                       const float* __restrict__ beta, float eps, void* __restrict__ y, float* __restrict__ stats) {
  __shared__ float buf[2][32];
  pdl_wait();
  pdl_trigger();
  const long long row = blockIdx.x, at = row * channels;
  const float inv_c = 1.0f / static_cast<float>(channels);
  float f[1], s = 0.0f, q = 0.0f;
  for (int c = threadIdx.x; c < channels; c += 1024) {
    load_elems<DT, 1>(x, at + c, f);
    s += f[0];
  }
  const float mean = row_sum<1024>(s, buf[0]) * inv_c;
  for (int c = threadIdx.x; c < channels; c += 1024) {
    load_elems<DT, 1>(x, at + c, f);
    q += (f[0] - mean) * (f[0] - mean);
  }
  const float r = rsqrtf(row_sum<1024>(q, buf[1]) * inv_c + eps);
  if (stats && threadIdx.x == 0) {
    stats[row] = mean;
    stats[rows + row] = r;
  }
  for (int c = threadIdx.x; c < channels; c += 1024) {
    load_elems<DT, 1>(x, at + c, f);
    f[0] = (f[0] - mean) * r;
    if (gamma) f[0] *= gamma[c];
    if (beta) f[0] += beta[c];
    store_elems<DT, 1>(y, at + c, f);
  }
}

// Rows too long for registers: the row's two sums, then dx; the columns' sums are another kernel's.
template <int XDT, int GDT>
__global__ void __launch_bounds__(1024)
ln_backward_long_kernel(const void* __restrict__ x, const void* __restrict__ dy, long long rows, int channels,
                        const float* __restrict__ gamma, const float* __restrict__ stats,
                        const void* __restrict__ residual, void* __restrict__ dx) {
  __shared__ float buf[2][32];
  pdl_wait();
  pdl_trigger();
  const long long row = blockIdx.x, at = row * channels;
  const float inv_c = 1.0f / static_cast<float>(channels);
  const float mean = stats[row], r = stats[rows + row];
  float a[1], d[1], c1 = 0.0f, c2 = 0.0f;
  for (int c = threadIdx.x; c < channels; c += 1024) {
    load_elems<XDT, 1>(x, at + c, a);
    load_elems<GDT, 1>(dy, at + c, d);
    if (gamma) d[0] *= gamma[c];
    c1 += d[0];
    c2 += d[0] * ((a[0] - mean) * r);
  }
  c1 = row_sum<1024>(c1, buf[0]) * inv_c;
  c2 = row_sum<1024>(c2, buf[1]) * inv_c;
  for (int c = threadIdx.x; c < channels; c += 1024) {
    load_elems<XDT, 1>(x, at + c, a);
    load_elems<GDT, 1>(dy, at + c, d);
    if (gamma) d[0] *= gamma[c];
    d[0] = r * (d[0] - c1 - ((a[0] - mean) * r) * c2);
    if (residual) {
      float k[1];
      load_elems<GDT, 1>(residual, at + c, k);
      d[0] += k[0];
    }
    store_elems<GDT, 1>(dx, at + c, d);
  }
}

// Column sums of a slab of rows (blockIdx.y), a thread per column.
template <int XDT, int GDT>
__global__ void __launch_bounds__(kLnThreads)
ln_columns_kernel(const void* __restrict__ x, const void* __restrict__ dy, long long rows, int channels,
                  const float* __restrict__ stats, long long rows_per, float* __restrict__ partial) {
  pdl_wait();
  pdl_trigger();
  const int c = blockIdx.x * kLnThreads + threadIdx.x;
  if (c >= channels) return;
  const long long begin = blockIdx.y * rows_per, end = begin + rows_per < rows ? begin + rows_per : rows;
  float dg = 0.0f, db = 0.0f, a[1], d[1];
#pragma unroll 4
  for (long long t = begin; t < end; ++t) {
    load_elems<XDT, 1>(x, t * channels + c, a);
    load_elems<GDT, 1>(dy, t * channels + c, d);
    dg += d[0] * ((a[0] - stats[t]) * stats[rows + t]);
    db += d[0];
  }
  partial[static_cast<long long>(blockIdx.y) * 2 * channels + c] = dg;
  partial[(static_cast<long long>(blockIdx.y) * 2 + 1) * channels + c] = db;
}

// The partial sums' rows, added in order: 32 columns per CTA, 32 slices of the rows (each a few loads that are on their way
// together).
constexpr int kFinalThreads = 1024;
__global__ void __launch_bounds__(kFinalThreads)
ln_final_kernel(const float* __restrict__ partial, int n_partials, int channels, float* __restrict__ dgamma,
                float* __restrict__ dbeta, int accumulate) {
  __shared__ float part[kFinalThreads / 32][33];
  pdl_wait();
  pdl_trigger();
  const int k = blockIdx.y;
  float* out = k ? dbeta : dgamma;
  if (!out) return;
  const int c = blockIdx.x * 32 + (threadIdx.x & 31), slice = threadIdx.x >> 5;
  float t = 0.0f;
  if (c < channels) {
#pragma unroll 5
    for (int i = slice; i < n_partials; i += kFinalThreads / 32) t += partial[(static_cast<long long>(i) * 2 + k) * channels + c];
  }
  part[slice][threadIdx.x & 31] = t;
  __syncthreads();
  if (slice == 0 && c < channels) {
    t = 0.0f;
#pragma unroll
    for (int i = 0; i < kFinalThreads / 32; ++i) t += part[i][threadIdx.x];
    out[c] = accumulate ? out[c] + t : t;
  }
}

// ---- a ring of chunks in shared memory ----
//
// A chunk is some consecutive rows, one contiguous piece of memory.  A producer warp fetches chunks of x (and dy,
// residual_grad) with bulk copies, rounded to 16-byte boundaries on either side, so that rows of any width arrive with wide
// asynchronous loads and some 150 KB per SM are in flight.  Two groups of eight warps take the chunks in turn.  One CTA per SM.

constexpr int kRingGroups = 2, kGroupThreads = 256;
constexpr int kRingThreads = kRingGroups * kGroupThreads + 32;
constexpr int kSmemBytes = 224 * 1024;           // ring and parameters
constexpr int kMaxRing = 8;

struct RingArgs {
  const void* src[3];
  int elem[3];                                   // bytes of an element
  int at[3];                                     // where the array's rows lie in a stage
  int n_src;
  long long rows;
  int channels;
  int chunk_rows, stages, stage_bytes;
  int params;                                    // parameters' place in shared memory
  long long chunks;
};

// Where row `row` of array i starts behind the 16-byte boundary that its copy begins at.
__device__ __forceinline__ uint32_t ring_shift(const RingArgs& a, int i, long long row) {
  return static_cast<uint32_t>(row * a.channels * a.elem[i]) & 15u;
}

// A stage's barrier for a group's chunks.  A wait knows a phase from the one before it by its parity alone, so whoever waits on a
// barrier has to see all of its phases; with an odd number of stages a stage's chunks go to either group in turn.
__device__ __forceinline__ uint32_t ring_full(uint32_t full, int group, int stage) { return full + 8 * (group * kMaxRing + stage); }

// The producer warp: every gridDim.x-th chunk into the ring.
__device__ __forceinline__ void ring_produce(const RingArgs& a, unsigned char* ring, uint32_t full, uint32_t empty) {
  const bool leader = tc::elected();
  int s = 0, group = 0;
  uint32_t phase = 1;
  for (long long chunk = blockIdx.x; chunk < a.chunks; chunk += gridDim.x) {
    if (!__all_sync(0xFFFFFFFFu, tc::mbar_wait_suspend(empty + 8 * s, phase))) return;
    const uint32_t bar = ring_full(full, group, s);
    const long long row = chunk * a.chunk_rows;
    const long long here = a.rows - row < a.chunk_rows ? a.rows - row : a.chunk_rows;
    if (leader) {
      uint32_t bytes[3], total = 0;
#pragma unroll
      for (int i = 0; i < 3; ++i) {
        if (i >= a.n_src) break;
        const long long pitch = static_cast<long long>(a.channels) * a.elem[i];
        const long long begin = row * pitch, end = begin + here * pitch, lo = begin & ~15LL, last = (a.rows * pitch) & ~15LL;
        long long hi = (end + 15) & ~15LL;
        if (hi > last) hi = last > lo ? last : lo;              // the tensor's last bytes, below 16, one by one
        for (long long b = hi > begin ? hi : begin; b < end; b += 2)
          *reinterpret_cast<unsigned short*>(ring + s * a.stage_bytes + a.at[i] + (b - lo)) =
              *reinterpret_cast<const unsigned short*>(static_cast<const unsigned char*>(a.src[i]) + b);
        bytes[i] = static_cast<uint32_t>(hi - lo);
        total += bytes[i];
      }
      tc::mbar_arrive_expect_tx(bar, total);
#pragma unroll
      for (int i = 0; i < 3; ++i) {
        if (i >= a.n_src) break;
        if (bytes[i])
          tc::bulk_load(tc::smem_u32(ring + s * a.stage_bytes + a.at[i]),
                        static_cast<const unsigned char*>(a.src[i]) + ((row * a.channels * a.elem[i]) & ~15LL), bytes[i], bar);
      }
    }
    __syncwarp();
    if (++group == kRingGroups) group = 0;
    if (++s == a.stages) { s = 0; phase ^= 1; }
  }
}

// A chunk's place given back: every number of it has gone into a sum or a store by now, and the fence orders these reads before
// the next bulk copy, which is of another proxy.
__device__ __forceinline__ void ring_release(uint32_t bar) {
  tc::fence_proxy_async();
  __syncwarp();
  if (lane_id() == 0) tc::mbar_arrive(bar);
}

// Sum over the TPR threads of a row inside a group of 256; `buf` [2][8], `turn` flips with every call.
template <int TPR>
__device__ __forceinline__ float ring_sum(float v, float* buf, int& turn, int group) {
  v = lanes_sum<(TPR < 32 ? TPR : 32)>(v);
  if constexpr (TPR > 32) {
    float* b = buf + (group * 2 + turn) * 8;
    if ((threadIdx.x & 31) == 0) b[(threadIdx.x >> 5) & 7] = v;
    named_barrier(group + 1, kGroupThreads);
    v = 0.0f;
#pragma unroll
    for (int w = 0; w < 8; ++w) v += b[w];
    turn ^= 1;
  }
  return v;
}

// Two sums at once: one barrier.  `buf` [2][16].
template <int TPR>
__device__ __forceinline__ void ring_sums(float& u, float& v, float* buf, int& turn, int group) {
  u = lanes_sum<(TPR < 32 ? TPR : 32)>(u);
  v = lanes_sum<(TPR < 32 ? TPR : 32)>(v);
  if constexpr (TPR > 32) {
    float2* b = reinterpret_cast<float2*>(buf) + (group * 2 + turn) * 8;
    if ((threadIdx.x & 31) == 0) b[(threadIdx.x >> 5) & 7] = make_float2(u, v);
    named_barrier(group + 1, kGroupThreads);
    u = v = 0.0f;
#pragma unroll
    for (int w = 0; w < 8; ++w) {
      const float2 q = b[w];
      u += q.x;
      v += q.y;
    }
    turn ^= 1;
  }
}

__device__ __forceinline__ void ring_begin(const RingArgs& a, uint32_t full, uint32_t empty) {
  if (threadIdx.x == 0) {
    for (int s = 0; s < a.stages; ++s) {
      for (int g = 0; g < kRingGroups; ++g) tc::mbar_init(ring_full(full, g, s), 1);
      tc::mbar_init(empty + 8 * s, kGroupThreads / 32);
    }
    tc::fence_barrier_init();
  }
  __syncthreads();
  pdl_wait();
  pdl_trigger();
}

__device__ __forceinline__ void consumers_sync() { named_barrier(3, kRingGroups * kGroupThreads); }

template <int DT, int E, int V, int TPR>
__global__ void __launch_bounds__(kRingThreads, 1)
ln_forward_ring_kernel(const __grid_constant__ RingArgs a, const float* __restrict__ gamma, const float* __restrict__ beta, float eps,
                       void* __restrict__ y, float* __restrict__ stats) {
  extern __shared__ __align__(128) unsigned char ring[];
  __shared__ __align__(8) unsigned long long bars[(kRingGroups + 1) * kMaxRing];
  __shared__ float buf[kRingGroups * 2 * 8];
  constexpr int kRows = kGroupThreads / TPR;     // rows of a group at a time
  const uint32_t full = tc::smem_u32(bars), empty = full + 8 * kRingGroups * kMaxRing;
  ring_begin(a, full, empty);
  if (threadIdx.x >= kRingGroups * kGroupThreads) {
    ring_produce(a, ring, full, empty);
    return;
  }
  float* s_gamma = reinterpret_cast<float*>(ring + a.params);
  float* s_beta = s_gamma + V * TPR * E;
  fill_params<E, TPR>(kRingGroups * kGroupThreads, s_gamma, gamma, 1.0f, a.channels);
  fill_params<E, TPR>(kRingGroups * kGroupThreads, s_beta, beta, 0.0f, a.channels);
  consumers_sync();
  const int group = threadIdx.x / kGroupThreads;
  const int l = static_cast<int>(threadIdx.x) % TPR, sub = static_cast<int>(threadIdx.x) % kGroupThreads / TPR;
  const float inv_c = 1.0f / static_cast<float>(a.channels);
  int turn = 0, i = 0;
    uint32_t phases = 0;                         // of the group's barriers, a bit per stage
  for (long long chunk = blockIdx.x; chunk < a.chunks; chunk += gridDim.x, ++i) {
    if (i % kRingGroups != group) continue;
    const int s = i % a.stages;
    const long long row0 = chunk * a.chunk_rows;
    const bool there = tc::mbar_wait_suspend(ring_full(full, group, s), (phases >> s) & 1);
    phases ^= 1u << s;
    const unsigned char* x = ring + s * a.stage_bytes + (E == 1 ? ring_shift(a, 0, row0) : 0);
    const int here = static_cast<int>(a.rows - row0 < a.chunk_rows ? a.rows - row0 : a.chunk_rows);
    for (int first = 0; first < here; first += kRows) {
      const int k = first + sub;
      const bool on = k < here;
      float f[V][E], sum = 0.0f, q = 0.0f;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const int c = (v * TPR + l) * E;
        if (on && c < a.channels) load_elems<DT, E>(x, k * a.channels + c, f[v]);
        else {
#pragma unroll
          for (int e = 0; e < E; ++e) f[v][e] = 0.0f;
        }
#pragma unroll
        for (int e = 0; e < E; ++e) sum += f[v][e];
      }
      const float mean = ring_sum<TPR>(sum, buf, turn, group) * inv_c;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        if ((v * TPR + l) * E < a.channels) {
#pragma unroll
          for (int e = 0; e < E; ++e) {
            f[v][e] -= mean;
            q += f[v][e] * f[v][e];
          }
        }
      }
      q = ring_sum<TPR>(q, buf, turn, group);
      const float r = there ? rsqrtf(q * inv_c + eps) : __int_as_float(0x7FC00000);   // a copy that never came shows as NaN
      if (on) {
        const long long row = row0 + k;
        if (stats && l == 0) {
          stats[row] = mean;
          stats[a.rows + row] = r;
        }
#pragma unroll
        for (int v = 0; v < V; ++v) {
          const int c = (v * TPR + l) * E;
          if (c < a.channels) {
            float w[E], b[E];
            load_params<E, TPR>(s_gamma, v, l, w);
            load_params<E, TPR>(s_beta, v, l, b);
#pragma unroll
            for (int e = 0; e < E; ++e) f[v][e] = fmaf(f[v][e] * r, w[e], b[e]);
            store_elems<DT, E>(y, row * a.channels + c, f[v]);
          }
        }
      }
    }
    ring_release(empty + 8 * s);
  }
}

// The columns' sums stay in registers over all chunks of the CTA; x and dy are read twice from shared memory.  At the end a CTA
// leaves one row of partial sums per array, partial[cta][0: dgamma, 1: dbeta][channels].
template <int XDT, int GDT, int E, int V, int TPR>
__global__ void __launch_bounds__(kRingThreads, 1)
ln_backward_ring_kernel(const __grid_constant__ RingArgs a, const float* __restrict__ gamma, const float* __restrict__ stats,
                        void* __restrict__ dx, float* __restrict__ partial) {
  extern __shared__ __align__(128) unsigned char ring[];
  __shared__ __align__(8) unsigned long long bars[(kRingGroups + 1) * kMaxRing];
  __shared__ __align__(8) float buf[kRingGroups * 2 * 16];
  constexpr int kRows = kGroupThreads / TPR, kWidth = V * TPR * E;
  const uint32_t full = tc::smem_u32(bars), empty = full + 8 * kRingGroups * kMaxRing;
  ring_begin(a, full, empty);
  const bool producer = threadIdx.x >= kRingGroups * kGroupThreads;
  float dg[V][E], db[V][E];
#pragma unroll
  for (int v = 0; v < V; ++v)
#pragma unroll
    for (int e = 0; e < E; ++e) dg[v][e] = db[v][e] = 0.0f;
  const int group = threadIdx.x / kGroupThreads;
  const int l = static_cast<int>(threadIdx.x) % TPR, sub = static_cast<int>(threadIdx.x) % kGroupThreads / TPR;
  if (producer) {
    ring_produce(a, ring, full, empty);
  } else {
    float* s_gamma = reinterpret_cast<float*>(ring + a.params);
    fill_params<E, TPR>(kRingGroups * kGroupThreads, s_gamma, gamma, 1.0f, a.channels);
    consumers_sync();
    const float inv_c = 1.0f / static_cast<float>(a.channels);
    int turn = 0, i = 0;
    uint32_t phases = 0;                         // of the group's barriers, a bit per stage
    for (long long chunk = blockIdx.x; chunk < a.chunks; chunk += gridDim.x, ++i) {
      if (i % kRingGroups != group) continue;
      const int s = i % a.stages;
      const long long row0 = chunk * a.chunk_rows;
      const int here = static_cast<int>(a.rows - row0 < a.chunk_rows ? a.rows - row0 : a.chunk_rows);
      // a row's statistics are asked for one turn ahead (the first: while the chunk is on its way)
      float next_mean = sub < here ? __ldg(stats + row0 + sub) : 0.0f, next_r = sub < here ? __ldg(stats + a.rows + row0 + sub) : 0.0f;
      const bool there = tc::mbar_wait_suspend(ring_full(full, group, s), (phases >> s) & 1);
      phases ^= 1u << s;
      const unsigned char* stage = ring + s * a.stage_bytes;
      const unsigned char* x = stage + (E == 1 ? ring_shift(a, 0, row0) : 0);
      const unsigned char* dy = stage + a.at[1] + (E == 1 ? ring_shift(a, 1, row0) : 0);
      const unsigned char* res = stage + a.at[2] + (E == 1 ? ring_shift(a, 2, row0) : 0);
      for (int first = 0; first < here; first += kRows) {
        const int k = first + sub;
        const bool on = k < here;
        const float mean = next_mean, r = there ? next_r : __int_as_float(0x7FC00000);   // (a copy that never came shows as NaN)
        if (k + kRows < here) {
          next_mean = __ldg(stats + row0 + k + kRows);
          next_r = __ldg(stats + a.rows + row0 + k + kRows);
        }
        float c1 = 0.0f, c2 = 0.0f;
        if (on) {
#pragma unroll
          for (int v = 0; v < V; ++v) {
            const int c = (v * TPR + l) * E;
            if (c < a.channels) {
              float xh[E], g[E], w[E];
              load_elems<XDT, E>(x, k * a.channels + c, xh);
              load_elems<GDT, E>(dy, k * a.channels + c, g);
              load_params<E, TPR>(s_gamma, v, l, w);
#pragma unroll
              for (int e = 0; e < E; ++e) {
                xh[e] = (xh[e] - mean) * r;
                dg[v][e] += g[e] * xh[e];
                db[v][e] += g[e];
                g[e] *= w[e];
                c1 += g[e];
                c2 += g[e] * xh[e];
              }
            }
          }
        }
        ring_sums<TPR>(c1, c2, buf, turn, group);
        c1 *= inv_c;
        c2 *= inv_c;
        if (on && dx) {
          const long long row = row0 + k;
#pragma unroll
          for (int v = 0; v < V; ++v) {
            const int c = (v * TPR + l) * E;
            if (c < a.channels) {
              float xh[E], g[E], w[E];
              load_elems<XDT, E>(x, k * a.channels + c, xh);
              load_elems<GDT, E>(dy, k * a.channels + c, g);
              load_params<E, TPR>(s_gamma, v, l, w);
#pragma unroll
              for (int e = 0; e < E; ++e) g[e] = r * (g[e] * w[e] - c1 - (xh[e] - mean) * r * c2);
              if (a.n_src > 2) {
                float q[E];
                load_elems<GDT, E>(res, k * a.channels + c, q);
#pragma unroll
                for (int e = 0; e < E; ++e) g[e] += q[e];
              }
              store_elems<GDT, E>(dx, row * a.channels + c, g);
            }
          }
        }
      }
      ring_release(empty + 8 * s);
    }
  }
  if (!partial) return;
  // the rows' shares of each column, added in order in the place of the ring
  float* sums = reinterpret_cast<float*>(ring);
  float* out = partial + static_cast<long long>(blockIdx.x) * 2 * a.channels;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    __syncthreads();
    if (!producer) {
#pragma unroll
      for (int v = 0; v < V; ++v)
#pragma unroll
        for (int e = 0; e < E; ++e)
          sums[(group * kRows + sub) * kWidth + (v * TPR + l) * E + e] = k ? db[v][e] : dg[v][e];
    }
    __syncthreads();
    for (int c = threadIdx.x; c < a.channels; c += kRingThreads) {
      float t = 0.0f;
#pragma unroll 8
      for (int j = 0; j < kRingGroups * kRows; ++j) t += sums[j * kWidth + c];
      out[k * a.channels + c] = t;
    }
  }
}

bool whole_vectors(int channels, int elems) { return channels % elems == 0; }

template <int DT, int E, int V, int TPR>
void forward_as(const void* x, long long rows, int channels, const float* gamma, const float* beta, float eps, void* y,
                float* stats, cudaStream_t stream) {
  constexpr int kRows = TPR > 32 ? 1 : kLnThreads / TPR;
  // (short fp32 rows are better off without: 65536 x 64 7.4 us against 8.2, 12608 x 384 8.4 against 8.7; 4096 x 1024 9.8 against 8.6)
  if constexpr (E > 1 && TPR <= 32 && (DT == 1 || V >= 6)) {
    const long long most = static_cast<long long>(rows_ctas<DT, V, TPR>()) * sm_count();
    if (rows > most * kRows) {
      launch_kernel(ln_forward_rows_kernel<DT, V, TPR>, dim3(static_cast<unsigned>(most)), dim3(kLnThreads), 0, stream, true, x, rows,
                    channels, gamma, beta, eps, y, stats);
      return;
    }
  }
  launch_kernel(ln_forward_kernel<DT, E, V, TPR>, dim3(static_cast<unsigned>((rows + kRows - 1) / kRows)),
                dim3(TPR > 32 ? TPR : kLnThreads), 0, stream, true, x, rows, channels, gamma, beta, eps, y, stats);
}

// Rows that no ring holds.  Returns how many rows of partial sums there are.
template <int XDT, int GDT>
int backward_long(const void* x, const void* dy, long long rows, int channels, const float* gamma, const float* stats,
                  const void* residual, void* dx, float* partial, cudaStream_t stream) {
  int slabs = 0;
  if (partial) {                                 // (before dx, which may take the place of dy)
    const long long per = (rows + kLnPartials - 1) / kLnPartials;
    slabs = static_cast<int>((rows + per - 1) / per);
    launch_kernel(ln_columns_kernel<XDT, GDT>, dim3((channels + kLnThreads - 1) / kLnThreads, slabs), dim3(kLnThreads), 0, stream,
                  true, x, dy, rows, channels, stats, per, partial);
    note_launches(1);
  }
  if (dx) {
    launch_kernel(ln_backward_long_kernel<XDT, GDT>, dim3(static_cast<unsigned>(rows)), dim3(1024), 0, stream, true, x, dy, rows,
                  channels, gamma, stats, residual, dx);
    note_launches(1);
  }
  return slabs;
}

// The ring of a call, or false where not even two chunks of one row fit.  `parallel`: rows that a group takes at a time;
// `arrays`: what the call may read at most, by which the chunks go (so that the columns' sums are the same whether dx and the
// residual's gradient are wanted or not); `param_bytes`: of the parameters behind the ring.
bool plan_ring(RingArgs* a, int parallel, int arrays, int param_bytes) {
  long long bytes = 0;
  for (int i = 0; i < arrays; ++i) bytes += static_cast<long long>(a->channels) * a->elem[i];
  const long long room = kSmemBytes - param_bytes;
  // whole turns of the group while three stages of them fit; more rows where rows are short and every CTA still has work
  long long rows = parallel;
  if (rows * bytes > room / 3 - 512) rows = (room / 3 - 512) / bytes > 1 ? (room / 3 - 512) / bytes : 1;
  while (2 * rows * bytes <= 24 * 1024 && 4 * rows * sm_count() <= a->rows) rows *= 2;
  long long stage = 0, most = 0;
  for (int i = 0; i < arrays; ++i) {
    a->at[i] = static_cast<int>(most);
    most += (rows * a->channels * a->elem[i] + 16 + 127) & ~127LL;
    if (most > room / 2) return false;
    if (i < a->n_src) stage = most;
  }
  a->chunk_rows = static_cast<int>(rows);
  a->stage_bytes = static_cast<int>(stage);
  a->stages = static_cast<int>(room / stage);
  if (a->stages > kMaxRing) a->stages = kMaxRing;
  a->params = a->stages * a->stage_bytes;
  a->chunks = (a->rows + rows - 1) / rows;
  return true;
}

template <int DT, int E, int V, int TPR>
bool forward_ring_as(const void* x, long long rows, int channels, const float* gamma, const float* beta, float eps, void* y,
                     float* stats, cudaStream_t stream) {
  RingArgs a = {};
  a.src[0] = x; a.elem[0] = DT ? 2 : 4; a.n_src = 1;
  a.rows = rows; a.channels = channels;
  constexpr int kParams = 2 * V * TPR * E * 4;
  if (!plan_ring(&a, kGroupThreads / TPR, 1, kParams)) return false;
  const auto kernel = ln_forward_ring_kernel<DT, E, V, TPR>;
  const int smem = a.params + kParams;
  if (allow_dynamic_smem(reinterpret_cast<const void*>(kernel), smem) != cudaSuccess) return false;
  const int ctas = static_cast<int>(a.chunks < sm_count() ? a.chunks : sm_count());
  launch_kernel(kernel, dim3(ctas), dim3(kRingThreads), smem, stream, true, a, gamma, beta, eps, y, stats);
  return true;
}

template <int XDT, int GDT, int E, int V, int TPR>
int backward_ring_as(const void* x, const void* dy, long long rows, int channels, const float* gamma, const float* stats,
                     const void* residual, void* dx, float* partial, cudaStream_t stream) {
  RingArgs a = {};
  a.src[0] = x; a.src[1] = dy; a.src[2] = residual;
  a.elem[0] = XDT ? 2 : 4; a.elem[1] = a.elem[2] = GDT ? 2 : 4;
  a.n_src = residual && dx ? 3 : 2;
  a.rows = rows; a.channels = channels;
  constexpr int kParams = V * TPR * E * 4;
  if (!plan_ring(&a, kGroupThreads / TPR, 3, kParams)) return 0;
  const auto kernel = ln_backward_ring_kernel<XDT, GDT, E, V, TPR>;
  int smem = a.params + kParams;
  const int sums = kRingGroups * (kGroupThreads / TPR) * V * TPR * E * 4;
  if (smem < sums) smem = sums;
  if (allow_dynamic_smem(reinterpret_cast<const void*>(kernel), smem) != cudaSuccess) return 0;
  const int ctas = static_cast<int>(a.chunks < sm_count() ? a.chunks : sm_count());
  launch_kernel(kernel, dim3(ctas), dim3(kRingThreads), smem, stream, true, a, gamma, stats, dx, partial);
  note_launches(1);
  return ctas;
}

// E: elements of a vector, 1 where rows start at no 16-byte boundary; N elements per thread.  Whole vectors need no ring
// (12608 x 768 bf16 13.0 us with one, 8.2 without), nor do odd widths of fp32, where a warp reads 128 bytes an element each (3000 x
// 2047 15.7 us against 18.7, 12608 x 767 18.8 against 26.3); those of bf16 go through it, which reads them in wide pieces (3000 x
// 2047 16.7 us against 32.4).
template <int DT, int E>
void forward_of(const void* x, long long rows, int channels, const float* gamma, const float* beta, float eps, void* y,
                float* stats, cudaStream_t stream) {
  if constexpr (E > 1) {
#define SURGEON_LN(TPR, N)                                                                                \
  if (channels <= TPR * N) return forward_as<DT, E, N / E, TPR>(x, rows, channels, gamma, beta, eps, y, stats, stream)
    SURGEON_LN(8, 8);
    SURGEON_LN(16, 8);
    SURGEON_LN(32, 8);
    SURGEON_LN(32, 16);
    SURGEON_LN(32, 24);
    SURGEON_LN(32, 32);
    SURGEON_LN(128, 16);
    SURGEON_LN(256, 16);
    SURGEON_LN(512, 16);
#undef SURGEON_LN
  } else if constexpr (DT == 0) {
#define SURGEON_LN(TPR, N)                                                                                \
  if (channels <= TPR * N) return forward_as<DT, 1, N, TPR>(x, rows, channels, gamma, beta, eps, y, stats, stream)
    SURGEON_LN(16, 4);
    SURGEON_LN(16, 8);
    SURGEON_LN(32, 8);
    SURGEON_LN(32, 12);
    SURGEON_LN(128, 6);
    SURGEON_LN(256, 4);
    SURGEON_LN(256, 8);
    SURGEON_LN(512, 8);
    SURGEON_LN(512, 12);
    if (rows > 2 * sm_count()) SURGEON_LN(512, 16);              // (2000 x 7001 34.4 us, 51.7 by 1024 threads; 100 x 7001 10.4 against 6.9)
    SURGEON_LN(1024, 8);
#undef SURGEON_LN
  } else {
#define SURGEON_LN(TPR, N)                                                                                            \
  if (channels <= TPR * N && forward_ring_as<DT, 1, N, TPR>(x, rows, channels, gamma, beta, eps, y, stats, stream)) return
    SURGEON_LN(8, 8);
    SURGEON_LN(16, 8);
    SURGEON_LN(32, 8);
    SURGEON_LN(32, 16);
    SURGEON_LN(32, 32);
    SURGEON_LN(256, 8);
    SURGEON_LN(256, 16);
    SURGEON_LN(256, 32);
#undef SURGEON_LN
  }
  launch_kernel(ln_forward_long_kernel<DT>, dim3(static_cast<unsigned>(rows)), dim3(1024), 0, stream, true, x, rows, channels,
                gamma, beta, eps, y, stats);
}

// Returns how many rows of partial sums there are.  A warp to a row, but for a few long ones, which 256 threads share: 197 x
// 1021 fp32 8.1 us against 11.9, 2000 x 1024 12.8 against 18.0; 4000 x 768 17.9 against 16.8, 1024 x 512 8.4 against 7.0.
template <int XDT, int GDT, int E>
int backward_of(const void* x, const void* dy, long long rows, int channels, const float* gamma, const float* stats,
                const void* residual, void* dx, float* partial, cudaStream_t stream) {
  int n = 0;
  const bool shared = channels > 512 && rows <= 2048;
#define SURGEON_LN(TPR, N)                                                                                                         \
  if (n == 0 && channels <= TPR * N && (TPR == 256 || !shared))                                                                                               \
    n = backward_ring_as<XDT, GDT, E, N / E, TPR>(x, dy, rows, channels, gamma, stats, residual, dx, partial, stream)
  SURGEON_LN(8, 8);
  SURGEON_LN(16, 8);
  SURGEON_LN(32, 8);
  SURGEON_LN(32, 16);
  SURGEON_LN(32, 24);
  SURGEON_LN(32, 32);
  SURGEON_LN(256, 8);
  SURGEON_LN(256, 16);
  SURGEON_LN(256, 32);
#undef SURGEON_LN
  return n ? n : backward_long<XDT, GDT>(x, dy, rows, channels, gamma, stats, residual, dx, partial, stream);
}

}  // namespace

cudaError_t launch_layer_norm(const void* x, long long rows, int channels, int dt, const float* gamma, const float* beta,
                              float eps, void* y, float* stats, cudaStream_t stream) {
  if (rows == 0) return cudaSuccess;
  if (dt == 0) {
    if (whole_vectors(channels, 4)) forward_of<0, 4>(x, rows, channels, gamma, beta, eps, y, stats, stream);
    else forward_of<0, 1>(x, rows, channels, gamma, beta, eps, y, stats, stream);
  } else {
    if (whole_vectors(channels, 8)) forward_of<1, 8>(x, rows, channels, gamma, beta, eps, y, stats, stream);
    else forward_of<1, 1>(x, rows, channels, gamma, beta, eps, y, stats, stream);
  }
  note_launches(1);
  return cudaGetLastError();
}

size_t layer_norm_grad_workspace(long long rows, int channels) {
  const long long n = rows < kLnPartials ? rows : kLnPartials;
  return static_cast<size_t>(n) * 2 * channels * sizeof(float);
}

cudaError_t launch_layer_norm_grad(const void* x, const void* dy, long long rows, int channels, int dt, int grad_dt,
                                   const float* gamma, const float* stats, const void* residual, void* dx, float* dgamma,
                                   float* dbeta, int accumulate, void* workspace, cudaStream_t stream) {
  float* partial = dgamma || dbeta ? static_cast<float*>(workspace) : nullptr;
  int n = 0;
  if (rows > 0) {
#define SURGEON_LN(XDT, GDT, E) n = backward_of<XDT, GDT, E>(x, dy, rows, channels, gamma, stats, residual, dx, partial, stream)
    if (dt == 0) {
      if (whole_vectors(channels, 4)) SURGEON_LN(0, 0, 4);
      else SURGEON_LN(0, 0, 1);
    } else if (grad_dt == 0) {
      if (whole_vectors(channels, 8)) SURGEON_LN(1, 0, 4);
      else SURGEON_LN(1, 0, 1);
    } else {
      if (whole_vectors(channels, 8)) SURGEON_LN(1, 1, 8);
      else SURGEON_LN(1, 1, 1);
    }
#undef SURGEON_LN
  }
  if (dgamma || dbeta) {                         // (of no rows too, which need no scratch)
    launch_kernel(ln_final_kernel, dim3((channels + 31) / 32, 2), dim3(kFinalThreads), 0, stream, true, partial, n, channels, dgamma,
                  dbeta, accumulate);
    note_launches(1);
  }
  return cudaGetLastError();
}

}  // namespace surgeon
