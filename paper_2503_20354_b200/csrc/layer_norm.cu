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

// A CTA takes every gridDim.x-th group of rows and keeps its columns' sums in registers; at the end it leaves one row
// of partial sums per array, partial[cta][0: dgamma, 1: dbeta][channels].
template <int XDT, int GDT, int E, int V, int TPR>
__global__ void __launch_bounds__(TPR > 32 ? TPR : kLnThreads)
ln_backward_kernel(const void* __restrict__ x, const void* __restrict__ dy, long long rows, int channels,
                   const float* __restrict__ gamma, const float* __restrict__ stats,
                   const void* __restrict__ residual, void* __restrict__ dx, float* __restrict__ partial) {
  constexpr int kThreads = TPR > 32 ? TPR : kLnThreads;
  constexpr int kRows = kThreads / TPR;
  __shared__ float buf[4][TPR > 32 ? TPR / 32 : 1];
  __shared__ float sums[kRows > 1 ? kThreads * V * E : 1];
  pdl_wait();
  pdl_trigger();
  const int l = static_cast<int>(threadIdx.x) % TPR, group = static_cast<int>(threadIdx.x) / TPR;
  const float inv_c = 1.0f / static_cast<float>(channels);
  float dg[V][E], db[V][E];
#pragma unroll
  for (int v = 0; v < V; ++v)
#pragma unroll
    for (int e = 0; e < E; ++e) dg[v][e] = db[v][e] = 0.0f;
  int turn = 0;
  for (long long first = static_cast<long long>(blockIdx.x) * kRows; first < rows;
       first += static_cast<long long>(gridDim.x) * kRows) {
    const long long row = first + group;
    const bool on = row < rows;
    const float mean = on ? stats[row] : 0.0f, r = on ? stats[rows + row] : 0.0f;
    float xh[V][E], g[V][E];
    float c1 = 0.0f, c2 = 0.0f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int c = (v * TPR + l) * E;
      if (on && c < channels) {
        load_elems<XDT, E>(x, row * channels + c, xh[v]);
        load_elems<GDT, E>(dy, row * channels + c, g[v]);
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e) xh[v][e] = mean, g[v][e] = 0.0f;
      }
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int c = (v * TPR + l) * E;
      float w[E];
#pragma unroll
      for (int e = 0; e < E; ++e) w[e] = 1.0f;
      if (gamma && c < channels) load_elems<0, E>(gamma, c, w);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        xh[v][e] = (xh[v][e] - mean) * r;
        dg[v][e] += g[v][e] * xh[v][e];
        db[v][e] += g[v][e];
        g[v][e] *= w[e];
        c1 += g[v][e];
        c2 += g[v][e] * xh[v][e];
      }
    }
    c1 = row_sum<TPR>(c1, buf[turn]) * inv_c;
    c2 = row_sum<TPR>(c2, buf[turn + 1]) * inv_c;
    turn ^= 2;
    if (on && dx) {
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const int c = (v * TPR + l) * E;
        if (c < channels) {
          float o[E];
#pragma unroll
          for (int e = 0; e < E; ++e) o[e] = r * (g[v][e] - c1 - xh[v][e] * c2);
          if (residual) {
            float k[E];
            load_elems<GDT, E>(residual, row * channels + c, k);
#pragma unroll
            for (int e = 0; e < E; ++e) o[e] += k[e];
          }
          store_elems<GDT, E>(dx, row * channels + c, o);
        }
      }
    }
  }
  if (!partial) return;
  float* out = partial + static_cast<long long>(blockIdx.x) * 2 * channels;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    if constexpr (kRows == 1) {
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const int c = (v * TPR + l) * E;
        if (c < channels) {
#pragma unroll
          for (int e = 0; e < E; ++e) out[k * channels + c + e] = k ? db[v][e] : dg[v][e];
        }
      }
    } else {
      __syncthreads();
#pragma unroll
      for (int v = 0; v < V; ++v)
#pragma unroll
        for (int e = 0; e < E; ++e) sums[group * (V * TPR * E) + (v * TPR + l) * E + e] = k ? db[v][e] : dg[v][e];
      __syncthreads();
      for (int c = threadIdx.x; c < channels; c += kThreads) {
        float t = 0.0f;
#pragma unroll
        for (int i = 0; i < kRows; ++i) t += sums[i * (V * TPR * E) + c];
        out[k * channels + c] = t;
      }
    }
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

// The partial sums' rows, added in order: 32 columns per CTA, eight slices of the rows.
__global__ void __launch_bounds__(kLnThreads)
ln_final_kernel(const float* __restrict__ partial, int n_partials, int channels, float* __restrict__ dgamma,
                float* __restrict__ dbeta, int accumulate) {
  __shared__ float part[kLnThreads / 32][33];
  pdl_wait();
  pdl_trigger();
  const int k = blockIdx.y;
  float* out = k ? dbeta : dgamma;
  if (!out) return;
  const int c = blockIdx.x * 32 + (threadIdx.x & 31), slice = threadIdx.x >> 5;
  float t = 0.0f;
  if (c < channels) {
#pragma unroll 8
    for (int i = slice; i < n_partials; i += kLnThreads / 32) t += partial[(static_cast<long long>(i) * 2 + k) * channels + c];
  }
  part[slice][threadIdx.x & 31] = t;
  __syncthreads();
  if (slice == 0 && c < channels) {
    t = 0.0f;
#pragma unroll
    for (int i = 0; i < kLnThreads / 32; ++i) t += part[i][threadIdx.x];
    out[c] = accumulate ? out[c] + t : t;
  }
}

bool whole_vectors(int channels, int elems) { return channels % elems == 0; }

template <int DT, int E, int V, int TPR>
void forward_as(const void* x, long long rows, int channels, const float* gamma, const float* beta, float eps, void* y,
                float* stats, cudaStream_t stream) {
  constexpr int kRows = TPR > 32 ? 1 : kLnThreads / TPR;
  launch_kernel(ln_forward_kernel<DT, E, V, TPR>, dim3(static_cast<unsigned>((rows + kRows - 1) / kRows)),
                dim3(TPR > 32 ? TPR : kLnThreads), 0, stream, true, x, rows, channels, gamma, beta, eps, y, stats);
}

// E: elements of a vector; N = V * E elements per thread.
template <int DT, int E>
void forward_of(const void* x, long long rows, int channels, const float* gamma, const float* beta, float eps, void* y,
                float* stats, cudaStream_t stream) {
#define SURGEON_LN(TPR, N)                                                                                \
  if (channels <= TPR * N) return forward_as<DT, E, N / E, TPR>(x, rows, channels, gamma, beta, eps, y, stats, stream)
  SURGEON_LN(8, 8);
  SURGEON_LN(32, 8);
  SURGEON_LN(32, 16);
  SURGEON_LN(32, 24);
  SURGEON_LN(32, 32);
  SURGEON_LN(128, 16);
  SURGEON_LN(256, 16);
  SURGEON_LN(512, 16);
#undef SURGEON_LN
  launch_kernel(ln_forward_long_kernel<DT>, dim3(static_cast<unsigned>(rows)), dim3(1024), 0, stream, true, x, rows, channels,
                gamma, beta, eps, y, stats);
}

template <int XDT, int GDT, int E, int V, int TPR>
int backward_as(const void* x, const void* dy, long long rows, int channels, const float* gamma, const float* stats,
                const void* residual, void* dx, float* partial, cudaStream_t stream) {
  constexpr int kRows = TPR > 32 ? 1 : kLnThreads / TPR;
  const long long groups = (rows + kRows - 1) / kRows;
  const int ctas = static_cast<int>(groups < kLnPartials ? groups : kLnPartials);
  launch_kernel(ln_backward_kernel<XDT, GDT, E, V, TPR>, dim3(ctas), dim3(TPR > 32 ? TPR : kLnThreads), 0, stream, true, x, dy,
                rows, channels, gamma, stats, residual, dx, partial);
  note_launches(1);
  return ctas;
}

// Returns how many rows of partial sums there are.
template <int XDT, int GDT, int E>
int backward_of(const void* x, const void* dy, long long rows, int channels, const float* gamma, const float* stats,
                const void* residual, void* dx, float* partial, cudaStream_t stream) {
#define SURGEON_LN(TPR, N)                                                                                         \
  if (channels <= TPR * N)                                                                                         \
    return backward_as<XDT, GDT, E, N / E, TPR>(x, dy, rows, channels, gamma, stats, residual, dx, partial, stream)
  SURGEON_LN(8, 8);
  SURGEON_LN(32, 8);
  SURGEON_LN(32, 16);
  SURGEON_LN(32, 24);
  SURGEON_LN(64, 16);
  SURGEON_LN(128, 16);
  SURGEON_LN(256, 16);
  SURGEON_LN(512, 16);
#undef SURGEON_LN
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
      if (whole_vectors(channels, 8)) SURGEON_LN(1, 0, 8);
      else SURGEON_LN(1, 0, 1);
    } else {
      if (whole_vectors(channels, 8)) SURGEON_LN(1, 1, 8);
      else SURGEON_LN(1, 1, 1);
    }
#undef SURGEON_LN
  }
  if (partial) {
    launch_kernel(ln_final_kernel, dim3((channels + 31) / 32, 2), dim3(kLnThreads), 0, stream, true, partial, n, channels, dgamma,
                  dbeta, accumulate);
    note_launches(1);
  }
  return cudaGetLastError();
}

}  // namespace surgeon
