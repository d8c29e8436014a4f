// Group norm with an activation over channels-last tensors, and its backward pass.
//
//   z = (x - mean) r gamma + beta;  y = act(z);  mean, r = 1 / sqrt(var + eps) of a group: all positions of an image, C / G channels
//   dz = dy act'(z), z made again;  A_c = sum dz, B_c = sum dz xh over an image's positions;  dbeta = sum A, dgamma = sum B over images
//   dx = r (gamma dz - c1 - xh c2),  c1 = sum_c gamma A / m,  c2 = sum_c gamma B / m,  m = positions * C / G
//
// z is computed with the same roundings in both directions, a rounding per operation, so that ReLU's slope is that of the sign the
// forward pass saw.
//
// Three steps: sums of a chunk of positions per channel, sums of the chunks per group, the outputs.  In the first and the last a
// thread keeps its vector of channels, so that their parameters stay in registers, and walks down the positions.
// The last step takes the chunks in the opposite order: what the first read last is still in L2.
#include "linear.cuh"

namespace surgeon {

namespace {

constexpr int kActSilu = 3;
constexpr int kMaxThreads = 256;                 // vectors of channels a CTA takes at once
constexpr int kUnroll = 4;                       // rows on their way

template <int ACT>
__device__ __forceinline__ float gn_activate(float z) {
  if constexpr (ACT == kActSilu) {
    float e, s;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(z * -1.4426950408889634f));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(s) : "f"(1.0f + e));
    return fmaxf(z, -3.0e38f) * s;               // (0 at -infinity; s is NaN for a NaN)
  } else {
    return activate<ACT>(z);
  }
}
template <int ACT>
__device__ __forceinline__ float gn_slope(float z) {
  if constexpr (ACT == kActSilu) {
    float e, s;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(z * -1.4426950408889634f));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(s) : "f"(1.0f + e));
    return fmaf(fminf(fmaxf(z, -3.0e38f), 3.0e38f) * s, 1.0f - s, s);
  } else {
    return slope<ACT>(z);
  }
}

struct Geometry {
  int positions, channels, groups, per_group;    // per_group: channels of a group
  int vectors, cols, lanes;                      // vectors of a row; of them a CTA's; rows that a CTA takes at once
  int chunk, chunks;                             // positions of a chunk, chunks of an image
  long long image;                               // elements of an image
};

// xh and z of one element, a rounding per operation
__device__ __forceinline__ float normal(float x, float mean, float r) { return __fmul_rn(__fsub_rn(x, mean), r); }
__device__ __forceinline__ float affine(float xh, float gamma, float beta) { return __fadd_rn(__fmul_rn(xh, gamma), beta); }

template <int E>
struct Params {
  float mean[E], r[E], gamma[E], beta[E];
};
// The parameters of channels c, ..., c + E - 1 of image b.
template <int E>
__device__ __forceinline__ void load_params(Params<E>& p, const Geometry& g, int b, int c, const float* stats, int images, const float* gamma,
                                            const float* beta) {
#pragma unroll
  for (int i = 0; i < E; ++i) {
    const int at = b * g.groups + (c + i) / g.per_group;
    p.mean[i] = stats[at];
    p.r[i] = stats[images * g.groups + at];
    p.gamma[i] = gamma ? gamma[c + i] : 1.0f;
    p.beta[i] = beta ? beta[c + i] : 0.0f;
  }
}

// Rows of a chunk that lane `lane` takes: lane, lane + lanes, ...
__device__ __forceinline__ int rows_of(int rows, int lane, int lanes) { return rows > lane ? (rows - lane + lanes - 1) / lanes : 0; }

// What a thread of the first and the last step works on: a vector of channels and every lanes-th position of a chunk.
template <int E>
struct Place {
  int b, chunk, col, lane, v, mine, rows;
  long long at, step;
  bool on;
  __device__ __forceinline__ Place(const Geometry& g, int item) {
    col = threadIdx.x % g.cols;
    lane = threadIdx.x / g.cols;
    v = blockIdx.y * g.cols + col;
    chunk = item % g.chunks;
    b = item / g.chunks;
    const int first = chunk * g.chunk;
    rows = min(g.chunk, g.positions - first);
    on = lane < g.lanes && v < g.vectors;
    mine = on ? rows_of(rows, lane, g.lanes) : 0;
    at = b * g.image + static_cast<long long>(first + lane) * g.channels + static_cast<long long>(v) * E;
    step = static_cast<long long>(g.lanes) * g.channels;
  }
};

// ---- step 1, forward: mean and centred sum of squares of every channel of a chunk ----
// A thread sums x - s and (x - s)^2, s its first number of the channel.  What the difference of the n squares and their mean's loses is
// below n roundings of the result, wherever s lies.
template <int DT, int E>
__global__ void __launch_bounds__(kMaxThreads)
group_sums_kernel(const void* x, float2* partial, const Geometry g) {
  extern __shared__ float2 s_pairs[];            // [lanes - 1][E][cols]
  pdl_trigger();
  pdl_wait();
  const Place<E> p(g, blockIdx.x);
  float2 sum[E];
#pragma unroll
  for (int i = 0; i < E; ++i) sum[i] = make_float2(0.0f, 0.0f);
  if (p.mine > 0) {
    float shift[E];
    load_elems<DT, E>(x, p.at, shift);
    const auto add = [&](const float (&f)[E]) {
#pragma unroll
      for (int i = 0; i < E; ++i) {
        const float d = f[i] - shift[i];
        sum[i].x += d;
        sum[i].y = fmaf(d, d, sum[i].y);
      }
    };
    long long at = p.at;
    int t = 0;
    for (; t + kUnroll <= p.mine; t += kUnroll, at += kUnroll * p.step) {
      float f[kUnroll][E];
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) load_elems<DT, E>(x, at + u * p.step, f[u]);
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) add(f[u]);
    }
    for (; t < p.mine; ++t, at += p.step) {
      float f[E];
      load_elems<DT, E>(x, at, f);
      add(f);
    }
    const float inv = 1.0f / static_cast<float>(p.mine);
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const float m = sum[i].x * inv;
      sum[i] = make_float2(shift[i] + m, sum[i].y - sum[i].x * m);
    }
  }
  if (g.lanes > 1) {                             // (Chan, Golub and LeVeque's update, lane by lane)
    if (p.on && p.lane > 0)
#pragma unroll
      for (int i = 0; i < E; ++i) s_pairs[((p.lane - 1) * E + i) * g.cols + p.col] = sum[i];
    __syncthreads();
    if (p.on && p.lane == 0) {
      int before = p.mine;
      for (int l = 1; l < g.lanes; ++l) {
        const int k = rows_of(p.rows, l, g.lanes);
        if (k == 0) break;
        const float w = static_cast<float>(k) / static_cast<float>(before + k), n = static_cast<float>(before);
#pragma unroll
        for (int i = 0; i < E; ++i) {
          const float2 o = s_pairs[((l - 1) * E + i) * g.cols + p.col];
          const float d = o.x - sum[i].x;
          sum[i].x = fmaf(d, w, sum[i].x);
          sum[i].y += o.y + d * d * n * w;
        }
        before += k;
      }
    }
  }
  if (p.on && p.lane == 0) {
    float2* to = partial + (static_cast<long long>(p.b) * g.chunks + p.chunk) * g.channels + static_cast<long long>(p.v) * E;
#pragma unroll
    for (int i = 0; i < E; ++i) to[i] = sum[i];
  }
}

// Sum of a double over a CTA's threads in a fixed order, in every thread.
__device__ __forceinline__ double cta_sum(double v, double* buf) {
  v = lanes_sum<32>(v);
  __syncthreads();
  if (lane_id() == 0) buf[threadIdx.x >> 5] = v;
  __syncthreads();
  double t = 0.0;
  for (int i = 0; i < static_cast<int>(blockDim.x >> 5); ++i) t += buf[i];
  return t;
}

// ---- step 2, forward: a group's mean and r from the chunks', in double ----
__global__ void __launch_bounds__(256)
group_stats_kernel(const float2* partial, float* stats, int images, float eps, const Geometry g) {
  __shared__ double buf[8];
  pdl_trigger();
  pdl_wait();
  const int b = blockIdx.x / g.groups, group = blockIdx.x % g.groups;
  double s = 0.0, q = 0.0;
  const long long total = static_cast<long long>(g.chunks) * g.per_group;
  const float2* from = partial + static_cast<long long>(b) * g.chunks * g.channels + group * g.per_group;
  for (long long i = threadIdx.x; i < total; i += blockDim.x) {
    const int chunk = static_cast<int>(i / g.per_group), c = static_cast<int>(i % g.per_group);
    const float2 v = from[static_cast<long long>(chunk) * g.channels + c];
    const double n = min(g.chunk, g.positions - chunk * g.chunk), m = v.x;
    s += n * m;
    q += v.y + n * m * m;
  }
  s = cta_sum(s, buf);
  q = cta_sum(q, buf);
  if (threadIdx.x == 0) {
    const double n = static_cast<double>(g.positions) * g.per_group, mean = s / n;
    double var = q / n - mean * mean;
    if (var < 0.0) var = 0.0;                    // (a NaN stays one)
    stats[blockIdx.x] = static_cast<float>(mean);
    stats[images * g.groups + blockIdx.x] = static_cast<float>(1.0 / sqrt(var + eps));
  }
}

// ---- step 3, forward ----
template <int DT, int E, int ACT>
__global__ void __launch_bounds__(kMaxThreads)
group_apply_kernel(const void* x, void* y, const float* stats, int images, const float* gamma, const float* beta, const Geometry g) {
  pdl_trigger();
  pdl_wait();
  const Place<E> p(g, gridDim.x - 1 - blockIdx.x);
  if (p.mine == 0) return;
  Params<E> k;
  load_params<E>(k, g, p.b, p.v * E, stats, images, gamma, beta);
  const auto finish = [&](long long at, float (&f)[E]) {
#pragma unroll
    for (int i = 0; i < E; ++i) f[i] = gn_activate<ACT>(affine(normal(f[i], k.mean[i], k.r[i]), k.gamma[i], k.beta[i]));
    store_elems<DT, E>(y, at, f);
  };
  long long at = p.at;
  int t = 0;
  for (; t + kUnroll <= p.mine; t += kUnroll, at += kUnroll * p.step) {
    float f[kUnroll][E];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) load_elems<DT, E>(x, at + u * p.step, f[u]);
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) finish(at + u * p.step, f[u]);
  }
  for (; t < p.mine; ++t, at += p.step) {
    float f[E];
    load_elems<DT, E>(x, at, f);
    finish(at, f);
  }
}

// ---- step 1, backward: A and B of every channel of a chunk ----
template <int DT, int GDT, int E, int ACT>
__global__ void __launch_bounds__(kMaxThreads)
group_grad_sums_kernel(const void* x, const void* dy, float2* partial, const float* stats, int images, const float* gamma, const float* beta,
                       const Geometry g) {
  extern __shared__ float2 s_pairs[];
  pdl_trigger();
  pdl_wait();
  const Place<E> p(g, blockIdx.x);
  float2 sum[E];
#pragma unroll
  for (int i = 0; i < E; ++i) sum[i] = make_float2(0.0f, 0.0f);
  if (p.mine > 0) {
    Params<E> k;
    load_params<E>(k, g, p.b, p.v * E, stats, images, gamma, beta);
    const auto add = [&](const float (&f)[E], const float (&d)[E]) {
#pragma unroll
      for (int i = 0; i < E; ++i) {
        const float xh = normal(f[i], k.mean[i], k.r[i]);
        const float dz = ACT == kActNone ? d[i] : d[i] * gn_slope<ACT>(affine(xh, k.gamma[i], k.beta[i]));
        sum[i].x += dz;
        sum[i].y = fmaf(dz, xh, sum[i].y);
      }
    };
    long long at = p.at;
    int t = 0;
    for (; t + 2 <= p.mine; t += 2, at += 2 * p.step) {
      float f[2][E], d[2][E];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        load_elems<DT, E>(x, at + u * p.step, f[u]);
        load_elems<GDT, E>(dy, at + u * p.step, d[u]);
      }
#pragma unroll
      for (int u = 0; u < 2; ++u) add(f[u], d[u]);
    }
    if (t < p.mine) {
      float f[E], d[E];
      load_elems<DT, E>(x, at, f);
      load_elems<GDT, E>(dy, at, d);
      add(f, d);
    }
  }
  if (g.lanes > 1) {
    if (p.on && p.lane > 0)
#pragma unroll
      for (int i = 0; i < E; ++i) s_pairs[((p.lane - 1) * E + i) * g.cols + p.col] = sum[i];
    __syncthreads();
    if (p.on && p.lane == 0)
      for (int l = 1; l < g.lanes; ++l)
#pragma unroll
        for (int i = 0; i < E; ++i) {
          const float2 o = s_pairs[((l - 1) * E + i) * g.cols + p.col];
          sum[i].x += o.x;
          sum[i].y += o.y;
        }
  }
  if (p.on && p.lane == 0) {
    float2* to = partial + (static_cast<long long>(p.b) * g.chunks + p.chunk) * g.channels + static_cast<long long>(p.v) * E;
#pragma unroll
    for (int i = 0; i < E; ++i) to[i] = sum[i];
  }
}

// ---- step 2, backward: A and B of every channel of an image, c1 and c2 of every group ----
// `width` threads side by side on channels, 256 / width on the chunks.
__global__ void __launch_bounds__(256)
group_grad_terms_kernel(const float2* partial, double2* sums, float2* terms, const float* gamma, int width, const Geometry g) {
  __shared__ double2 buf[256];
  __shared__ double total[8];
  pdl_trigger();
  pdl_wait();
  const int b = blockIdx.x / g.groups, group = blockIdx.x % g.groups;
  const int col = threadIdx.x % width, row = threadIdx.x / width, rows = 256 / width;
  double c1 = 0.0, c2 = 0.0;
  for (int c0 = 0; c0 < g.per_group; c0 += width) {
    const int c = c0 + col, channel = group * g.per_group + c;
    double2 s = make_double2(0.0, 0.0);
    if (c < g.per_group)
      for (int i = row; i < g.chunks; i += rows) {
        const float2 v = partial[(static_cast<long long>(b) * g.chunks + i) * g.channels + channel];
        s.x += v.x;
        s.y += v.y;
      }
    __syncthreads();
    buf[threadIdx.x] = s;
    __syncthreads();
    if (row == 0 && c < g.per_group) {
      for (int i = 1; i < rows; ++i) {
        s.x += buf[i * width + col].x;
        s.y += buf[i * width + col].y;
      }
      sums[static_cast<long long>(b) * g.channels + channel] = s;
      const double w = gamma ? gamma[channel] : 1.0;
      c1 += w * s.x;
      c2 += w * s.y;
    }
  }
  c1 = cta_sum(c1, total);
  c2 = cta_sum(c2, total);
  const double m = static_cast<double>(g.positions) * g.per_group;
  if (threadIdx.x == 0) terms[blockIdx.x] = make_float2(static_cast<float>(c1 / m), static_cast<float>(c2 / m));
}

// ---- step 3, backward: dx, and (the first CTAs) dgamma and dbeta over the images ----
struct Columns {
  const double2* sums;
  float* dgamma;
  float* dbeta;
  int accumulate, images;
};

template <int DT, int GDT, int E, int ACT>
__global__ void __launch_bounds__(kMaxThreads)
group_grad_apply_kernel(const void* x, const void* dy, void* dx, const float* stats, const float2* terms, int images, const float* gamma,
                        const float* beta, const Columns cols, int items, const Geometry g) {
  pdl_trigger();
  pdl_wait();
  if (blockIdx.y == 0) {
    for (int c = blockIdx.x * blockDim.x + threadIdx.x; c < g.channels; c += gridDim.x * blockDim.x) {
      double a = 0.0, s = 0.0;
#pragma unroll 4
      for (int b = 0; b < images; ++b) {
        const double2 v = cols.sums[static_cast<long long>(b) * g.channels + c];
        a += v.x;
        s += v.y;
      }
      if (cols.dbeta) cols.dbeta[c] = static_cast<float>(cols.accumulate ? cols.dbeta[c] + a : a);
      if (cols.dgamma) cols.dgamma[c] = static_cast<float>(cols.accumulate ? cols.dgamma[c] + s : s);
    }
  }
  if (static_cast<int>(blockIdx.x) >= items) return;
  const Place<E> p(g, items - 1 - blockIdx.x);
  if (p.mine == 0) return;
  Params<E> k;
  load_params<E>(k, g, p.b, p.v * E, stats, images, gamma, beta);
  float c1[E], c2[E];
#pragma unroll
  for (int i = 0; i < E; ++i) {
    const float2 v = terms[p.b * g.groups + (p.v * E + i) / g.per_group];
    c1[i] = v.x;
    c2[i] = v.y;
  }
  const auto finish = [&](long long at, const float (&f)[E], float (&d)[E]) {
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const float xh = normal(f[i], k.mean[i], k.r[i]);
      const float dz = ACT == kActNone ? d[i] : d[i] * gn_slope<ACT>(affine(xh, k.gamma[i], k.beta[i]));
      d[i] = k.r[i] * (__fmul_rn(dz, k.gamma[i]) - c1[i] - xh * c2[i]);
    }
    store_elems<GDT, E>(dx, at, d);
  };
  long long at = p.at;
  int t = 0;
  for (; t + 2 <= p.mine; t += 2, at += 2 * p.step) {
    float f[2][E], d[2][E];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      load_elems<DT, E>(x, at + u * p.step, f[u]);
      load_elems<GDT, E>(dy, at + u * p.step, d[u]);
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) finish(at + u * p.step, f[u], d[u]);
  }
  if (t < p.mine) {
    float f[E], d[E];
    load_elems<DT, E>(x, at, f);
    load_elems<GDT, E>(dy, at, d);
    finish(at, f, d);
  }
}

// ---- host ----
constexpr int kPartials = 148 * 6;               // CTAs of the first step, about: enough for two or three on every SM to take turns

Geometry geometry(long long batch, long long positions, int channels, int groups, int vec) {
  Geometry g = {};
  g.positions = static_cast<int>(positions);
  g.channels = channels;
  g.groups = groups;
  g.per_group = channels / groups;
  g.vectors = channels / vec;
  const int blocks = (g.vectors + kMaxThreads - 1) / kMaxThreads;
  g.cols = (g.vectors + blocks - 1) / blocks;
  g.lanes = kMaxThreads / g.cols;
  if (g.lanes > positions) g.lanes = static_cast<int>(positions > 0 ? positions : 1);
  g.image = positions * channels;
  const long long items = batch * blocks;
  long long chunks = items > 0 ? (kPartials + items - 1) / items : 1;
  const long long most = (positions + 2 * g.lanes - 1) / (2 * g.lanes);      // two rows a thread at least
  if (chunks > most) chunks = most;
  if (chunks < 1) chunks = 1;
  g.chunk = static_cast<int>((positions + chunks - 1) / chunks);
  g.chunk = (g.chunk + g.lanes - 1) / g.lanes * g.lanes;
  g.chunks = static_cast<int>((positions + g.chunk - 1) / g.chunk);
  return g;
}
int vector_of(int channels, int dt, int grad_dt) {               // elements of a thread's vector: 16 bytes of the narrower type
  const int e = dt || grad_dt ? 8 : 4;
  return channels % e == 0 ? e : 1;
}
dim3 grid_of(const Geometry& g, long long batch) {
  return dim3(static_cast<unsigned>(batch * g.chunks), static_cast<unsigned>((g.vectors + g.cols - 1) / g.cols));
}
dim3 block_of(const Geometry& g) { return dim3(static_cast<unsigned>((g.cols * g.lanes + 31) / 32 * 32)); }

// The scratch: partial sums, then (forward) the statistics, (backward) the sums of every image's channels and the groups' terms.
struct Scratch {
  size_t partial, second, terms, total;
};
size_t up(size_t n) { return (n + 255) & ~static_cast<size_t>(255); }
Scratch scratch_of(long long batch, long long positions, int channels, int groups, bool grad) {
  // (the most of either width of vectors)
  long long chunks = 0;
  for (int e : {1, 4, 8})
    if (channels % e == 0) {
      const Geometry g = geometry(batch, positions, channels, groups, e);
      if (g.chunks > chunks) chunks = g.chunks;
    }
  Scratch s = {};
  s.second = up(static_cast<size_t>(batch) * chunks * channels * 8);
  s.terms = s.second + (grad ? up(static_cast<size_t>(batch) * channels * 16) : up(static_cast<size_t>(batch) * groups * 8));
  s.total = s.terms + (grad ? up(static_cast<size_t>(batch) * groups * 8) : 0);
  return s;
}

}  // namespace

size_t group_norm_workspace(long long batch, long long positions, int channels, int groups) {
  return scratch_of(batch, positions, channels, groups, false).total;
}
size_t group_norm_grad_workspace(long long batch, long long positions, int channels, int groups) {
  return scratch_of(batch, positions, channels, groups, true).total;
}

cudaError_t launch_group_norm(const void* x, long long batch, long long positions, int channels, int groups, int dt, const float* gamma,
                              const float* beta, float eps, int act, void* y, float* stats, void* workspace, cudaStream_t stream) {
  if (batch == 0 || positions == 0) return cudaSuccess;
  const int e = vector_of(channels, dt, dt), images = static_cast<int>(batch);
  const Geometry g = geometry(batch, positions, channels, groups, e);
  const Scratch s = scratch_of(batch, positions, channels, groups, false);
  char* ws = static_cast<char*>(workspace);
  float2* partial = reinterpret_cast<float2*>(ws);
  if (!stats) stats = reinterpret_cast<float*>(ws + s.second);
  const size_t smem = static_cast<size_t>(g.lanes - 1) * e * g.cols * sizeof(float2);
  const auto sums = dt ? (e == 8 ? group_sums_kernel<1, 8> : group_sums_kernel<1, 1>) : (e == 4 ? group_sums_kernel<0, 4> : group_sums_kernel<0, 1>);
  cudaError_t st = launch_kernel(sums, grid_of(g, batch), block_of(g), smem, stream, true, x, partial, g);
  if (st != cudaSuccess) return st;
  st = launch_kernel(group_stats_kernel, dim3(static_cast<unsigned>(batch * groups)), dim3(256), 0, stream, true,
                     static_cast<const float2*>(partial), stats, images, eps, g);
  if (st != cudaSuccess) return st;
#define SURGEON_APPLY(ACT)                                                                      \
  (dt ? (e == 8 ? group_apply_kernel<1, 8, ACT> : group_apply_kernel<1, 1, ACT>)                \
      : (e == 4 ? group_apply_kernel<0, 4, ACT> : group_apply_kernel<0, 1, ACT>))
  const auto apply = act == kActNone ? SURGEON_APPLY(kActNone) : act == kActRelu ? SURGEON_APPLY(kActRelu)
                     : act == kActGelu ? SURGEON_APPLY(kActGelu) : SURGEON_APPLY(kActSilu);
#undef SURGEON_APPLY
  st = launch_kernel(apply, grid_of(g, batch), block_of(g), 0, stream, true, x, y, static_cast<const float*>(stats), images, gamma, beta, g);
  note_launches(3);
  return st;
}

namespace {

template <int DT, int GDT, int E, int ACT>
cudaError_t launch_grad(const void* x, const void* dy, long long batch, const Geometry& g, const Scratch& s, const float* gamma,
                        const float* beta, const float* stats, void* dx, const Columns& cols, char* ws, cudaStream_t stream) {
  float2* partial = reinterpret_cast<float2*>(ws);
  double2* sums = reinterpret_cast<double2*>(ws + s.second);
  float2* terms = reinterpret_cast<float2*>(ws + s.terms);
  const int images = static_cast<int>(batch);
  const size_t smem = static_cast<size_t>(g.lanes - 1) * E * g.cols * sizeof(float2);
  cudaError_t st = launch_kernel(group_grad_sums_kernel<DT, GDT, E, ACT>, grid_of(g, batch), block_of(g), smem, stream, true, x, dy, partial,
                                 stats, images, gamma, beta, g);
  if (st != cudaSuccess) return st;
  int width = 1;
  while (width < g.per_group && width < 32) width *= 2;
  st = launch_kernel(group_grad_terms_kernel, dim3(static_cast<unsigned>(batch * g.groups)), dim3(256), 0, stream, true,
                     static_cast<const float2*>(partial), sums, terms, gamma, width, g);
  if (st != cudaSuccess) return st;
  dim3 grid = grid_of(g, batch);
  const int items = dx ? static_cast<int>(grid.x) : 0;
  if (!dx) grid = dim3((g.channels + block_of(g).x - 1) / block_of(g).x);
  Columns c = cols;
  c.sums = sums;
  st = launch_kernel(group_grad_apply_kernel<DT, GDT, E, ACT>, grid, block_of(g), 0, stream, true, x, dy, dx, stats,
                     static_cast<const float2*>(terms), images, gamma, beta, c, items, g);
  note_launches(3);
  return st;
}

template <int DT, int GDT, int E>
cudaError_t launch_grad_act(int act, const void* x, const void* dy, long long batch, const Geometry& g, const Scratch& s, const float* gamma,
                            const float* beta, const float* stats, void* dx, const Columns& cols, char* ws, cudaStream_t stream) {
  return (act == kActNone ? launch_grad<DT, GDT, E, kActNone> : act == kActRelu ? launch_grad<DT, GDT, E, kActRelu>
          : act == kActGelu ? launch_grad<DT, GDT, E, kActGelu> : launch_grad<DT, GDT, E, kActSilu>)(x, dy, batch, g, s, gamma, beta, stats, dx,
                                                                                                     cols, ws, stream);
}

__global__ void group_no_rows_kernel(float* dgamma, float* dbeta, int channels) {
  const int c = blockIdx.x * blockDim.x + threadIdx.x;
  if (c >= channels) return;
  if (dgamma) dgamma[c] = 0.0f;
  if (dbeta) dbeta[c] = 0.0f;
}

}  // namespace

cudaError_t launch_group_norm_grad(const void* x, const void* dy, long long batch, long long positions, int channels, int groups, int dt,
                                   int grad_dt, const float* gamma, const float* beta, const float* stats, int act, void* dx, float* dgamma,
                                   float* dbeta, int accumulate, void* workspace, cudaStream_t stream) {
  if (!dx && !dgamma && !dbeta) return cudaSuccess;
  if (batch == 0 || positions == 0) {            // sums over nothing
    if (accumulate || (!dgamma && !dbeta)) return cudaSuccess;
    group_no_rows_kernel<<<(channels + 255) / 256, 256, 0, stream>>>(dgamma, dbeta, channels);
    note_launches(1);
    return cudaGetLastError();
  }
  const int e = vector_of(channels, dt, grad_dt);
  const Geometry g = geometry(batch, positions, channels, groups, e);
  const Scratch s = scratch_of(batch, positions, channels, groups, true);
  const Columns cols = {nullptr, dgamma, dbeta, accumulate, static_cast<int>(batch)};
  char* ws = static_cast<char*>(workspace);
#define SURGEON_GRAD(DT, GDT, E) launch_grad_act<DT, GDT, E>(act, x, dy, batch, g, s, gamma, beta, stats, dx, cols, ws, stream)
  if (dt == 0) return e == 4 ? SURGEON_GRAD(0, 0, 4) : SURGEON_GRAD(0, 0, 1);
  if (grad_dt == 0) return e == 8 ? SURGEON_GRAD(1, 0, 8) : SURGEON_GRAD(1, 0, 1);
  return e == 8 ? SURGEON_GRAD(1, 1, 8) : SURGEON_GRAD(1, 1, 1);
#undef SURGEON_GRAD
}

}  // namespace surgeon
