// Linear layers: host side, the passes around the matrix product (linear_tc.cu), and the kernels for few rows.
#include "linear.cuh"

namespace surgeon {

namespace {

constexpr int kThreads = 256;
constexpr int kFewRows = 4;                      // rows up to which the weights' bytes are all there is: no tensor cores
constexpr int kMaxSlabs = 296;

// Up to two matrices of bf16 with `cols` columns copied to rows of `pitch` (a multiple of 8), zeros behind: what TMA can read.
struct PadArgs {
  const unsigned short* src[2];
  uint4* dst[2];
  uint32_t vecs[2];                              // 16-byte vectors of each
  FastDiv per_row;                               // by a row's vectors
  int cols, row_vecs;
};
__global__ void __launch_bounds__(kThreads)
pad_rows_kernel(const __grid_constant__ PadArgs a) {
  pdl_wait();
  pdl_trigger();
  for (uint32_t i = blockIdx.x * kThreads + threadIdx.x; i < a.vecs[0] + a.vecs[1]; i += gridDim.x * kThreads) {
    const int which = i >= a.vecs[0];
    const uint32_t j = which ? i - a.vecs[0] : i, row = divide(j, a.per_row);
    const int c = static_cast<int>(j - row * a.row_vecs) * 8;
    const unsigned short* from = a.src[which] + static_cast<long long>(row) * a.cols + c;
    uint32_t v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = c + e < a.cols ? from[e] : 0u;
    a.dst[which][j] = make_uint4(v[0] | v[1] << 16, v[2] | v[3] << 16, v[4] | v[5] << 16, v[6] | v[7] << 16);
  }
}

// dz = dy act'(pre) for a slab of rows (blockIdx.y) of 32 E columns: to dz in fp32, to dz16 in bf16 (rows `pitch` apart), and the
// slab's column sums to partial[slab][cols] (added to what is there with `accumulate`); each where wanted.  A warp takes
// every eighth row of the slab.  Bound by HBM for wide layers (12608 x 2304 in bf16 with z, dz in fp32: 41-43 us, 5.5 TB/s), by the
// launch and the first loads for small ones (4037 x 1280: 11.6 us, its bytes 6.3).
template <int GDT, int E, int ACT>
__global__ void __launch_bounds__(kThreads, ACT == kActGelu ? 4 : 1)
act_grad_kernel(const void* __restrict__ dy, const unsigned short* __restrict__ pre, long long rows, int cols,
                long long rows_per, float* __restrict__ dz, unsigned short* __restrict__ dz16, int pitch, float* __restrict__ partial,
                int accumulate) {
  __shared__ float sums[kThreads / 32][32 * E];
  pdl_wait();
  pdl_trigger();
  const int lane = static_cast<int>(lane_id()), warp = threadIdx.x >> 5;
  const int c = (blockIdx.x * 32 + lane) * E;
  const long long begin = blockIdx.y * rows_per, end = begin + rows_per < rows ? begin + rows_per : rows;
  float acc[E];
#pragma unroll
  for (int e = 0; e < E; ++e) acc[e] = 0.0f;
  if (c < cols) {
    const auto finish = [&](long long t, float (&g)[E], const float (&z)[E]) {
      if constexpr (ACT != kActNone) {
#pragma unroll
        for (int e = 0; e < E; ++e) g[e] = __fmul_rn(g[e], slope<ACT>(z[e]));      // (rounded also where only the sum takes it:
      }                                                                            // the same bits whichever outputs are wanted)
#pragma unroll
      for (int e = 0; e < E; ++e) acc[e] += g[e];
      if (dz) store_elems<0, E>(dz, t * cols + c, g);
      if (dz16) store_elems<1, E>(dz16, t * pitch + c, g);
    };
    // Rows whose loads are on their way together. GELU's slope is long enough that two rows and four CTAs per SM
    // pass four rows and the two CTAs that their registers leave (12608 x 2304, dz and its sums: 42 us, else 52);
    // without it four rows are the faster (ReLU: 41 us, 50 with two).
    constexpr int kBatch = E == 1 ? 8 : ACT == kActGelu ? 2 : 4;
    long long t = begin + warp;
    for (; t + (kBatch - 1) * (kThreads / 32) < end; t += kBatch * (kThreads / 32)) {
      float g[kBatch][E], z[kBatch][E];
#pragma unroll
      for (int b = 0; b < kBatch; ++b) load_elems<GDT, E>(dy, (t + b * (kThreads / 32)) * cols + c, g[b]);
      if constexpr (ACT != kActNone) {
#pragma unroll
        for (int b = 0; b < kBatch; ++b) load_elems<1, E>(pre, (t + b * (kThreads / 32)) * cols + c, z[b]);
      }
#pragma unroll
      for (int b = 0; b < kBatch; ++b) finish(t + b * (kThreads / 32), g[b], z[b]);
    }
    for (; t < end; t += kThreads / 32) {
      float g[E], z[E];
      load_elems<GDT, E>(dy, t * cols + c, g);
      if constexpr (ACT != kActNone) load_elems<1, E>(pre, t * cols + c, z);
      finish(t, g, z);
    }
  }
  if (!partial) return;
#pragma unroll
  for (int e = 0; e < E; ++e) sums[warp][lane * E + e] = acc[e];
  __syncthreads();
  for (int i = threadIdx.x; i < 32 * E; i += kThreads) {
    const int col = blockIdx.x * 32 * E + i;
    float s = 0.0f;
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w) s += sums[w][i];
    if (col < cols) {
      float* to = partial + blockIdx.y * static_cast<long long>(cols) + col;
      *to = accumulate ? *to + s : s;
    }
  }
}

// The slabs' column sums where no product follows.
__global__ void __launch_bounds__(1024)
column_sums_kernel(const __grid_constant__ ColumnSums s) {
  __shared__ float buf[kSumSlices][32];
  pdl_wait();
  pdl_trigger();
  add_columns<32>(s, blockIdx.x, gridDim.x, threadIdx.x >> 5, buf);
}

// Few rows, forward: a warp per output, the weights read once.  Latency: 1 x 2048 -> 1000 in 3.3 us, of which a launch is 2 and the 4 MB
// of weights from HBM 0.6; tiles of 128 rows would be empty but for four.
template <int E, int R>
__global__ void __launch_bounds__(kThreads)
few_rows_kernel(const unsigned short* __restrict__ x, const unsigned short* __restrict__ weight, int c_in, int c_out,
                const float* __restrict__ bias, const void* __restrict__ residual, int act, int dt, void* __restrict__ y,
                unsigned short* __restrict__ pre) {
  pdl_wait();
  pdl_trigger();
  const int lane = static_cast<int>(lane_id());
  const int o = blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
  if (o >= c_out) return;
  float acc[R];
#pragma unroll
  for (int r = 0; r < R; ++r) acc[r] = 0.0f;
#pragma unroll 4
  for (int k = lane * E; k < c_in; k += 32 * E) {
    float w[E];
    load_elems<1, E>(weight, static_cast<long long>(o) * c_in + k, w);
#pragma unroll
    for (int r = 0; r < R; ++r) {
      float a[E];
      load_elems<1, E>(x, static_cast<long long>(r) * c_in + k, a);
#pragma unroll
      for (int e = 0; e < E; ++e) acc[r] = fmaf(w[e], a[e], acc[r]);
    }
  }
#pragma unroll
  for (int r = 0; r < R; ++r) acc[r] = lanes_sum<32>(acc[r]);
  if (lane < R) {
    float z = acc[0];
#pragma unroll
    for (int r = 1; r < R; ++r) z = lane == r ? acc[r] : z;
    const long long at = static_cast<long long>(lane) * c_out + o;
    if (bias) z += bias[o];
    float f[1] = {z};
    if (pre) store_elems<1, 1>(pre, at, f);
    f[0] = activate(z, act);
    if (residual) {
      float q[1];
      if (dt == 0) load_elems<0, 1>(residual, at, q);
      else load_elems<1, 1>(residual, at, q);
      f[0] += q[0];
    }
    if (dt == 0) store_elems<0, 1>(y, at, f);
    else store_elems<1, 1>(y, at, f);
  }
}

// Few rows, the input's gradient: 2 E columns per CTA, the outputs shared out among 128 pairs of lanes; dz from fp32.
template <int E, int R>
__global__ void __launch_bounds__(kThreads)
few_rows_grad_kernel(const float* __restrict__ dz, const unsigned short* __restrict__ weight, int c_in, int c_out, int dt,
                     void* __restrict__ dx) {
  __shared__ float part[kThreads / 32][R][2 * E];
  pdl_wait();
  pdl_trigger();
  const int half = threadIdx.x & 1;
  const int c = (blockIdx.x * 2 + half) * E;
  float acc[R][E];
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int e = 0; e < E; ++e) acc[r][e] = 0.0f;
  if (c < c_in) {
#pragma unroll 4
    for (int o = threadIdx.x >> 1; o < c_out; o += kThreads / 2) {
      float w[E];
      load_elems<1, E>(weight, static_cast<long long>(o) * c_in + c, w);
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const float g = dz[static_cast<long long>(r) * c_out + o];
#pragma unroll
        for (int e = 0; e < E; ++e) acc[r][e] = fmaf(w[e], g, acc[r][e]);
      }
    }
  }
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int e = 0; e < E; ++e) {
#pragma unroll
      for (int s = 16; s > 1; s >>= 1) acc[r][e] += __shfl_xor_sync(0xFFFFFFFFu, acc[r][e], s);
      if ((threadIdx.x & 31) < 2) part[threadIdx.x >> 5][r][half * E + e] = acc[r][e];
    }
  __syncthreads();
  for (int i = threadIdx.x; i < R * 2 * E; i += kThreads) {
    const int r = i / (2 * E), col = blockIdx.x * 2 * E + i % (2 * E);
    float f[1] = {0.0f};
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w) f[0] += part[w][r][i % (2 * E)];
    if (col < c_in) {
      const long long at = static_cast<long long>(r) * c_in + col;
      if (dt == 0) store_elems<0, 1>(dx, at, f);
      else store_elems<1, 1>(dx, at, f);
    }
  }
}

constexpr size_t kHead = 256;                    // the status word
size_t up(size_t bytes) { return (bytes + 255) & ~static_cast<size_t>(255); }
int pitch_of(int cols) { return (cols + 7) & ~7; }

void pad_rows(const void* a, long long a_rows, void* a_to, const void* b, long long b_rows, void* b_to, int cols, cudaStream_t stream) {
  PadArgs p = {{static_cast<const unsigned short*>(a), static_cast<const unsigned short*>(b)},
               {static_cast<uint4*>(a_to), static_cast<uint4*>(b_to)}, {0, 0}, make_div(pitch_of(cols) / 8), cols, pitch_of(cols) / 8};
  p.vecs[0] = static_cast<uint32_t>(a_rows * p.row_vecs);
  p.vecs[1] = static_cast<uint32_t>(b_rows * p.row_vecs);
  const long long blocks = (static_cast<long long>(p.vecs[0]) + p.vecs[1] + kThreads - 1) / kThreads;
  launch_kernel(pad_rows_kernel, dim3(static_cast<unsigned>(blocks < 148 * 8 ? blocks : 148 * 8)), dim3(kThreads), 0, stream, true, p);
  note_launches(1);
}

// Rows of a slab in the pass over dy: enough CTAs for the SMs, at least 8 rows each.  Up to 64 rows are one slab, whose sums
// need no second kernel.
long long slab_rows(long long rows, int cols) {
  if (rows <= 64) return 64;
  const int wide = cols % 8 == 0 ? 256 : 32;     // columns of a CTA
  const long long across = (cols + wide - 1) / wide;
  long long slabs = kMaxSlabs * 2 / across > 0 ? kMaxSlabs * 2 / across : 1;
  if (slabs > kMaxSlabs) slabs = kMaxSlabs;
  const long long per = (rows + slabs - 1) / slabs;
  return (per + 7) / 8 * 8;
}

// Parts of surgeon_linear_grad's scratch behind the status word.
struct GradScratch {
  size_t dz, weight, partial, total;
  long long per;                                 // rows of a slab
  int slabs, tiles;                              // slabs of the pass over dy, of 128 rows of the product
};
GradScratch grad_scratch(const surgeon_layer_desc& d) {
  GradScratch s{};
  size_t at = kHead;
  s.dz = at;                                     // bf16 rows for the product, or fp32 for few rows
  at += up(d.batch <= kFewRows ? static_cast<size_t>(d.batch) * d.c_out * 4 : static_cast<size_t>(d.batch) * pitch_of(d.c_out) * 2);
  s.weight = at;
  if (d.c_in % 8 != 0 && d.batch > kFewRows) at += up(static_cast<size_t>(d.c_out) * pitch_of(d.c_in) * 2);
  s.partial = at;
  s.per = slab_rows(d.batch, d.c_out);
  s.slabs = static_cast<int>((d.batch + s.per - 1) / s.per);
  s.tiles = (d.batch + 127) / 128;
  at += up(static_cast<size_t>(s.slabs > s.tiles ? s.slabs : s.tiles) * d.c_out * 4);
  s.total = at;
  return s;
}

}  // namespace

size_t linear_workspace(const surgeon_layer_desc& d) {
  size_t b = kHead;
  if (d.c_in % 8 != 0 && d.batch > kFewRows) {
    b += up(static_cast<size_t>(d.batch) * pitch_of(d.c_in) * 2);
    b += up(static_cast<size_t>(d.c_out) * pitch_of(d.c_in) * 2);
  }
  return b;
}

cudaError_t launch_linear(const surgeon_layer_desc& d, const void* x, const void* weight, const float* bias, const void* residual,
                          int act, int dt, void* y, void* pre, void* workspace, cudaStream_t stream) {
  if (d.batch <= kFewRows) {
    const auto launch = [&](auto kernel) {
      launch_kernel(kernel, dim3((d.c_out + kThreads / 32 - 1) / (kThreads / 32)), dim3(kThreads), 0, stream, true,
                    static_cast<const unsigned short*>(x), static_cast<const unsigned short*>(weight), d.c_in, d.c_out, bias,
                    residual, act, dt, y, static_cast<unsigned short*>(pre));
      note_launches(1);
    };
    if (d.c_in % 8 == 0) {
      if (d.batch == 1) launch(few_rows_kernel<8, 1>);
      else if (d.batch == 2) launch(few_rows_kernel<8, 2>);
      else if (d.batch == 3) launch(few_rows_kernel<8, 3>);
      else launch(few_rows_kernel<8, 4>);
    } else {
      if (d.batch == 1) launch(few_rows_kernel<1, 1>);
      else if (d.batch == 2) launch(few_rows_kernel<1, 2>);
      else if (d.batch == 3) launch(few_rows_kernel<1, 3>);
      else launch(few_rows_kernel<1, 4>);
    }
    return cudaGetLastError();
  }
  unsigned char* at = static_cast<unsigned char*>(workspace);
  uint32_t* status = reinterpret_cast<uint32_t*>(at);
  at += kHead;
  Product p = {x, weight, d.batch, d.c_out, d.c_in, d.c_in, d.c_in, 0, bias, residual, y, pre, act, dt, {}, 0, {}};
  if (d.c_in % 8 != 0) {
    p.lda = p.ldb = pitch_of(d.c_in);
    unsigned char* b_at = at + up(static_cast<size_t>(d.batch) * p.lda * 2);
    pad_rows(x, d.batch, at, weight, d.c_out, b_at, d.c_in, stream);
    p.a = at;
    p.b = b_at;
  }
  const cudaError_t e = launch_product(p, status, stream);
  return e == cudaSuccess ? cudaGetLastError() : e;
}

size_t linear_grad_workspace(const surgeon_layer_desc& d) { return grad_scratch(d).total; }

cudaError_t launch_linear_grad(const surgeon_layer_desc& d, const void* dy, int grad_dt, const void* weight, const void* pre, int act,
                               int dx_dt, void* dx, float* dz, float* dbias, int accumulate, void* workspace, cudaStream_t stream) {
  const GradScratch s = grad_scratch(d);
  unsigned char* base = static_cast<unsigned char*>(workspace);
  uint32_t* status = reinterpret_cast<uint32_t*>(base);
  float* partial = reinterpret_cast<float*>(base + s.partial);
  if (act == kActNone) pre = nullptr;
  const bool few = d.batch <= kFewRows;
  // the product's operand: dy itself where that is dz and lies as TMA reads it
  const bool direct = !few && !pre && grad_dt == SURGEON_BF16 && d.c_out % 8 == 0;
  // Then dz and the column sums come from the product's tiles, without a pass over dy: 12608 x 768 <- 2304 57 us against 82, 37000 x 64 <-
  // 256 18 against 27, 64 x 320 <- 4096 8.3 against 10.5, 16384 x 2048 <- 2048 123 against 129 (whose product by itself is the faster in
  // pairs of CTAs); 12608 x 3200 <- 768 62 against 60.5, 1000 x 768 <- 768 8.8 against 8.3.
  const bool copied = direct && dx && (dz || dbias);
  float* dz32 = dz;
  if (few && dx && !dz) dz32 = reinterpret_cast<float*>(base + s.dz);
  // (dz in bf16, off by 2^-8 of itself at most: the tensor cores' operand.  In fp32 it would be two products, or one at half their rate of
  // tf32 with a pass over the weights; dx errs by 0.0023 of its norm so, where its own rounding to bf16 alone gives 0.0017.)
  void* dz16 = dx && !few && !direct ? base + s.dz : nullptr;
  if (!copied && (dz32 || dz16 || dbias)) {
    const auto launch = [&](auto kernel, int elems) {
      launch_kernel(kernel, dim3((d.c_out + 32 * elems - 1) / (32 * elems), s.slabs), dim3(kThreads), 0, stream, true, dy,
                    static_cast<const unsigned short*>(pre), static_cast<long long>(d.batch), d.c_out, s.per, dz32,
                    static_cast<unsigned short*>(dz16), pitch_of(d.c_out), !dbias ? nullptr : s.slabs == 1 ? dbias : partial,
                    s.slabs == 1 ? accumulate : 0);
      note_launches(1);
    };
#define SURGEON_ACT_GRAD(GDT, E)                                                \
  (act == kActNone ? launch(act_grad_kernel<GDT, E, kActNone>, E)               \
   : act == kActRelu ? launch(act_grad_kernel<GDT, E, kActRelu>, E)             \
                     : launch(act_grad_kernel<GDT, E, kActGelu>, E))
    if (grad_dt == SURGEON_F32) {
      if (d.c_out % 8 == 0) SURGEON_ACT_GRAD(0, 8);
      else SURGEON_ACT_GRAD(0, 1);
    } else {
      if (d.c_out % 8 == 0) SURGEON_ACT_GRAD(1, 8);
      else SURGEON_ACT_GRAD(1, 1);
    }
#undef SURGEON_ACT_GRAD
  }
  ColumnSums sums = {};
  if (!copied && dbias && s.slabs > 1) sums = {partial, dbias, s.slabs, d.c_out, accumulate};
  if (sums.out && !dx) {
    launch_kernel(column_sums_kernel, dim3((d.c_out + 31) / 32), dim3(1024), 0, stream, true, sums);
    note_launches(1);
  }
  if (!dx) return cudaGetLastError();
  if (few) {
    const auto launch = [&](auto kernel, int elems) {
      launch_kernel(kernel, dim3((d.c_in + 2 * elems - 1) / (2 * elems)), dim3(kThreads), 0, stream, true, dz32,
                    static_cast<const unsigned short*>(weight), d.c_in, d.c_out, dx_dt, dx);
      note_launches(1);
    };
    if (d.c_in % 8 == 0) {
      if (d.batch == 1) launch(few_rows_grad_kernel<8, 1>, 8);
      else if (d.batch == 2) launch(few_rows_grad_kernel<8, 2>, 8);
      else if (d.batch == 3) launch(few_rows_grad_kernel<8, 3>, 8);
      else launch(few_rows_grad_kernel<8, 4>, 8);
    } else {
      if (d.batch == 1) launch(few_rows_grad_kernel<1, 1>, 1);
      else if (d.batch == 2) launch(few_rows_grad_kernel<1, 2>, 1);
      else if (d.batch == 3) launch(few_rows_grad_kernel<1, 3>, 1);
      else launch(few_rows_grad_kernel<1, 4>, 1);
    }
    return cudaGetLastError();
  }
  Product p = {direct ? dy : dz16, weight, d.batch, d.c_in, d.c_out, direct ? d.c_out : pitch_of(d.c_out), d.c_in, 1,
               nullptr, nullptr, dx, nullptr, kActNone, dx_dt, sums, copied ? 1 : 0,
               {dz, dbias && s.tiles > 1 ? partial : nullptr, dbias && s.tiles == 1 ? dbias : nullptr, accumulate}};
  if (d.c_in % 8 != 0) {
    pad_rows(weight, d.c_out, base + s.weight, nullptr, 0, nullptr, d.c_in, stream);
    p.b = base + s.weight;
    p.ldb = pitch_of(d.c_in);
  }
  const cudaError_t e = launch_product(p, status, stream);
  if (e == cudaSuccess && copied && dbias && s.tiles > 1) {
    sums = {partial, dbias, s.tiles, d.c_out, accumulate};
    launch_kernel(column_sums_kernel, dim3((d.c_out + 31) / 32), dim3(1024), 0, stream, true, sums);
    note_launches(1);
  }
  return e == cudaSuccess ? cudaGetLastError() : e;
}

}  // namespace surgeon
