// Global norm over a list of gradients, Gradient Importance (Eq. 4) of each of them in the same pass, and clipping.
//
//   S_i = sum_j g_ij^2;  G_i = sqrt(S_i / n_i);  norm = sqrt(sum_i S_i);  out = g * min(1, max_norm / (norm + 1e-6))
//
// A tensor is cut into units of kUnit elements whose places start at 16-byte boundaries, and the units of the whole list,
// in order, into one contiguous range per CTA.  A CTA leaves one sum per tensor that it meets, at slot (CTA + tensor): the
// path through the list moves by one CTA or by one tensor at a time, so the slots are distinct.  The second kernel adds
// the slots in a fixed order (every CTA for itself, some 5 KB from L2 for a list of one launch; a list of several launches has all
// its slots added by every CTA of each, which grows with the square of its length: 10000 tensors of 100 take 0.16 ms to clip, the
// longest list, 65536 of them, 1.8, their norms alone 0.08 and 0.49) and scales the same ranges, last unit first: what
// the first kernel read last is still in L2.  For that the first kernel reads all but the last 80 MB as data that leaves L2
// first, and so does the second with all that it reads and writes: 86 million fp32 gradients clipped into other tensors 173 us, 181
// without, in place the same 179 (48 MB: 174; the 80 MB asked for by a policy that keeps them: 175); three passes over HBM take
// 158, the norm alone takes 55 of 53.  Squares and sums are double (a product of two fp32 numbers is exact in double, and no fp32
// number's square overflows).  Both kernels are bound by HBM; a list of short tensors (106, 213 KB: 8-9 us) by two launches and
// by the ends of its tensors: a unit that is not whole is read element by element, one load after the other.
#include "row_vectors.cuh"

#include <algorithm>
#include <new>

namespace surgeon {

namespace {

constexpr int kThreads = 256;
constexpr int kUnitBytes = 16384;            // of fp32 or bf16 elements: 64 bytes a thread
constexpr int kMaxCtas = 592;                // four per SM (eight: 86 million fp32 gradients clipped in 181 us, four 179)
constexpr uint32_t kKeptUnits = (80 << 20) / kUnitBytes;       // of the list's, that L2 is to hold from one kernel to the next
constexpr double kClipEps = 1e-6;

// One launch's part of the list, passed by value (a kernel's parameters hold up to 32764 bytes).
template <int N>
struct Table {
  const void* grad[N];
  void* out[N];
  long long n[N];
  uint32_t first[N + 1];                     // units before each tensor
  uint32_t types[N / 32];                    // bit i: tensor i is bf16
  int count;                                 // tensors
  uint32_t per;                              // units of a CTA
  int ctas;
  uint32_t keep;                             // of a CTA's units, the last to be read and the first to be scaled
  long long slot;                            // this launch's first slot
  int index;                                 // this launch's first tensor in the whole list
};

__device__ __forceinline__ double block_sum(double v, double* buf) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
  __syncthreads();                           // (the buffer has been read)
  if ((threadIdx.x & 31) == 0) buf[threadIdx.x >> 5] = v;
  __syncthreads();
  v = 0.0;
#pragma unroll
  for (int w = 0; w < kThreads / 32; ++w) v += buf[w];
  return v;
}

template <typename T>
__device__ __forceinline__ int tensor_of(const T& t, uint32_t unit) {
  int lo = 0, hi = t.count - 1;              // the last tensor that begins at `unit` or before
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (t.first[mid] <= unit) lo = mid; else hi = mid - 1;
  }
  return lo;
}

// First element of unit `u` (below 0 in front of a tensor that starts behind a 16-byte boundary) and whether all of the unit's
// elements are the tensor's.
template <int DT>
struct Unit {
  static constexpr int kSize = DT == 0 ? 4 : 2, kElems = 16 / kSize, kUnit = kUnitBytes / kSize, kVecs = kUnitBytes / 16 / kThreads;
  long long at;
  bool whole;
  __device__ __forceinline__ Unit(const void* grad, long long n, uint32_t u) {
    at = static_cast<long long>(u) * kUnit - static_cast<int>(reinterpret_cast<uintptr_t>(grad) & 15) / kSize;
    whole = at >= 0 && at + kUnit <= n;
  }
  // this thread's i-th vector
  __device__ __forceinline__ long long vec(int i) const { return at + (i * kThreads + static_cast<int>(threadIdx.x)) * kElems; }
};

template <int DT>
__device__ __forceinline__ double unit_squares(const void* grad, long long n, uint32_t u, bool keep) {
  using T = typename Elem<DT>::type;
  const Unit<DT> unit(grad, n, u);
  constexpr int E = Unit<DT>::kElems;
  double acc = 0.0;
  if (unit.whole) {                          // (a branch around each load would let one load at a time be on its way)
    uint4 v[Unit<DT>::kVecs];
#pragma unroll
    for (int i = 0; i < Unit<DT>::kVecs; ++i) {
      const uint4* from = reinterpret_cast<const uint4*>(static_cast<const T*>(grad) + unit.vec(i));
      v[i] = keep ? *from : __ldcs(from);
    }
#pragma unroll
    for (int i = 0; i < Unit<DT>::kVecs; ++i) {
      float f[E];
      vector_elems<DT>(v[i], f);
#pragma unroll
      for (int e = 0; e < E; ++e) acc = fma(static_cast<double>(f[e]), static_cast<double>(f[e]), acc);
    }
    return acc;
  }
#pragma unroll 1
  for (int i = 0; i < Unit<DT>::kVecs; ++i) {
    const long long j = unit.vec(i);
#pragma unroll 1
    for (int e = 0; e < E; ++e) {
      if (j + e < 0 || j + e >= n) continue;
      float f[1];
      load_elems<DT, 1>(grad, j + e, f);
      acc = fma(static_cast<double>(f[0]), static_cast<double>(f[0]), acc);
    }
  }
  return acc;
}

template <int N>
__global__ void __launch_bounds__(kThreads)
list_squares_kernel(const __grid_constant__ Table<N> t, double* __restrict__ slots) {
  __shared__ double buf[kThreads / 32];
  pdl_wait();
  pdl_trigger();
  const uint32_t units = t.first[t.count];
  const uint32_t begin = blockIdx.x * t.per, end = begin + t.per < units ? begin + t.per : units;
  int i = tensor_of(t, begin);
  // a tensor that begins with this CTA: the slot before its own belongs to no one
  if (blockIdx.x > 0 && t.first[i] == begin && threadIdx.x == 0) slots[t.slot + blockIdx.x + i - 1] = 0.0;
  double acc = 0.0;
  for (uint32_t u = begin; u < end; ++u) {
    const bool keep = end - u <= t.keep;
    acc += (t.types[i >> 5] >> (i & 31)) & 1 ? unit_squares<1>(t.grad[i], t.n[i], u - t.first[i], keep)
                                             : unit_squares<0>(t.grad[i], t.n[i], u - t.first[i], keep);
    if (u + 1 == end || u + 1 == t.first[i + 1]) {
      acc = block_sum(acc, buf);
      if (threadIdx.x == 0) slots[t.slot + blockIdx.x + i] = acc;
      acc = 0.0;
      ++i;
    }
  }
}

// Sum of all slots of the call, the same bits in every CTA.
__device__ __forceinline__ double total_of(const double* slots, long long n_slots, double* buf) {
  double acc = 0.0;
#pragma unroll 4
  for (long long j = threadIdx.x; j < n_slots; j += kThreads) acc += slots[j];
  return block_sum(acc, buf);
}

// G_i of the launch's tensors: a warp per tensor.
template <typename T>
__device__ __forceinline__ void write_importance(const T& t, const double* slots, double* gi_out) {
  for (int i = blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5); i < t.count; i += gridDim.x * (kThreads / 32)) {
    const uint32_t c0 = t.first[i] / t.per, c1 = (t.first[i + 1] - 1) / t.per;
    double acc = 0.0;
    for (uint32_t c = c0 + (threadIdx.x & 31); c <= c1; c += 32) acc += slots[t.slot + c + i];
    acc = lanes_sum<32>(acc);
    if ((threadIdx.x & 31) == 0) gi_out[t.index + i] = t.n[i] > 0 ? sqrt(acc / static_cast<double>(t.n[i])) : 0.0;
  }
}

template <int N>
__global__ void __launch_bounds__(kThreads)
list_norm_kernel(const __grid_constant__ Table<N> t, const double* __restrict__ slots, long long n_slots,
                 double* __restrict__ norm_out, double* __restrict__ gi_out) {
  __shared__ double buf[kThreads / 32];
  pdl_wait();
  pdl_trigger();
  if (gi_out) write_importance(t, slots, gi_out);
  if (norm_out && blockIdx.x == 0) {
    const double total = total_of(slots, n_slots, buf);
    if (threadIdx.x == 0) *norm_out = sqrt(total);
  }
}

// Elements as they are: with nothing to clip the output is a copy to the last bit, NaNs included.
template <int DT>
__device__ __forceinline__ void scale_one(const void* grad, void* out, long long j, float coef, bool copy) {
  using T = typename Elem<DT>::type;
  if (copy) {
    static_cast<T*>(out)[j] = static_cast<const T*>(grad)[j];
  } else {
    float f[1];
    load_elems<DT, 1>(grad, j, f);
    f[0] *= coef;
    store_elems<DT, 1>(out, j, f);
  }
}

template <int DT>
__device__ __forceinline__ void scale_unit(const void* grad, void* out, long long n, uint32_t u, float coef, bool copy) {
  using T = typename Elem<DT>::type;
  const Unit<DT> unit(grad, n, u);
  constexpr int E = Unit<DT>::kElems;
  if (unit.whole && ((reinterpret_cast<uintptr_t>(grad) ^ reinterpret_cast<uintptr_t>(out)) & 15) == 0) {
    uint4 v[Unit<DT>::kVecs];
#pragma unroll
    for (int i = 0; i < Unit<DT>::kVecs; ++i) v[i] = __ldcs(reinterpret_cast<const uint4*>(static_cast<const T*>(grad) + unit.vec(i)));
#pragma unroll
    for (int i = 0; i < Unit<DT>::kVecs; ++i) {
      if (!copy) {
        float f[E];
        vector_elems<DT>(v[i], f);
#pragma unroll
        for (int e = 0; e < E; ++e) f[e] *= coef;
        if constexpr (DT == 0)
          v[i] = make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
        else
          v[i] = make_uint4(to_bf16x2(f[0], f[1]), to_bf16x2(f[2], f[3]), to_bf16x2(f[4], f[5]), to_bf16x2(f[6], f[7]));
      }
      // (written through: the gradients that are still to be read keep their place in L2)
      __stcs(reinterpret_cast<uint4*>(static_cast<T*>(out) + unit.vec(i)), v[i]);
    }
    return;
  }
#pragma unroll 1
  for (int i = 0; i < Unit<DT>::kVecs; ++i) {
    const long long j = unit.vec(i);
#pragma unroll 1
    for (int e = 0; e < E; ++e)
      if (j + e >= 0 && j + e < n) scale_one<DT>(grad, out, j + e, coef, copy);
  }
}

template <int N>
__global__ void __launch_bounds__(kThreads)
list_scale_kernel(const __grid_constant__ Table<N> t, const double* __restrict__ slots, long long n_slots, double max_norm,
                  int first_launch, double* __restrict__ norm_out, double* __restrict__ gi_out) {
  __shared__ double buf[kThreads / 32];
  pdl_wait();
  pdl_trigger();
  const double norm = sqrt(total_of(slots, n_slots, buf));
  if (norm_out && first_launch && blockIdx.x == 0 && threadIdx.x == 0) *norm_out = norm;
  if (gi_out) write_importance(t, slots, gi_out);
  // nothing to clip, or a norm that is infinite or no number
  const double c = max_norm / (norm + kClipEps);
  const bool copy = !(c < 1.0 && norm <= 1.7976931348623157e308);
  const float coef = static_cast<float>(c);
  const uint32_t units = t.first[t.count];
  const uint32_t begin = blockIdx.x * t.per, end = begin + t.per < units ? begin + t.per : units;
  int i = tensor_of(t, end - 1);
  for (uint32_t u = end; u-- > begin;) {
    while (u < t.first[i]) --i;
    if (copy && t.out[i] == t.grad[i]) continue;
    if ((t.types[i >> 5] >> (i & 31)) & 1) scale_unit<1>(t.grad[i], t.out[i], t.n[i], u - t.first[i], coef, copy);
    else scale_unit<0>(t.grad[i], t.out[i], t.n[i], u - t.first[i], coef, copy);
  }
}

constexpr int kLarge = 1024;                 // tensors per launch: all that fit
static_assert(sizeof(Table<96>) <= 4000 && sizeof(Table<kLarge>) <= 32000, "a launch's parameters");

inline uint32_t units_of(const surgeon_gradient& g) {
  const int size = g.dt == SURGEON_F32 ? 4 : 2;
  const long long shift = static_cast<long long>(reinterpret_cast<uintptr_t>(g.grad) & 15) / size;
  const long long unit = kUnitBytes / size;
  return g.n == 0 ? 1u : static_cast<uint32_t>((g.n + shift + unit - 1) / unit);
}

// CTAs for `units` units, and how many units each takes.
inline int ctas_for(uint32_t units, uint32_t* per) {
  *per = (units + kMaxCtas - 1) / kMaxCtas;
  return static_cast<int>((units + *per - 1) / *per);
}

template <int N>
cudaError_t launch_list_as(const surgeon_gradient* list, int count, int clip, double max_norm, double* norm_out,
                           double* gi_out, double* slots, cudaStream_t stream) {
  Table<N> t;
  long long n_slots = 0;
  for (int pass = 0; pass < 2; ++pass) {                    // squares of the whole list, then norms or scaling
    long long slot = 0;
    for (int at = 0; at < count; at += N) {
      const int n = std::min(N, count - at);
      if (pass == 0 || count > N) {                         // (one launch's table serves both passes)
        uint32_t units = 0;
        for (int w = 0; w < N / 32; ++w) t.types[w] = 0;
        for (int i = 0; i < n; ++i) {
          const surgeon_gradient& g = list[at + i];
          t.grad[i] = g.grad;
          t.out[i] = g.out;
          t.n[i] = g.n;
          t.first[i] = units;
          if (g.dt == SURGEON_BF16) t.types[i >> 5] |= 1u << (i & 31);
          units += units_of(g);
        }
        t.first[n] = units;
        t.count = n;
        t.ctas = ctas_for(units, &t.per);
        t.keep = kKeptUnits / t.ctas;
        t.slot = slot;
        t.index = at;
      }
      slot += t.ctas + n - 1;
      if (pass == 0)
        launch_kernel(list_squares_kernel<N>, dim3(t.ctas), dim3(kThreads), 0, stream, true, t, slots);
      else if (clip)
        launch_kernel(list_scale_kernel<N>, dim3(t.ctas), dim3(kThreads), 0, stream, true, t, slots, n_slots, max_norm,
                      at == 0 ? 1 : 0, norm_out, gi_out);
      else
        launch_kernel(list_norm_kernel<N>, dim3(gi_out ? (n + 7) / 8 : 1), dim3(kThreads), 0, stream, true, t, slots, n_slots,
                      at == 0 ? norm_out : nullptr, gi_out);
      note_launches(1);
    }
    n_slots = slot;
  }
  return cudaGetLastError();
}

struct Range {
  uintptr_t begin, end;
  int out;
};

}  // namespace

size_t gradient_list_workspace(int count) {
  const long long launches = (count + kLarge - 1) / kLarge;
  return static_cast<size_t>(count + launches * kMaxCtas + 1) * sizeof(double);
}

// Whether an output overlaps another output, or a gradient that is not its own; 2 when there was no memory to find out.
int gradient_list_overlaps(const surgeon_gradient* list, int count) {
  Range* r = new (std::nothrow) Range[2 * static_cast<size_t>(count) + 1];
  if (!r) return 2;
  size_t k = 0;
  for (int pass = 0; pass < 2; ++pass)                      // outputs in one run, gradients in the next: either is mostly in order
    for (int i = 0; i < count; ++i) {
      const surgeon_gradient& g = list[i];
      if (g.n == 0 || (pass == 1 && g.grad == g.out)) continue;
      const uintptr_t at = reinterpret_cast<uintptr_t>(pass == 0 ? g.out : g.grad);
      r[k++] = {at, at + static_cast<uintptr_t>(g.n) * (g.dt == SURGEON_F32 ? 4 : 2), pass == 0};
    }
  const auto before = [](const Range& a, const Range& b) { return a.begin < b.begin; };
  if (!std::is_sorted(r, r + k, before)) std::sort(r, r + k, before);
  uintptr_t any = 0, outs = 0;                              // ends of what lies behind: of all ranges, and of the outputs
  int bad = 0;
  for (size_t i = 0; i < k && !bad; ++i) {
    if (r[i].begin < (r[i].out ? any : outs)) bad = 1;
    any = std::max(any, r[i].end);
    if (r[i].out) outs = std::max(outs, r[i].end);
  }
  delete[] r;
  return bad;
}

cudaError_t launch_gradient_list(const surgeon_gradient* list, int count, int clip, double max_norm, double* norm_out,
                                 double* gi_out, void* workspace, cudaStream_t stream) {
  double* slots = static_cast<double*>(workspace);
  if (count == 0) {                                         // the norm of nothing
    return norm_out ? cudaMemsetAsync(norm_out, 0, sizeof(double), stream) : cudaSuccess;
  }
  // (a launch copies its parameters: short lists take small tables)
  if (count <= 96) return launch_list_as<96>(list, count, clip, max_norm, norm_out, gi_out, slots, stream);
  if (count <= 320) return launch_list_as<320>(list, count, clip, max_norm, norm_out, gi_out, slots, stream);
  return launch_list_as<kLarge>(list, count, clip, max_norm, norm_out, gi_out, slots, stream);
}

}  // namespace surgeon
