// extern "C" entry points of libsurgeon: argument checks and host-side arithmetic; every step
// that touches tensor data is a kernel launched from the other translation units.
#include <math.h>
#include <stdio.h>
#include <stdlib.h>

#include <atomic>
#include <initializer_list>

#include "smem_table.h"
#include "surgeon_internal.cuh"

namespace surgeon {

static std::atomic<unsigned long long> g_launches{0};
void note_launches(int n) { g_launches.fetch_add(static_cast<unsigned long long>(n), std::memory_order_relaxed); }
unsigned long long launches_so_far() { return g_launches.load(std::memory_order_relaxed); }

void* tensor_map_encode_fn() {
  static void* fn = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) != cudaSuccess ||
        q != cudaDriverEntryPointSuccess)
      p = nullptr;
    return p;
  }();
  return fn;
}

cudaError_t allow_dynamic_smem(const void* kernel, int bytes) {
  static SmemTable table;
  int dev = 0;
  const cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const int st = table.allow(kernel, dev, bytes, [kernel](int n) {
    return static_cast<int>(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, n));
  });
  return st == SmemTable::kNoRoom ? cudaErrorNotSupported : static_cast<cudaError_t>(st);
}

int sm_count() {
  static int cached[64] = {0};
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 148;
  if (cached[dev] == 0) {
    int n = 0;
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n <= 0)
      n = 148;
    cached[dev] = n;
  }
  return cached[dev];
}

namespace {

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

// Algorithm 1: prune step: kept count for `ratio`; one double multiply, one floor.
inline int64_t kept_count(int64_t n, double ratio) {
  double pruned = floor(ratio * static_cast<double>(n));
  if (pruned < 0.0) pruned = 0.0;
  int64_t np = static_cast<int64_t>(pruned);
  if (np > n) np = n;
  return n - np;
}

bool desc_ok(const surgeon_layer_desc* d, surgeon_status* why) {
  *why = SURGEON_ERR_INVALID_ARG;
  if (!d) return false;
  if (d->kind != 0 && d->kind != 1) return false;
  if (d->path != 0 && d->path != 1) return false;
  if (d->batch <= 0 || d->c_in <= 0 || d->c_out <= 0 || d->h <= 0 || d->w <= 0) return false;
  if (d->kh <= 0 || d->kw <= 0 || d->stride <= 0 || d->pad < 0) return false;
  if (d->kind == 0 && (d->h != 1 || d->w != 1 || d->kh != 1 || d->kw != 1 || d->stride != 1 ||
                       d->pad != 0))
    return false;
  if (d->h + 2 * d->pad < d->kh || d->w + 2 * d->pad < d->kw) return false;
  if (d->groups < 0) return false;
  if (d->groups > 1 && (d->kind != 1 || d->c_in % d->groups != 0 || d->c_out % d->groups != 0)) return false;
  *why = SURGEON_ERR_UNSUPPORTED;
  const long long oh = (d->h + 2 * d->pad - d->kh) / d->stride + 1;
  const long long ow = (d->w + 2 * d->pad - d->kw) / d->stride + 1;
  const long long lim = 2147483647LL;
  if (static_cast<long long>(d->batch) * d->c_in * d->h * d->w > lim) return false;
  if (static_cast<long long>(d->batch) * d->c_out * oh * ow > lim) return false;
  if (static_cast<long long>(d->c_out) * d->c_in * d->kh * d->kw > lim) return false;
  if (d->pad >= d->kh || d->pad >= d->kw) return false;  // windows entirely in the padding
  *why = SURGEON_OK;
  return true;
}

inline bool known_dtype(int dt) { return dt == SURGEON_F32 || dt == SURGEON_BF16; }

// Columns and rows are counted in 32 bits with a few CTAs' worth to spare.
constexpr int32_t kMaxExtent = 1 << 30;

surgeon_status rows_ok(int64_t rows, int32_t channels) {
  if (rows < 0 || channels <= 0) return SURGEON_ERR_INVALID_ARG;
  if (rows > SURGEON_MAX_N / channels || channels > kMaxExtent) return SURGEON_ERR_UNSUPPORTED;
  return SURGEON_OK;
}

surgeon_status linear_ok(const surgeon_layer_desc* d) {
  surgeon_status why;
  if (!desc_ok(d, &why)) return why;
  if (d->kind != 0) return SURGEON_ERR_INVALID_ARG;
  if (d->batch > kMaxExtent || d->c_in > kMaxExtent || d->c_out > kMaxExtent) return SURGEON_ERR_UNSUPPORTED;
  return d->path == 0 ? SURGEON_OK : SURGEON_ERR_UNSUPPORTED;
}
inline bool known_activation(int act) { return act == SURGEON_ACT_NONE || act == SURGEON_ACT_RELU || act == SURGEON_ACT_GELU; }

// Memory that a call writes or reads (none where `at` is null).
struct Span {
  const void* at;
  size_t bytes;
};
Span elems(const void* at, int64_t n, int dt) { return {at, static_cast<size_t>(n) * (dt == SURGEON_F32 ? 4 : 2)}; }
Span floats(const float* at, int64_t n) { return elems(at, n, SURGEON_F32); }
bool overlap(const Span& a, const Span& b) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a.at), y = reinterpret_cast<uintptr_t>(b.at);
  return a.at && b.at && a.bytes && b.bytes && x < y + b.bytes && y < x + a.bytes;
}
// Whether something that is written overlaps something that is read, or another thing that is written.
bool clash(std::initializer_list<Span> written, std::initializer_list<Span> read) {
  for (const Span* a = written.begin(); a != written.end(); ++a) {
    for (const Span* b = a + 1; b != written.end(); ++b)
      if (overlap(*a, *b)) return true;
    for (const Span& r : read)
      if (overlap(*a, r)) return true;
  }
  return false;
}
// An operand in whose place `out` may be written: nothing to compare where it is.
Span unless_place(Span operand, const void* out) { return operand.at == out ? Span{nullptr, 0} : operand; }

surgeon_status group_norm_ok(int64_t batch, int64_t positions, int32_t channels, int32_t groups) {
  if (batch < 0 || positions < 0 || channels <= 0 || groups <= 0 || channels % groups != 0) return SURGEON_ERR_INVALID_ARG;
  if (channels > (1 << 20)) return SURGEON_ERR_UNSUPPORTED;
  const int64_t most = SURGEON_MAX_N / channels;
  if (batch > most || positions > most || (batch > 0 && positions > most / batch)) return SURGEON_ERR_UNSUPPORTED;
  return SURGEON_OK;
}
inline bool known_norm_activation(int act) { return known_activation(act) || act == SURGEON_ACT_SILU; }

surgeon_status attention_ok(const surgeon_attention_desc* d) {
  if (!d || d->batch <= 0 || d->heads <= 0 || d->kv_heads <= 0 || d->heads % d->kv_heads != 0 || d->q_len < 0 || d->kv_len < 0 ||
      d->head_dim <= 0 || d->reserved != 0)
    return SURGEON_ERR_INVALID_ARG;
  const float s = static_cast<float>(d->scale);
  if (!(s > 0.0f) || !isfinite(s)) return SURGEON_ERR_INVALID_ARG;
  if (d->head_dim % 8 != 0 || d->head_dim > 128) return SURGEON_ERR_UNSUPPORTED;
  // (rows of all heads are counted in 31 bits, a tile's worth to spare)
  const int64_t most = (SURGEON_MAX_N / 2) / (static_cast<int64_t>(d->q_len > d->kv_len ? d->q_len : d->kv_len) + 256);
  if (static_cast<int64_t>(d->batch) * d->heads > most) return SURGEON_ERR_UNSUPPORTED;
  return SURGEON_OK;
}

// A tensor of heads with its extents, for comparing places.
struct View {
  const void* at;
  int64_t n[3], stride[3];                       // batch, rows, heads
  int64_t dim;
  int64_t span() const {                         // elements from the first to behind the last
    int64_t s = dim;
    for (int i = 0; i < 3; ++i) s += (n[i] - 1) * stride[i];
    return s;
  }
  bool empty() const { return n[1] == 0; }
};
// Takes a tensor of a call over: false for a bad pointer or stride.
bool view_of(const surgeon_heads* t, int64_t batch, int64_t rows, int64_t heads, int64_t dim, View* out) {
  if (!t) return false;
  *out = {t->data, {batch, rows, heads}, {t->batch_stride, t->row_stride, t->head_stride}, dim};
  if (rows == 0) return true;
  if (!t->data || !aligned16(t->data)) return false;
  for (int i = 0; i < 3; ++i) {
    if (out->n[i] == 1) out->stride[i] = 0;      // (not looked at)
    else if (out->stride[i] <= 0 || out->stride[i] % 8 != 0 || out->stride[i] >= (1LL << 38)) return false;
  }
  return true;
}
// Whether every element has a place of its own.
bool injective(const View& v) {
  if (v.empty()) return true;
  int64_t span = v.dim;
  bool used[3] = {v.n[0] == 1, v.n[1] == 1, v.n[2] == 1};
  for (;;) {
    int next = -1;
    for (int i = 0; i < 3; ++i)
      if (!used[i] && (next < 0 || v.stride[i] < v.stride[next])) next = i;
    if (next < 0) return true;
    if (v.stride[next] < span) return false;
    span += (v.n[next] - 1) * v.stride[next];
    used[next] = true;
  }
}
Span span_of(const View& v) { return {v.empty() ? nullptr : v.at, static_cast<size_t>(v.empty() ? 0 : v.span()) * 2}; }
// Elements of both, modulo one of the strides: those dimensions whose strides are multiples of it drop out, the others span less.
bool apart(const View& a, const View& b) {
  if (!overlap(span_of(a), span_of(b))) return true;
  const int64_t delta = (reinterpret_cast<intptr_t>(b.at) - reinterpret_cast<intptr_t>(a.at)) / 2;
  for (const View* from : {&a, &b})
    for (int64_t m : from->stride) {
      if (m == 0) continue;
      int64_t wide[2] = {a.dim, b.dim};
      const View* both[2] = {&a, &b};
      for (int w = 0; w < 2; ++w)
        for (int i = 0; i < 3; ++i)
          if (both[w]->n[i] > 1 && both[w]->stride[i] % m != 0) wide[w] += (both[w]->n[i] - 1) * both[w]->stride[i];
      const int64_t at = ((delta % m) + m) % m;
      if (at >= wide[0] && at + wide[1] <= m) return true;
    }
  return false;
}
// As clash(), of tensors of heads: `written` ones among themselves and against `read` ones, and all against `words`, which are written.
bool heads_clash(std::initializer_list<const View*> written, std::initializer_list<const View*> read, std::initializer_list<Span> words) {
  for (const View* const* a = written.begin(); a != written.end(); ++a) {
    if (!*a) continue;
    for (const View* const* b = a + 1; b != written.end(); ++b)
      if (*b && !apart(**a, **b)) return true;
    for (const View* r : read)
      if (!apart(**a, *r)) return true;
    for (const Span& w : words)
      if (overlap(span_of(**a), w)) return true;
  }
  for (const View* r : read)
    for (const Span& w : words)
      if (overlap(span_of(*r), w)) return true;
  return false;
}
// Strides that a tensor map takes, for extents of one too.
surgeon_heads plain(const View& v) {
  surgeon_heads t = {const_cast<void*>(v.at), v.stride[0], v.stride[1], v.stride[2]};
  if (!t.head_stride) t.head_stride = (v.dim + 7) / 8 * 8;
  if (!t.row_stride) t.row_stride = t.head_stride;
  if (!t.batch_stride) t.batch_stride = t.row_stride;
  return t;
}
Span ints(const int32_t* at, int64_t n) { return {at, static_cast<size_t>(n) * 4}; }

surgeon_status gradients_ok(const surgeon_gradient* list, int32_t count, bool outputs, const double* norm_out,
                            const double* gi_out, const void* workspace, size_t workspace_bytes) {
  if (count < 0 || (count > 0 && (!list || !workspace))) return SURGEON_ERR_INVALID_ARG;
  if (count > SURGEON_MAX_GRADIENTS) return SURGEON_ERR_UNSUPPORTED;
  if ((reinterpret_cast<uintptr_t>(norm_out) | reinterpret_cast<uintptr_t>(gi_out) |
       reinterpret_cast<uintptr_t>(workspace)) & 7u)
    return SURGEON_ERR_INVALID_ARG;
  for (int i = 0; i < count; ++i) {
    const surgeon_gradient& g = list[i];
    if (g.n < 0 || !known_dtype(g.dt)) return SURGEON_ERR_INVALID_ARG;
    if (g.n > 0 && (!g.grad || (outputs && !g.out))) return SURGEON_ERR_INVALID_ARG;
    const uintptr_t mask = g.dt == SURGEON_F32 ? 3u : 1u;
    if ((reinterpret_cast<uintptr_t>(g.grad) & mask) || (outputs && (reinterpret_cast<uintptr_t>(g.out) & mask)))
      return SURGEON_ERR_INVALID_ARG;
    if (g.n > SURGEON_MAX_N) return SURGEON_ERR_UNSUPPORTED;
  }
  if (count > 0 && workspace_bytes < gradient_list_workspace(count)) return SURGEON_ERR_BUFFER_TOO_SMALL;
  return SURGEON_OK;
}

}  // namespace
}  // namespace surgeon

using namespace surgeon;

extern "C" {

surgeon_status surgeon_layer_ratios(const double* gi, const double* lam, int32_t n_layers,
                                    double* ratios_out) {
  if (!gi || !lam || !ratios_out || n_layers <= 0) return SURGEON_ERR_INVALID_ARG;
  double total = 0.0, g_max = 0.0;
  for (int i = 0; i < n_layers; ++i) {
    if (!isfinite(gi[i]) || gi[i] < 0.0 || !isfinite(lam[i]) || !(lam[i] > 0.0))
      return SURGEON_ERR_INVALID_ARG;
    total += lam[i];
    if (gi[i] > g_max) g_max = gi[i];
  }
  // Eq. 5: M_i = -log(m_i / sum m); kept in ratios_out until Eq. 6 overwrites it.
  double m_max = 0.0;
  for (int i = 0; i < n_layers; ++i) {
    const double mi = -log(lam[i] / total);
    ratios_out[i] = mi;
    if (mi > m_max) m_max = mi;
  }
  // Eq. 6: I_i = (M_i / max M) * (G_i / max G).
  double i_max = 0.0;
  for (int i = 0; i < n_layers; ++i) {
    const double imp = (m_max > 0.0 && g_max > 0.0) ? (ratios_out[i] / m_max) * (gi[i] / g_max) : 0.0;
    ratios_out[i] = imp;
    if (imp > i_max) i_max = imp;
  }
  if (!(i_max > 0.0)) {
    for (int i = 0; i < n_layers; ++i) ratios_out[i] = 0.0;
    return SURGEON_ERR_DEGENERATE;
  }
  // Eq. 7: p_i = 1 - I_i / max I.
  for (int i = 0; i < n_layers; ++i) ratios_out[i] = 1.0 - ratios_out[i] / i_max;
  return SURGEON_OK;
}

surgeon_status surgeon_layer_ratios_rule(const double* gi, const double* lam, int32_t n_layers,
                                         surgeon_ratio_rule rule, double static_ratio,
                                         double* ratios_out) {
  if (!ratios_out || n_layers <= 0) return SURGEON_ERR_INVALID_ARG;
  if (rule == SURGEON_RULE_BOTH) return surgeon_layer_ratios(gi, lam, n_layers, ratios_out);
  if (rule == SURGEON_RULE_STATIC) {
    if (!(static_ratio >= 0.0 && static_ratio <= 1.0)) return SURGEON_ERR_INVALID_ARG;
    for (int i = 0; i < n_layers; ++i) ratios_out[i] = static_ratio;
    return SURGEON_OK;
  }
  double i_max = 0.0;
  if (rule == SURGEON_RULE_NO_GRADIENT) {
    // Eq. 5, then Eq. 6 with the gradient factor taken as 1: I_i = M_i / max M
    if (!lam) return SURGEON_ERR_INVALID_ARG;
    double total = 0.0;
    for (int i = 0; i < n_layers; ++i) {
      if (!isfinite(lam[i]) || !(lam[i] > 0.0)) return SURGEON_ERR_INVALID_ARG;
      total += lam[i];
    }
    for (int i = 0; i < n_layers; ++i) {
      ratios_out[i] = -log(lam[i] / total);
      if (ratios_out[i] > i_max) i_max = ratios_out[i];
    }
  } else if (rule == SURGEON_RULE_NO_MEMORY) {
    // Eq. 6 with the memory factor taken as 1: I_i = G_i / max G
    if (!gi) return SURGEON_ERR_INVALID_ARG;
    for (int i = 0; i < n_layers; ++i) {
      if (!isfinite(gi[i]) || gi[i] < 0.0) return SURGEON_ERR_INVALID_ARG;
      ratios_out[i] = gi[i];
      if (gi[i] > i_max) i_max = gi[i];
    }
  } else {
    return SURGEON_ERR_INVALID_ARG;
  }
  if (!(i_max > 0.0)) {
    for (int i = 0; i < n_layers; ++i) ratios_out[i] = 0.0;
    return SURGEON_ERR_DEGENERATE;
  }
  // Eq. 7 (the inner normalisation cancels against the outer one)
  for (int i = 0; i < n_layers; ++i) ratios_out[i] = 1.0 - ratios_out[i] / i_max;
  return SURGEON_OK;
}

surgeon_status surgeon_compact_sizes(int64_t n, surgeon_dtype dt, double ratio, int64_t* n_keep,
                                     size_t* bitmap_bytes, size_t* values_bytes,
                                     size_t* offsets_bytes, size_t* workspace_bytes) {
  if (n < 0 || !(ratio >= 0.0 && ratio <= 1.0) || (dt != SURGEON_F32 && dt != SURGEON_BF16))
    return SURGEON_ERR_INVALID_ARG;
  if (n > SURGEON_MAX_N) return SURGEON_ERR_UNSUPPORTED;
  const int64_t k = kept_count(n, ratio);
  if (n_keep) *n_keep = k;
  if (bitmap_bytes) *bitmap_bytes = static_cast<size_t>((n + 31) / 32) * 4;
  if (values_bytes) *values_bytes = static_cast<size_t>(k) * (dt == SURGEON_F32 ? 4 : 2);
  if (offsets_bytes)
    *offsets_bytes = static_cast<size_t>((n + SURGEON_BLOCK - 1) / SURGEON_BLOCK + 1) * 4;
  if (workspace_bytes) *workspace_bytes = prune_workspace_bytes(n, static_cast<int>(dt));
  return SURGEON_OK;
}

surgeon_status surgeon_prune_compact(const void* x, int64_t n, surgeon_dtype dt, double ratio,
                                     surgeon_compressed* out, void* workspace,
                                     size_t workspace_bytes, void* cuda_stream) {
  return surgeon_prune_compact_flags(x, n, dt, ratio, 0u, out, workspace, workspace_bytes, cuda_stream);
}

surgeon_status surgeon_prune_compact_flags(const void* x, int64_t n, surgeon_dtype dt, double ratio,
                                           uint32_t flags, surgeon_compressed* out, void* workspace,
                                           size_t workspace_bytes, void* cuda_stream) {
  if (flags & ~static_cast<uint32_t>(SURGEON_STORE_DROP_ZEROS | SURGEON_SHARE_GPU | SURGEON_DEBUG_STALL_BARRIER))
    return SURGEON_ERR_INVALID_ARG;
  if (!out || n < 0 || !(ratio >= 0.0 && ratio <= 1.0) ||
      (dt != SURGEON_F32 && dt != SURGEON_BF16))
    return SURGEON_ERR_INVALID_ARG;
  if (n > SURGEON_MAX_N) return SURGEON_ERR_UNSUPPORTED;
  const int64_t k = kept_count(n, ratio);
  if (!out->header || !out->block_offsets || !workspace) return SURGEON_ERR_INVALID_ARG;
  if (n > 0 && (!x || !out->bitmap)) return SURGEON_ERR_INVALID_ARG;
  if (k > 0 && !out->values) return SURGEON_ERR_INVALID_ARG;
  if (!aligned16(x) || !aligned16(out->bitmap) || !aligned16(out->values) ||
      !aligned16(out->block_offsets) || !aligned16(out->header) || !aligned16(workspace))
    return SURGEON_ERR_INVALID_ARG;
  if (workspace_bytes < prune_workspace_bytes(n, static_cast<int>(dt))) return SURGEON_ERR_BUFFER_TOO_SMALL;
  out->n = n;
  out->dt = static_cast<int32_t>(dt);
  out->reserved = 0;
  const cudaError_t e = launch_prune_compact(x, n, static_cast<int>(dt), k, *out, workspace,
                                             static_cast<cudaStream_t>(cuda_stream),
                                             (flags & SURGEON_STORE_DROP_ZEROS) ? 1 : 0,
                                             (flags & SURGEON_DEBUG_STALL_BARRIER) ? 1 : 0,
                                             (flags & SURGEON_SHARE_GPU) ? 1 : 0);
  return e == cudaSuccess ? SURGEON_OK : SURGEON_ERR_CUDA;
}

size_t surgeon_weight_grad_workspace(const surgeon_layer_desc* d) {
  surgeon_status why;
  if (!desc_ok(d, &why)) return 0;
  const size_t b = d->groups > 1 ? weight_grad_grouped_workspace(*d)
                   : (d->path == 1 ? weight_grad_fp32_workspace(*d) : weight_grad_tc_workspace(*d));
  return (b + 255) & ~static_cast<size_t>(255);
}

surgeon_status surgeon_weight_grad(const surgeon_compressed* act, const surgeon_layer_desc* d,
                                   const float* grad_out, float* dw, int32_t accumulate,
                                   void* workspace, size_t workspace_bytes, void* cuda_stream) {
  return surgeon_weight_grad_flags(act, d, grad_out, dw, accumulate, 0u, workspace, workspace_bytes, cuda_stream);
}

surgeon_status surgeon_weight_grad_flags(const surgeon_compressed* act, const surgeon_layer_desc* d,
                                         const float* grad_out, float* dw, int32_t accumulate, uint32_t flags,
                                         void* workspace, size_t workspace_bytes, void* cuda_stream) {
  surgeon_status why;
  if (!desc_ok(d, &why)) return why;
  if (flags & ~static_cast<uint32_t>(SURGEON_SHARE_GPU)) return SURGEON_ERR_INVALID_ARG;
  if (!act || !grad_out || !dw || !act->bitmap || !act->block_offsets) return SURGEON_ERR_INVALID_ARG;
  if (act->dt != SURGEON_F32 && act->dt != SURGEON_BF16) return SURGEON_ERR_INVALID_ARG;
  if (act->n != static_cast<int64_t>(d->batch) * d->c_in * d->h * d->w) return SURGEON_ERR_INVALID_ARG;
  if (!aligned16(act->bitmap) || !aligned16(act->values) || !aligned16(act->block_offsets) ||
      !aligned16(grad_out) || !aligned16(dw) || !aligned16(workspace))
    return SURGEON_ERR_INVALID_ARG;
  const size_t need = surgeon_weight_grad_workspace(d);
  if (need > 0 && (!workspace || workspace_bytes < need)) return SURGEON_ERR_BUFFER_TOO_SMALL;
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  if (d->groups > 1 && need == 0) return SURGEON_ERR_UNSUPPORTED;
  const cudaError_t e =
      d->groups > 1 ? launch_weight_grad_grouped(*act, *d, grad_out, dw, accumulate ? 1 : 0, workspace, s)
      : d->path == 1 ? launch_weight_grad_fp32(*act, *d, grad_out, dw, accumulate ? 1 : 0, workspace, s)
                     : launch_weight_grad_tc(*act, *d, grad_out, dw, accumulate ? 1 : 0, flags & SURGEON_SHARE_GPU ? 1 : 0,
                                             workspace, s);
  if (e == cudaErrorNotSupported) return SURGEON_ERR_UNSUPPORTED;
  if (e != cudaSuccess && getenv("SURGEON_VERBOSE"))
    fprintf(stderr, "surgeon_weight_grad: %s\n", cudaGetErrorString(e));
  return e == cudaSuccess ? SURGEON_OK : SURGEON_ERR_CUDA;
}

surgeon_status surgeon_decompress(const surgeon_compressed* act, void* x_out, void* cuda_stream) {
  if (!act || act->n < 0 || (act->dt != SURGEON_F32 && act->dt != SURGEON_BF16))
    return SURGEON_ERR_INVALID_ARG;
  if (act->n > 0 && (!x_out || !act->bitmap || !act->block_offsets)) return SURGEON_ERR_INVALID_ARG;
  if (!aligned16(x_out) || !aligned16(act->bitmap) || !aligned16(act->values) ||
      !aligned16(act->block_offsets))
    return SURGEON_ERR_INVALID_ARG;
  const cudaError_t e = launch_decompress(*act, x_out, static_cast<cudaStream_t>(cuda_stream));
  return e == cudaSuccess ? SURGEON_OK : SURGEON_ERR_CUDA;
}

surgeon_status surgeon_gradient_importance(const float* dw, int64_t n_weights, double* gi_out,
                                           void* workspace, size_t workspace_bytes,
                                           void* cuda_stream) {
  if (!gi_out || !workspace || n_weights < 0 || (n_weights > 0 && !dw)) return SURGEON_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(workspace) & 7u) || (reinterpret_cast<uintptr_t>(gi_out) & 7u) ||
      (reinterpret_cast<uintptr_t>(dw) & 3u))
    return SURGEON_ERR_INVALID_ARG;
  if (workspace_bytes < SURGEON_GI_WORKSPACE_BYTES) return SURGEON_ERR_BUFFER_TOO_SMALL;
  const cudaError_t e = launch_gradient_importance(dw, n_weights, gi_out, workspace,
                                                   static_cast<cudaStream_t>(cuda_stream));
  return e == cudaSuccess ? SURGEON_OK : SURGEON_ERR_CUDA;
}

surgeon_status surgeon_layer_norm(const void* x, int64_t rows, int32_t channels, surgeon_dtype dt,
                                  const float* gamma, const float* beta, double eps, void* y,
                                  float* stats, void* cuda_stream) {
  const surgeon_status st = rows_ok(rows, channels);
  if (st != SURGEON_OK) return st;
  const float e = static_cast<float>(eps);
  if (!known_dtype(dt) || !(e > 0.0f) || !isfinite(e)) return SURGEON_ERR_INVALID_ARG;
  if (rows > 0 && (!x || !y)) return SURGEON_ERR_INVALID_ARG;
  if (!aligned16(x) || !aligned16(y) || !aligned16(gamma) || !aligned16(beta) || !aligned16(stats))
    return SURGEON_ERR_INVALID_ARG;
  const int64_t n = rows * channels;
  if (rows > 0 && clash({elems(y, n, dt), floats(stats, 2 * rows)},
                        {unless_place(elems(x, n, dt), y), floats(gamma, channels), floats(beta, channels)}))
    return SURGEON_ERR_INVALID_ARG;
  return launch_layer_norm(x, rows, channels, static_cast<int>(dt), gamma, beta, e, y, stats,
                           static_cast<cudaStream_t>(cuda_stream)) == cudaSuccess ? SURGEON_OK : SURGEON_ERR_CUDA;
}

size_t surgeon_layer_norm_grad_workspace(int64_t rows, int32_t channels) {
  return rows_ok(rows, channels) == SURGEON_OK ? layer_norm_grad_workspace(rows, channels) : 0;
}

surgeon_status surgeon_layer_norm_grad(const void* x, const void* dy, int64_t rows, int32_t channels,
                                       surgeon_dtype dt, surgeon_dtype grad_dt, const float* gamma,
                                       const float* stats, const void* residual_grad, void* dx,
                                       float* dgamma, float* dbeta, int32_t accumulate,
                                       void* workspace, size_t workspace_bytes, void* cuda_stream) {
  const surgeon_status st = rows_ok(rows, channels);
  if (st != SURGEON_OK) return st;
  if (!known_dtype(dt) || !known_dtype(grad_dt)) return SURGEON_ERR_INVALID_ARG;
  if (rows > 0 && (!x || !dy || !stats)) return SURGEON_ERR_INVALID_ARG;
  if (!aligned16(x) || !aligned16(dy) || !aligned16(gamma) || !aligned16(stats) || !aligned16(residual_grad) ||
      !aligned16(dx) || !aligned16(dgamma) || !aligned16(dbeta) || !aligned16(workspace))
    return SURGEON_ERR_INVALID_ARG;
  if (dt == SURGEON_F32 && grad_dt == SURGEON_BF16) return SURGEON_ERR_UNSUPPORTED;
  if ((dgamma || dbeta) && rows > 0) {
    if (!workspace) return SURGEON_ERR_INVALID_ARG;
    if (workspace_bytes < layer_norm_grad_workspace(rows, channels)) return SURGEON_ERR_BUFFER_TOO_SMALL;
  }
  const int64_t n = rows * channels;
  const size_t scratch = dgamma || dbeta ? layer_norm_grad_workspace(rows, channels) : 0;
  if (rows > 0 && clash({elems(dx, n, grad_dt), floats(dgamma, channels), floats(dbeta, channels), {workspace, scratch}},
                        {elems(x, n, dt), unless_place(elems(dy, n, grad_dt), dx), floats(gamma, channels), floats(stats, 2 * rows),
                         unless_place(elems(dx ? residual_grad : nullptr, n, grad_dt), dx)}))
    return SURGEON_ERR_INVALID_ARG;
  return launch_layer_norm_grad(x, dy, rows, channels, static_cast<int>(dt), static_cast<int>(grad_dt), gamma, stats,
                                residual_grad, dx, dgamma, dbeta, accumulate ? 1 : 0, workspace,
                                static_cast<cudaStream_t>(cuda_stream)) == cudaSuccess ? SURGEON_OK : SURGEON_ERR_CUDA;
}

size_t surgeon_linear_workspace(const surgeon_layer_desc* d) {
  return linear_ok(d) == SURGEON_OK ? linear_workspace(*d) : 0;
}

surgeon_status surgeon_linear(const surgeon_layer_desc* d, const void* x, const void* weight,
                              const float* bias, surgeon_activation act, const void* residual,
                              surgeon_dtype out_dt, void* y, void* pre, void* workspace,
                              size_t workspace_bytes, void* cuda_stream) {
  const surgeon_status st = linear_ok(d);
  if (st != SURGEON_OK) return st;
  if (!x || !weight || !y || !workspace || !known_activation(act) || !known_dtype(out_dt)) return SURGEON_ERR_INVALID_ARG;
  if (!aligned16(x) || !aligned16(weight) || !aligned16(bias) || !aligned16(residual) || !aligned16(y) || !aligned16(pre) ||
      !aligned16(workspace))
    return SURGEON_ERR_INVALID_ARG;
  if (workspace_bytes < linear_workspace(*d)) return SURGEON_ERR_BUFFER_TOO_SMALL;
  const int64_t in = static_cast<int64_t>(d->batch) * d->c_in, out = static_cast<int64_t>(d->batch) * d->c_out;
  const int64_t weights = static_cast<int64_t>(d->c_out) * d->c_in;
  if (clash({elems(y, out, out_dt), elems(pre, out, SURGEON_BF16), {workspace, linear_workspace(*d)}},
            {elems(x, in, SURGEON_BF16), elems(weight, weights, SURGEON_BF16), floats(bias, d->c_out),
             unless_place(elems(residual, out, out_dt), y)}))
    return SURGEON_ERR_INVALID_ARG;
  return launch_linear(*d, x, weight, bias, residual, static_cast<int>(act), static_cast<int>(out_dt), y, pre, workspace,
                       static_cast<cudaStream_t>(cuda_stream)) == cudaSuccess ? SURGEON_OK : SURGEON_ERR_CUDA;
}

size_t surgeon_linear_grad_workspace(const surgeon_layer_desc* d) {
  return linear_ok(d) == SURGEON_OK ? linear_grad_workspace(*d) : 0;
}

surgeon_status surgeon_linear_grad(const surgeon_layer_desc* d, const void* dy, surgeon_dtype grad_dt,
                                   const void* weight, const void* pre, surgeon_activation act,
                                   surgeon_dtype dx_dt, void* dx, float* dz, float* dbias,
                                   int32_t accumulate, void* workspace, size_t workspace_bytes,
                                   void* cuda_stream) {
  const surgeon_status st = linear_ok(d);
  if (st != SURGEON_OK) return st;
  if (!dy || !workspace || !known_activation(act) || !known_dtype(grad_dt) || !known_dtype(dx_dt)) return SURGEON_ERR_INVALID_ARG;
  if ((dx && !weight) || (act != SURGEON_ACT_NONE && !pre)) return SURGEON_ERR_INVALID_ARG;
  if (!aligned16(dy) || !aligned16(weight) || !aligned16(pre) || !aligned16(dx) || !aligned16(dz) || !aligned16(dbias) ||
      !aligned16(workspace))
    return SURGEON_ERR_INVALID_ARG;
  if (workspace_bytes < linear_grad_workspace(*d)) return SURGEON_ERR_BUFFER_TOO_SMALL;
  const int64_t in = static_cast<int64_t>(d->batch) * d->c_in, out = static_cast<int64_t>(d->batch) * d->c_out;
  const int64_t weights = static_cast<int64_t>(d->c_out) * d->c_in;
  if (clash({elems(dx, in, dx_dt), floats(dz, out), floats(dbias, d->c_out), {workspace, linear_grad_workspace(*d)}},
            {elems(dy, out, grad_dt), elems(dx ? weight : nullptr, weights, SURGEON_BF16),
             elems(act != SURGEON_ACT_NONE ? pre : nullptr, out, SURGEON_BF16)}))
    return SURGEON_ERR_INVALID_ARG;
  return launch_linear_grad(*d, dy, static_cast<int>(grad_dt), weight, pre, static_cast<int>(act), static_cast<int>(dx_dt), dx, dz,
                            dbias, accumulate ? 1 : 0, workspace, static_cast<cudaStream_t>(cuda_stream)) == cudaSuccess
             ? SURGEON_OK : SURGEON_ERR_CUDA;
}

size_t surgeon_gradient_norm_workspace(int32_t count) {
  return count < 0 || count > SURGEON_MAX_GRADIENTS ? 0 : gradient_list_workspace(count);
}

surgeon_status surgeon_gradient_norm(const surgeon_gradient* list, int32_t count, double* norm_out,
                                     double* gi_out, void* workspace, size_t workspace_bytes,
                                     void* cuda_stream) {
  if (!norm_out && !gi_out) return SURGEON_ERR_INVALID_ARG;
  const surgeon_status st = gradients_ok(list, count, false, norm_out, gi_out, workspace, workspace_bytes);
  if (st != SURGEON_OK) return st;
  return launch_gradient_list(list, count, 0, 0.0, norm_out, gi_out, workspace,
                              static_cast<cudaStream_t>(cuda_stream)) == cudaSuccess ? SURGEON_OK : SURGEON_ERR_CUDA;
}

surgeon_status surgeon_clip_gradients(const surgeon_gradient* list, int32_t count, double max_norm,
                                      double* norm_out, double* gi_out, void* workspace,
                                      size_t workspace_bytes, void* cuda_stream) {
  if (!(max_norm >= 0.0)) return SURGEON_ERR_INVALID_ARG;
  const surgeon_status st = gradients_ok(list, count, true, norm_out, gi_out, workspace, workspace_bytes);
  if (st != SURGEON_OK) return st;
  if (gradient_list_overlaps(list, count)) return SURGEON_ERR_INVALID_ARG;
  return launch_gradient_list(list, count, 1, max_norm, norm_out, gi_out, workspace,
                              static_cast<cudaStream_t>(cuda_stream)) == cudaSuccess ? SURGEON_OK : SURGEON_ERR_CUDA;
}

size_t surgeon_attention_workspace(const surgeon_attention_desc* d) { return attention_ok(d) == SURGEON_OK ? attention_workspace(*d) : 0; }

surgeon_status surgeon_attention(const surgeon_attention_desc* d, const surgeon_heads* q, const surgeon_heads* k,
                                 const surgeon_heads* v, const int32_t* q_lengths, const int32_t* kv_lengths,
                                 const surgeon_heads* o, float* lse, void* workspace, size_t workspace_bytes,
                                 void* cuda_stream) {
  const surgeon_status st = attention_ok(d);
  if (st != SURGEON_OK) return st;
  View vq, vk, vv, vo;
  if (!view_of(q, d->batch, d->q_len, d->heads, d->head_dim, &vq) || !view_of(k, d->batch, d->kv_len, d->kv_heads, d->head_dim, &vk) ||
      !view_of(v, d->batch, d->kv_len, d->kv_heads, d->head_dim, &vv) || !view_of(o, d->batch, d->q_len, d->heads, d->head_dim, &vo) ||
      !injective(vo))
    return SURGEON_ERR_INVALID_ARG;
  const size_t need = attention_workspace(*d);
  if (!aligned16(lse) || !aligned16(workspace) || !aligned4(q_lengths) || !aligned4(kv_lengths) || (need && !workspace)) return SURGEON_ERR_INVALID_ARG;
  if (workspace_bytes < need) return SURGEON_ERR_BUFFER_TOO_SMALL;
  if (d->q_len == 0) return SURGEON_OK;
  const Span ls = floats(lse, static_cast<int64_t>(d->batch) * d->heads * d->q_len), ws = {workspace, need};
  const Span ql = ints(q_lengths, d->batch), kl = ints(kv_lengths, d->batch);
  if (heads_clash({&vo}, {&vq, &vk, &vv}, {ls, ws}) || clash({ls, ws, span_of(vo)}, {ql, kl})) return SURGEON_ERR_INVALID_ARG;
  return launch_attention(*d, plain(vq), plain(vk), plain(vv), q_lengths, kv_lengths, plain(vo), lse, workspace,
                          static_cast<cudaStream_t>(cuda_stream)) == cudaSuccess ? SURGEON_OK : SURGEON_ERR_CUDA;
}

size_t surgeon_attention_grad_workspace(const surgeon_attention_desc* d) {
  return attention_ok(d) == SURGEON_OK ? attention_grad_workspace(*d) : 0;
}

surgeon_status surgeon_attention_grad(const surgeon_attention_desc* d, const surgeon_heads* q, const surgeon_heads* k,
                                      const surgeon_heads* v, const surgeon_heads* o, const surgeon_heads* dout,
                                      const float* lse, const int32_t* q_lengths, const int32_t* kv_lengths,
                                      const surgeon_heads* dq, const surgeon_heads* dk, const surgeon_heads* dv,
                                      void* workspace, size_t workspace_bytes, void* cuda_stream) {
  const surgeon_status st = attention_ok(d);
  if (st != SURGEON_OK) return st;
  View vq, vk, vv, vo, vd, gq, gk, gv;
  if (!view_of(q, d->batch, d->q_len, d->heads, d->head_dim, &vq) || !view_of(k, d->batch, d->kv_len, d->kv_heads, d->head_dim, &vk) ||
      !view_of(v, d->batch, d->kv_len, d->kv_heads, d->head_dim, &vv) || !view_of(o, d->batch, d->q_len, d->heads, d->head_dim, &vo) ||
      !view_of(dout, d->batch, d->q_len, d->heads, d->head_dim, &vd))
    return SURGEON_ERR_INVALID_ARG;
  if (dq && (!view_of(dq, d->batch, d->q_len, d->heads, d->head_dim, &gq) || !injective(gq))) return SURGEON_ERR_INVALID_ARG;
  if ((dk != nullptr) != (dv != nullptr)) return SURGEON_ERR_INVALID_ARG;
  if (dk && (!view_of(dk, d->batch, d->kv_len, d->kv_heads, d->head_dim, &gk) || !injective(gk) ||
             !view_of(dv, d->batch, d->kv_len, d->kv_heads, d->head_dim, &gv) || !injective(gv)))
    return SURGEON_ERR_INVALID_ARG;
  if (!workspace || !aligned16(workspace) || !aligned16(lse) || (d->q_len > 0 && !lse) || !aligned4(q_lengths) || !aligned4(kv_lengths))
    return SURGEON_ERR_INVALID_ARG;
  const size_t need = attention_grad_workspace(*d);
  if (workspace_bytes < need) return SURGEON_ERR_BUFFER_TOO_SMALL;
  const Span ws = {workspace, need}, ls = floats(lse, static_cast<int64_t>(d->batch) * d->heads * d->q_len);
  const Span ql = ints(q_lengths, d->batch), kl = ints(kv_lengths, d->batch);
  if (heads_clash({dq ? &gq : nullptr, dk ? &gk : nullptr, dv ? &gv : nullptr}, {&vq, &vk, &vv, &vo, &vd}, {ws}) ||
      clash({ws}, {ls, ql, kl}))
    return SURGEON_ERR_INVALID_ARG;
  for (const View* g : {dq ? &gq : nullptr, dk ? &gk : nullptr, dv ? &gv : nullptr})
    if (g && clash({span_of(*g)}, {ls, ql, kl})) return SURGEON_ERR_INVALID_ARG;
  surgeon_heads pq, pk, pv;
  if (dq) pq = plain(gq);
  if (dk) { pk = plain(gk); pv = plain(gv); }
  return launch_attention_grad(*d, plain(vq), plain(vk), plain(vv), plain(vo), plain(vd), lse, q_lengths, kv_lengths, dq ? &pq : nullptr,
                               dk ? &pk : nullptr, dk ? &pv : nullptr, workspace, static_cast<cudaStream_t>(cuda_stream)) == cudaSuccess
             ? SURGEON_OK : SURGEON_ERR_CUDA;
}

size_t surgeon_group_norm_workspace(int64_t batch, int64_t positions, int32_t channels, int32_t groups) {
  return group_norm_ok(batch, positions, channels, groups) == SURGEON_OK ? group_norm_workspace(batch, positions, channels, groups) : 0;
}

surgeon_status surgeon_group_norm(const void* x, int64_t batch, int64_t positions, int32_t channels,
                                  int32_t groups, surgeon_dtype dt, const float* gamma, const float* beta,
                                  double eps, int32_t act, void* y, float* stats, void* workspace,
                                  size_t workspace_bytes, void* cuda_stream) {
  const surgeon_status st = group_norm_ok(batch, positions, channels, groups);
  if (st != SURGEON_OK) return st;
  const float e = static_cast<float>(eps);
  if (!known_dtype(dt) || !known_norm_activation(act) || !(e > 0.0f) || !isfinite(e)) return SURGEON_ERR_INVALID_ARG;
  const int64_t n = batch * positions * channels;
  if (n > 0 && (!x || !y || !workspace)) return SURGEON_ERR_INVALID_ARG;
  if (!aligned16(x) || !aligned16(y) || !aligned16(gamma) || !aligned16(beta) || !aligned16(stats) || !aligned16(workspace))
    return SURGEON_ERR_INVALID_ARG;
  if (n == 0) return SURGEON_OK;
  const size_t need = group_norm_workspace(batch, positions, channels, groups);
  if (workspace_bytes < need) return SURGEON_ERR_BUFFER_TOO_SMALL;
  if (clash({elems(y, n, dt), floats(stats, 2 * batch * groups), {workspace, need}},
            {unless_place(elems(x, n, dt), y), floats(gamma, channels), floats(beta, channels)}))
    return SURGEON_ERR_INVALID_ARG;
  return launch_group_norm(x, batch, positions, channels, groups, static_cast<int>(dt), gamma, beta, e, act, y, stats, workspace,
                           static_cast<cudaStream_t>(cuda_stream)) == cudaSuccess ? SURGEON_OK : SURGEON_ERR_CUDA;
}

size_t surgeon_group_norm_grad_workspace(int64_t batch, int64_t positions, int32_t channels, int32_t groups) {
  return group_norm_ok(batch, positions, channels, groups) == SURGEON_OK ? group_norm_grad_workspace(batch, positions, channels, groups) : 0;
}

surgeon_status surgeon_group_norm_grad(const void* x, const void* dy, int64_t batch, int64_t positions,
                                       int32_t channels, int32_t groups, surgeon_dtype dt, surgeon_dtype grad_dt,
                                       const float* gamma, const float* beta, const float* stats, int32_t act,
                                       void* dx, float* dgamma, float* dbeta, int32_t accumulate,
                                       void* workspace, size_t workspace_bytes, void* cuda_stream) {
  const surgeon_status st = group_norm_ok(batch, positions, channels, groups);
  if (st != SURGEON_OK) return st;
  if (!known_dtype(dt) || !known_dtype(grad_dt) || !known_norm_activation(act)) return SURGEON_ERR_INVALID_ARG;
  const int64_t n = batch * positions * channels;
  if (n > 0 && (!x || !dy || !stats || !workspace)) return SURGEON_ERR_INVALID_ARG;
  if (!aligned16(x) || !aligned16(dy) || !aligned16(gamma) || !aligned16(beta) || !aligned16(stats) || !aligned16(dx) || !aligned16(dgamma) ||
      !aligned16(dbeta) || !aligned16(workspace))
    return SURGEON_ERR_INVALID_ARG;
  if (dt == SURGEON_F32 && grad_dt == SURGEON_BF16) return SURGEON_ERR_UNSUPPORTED;
  const size_t need = n > 0 ? group_norm_grad_workspace(batch, positions, channels, groups) : 0;
  if (workspace_bytes < need) return SURGEON_ERR_BUFFER_TOO_SMALL;
  if (clash({elems(dx, n, grad_dt), floats(dgamma, channels), floats(dbeta, channels), {workspace, need}},
            {elems(x, n, dt), unless_place(elems(dy, n, grad_dt), dx), floats(gamma, channels), floats(beta, channels),
             floats(stats, 2 * batch * groups)}))
    return SURGEON_ERR_INVALID_ARG;
  return launch_group_norm_grad(x, dy, batch, positions, channels, groups, static_cast<int>(dt), static_cast<int>(grad_dt), gamma, beta, stats,
                                act, dx, dgamma, dbeta, accumulate ? 1 : 0, workspace, static_cast<cudaStream_t>(cuda_stream)) == cudaSuccess
             ? SURGEON_OK : SURGEON_ERR_CUDA;
}

surgeon_status surgeon_dropout(const void* x, int64_t n, surgeon_dtype dt, double p, uint64_t seed, uint64_t offset,
                               const uint64_t* device_offset, const void* residual, void* y, void* cuda_stream) {
  if (n < 0 || !known_dtype(dt) || !(p >= 0.0 && p <= 1.0) || (n > 0 && (!x || !y))) return SURGEON_ERR_INVALID_ARG;
  if (!aligned16(x) || !aligned16(residual) || !aligned16(y) || (reinterpret_cast<uintptr_t>(device_offset) & 7u)) return SURGEON_ERR_INVALID_ARG;
  if (n > SURGEON_MAX_N) return SURGEON_ERR_UNSUPPORTED;
  if (clash({elems(y, n, dt)}, {unless_place(elems(x, n, dt), y), unless_place(elems(residual, n, dt), y), {device_offset, 8}}))
    return SURGEON_ERR_INVALID_ARG;
  return launch_dropout(x, n, static_cast<int>(dt), static_cast<uint32_t>(floor(p * 65536.0 + 0.5)), seed, offset, device_offset, residual, y,
                        static_cast<cudaStream_t>(cuda_stream)) == cudaSuccess ? SURGEON_OK : SURGEON_ERR_CUDA;
}

uint64_t surgeon_launch_count(void) { return launches_so_far(); }

const char* surgeon_status_string(surgeon_status s) {
  switch (s) {
    case SURGEON_OK: return "ok";
    case SURGEON_ERR_INVALID_ARG: return "invalid argument";
    case SURGEON_ERR_BUFFER_TOO_SMALL: return "buffer too small";
    case SURGEON_ERR_DEGENERATE: return "degenerate input (ratio rule is 0/0)";
    case SURGEON_ERR_UNSUPPORTED: return "unsupported geometry, dtype or size";
    case SURGEON_ERR_CUDA: return "CUDA runtime error";
    case SURGEON_ERR_TIMEOUT: return "device-side bounded wait expired";
    case SURGEON_ERR_INTERNAL: return "device-side self-check failed";
  }
  return "unknown status";
}

}  // extern "C"
