// The calls of the layers around the store, marshalled in C++.  They are short: a layer norm of one row runs for 2 us, and
// checking its tensors one attribute at a time from Python and passing the arguments through ctypes took 4 us more than
// the launch.  A function here makes the call if every argument is the ordinary case (the types, shapes and device that
// binding.py asks for, contiguous, all buffers given, the current stream) and returns the library's status; for
// anything else it returns None and binding.py, which holds the rules and their errors, takes the call.
#include <Python.h>

#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <initializer_list>

#include "surgeon.h"

namespace {

// The library's entry points, by the addresses that the binding loaded them at (bind()).
decltype(&surgeon_layer_norm) layer_norm_fn = nullptr;
decltype(&surgeon_layer_norm_grad) layer_norm_grad_fn = nullptr;
decltype(&surgeon_linear) linear_fn = nullptr;
decltype(&surgeon_linear_grad) linear_grad_fn = nullptr;
decltype(&surgeon_gradient_norm) gradient_norm_fn = nullptr;
decltype(&surgeon_clip_gradients) clip_gradients_fn = nullptr;

using Shape = std::initializer_list<int64_t>;

// The checks of one call: `ok` turns false at the first argument that is not the ordinary case.
struct Args {
  const int device = c10::cuda::current_device();
  bool ok = true;

  const at::Tensor* tensor(PyObject* o) {
    if (!ok || !THPVariable_Check(o)) {
      ok = false;
      return nullptr;
    }
    return &THPVariable_Unpack(o);
  }
  void* plain(const at::Tensor& t) {
    if (!t.is_cuda() || t.get_device() != device || !t.is_contiguous()) ok = false;
    return ok ? t.data_ptr() : nullptr;
  }
  // A tensor of this type and shape; Py_None: a null pointer, where it may be left out.
  void* operand(PyObject* o, at::ScalarType type, at::IntArrayRef shape, bool optional = true) {
    if (o == Py_None) {
      ok = ok && optional;
      return nullptr;
    }
    const at::Tensor* t = tensor(o);
    if (!t || t->scalar_type() != type || t->sizes() != shape) {
      ok = false;
      return nullptr;
    }
    return plain(*t);
  }
  void* operand(PyObject* o, at::ScalarType type, Shape shape, bool optional = true) {
    return operand(o, type, at::IntArrayRef(shape.begin(), shape.size()), optional);
  }
  void* workspace(PyObject* o, size_t* bytes) {
    const at::Tensor* t = tensor(o);
    if (!t) return nullptr;
    *bytes = t->nbytes();
    return plain(*t);
  }
  surgeon_dtype type(const at::Tensor& t) {
    if (t.scalar_type() == at::kFloat) return SURGEON_F32;
    if (t.scalar_type() != at::kBFloat16) ok = false;
    return SURGEON_BF16;
  }
  int64_t integer(PyObject* o) {
    const int64_t v = PyLong_Check(o) ? PyLong_AsLongLong(o) : (ok = false, 0);
    if (PyErr_Occurred()) {
      PyErr_Clear();
      ok = false;
    }
    return v;
  }
  bool truth(PyObject* o) {                      // (as Python's `if`: any number, not True alone)
    const int v = PyObject_IsTrue(o);
    if (v < 0) {
      PyErr_Clear();
      ok = false;
    }
    return v > 0;
  }
  double number(PyObject* o) {
    const double v = PyFloat_AsDouble(o);
    if (PyErr_Occurred()) {
      PyErr_Clear();
      ok = false;
    }
    return v;
  }
  void* stream() const { return c10::cuda::getCurrentCUDAStream(static_cast<c10::DeviceIndex>(device)).stream(); }
};

PyObject* answer(surgeon_status s) { return PyLong_FromLong(s); }

// A linear layer's descriptor: a ctypes structure of the binding's.
struct Desc {
  Py_buffer view;
  const surgeon_layer_desc* d = nullptr;
  explicit Desc(PyObject* o) {
    if (PyObject_GetBuffer(o, &view, PyBUF_SIMPLE) != 0) PyErr_Clear();
    else if (view.len == static_cast<Py_ssize_t>(sizeof(surgeon_layer_desc))) d = static_cast<const surgeon_layer_desc*>(view.buf);
    else PyBuffer_Release(&view);
  }
  ~Desc() {
    if (d) PyBuffer_Release(&view);
  }
};

// The body of a call: no exception of the tensor library's leaves it.
template <typename F>
PyObject* guarded(F&& body) {
  try {
    return body();
  } catch (...) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
}

// x, gamma, beta, eps, out, stats
PyObject* layer_norm(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    Args c;
    if (n != 6 || !layer_norm_fn) Py_RETURN_NONE;
    const at::Tensor* x = c.tensor(a[0]);
    if (!x || x->dim() < 1 || x->size(-1) == 0) Py_RETURN_NONE;
    const int64_t channels = x->size(-1), rows = x->numel() / channels;
    const surgeon_dtype dt = c.type(*x);
    void* xp = c.plain(*x);
    void* gamma = c.operand(a[1], at::kFloat, {channels});
    void* beta = c.operand(a[2], at::kFloat, {channels});
    const double eps = c.number(a[3]);
    void* out = c.operand(a[4], x->scalar_type(), x->sizes(), false);
    void* stats = c.operand(a[5], at::kFloat, {2, rows});
    if (!c.ok || channels > INT32_MAX) Py_RETURN_NONE;
    return answer(layer_norm_fn(xp, rows, static_cast<int32_t>(channels), dt, static_cast<float*>(gamma), static_cast<float*>(beta),
                                eps, out, static_cast<float*>(stats), c.stream()));
  });
}

// x, dy, gamma, stats, residual_grad, dx, dgamma, dbeta, accumulate, workspace
PyObject* layer_norm_grad(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    Args c;
    if (n != 10 || !layer_norm_grad_fn) Py_RETURN_NONE;
    const at::Tensor* x = c.tensor(a[0]);
    const at::Tensor* dy = c.tensor(a[1]);
    if (!x || !dy || x->dim() < 1 || x->size(-1) == 0) Py_RETURN_NONE;
    const int64_t channels = x->size(-1), rows = x->numel() / channels;
    const surgeon_dtype dt = c.type(*x), gdt = c.type(*dy);
    const at::ScalarType g = dy->scalar_type();
    void* xp = c.plain(*x);
    void* dyp = c.operand(a[1], g, x->sizes(), false);
    void* gamma = c.operand(a[2], at::kFloat, {channels});
    void* stats = c.operand(a[3], at::kFloat, {2, rows}, false);
    void* res = c.operand(a[4], g, x->sizes());
    void* dx = c.operand(a[5], g, x->sizes(), false);
    void* dgamma = c.operand(a[6], at::kFloat, {channels});
    void* dbeta = c.operand(a[7], at::kFloat, {channels});
    const bool accumulate = c.truth(a[8]);
    size_t bytes = 0;
    void* ws = c.workspace(a[9], &bytes);
    if (!c.ok || channels > INT32_MAX) Py_RETURN_NONE;
    return answer(layer_norm_grad_fn(xp, dyp, rows, static_cast<int32_t>(channels), dt, gdt, static_cast<float*>(gamma),
                                     static_cast<float*>(stats), res, dx, static_cast<float*>(dgamma), static_cast<float*>(dbeta),
                                     accumulate, ws, bytes, c.stream()));
  });
}

// desc, x, weight, bias, act, residual, out, pre, workspace
PyObject* linear(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    Args c;
    if (n != 9 || !linear_fn) Py_RETURN_NONE;
    const Desc desc(a[0]);
    const at::Tensor* out = c.tensor(a[6]);
    if (!desc.d || !out) Py_RETURN_NONE;
    const int64_t rows = desc.d->batch, ci = desc.d->c_in, co = desc.d->c_out;
    void* x = c.operand(a[1], at::kBFloat16, {rows, ci}, false);
    void* w = c.operand(a[2], at::kBFloat16, {co, ci}, false);
    void* bias = c.operand(a[3], at::kFloat, {co});
    const int64_t act = c.integer(a[4]);
    const surgeon_dtype dt = c.type(*out);
    void* res = c.operand(a[5], out->scalar_type(), {rows, co});
    void* y = c.operand(a[6], out->scalar_type(), {rows, co}, false);
    void* pre = c.operand(a[7], at::kBFloat16, {rows, co});
    size_t bytes = 0;
    void* ws = c.workspace(a[8], &bytes);
    if (!c.ok) Py_RETURN_NONE;
    return answer(linear_fn(desc.d, x, w, static_cast<float*>(bias), static_cast<surgeon_activation>(act), res, dt, y, pre, ws, bytes,
                            c.stream()));
  });
}

// desc, dy, weight, pre, act, dx, dz, dbias, accumulate, workspace
PyObject* linear_grad(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    Args c;
    if (n != 10 || !linear_grad_fn) Py_RETURN_NONE;
    const Desc desc(a[0]);
    const at::Tensor* dy = c.tensor(a[1]);
    const at::Tensor* dx = c.tensor(a[5]);
    if (!desc.d || !dy || !dx) Py_RETURN_NONE;
    const int64_t rows = desc.d->batch, ci = desc.d->c_in, co = desc.d->c_out;
    const surgeon_dtype gdt = c.type(*dy), xdt = c.type(*dx);
    void* dyp = c.operand(a[1], dy->scalar_type(), {rows, co}, false);
    void* w = c.operand(a[2], at::kBFloat16, {co, ci}, false);
    void* pre = c.operand(a[3], at::kBFloat16, {rows, co});
    const int64_t act = c.integer(a[4]);
    void* dxp = c.operand(a[5], dx->scalar_type(), {rows, ci}, false);
    void* dz = c.operand(a[6], at::kFloat, {rows, co});
    void* dbias = c.operand(a[7], at::kFloat, {co});
    const bool accumulate = c.truth(a[8]);
    size_t bytes = 0;
    void* ws = c.workspace(a[9], &bytes);
    if (!c.ok) Py_RETURN_NONE;
    return answer(linear_grad_fn(desc.d, dyp, gdt, w, pre, static_cast<surgeon_activation>(act), xdt, dxp, static_cast<float*>(dz),
                                 static_cast<float*>(dbias), accumulate, ws, bytes, c.stream()));
  });
}

// list's address, count, device, max_norm (None: no clipping), norm, gi, workspace
PyObject* gradients(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    Args c;
    if (n != 7 || !gradient_norm_fn || !clip_gradients_fn) Py_RETURN_NONE;
    const auto* list = reinterpret_cast<const surgeon_gradient*>(static_cast<uintptr_t>(c.integer(a[0])));
    const int64_t count = c.integer(a[1]);
    if (c.integer(a[2]) != c.device || count > INT32_MAX) Py_RETURN_NONE;
    const bool clip = a[3] != Py_None;
    const double max_norm = clip ? c.number(a[3]) : 0.0;
    void* norm = c.operand(a[4], at::kDouble, {1}, false);
    void* gi = c.operand(a[5], at::kDouble, {count});
    size_t bytes = 0;
    void* ws = c.workspace(a[6], &bytes);
    if (!c.ok) Py_RETURN_NONE;
    return answer(clip ? clip_gradients_fn(list, static_cast<int32_t>(count), max_norm, static_cast<double*>(norm),
                                           static_cast<double*>(gi), ws, bytes, c.stream())
                       : gradient_norm_fn(list, static_cast<int32_t>(count), static_cast<double*>(norm), static_cast<double*>(gi), ws,
                                          bytes, c.stream()));
  });
}

template <typename F>
bool address(PyObject* o, F* to) {
  void* p = PyLong_AsVoidPtr(o);
  *to = reinterpret_cast<F>(p);
  return p != nullptr && !PyErr_Occurred();
}

// The entry points' addresses, in the order of their declarations above.
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 6) {
    PyErr_SetString(PyExc_TypeError, "bind takes six addresses");
    return nullptr;
  }
  if (!address(a[0], &layer_norm_fn) || !address(a[1], &layer_norm_grad_fn) || !address(a[2], &linear_fn) ||
      !address(a[3], &linear_grad_fn) || !address(a[4], &gradient_norm_fn) || !address(a[5], &clip_gradients_fn)) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "a null address");
    return nullptr;
  }
  Py_RETURN_NONE;
}

#define SURGEON_METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {SURGEON_METHOD(bind),        SURGEON_METHOD(layer_norm), SURGEON_METHOD(layer_norm_grad), SURGEON_METHOD(linear),
                         SURGEON_METHOD(linear_grad), SURGEON_METHOD(gradients),  {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__calls() { return PyModule_Create(&module); }
