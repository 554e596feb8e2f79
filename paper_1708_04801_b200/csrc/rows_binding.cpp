// Python entry of the operators on whole sets of rows (include/wpsgd.h): checks of tensors, output tensors, one call into the library. Marshalling
// only, as binding.py's, in C++ because these calls take a few microseconds on the GPU and as many in Python: the margins of one row on
// 1024 models took 13 us a call through ctypes and take 4.6 to 4.9 this way, 2.8 of them on the host.
//
// Every function takes the context's handle, device, stream and d first. A library error comes back as its status (an int).
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/wpsgd.h"

namespace {

constexpr int64_t kBlock = 128;

struct Call {
  wpsgd_ctx* ctx;
  int device;
  cudaStream_t stream;
  int64_t d;
};

bool number(PyObject* o, long long* v) {
  *v = PyLong_AsLongLong(o);
  return !(*v == -1 && PyErr_Occurred());
}
bool head(PyObject* const* args, Call* c) {
  long long h, dev, st, d;
  if (!number(args[0], &h) || !number(args[1], &dev) || !number(args[2], &st) || !number(args[3], &d)) return false;
  *c = {(wpsgd_ctx*)h, (int)dev, (cudaStream_t)st, d};
  return true;
}
bool count(Py_ssize_t n, Py_ssize_t want) {
  if (n != want) PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", want, n);
  return n == want;
}

// The tensor behind `o` if it is one on the context's device
const at::Tensor* on_device(PyObject* o, const Call& c, const char* what) {
  if (THPVariable_Check(o)) {
    const at::Tensor& t = THPVariable_Unpack(o);
    if (t.is_cuda() && t.get_device() == c.device) return &t;
  }
  PyErr_Format(PyExc_TypeError, "%s: expected a CUDA tensor on the context's device", what);
  return nullptr;
}

struct Matrix {
  void* p = nullptr;
  int64_t n = 0, ld = 0;
  at::ScalarType type = at::kFloat;
};
// rows of `cols` contiguous elements of one of two types; ld_of_one: the stride to pass for a single row
bool matrix(PyObject* o, const Call& c, at::ScalarType a, at::ScalarType b, int64_t cols, int64_t ld_of_one, const char* what, Matrix* m) {
  const at::Tensor* t = on_device(o, c, what);
  if (!t) return false;
  m->type = t->scalar_type();
  if (m->type != a && m->type != b) {
    PyErr_Format(PyExc_TypeError, "%s: expected dtype %s or %s, got %s", what, at::toString(a), at::toString(b), at::toString(m->type));
    return false;
  }
  if (t->dim() != 2 || t->size(1) != cols || (cols > 1 && t->stride(1) != 1)) {
    PyErr_Format(PyExc_ValueError, "%s: expected rows of %lld contiguous elements", what, (long long)cols);
    return false;
  }
  m->n = t->size(0);
  m->ld = m->n > 1 ? t->stride(0) : ld_of_one;
  m->p = t->data_ptr();
  return true;
}
// packed rows and their scales
bool packed(PyObject* q, PyObject* s, const Call& c, const char* what, const char* what_scales, Matrix* m, Matrix* scales) {
  const int64_t nb = (c.d + kBlock - 1) / kBlock;
  if (!matrix(q, c, at::kFloat8_e4m3fn, at::kByte, c.d, (c.d + 15) / 16 * 16, what, m)) return false;
  if (!matrix(s, c, at::kFloat, at::kFloat, nb, nb, what_scales, scales)) return false;
  if (m->n != scales->n) {
    PyErr_Format(PyExc_ValueError, "%s: %lld rows, but scales of %lld", what, (long long)m->n, (long long)scales->n);
    return false;
  }
  return true;
}
bool vector(PyObject* o, const Call& c, int64_t n, const char* what, float** p) {
  const at::Tensor* t = on_device(o, c, what);
  if (!t) return false;
  if (t->scalar_type() != at::kFloat || !t->is_contiguous()) {
    PyErr_Format(PyExc_TypeError, "%s: expected a contiguous float32 tensor", what);
    return false;
  }
  if (t->numel() < n) {
    PyErr_Format(PyExc_ValueError, "%s: %lld elements, expected %lld", what, (long long)t->numel(), (long long)n);
    return false;
  }
  *p = (float*)t->data_ptr();
  return true;
}

// A tensor for the context's stream to write: allocated for that stream, so that its memory is not reused under it.
at::Tensor empty(const Call& c, at::IntArrayRef sizes, at::IntArrayRef strides, at::ScalarType type) {
  const auto options = at::TensorOptions().dtype(type).device(at::kCUDA, (c10::DeviceIndex)c.device);
  if (c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)c.device).stream() == c.stream) return at::empty_strided(sizes, strides, options);
  const c10::cuda::CUDAStreamGuard guard(c10::cuda::getStreamFromExternal(c.stream, (c10::DeviceIndex)c.device));
  return at::empty_strided(sizes, strides, options);
}
// `o`, or a new tensor where it is None
struct Output {
  PyObject* o = nullptr;  // owned
  ~Output() { Py_XDECREF(o); }
  void take(PyObject* given) { Py_INCREF(o = given); }
  void take(at::Tensor&& t) { o = THPVariable_Wrap(std::move(t)); }
};
PyObject* pair(const Output& a, const Output& b) { return PyTuple_Pack(2, a.o, b.o); }

wpsgd_xtype element(at::ScalarType t) { return t == at::kBFloat16 ? WPSGD_X_BF16 : WPSGD_X_F32; }

// (head, X, out or None, scales or None) -> (out, scales)
PyObject* quantize_rows(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  Call c;
  Matrix x, q, s;
  if (!count(n_args, 7) || !head(args, &c) || !matrix(args[4], c, at::kFloat, at::kBFloat16, c.d, c.d, "X", &x)) return nullptr;
  const int64_t width = (c.d + 15) / 16 * 16, nb = (c.d + kBlock - 1) / kBlock;
  Output out, scales;
  if (args[5] == Py_None) out.take(empty(c, {x.n, c.d}, {width, 1}, at::kFloat8_e4m3fn));
  else out.take(args[5]);
  if (args[6] == Py_None) scales.take(empty(c, {x.n, nb}, {nb, 1}, at::kFloat));
  else scales.take(args[6]);
  if (!packed(out.o, scales.o, c, "out", "scales", &q, &s)) return nullptr;
  if (q.n != x.n) return PyErr_Format(PyExc_ValueError, "out has %lld rows, X %lld", (long long)q.n, (long long)x.n);
  const wpsgd_status st = wpsgd_quantize_rows(c.ctx, x.p, element(x.type), x.ld, x.n, (uint8_t*)q.p, q.ld, (float*)s.p, s.ld);
  return st ? PyLong_FromLong(st) : pair(out, scales);
  END_HANDLE_TH_ERRORS
}

// (head, Q, q_scales, M, m_scales, out or None, whether a new one is bf16) -> out
PyObject* margins_fp8(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  Call c;
  Matrix q, qs, m, ms, z;
  if (!count(n_args, 10) || !head(args, &c) || !packed(args[4], args[5], c, "Q", "Q scales", &q, &qs) || !packed(args[6], args[7], c, "M", "M scales", &m, &ms)) return nullptr;
  Output out;
  if (args[8] == Py_None) out.take(empty(c, {q.n, m.n}, {m.n, 1}, args[9] == Py_True ? at::kBFloat16 : at::kFloat));
  else out.take(args[8]);
  if (!matrix(out.o, c, at::kFloat, at::kBFloat16, m.n, m.n, "out", &z)) return nullptr;
  if (z.n != q.n) return PyErr_Format(PyExc_ValueError, "out has %lld rows, Q %lld", (long long)z.n, (long long)q.n);
  const wpsgd_status st = wpsgd_margins_fp8(c.ctx, (const uint8_t*)q.p, q.ld, (const float*)qs.p, qs.ld, q.n, (const uint8_t*)m.p, m.ld, (const float*)ms.p, ms.ld, m.n, z.p,
                                            element(z.type), z.ld);
  if (st) return PyLong_FromLong(st);
  Py_INCREF(out.o);
  return out.o;
  END_HANDLE_TH_ERRORS
}

// the arguments that both gradients share: y, w, lambda, loss, grad or None, out or None
struct GradientArgs {
  float *y, *w, *g, *o;
  double lambda;
  long long loss;
  Output grad, out;
  bool read(PyObject* const* a, const Call& c, int64_t n) {
    if (!vector(a[0], c, n, "y", &y) || !vector(a[1], c, c.d, "w", &w)) return false;
    lambda = PyFloat_AsDouble(a[2]);
    if ((lambda == -1.0 && PyErr_Occurred()) || !number(a[3], &loss)) return false;
    if (loss != (int)loss) loss = -1;  // unknown, as it is, and not what its low 32 bits are
    if (a[4] == Py_None) grad.take(empty(c, {c.d}, {1}, at::kFloat));
    else grad.take(a[4]);
    if (a[5] == Py_None) out.take(empty(c, {2}, {1}, at::kFloat));
    else out.take(a[5]);
    return vector(grad.o, c, c.d, "grad", &g) && vector(out.o, c, 2, "out", &o);
  }
};

// (head, X, y, w, lambda, loss, grad or None, out or None) -> (out, grad)
PyObject* objective_grad(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  Call c;
  Matrix x;
  GradientArgs a;
  if (!count(n_args, 11) || !head(args, &c) || !matrix(args[4], c, at::kFloat, at::kBFloat16, c.d, c.d, "X", &x) || !a.read(args + 5, c, x.n)) return nullptr;
  const wpsgd_status st = wpsgd_objective_grad(c.ctx, x.p, element(x.type), x.ld, a.y, x.n, a.w, (float)a.lambda, (wpsgd_loss)a.loss, a.g, a.o);
  return st ? PyLong_FromLong(st) : pair(a.out, a.grad);
  END_HANDLE_TH_ERRORS
}

// (head, Q, scales, y, w, lambda, loss, grad or None, out or None) -> (out, grad)
PyObject* objective_grad_fp8(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  Call c;
  Matrix q, s;
  GradientArgs a;
  if (!count(n_args, 12) || !head(args, &c) || !packed(args[4], args[5], c, "Q", "Q scales", &q, &s) || !a.read(args + 6, c, q.n)) return nullptr;
  const wpsgd_status st = wpsgd_objective_grad_fp8(c.ctx, (const uint8_t*)q.p, q.ld, (const float*)s.p, s.ld, a.y, q.n, a.w, (float)a.lambda, (wpsgd_loss)a.loss, a.g, a.o);
  return st ? PyLong_FromLong(st) : pair(a.out, a.grad);
  END_HANDLE_TH_ERRORS
}

// (head, list, max_norm or None for the norm alone, norm or None) -> norm
PyObject* grad_norm(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  Call c;
  long long list;
  if (!count(n_args, 7) || !head(args, &c) || !number(args[4], &list)) return nullptr;
  const double max_norm = args[5] == Py_None ? 0.0 : PyFloat_AsDouble(args[5]);
  if (max_norm == -1.0 && PyErr_Occurred()) return nullptr;
  Output norm;
  float* p;
  if (args[6] == Py_None) norm.take(empty(c, {1}, {1}, at::kFloat));
  else norm.take(args[6]);
  if (!vector(norm.o, c, 1, "norm", &p)) return nullptr;
  const wpsgd_status st = args[5] == Py_None ? wpsgd_grad_norm(c.ctx, (const wpsgd_grad_list*)list, p) : wpsgd_clip_grad_norm(c.ctx, (const wpsgd_grad_list*)list, max_norm, p);
  if (st) return PyLong_FromLong(st);
  Py_INCREF(norm.o);
  return norm.o;
  END_HANDLE_TH_ERRORS
}

PyMethodDef methods[] = {
    {"quantize_rows", (PyCFunction)(void*)quantize_rows, METH_FASTCALL, nullptr},
    {"margins_fp8", (PyCFunction)(void*)margins_fp8, METH_FASTCALL, nullptr},
    {"objective_grad", (PyCFunction)(void*)objective_grad, METH_FASTCALL, nullptr},
    {"objective_grad_fp8", (PyCFunction)(void*)objective_grad_fp8, METH_FASTCALL, nullptr},
    {"grad_norm", (PyCFunction)(void*)grad_norm, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_rows", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__rows() {
  PyObject* m = PyModule_Create(&module);
  if (m && PyModule_AddStringConstant(m, "built_for", ROWS_BUILT_FOR) < 0) Py_CLEAR(m);
  return m;
}
