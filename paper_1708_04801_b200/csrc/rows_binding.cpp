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

#include <cmath>

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

// contiguous [n, top] of one type
bool places(PyObject* o, const Call& c, at::ScalarType type, const char* what, Matrix* m) {
  const at::Tensor* t = on_device(o, c, what);
  if (!t) return false;
  if (t->scalar_type() != type || t->dim() != 2 || !t->is_contiguous()) {
    PyErr_Format(PyExc_TypeError, "%s: expected a contiguous 2-D %s tensor", what, at::toString(type));
    return false;
  }
  m->p = t->data_ptr();
  m->n = t->size(0);
  m->ld = t->size(1);
  return true;
}
bool same_places(const Matrix& a, const Matrix& b, const char* what) {
  if (a.n != b.n || a.ld != b.ld) PyErr_Format(PyExc_ValueError, "%s: [%lld, %lld], expected [%lld, %lld]", what, (long long)b.n, (long long)b.ld, (long long)a.n, (long long)a.ld);
  return a.n == b.n && a.ld == b.ld;
}
// the number of columns of a 2-D tensor, -1 with an error set
int64_t columns(PyObject* o, const Call& c, const char* what) {
  const at::Tensor* t = on_device(o, c, what);
  if (!t) return -1;
  if (t->dim() != 2) {
    PyErr_Format(PyExc_ValueError, "%s: expected a 2-D tensor", what);
    return -1;
  }
  return t->size(1);
}
// rows of either type, `cols` contiguous elements each, of the type of `like` where one is given
bool rows_like(PyObject* o, const Call& c, int64_t cols, const Matrix* like, const char* what, Matrix* m) {
  return matrix(o, c, like ? like->type : at::kFloat, like ? like->type : at::kBFloat16, cols, cols, what, m);
}
bool int32_of(PyObject* o, const char* what, int32_t* v) {
  long long n;
  if (!number(o, &n)) return false;
  if (n != (int32_t)n) PyErr_Format(PyExc_ValueError, "%s: %lld", what, n);
  *v = (int32_t)n;
  return n == (int32_t)n;
}

// A new tensor of rows that a call is about to write where a place has them: zeros elsewhere. 0, or the library's status
int cleared(const Call& c, const Matrix& where, const at::Tensor& rows) {
  const int64_t n = rows.size(0), d = rows.size(1);
  const at::Tensor marks = empty(c, {(n + 31) / 32}, {1}, at::kInt);
  return wpsgd_clear_rows(c.ctx, (const int32_t*)where.p, where.n, (int32_t)where.ld, rows.data_ptr(), element(rows.scalar_type()), d, d, n, (uint32_t*)marks.data_ptr());
}

// (head, node, n_nodes) -> (where, order, shard_off)
PyObject* sort_rows(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  Call c;
  Matrix node;
  int32_t n_nodes;
  if (!count(n_args, 6) || !head(args, &c) || !places(args[4], c, at::kInt, "node", &node) || !int32_of(args[5], "n_nodes", &n_nodes)) return nullptr;
  if (node.ld > INT32_MAX) return PyErr_Format(PyExc_ValueError, "node: too many places a row");
  at::Tensor where = empty(c, {node.n, node.ld}, {node.ld, 1}, at::kInt), order = empty(c, {node.n * node.ld}, {1}, at::kInt),
             off = empty(c, {std::max<int64_t>(n_nodes, 0) + 1}, {1}, at::kLong);
  const wpsgd_status st = wpsgd_sort_rows(c.ctx, (const int32_t*)node.p, node.n, (int32_t)node.ld, n_nodes, (int32_t*)where.data_ptr(), (int32_t*)order.data_ptr(), (int64_t*)off.data_ptr());
  if (st) return PyLong_FromLong(st);
  Output a, b, o;
  a.take(std::move(where));
  b.take(std::move(order));
  o.take(std::move(off));
  return PyTuple_Pack(3, a.o, b.o, o.o);
  END_HANDLE_TH_ERRORS
}

// (head, X, where, out or None) -> out
PyObject* gather_rows(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  Call c;
  Matrix x, where, to;
  int64_t d;
  if (!count(n_args, 7) || !head(args, &c) || (d = columns(args[4], c, "X")) < 0 || !rows_like(args[4], c, d, nullptr, "X", &x) || !places(args[5], c, at::kInt, "where", &where)) return nullptr;
  if (x.n != where.n) return PyErr_Format(PyExc_ValueError, "where has %lld rows, X %lld", (long long)where.n, (long long)x.n);
  Output out;
  if (args[6] == Py_None) {
    at::Tensor t = empty(c, {where.n * where.ld, d}, {d, 1}, x.type);
    if (const int st = cleared(c, where, t)) return PyLong_FromLong(st);
    out.take(std::move(t));
  } else {
    out.take(args[6]);
  }
  if (!rows_like(out.o, c, d, &x, "out", &to)) return nullptr;
  const wpsgd_status st = wpsgd_gather_rows(c.ctx, x.p, element(x.type), x.ld, d, (const int32_t*)where.p, where.n, (int32_t)where.ld, to.p, to.ld, to.n);
  if (st) return PyLong_FromLong(st);
  Py_INCREF(out.o);
  return out.o;
  END_HANDLE_TH_ERRORS
}

// (head, Y, where, weights or None, out or None) -> out
PyObject* combine_rows(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  Call c;
  Matrix y, where, weights, to;
  int64_t d;
  if (!count(n_args, 8) || !head(args, &c) || (d = columns(args[4], c, "Y")) < 0 || !rows_like(args[4], c, d, nullptr, "Y", &y) || !places(args[5], c, at::kInt, "where", &where)) return nullptr;
  if (args[6] != Py_None && (!places(args[6], c, at::kFloat, "weights", &weights) || !same_places(where, weights, "weights"))) return nullptr;
  Output out;
  if (args[7] == Py_None) out.take(empty(c, {where.n, d}, {d, 1}, y.type));
  else out.take(args[7]);
  if (!rows_like(out.o, c, d, &y, "out", &to)) return nullptr;
  if (to.n != where.n) return PyErr_Format(PyExc_ValueError, "out has %lld rows, where %lld", (long long)to.n, (long long)where.n);
  const wpsgd_status st = wpsgd_combine_rows(c.ctx, y.p, element(y.type), y.ld, d, y.n, (const int32_t*)where.p, (const float*)weights.p, where.n, (int32_t)where.ld, to.p, to.ld);
  if (st) return PyLong_FromLong(st);
  Py_INCREF(out.o);
  return out.o;
  END_HANDLE_TH_ERRORS
}

// (head, dout, Y, where, weights or None, dY or None, dweights or None) -> (dY, dweights)
PyObject* combine_rows_grad(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  Call c;
  Matrix y, dout, where, weights, to, tow;
  int64_t d;
  if (!count(n_args, 10) || !head(args, &c) || (d = columns(args[5], c, "Y")) < 0 || !rows_like(args[5], c, d, nullptr, "Y", &y) || !rows_like(args[4], c, d, &y, "dout", &dout) ||
      !places(args[6], c, at::kInt, "where", &where))
    return nullptr;
  if (args[7] != Py_None && (!places(args[7], c, at::kFloat, "weights", &weights) || !same_places(where, weights, "weights"))) return nullptr;
  if (dout.n != where.n) return PyErr_Format(PyExc_ValueError, "dout has %lld rows, where %lld", (long long)dout.n, (long long)where.n);
  Output dy, dw;
  if (args[8] == Py_None) {
    at::Tensor t = empty(c, {y.n, d}, {d, 1}, y.type);
    if (const int st = cleared(c, where, t)) return PyLong_FromLong(st);
    dy.take(std::move(t));
  } else {
    dy.take(args[8]);
  }
  if (args[9] == Py_None) dw.take(empty(c, {where.n, where.ld}, {where.ld, 1}, at::kFloat));
  else dw.take(args[9]);
  if (!rows_like(dy.o, c, d, &y, "dY", &to) || !places(dw.o, c, at::kFloat, "dweights", &tow) || !same_places(where, tow, "dweights")) return nullptr;
  if (to.n != y.n) return PyErr_Format(PyExc_ValueError, "dY has %lld rows, Y %lld", (long long)to.n, (long long)y.n);
  const wpsgd_status st = wpsgd_combine_rows_grad(c.ctx, dout.p, dout.ld, y.p, y.ld, element(y.type), d, y.n, (const int32_t*)where.p, (const float*)weights.p, where.n, (int32_t)where.ld,
                                                  to.p, to.ld, (float*)tow.p);
  return st ? PyLong_FromLong(st) : pair(dy, dw);
  END_HANDLE_TH_ERRORS
}

// rows [n, heads, width] of one type with heads one behind the other; ld: elements from row to row
struct Heads {
  const void* p = nullptr;
  int64_t n = 0, heads = 0, width = 0, ld = 0;
};
bool heads_of(PyObject* o, const Call& c, at::ScalarType type, int64_t dims, const char* what, Heads* m) {
  const at::Tensor* t = on_device(o, c, what);
  if (!t) return false;
  if (t->scalar_type() != type) {
    PyErr_Format(PyExc_TypeError, "%s: expected dtype %s, got %s", what, at::toString(type), at::toString(t->scalar_type()));
    return false;
  }
  if (t->dim() != dims) {
    PyErr_Format(PyExc_ValueError, "%s: expected %lld dimensions", what, (long long)dims);
    return false;
  }
  m->n = t->size(0);
  m->heads = t->size(1);
  m->width = dims == 3 ? t->size(2) : 1;
  if ((m->width > 1 && t->stride(2) != 1) || (m->heads > 1 && t->stride(1) != m->width)) {
    PyErr_Format(PyExc_ValueError, "%s: the heads of a row must lie one behind the other", what);
    return false;
  }
  m->ld = m->n > 1 ? t->stride(0) : m->heads * m->width;
  m->p = t->data_ptr();
  return true;
}
bool fits32(int64_t v) { return v >= 0 && v <= INT32_MAX; }
// q, k, v, g, beta, scale
bool delta_rows(PyObject* const* a, const Call& c, wpsgd_delta_rows* r, at::ScalarType* type) {
  if (!THPVariable_Check(a[0])) {
    PyErr_Format(PyExc_TypeError, "q: expected a tensor");
    return false;
  }
  *type = THPVariable_Unpack(a[0]).scalar_type();
  if (*type != at::kFloat && *type != at::kBFloat16) {
    PyErr_Format(PyExc_TypeError, "q: expected dtype Float or BFloat16, got %s", at::toString(*type));
    return false;
  }
  Heads q, k, v, g, beta;
  if (!heads_of(a[0], c, *type, 3, "q", &q) || !heads_of(a[1], c, *type, 3, "k", &k) || !heads_of(a[2], c, *type, 3, "v", &v) || !heads_of(a[3], c, *type, 2, "g", &g) ||
      !heads_of(a[4], c, *type, 2, "beta", &beta))
    return false;
  if (k.n != q.n || v.n != q.n || g.n != q.n || beta.n != q.n || k.heads != q.heads || k.width != q.width || g.heads != v.heads || beta.heads != v.heads || !fits32(q.heads) ||
      !fits32(q.width) || !fits32(v.heads) || !fits32(v.width)) {
    PyErr_Format(PyExc_ValueError, "q and k are [n, heads_k, dk], v [n, heads_v, dv], g and beta [n, heads_v]");
    return false;
  }
  double scale = 0.0;
  if (a[5] == Py_None) scale = 1.0 / std::sqrt((double)q.width);
  else scale = PyFloat_AsDouble(a[5]);
  if (scale == -1.0 && PyErr_Occurred()) return false;
  *r = {q.p, k.p, v.p, g.p, beta.p, q.ld, k.ld, v.ld, g.ld, beta.ld, nullptr, q.n, 0, (int32_t)q.heads, (int32_t)v.heads, (int32_t)q.width, (int32_t)v.width, element(*type), (float)scale};
  return true;
}
bool shards(PyObject* o, const Call& c, wpsgd_delta_rows* r) {
  const at::Tensor* t = on_device(o, c, "shard_off");
  if (!t) return false;
  if (t->scalar_type() != at::kLong || t->dim() != 1 || !t->is_contiguous() || t->numel() < 1 || !fits32(t->numel() - 1)) {
    PyErr_Format(PyExc_TypeError, "shard_off: expected a contiguous int64 tensor [n_chains + 1]");
    return false;
  }
  r->shard_off = (const int64_t*)t->data_ptr();
  r->n_chains = (int32_t)(t->numel() - 1);
  return true;
}
// models [n, heads_v, dv, dk], or None where that is allowed (then *p stays NULL)
bool models(PyObject* o, const Call& c, const wpsgd_delta_rows& r, int64_t n, const char* what, float** p, int64_t* got = nullptr) {
  if (o == Py_None && !got) return true;
  const at::Tensor* t = on_device(o, c, what);
  if (!t) return false;
  if (t->scalar_type() != at::kFloat || !t->is_contiguous()) {
    PyErr_Format(PyExc_TypeError, "%s: expected a contiguous float32 tensor", what);
    return false;
  }
  if (t->dim() != 4 || (n >= 0 && t->size(0) != n) || t->size(1) != r.heads_v || t->size(2) != r.dv || t->size(3) != r.dk) {
    PyErr_Format(PyExc_ValueError, "%s: expected [%s, heads_v, dv, dk]", what, n >= 0 ? "n_chains" : "n_slots");
    return false;
  }
  if (got) *got = t->size(0);
  *p = (float*)t->data_ptr();
  return true;
}
bool rows_out(PyObject* o, const Call& c, at::ScalarType type, const wpsgd_delta_rows& r, const char* what, Heads* m) {
  if (!heads_of(o, c, type, 3, what, m)) return false;
  if (m->n != r.n_rows || m->heads != r.heads_v || m->width != r.dv) {
    PyErr_Format(PyExc_ValueError, "%s: expected [n, heads_v, dv]", what);
    return false;
  }
  return true;
}
// Rows that have no workspace are refused by the call that it is for, with its text
void workspace(const Call& c, const wpsgd_delta_rows& r, wpsgd_delta_use use, at::Tensor* ws, int64_t* bytes) {
  if (wpsgd_delta_workspace(&r, use, bytes) == WPSGD_OK) *ws = empty(c, {*bytes}, {1}, at::kByte);
}

// (head, q, k, v, g, beta, scale or None, shard_off, W0 or None, W_out or None, out or None, save) -> (out, W, workspace or None)
PyObject* delta_run(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  Call c;
  wpsgd_delta_rows r;
  at::ScalarType type;
  if (!count(n_args, 15) || !head(args, &c) || !delta_rows(args + 4, c, &r, &type) || !shards(args[10], c, &r)) return nullptr;
  float *W0 = nullptr, *W1 = nullptr;
  Output W, out, saved;
  if (args[12] == Py_None) W.take(empty(c, {r.n_chains, r.heads_v, r.dv, r.dk}, {(int64_t)r.heads_v * r.dv * r.dk, (int64_t)r.dv * r.dk, r.dk, 1}, at::kFloat));
  else W.take(args[12]);
  if (args[13] == Py_None) out.take(empty(c, {r.n_rows, r.heads_v, r.dv}, {(int64_t)r.heads_v * r.dv, r.dv, 1}, type));
  else out.take(args[13]);
  Heads o;
  if (!models(args[11], c, r, r.n_chains, "W0", &W0) || !models(W.o, c, r, r.n_chains, "W_out", &W1) || !rows_out(out.o, c, type, r, "out", &o)) return nullptr;
  const wpsgd_delta_use use = args[14] == Py_True ? WPSGD_DELTA_RUN_SAVE : WPSGD_DELTA_RUN;
  at::Tensor ws;
  int64_t bytes = 0;
  workspace(c, r, use, &ws, &bytes);
  const wpsgd_delta_use whole = args[13] == Py_None ? (wpsgd_delta_use)(use | WPSGD_DELTA_NEW_OUT) : use;
  const wpsgd_status st = wpsgd_delta_run(c.ctx, &r, W0, W1, (void*)o.p, o.ld, whole, bytes ? ws.data_ptr() : nullptr, bytes);
  if (st) return PyLong_FromLong(st);
  if (use == WPSGD_DELTA_RUN_SAVE) saved.take(std::move(ws));
  else saved.take(Py_None);
  return PyTuple_Pack(3, out.o, W.o, saved.o);
  END_HANDLE_TH_ERRORS
}

// (head, q, k, v, g, beta, scale or None, shard_off, saved, dout, dW or None, whether dW0 is asked for) -> (dq, dk, dv, dg, dbeta, dW0 or None)
PyObject* delta_grad(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  Call c;
  wpsgd_delta_rows r;
  at::ScalarType type;
  if (!count(n_args, 15) || !head(args, &c) || !delta_rows(args + 4, c, &r, &type) || !shards(args[10], c, &r)) return nullptr;
  const at::Tensor* saved = on_device(args[11], c, "saved");
  if (!saved) return nullptr;
  Heads dout;
  float *dW = nullptr, *dW0 = nullptr;
  if (!rows_out(args[12], c, type, r, "dout", &dout) || !models(args[13], c, r, r.n_chains, "dW", &dW)) return nullptr;
  Output dq, dk, dv, dg, db, dw;
  const int64_t n = r.n_rows, hk = r.heads_k, hv = r.heads_v;
  const auto rows = [&](int64_t heads, int64_t width) { return empty(c, {n, heads, width}, {heads * width, width, 1}, type); };
  at::Tensor tq = rows(hk, r.dk), tk = rows(hk, r.dk), tv = rows(hv, r.dv), tg = empty(c, {n, hv}, {hv, 1}, type), tb = empty(c, {n, hv}, {hv, 1}, type), ws;
  if (args[14] == Py_True) {
    at::Tensor t = empty(c, {r.n_chains, hv, r.dv, r.dk}, {hv * r.dv * r.dk, (int64_t)r.dv * r.dk, r.dk, 1}, at::kFloat);
    dW0 = (float*)t.data_ptr();
    dw.take(std::move(t));
  } else {
    dw.take(Py_None);
  }
  int64_t bytes = 0;
  workspace(c, r, WPSGD_DELTA_GRAD, &ws, &bytes);
  const wpsgd_status st = wpsgd_delta_grad(c.ctx, &r, saved->data_ptr(), (int64_t)saved->numel(), dout.p, dout.ld, dW, tq.data_ptr(), tk.data_ptr(), tv.data_ptr(), tg.data_ptr(), tb.data_ptr(), dW0,
                        bytes ? ws.data_ptr() : nullptr, bytes);
  if (st) return PyLong_FromLong(st);
  dq.take(std::move(tq));
  dk.take(std::move(tk));
  dv.take(std::move(tv));
  dg.take(std::move(tg));
  db.take(std::move(tb));
  return PyTuple_Pack(6, dq.o, dk.o, dv.o, dg.o, db.o, dw.o);
  END_HANDLE_TH_ERRORS
}

// (head, q, k, v, g, beta, scale or None, W, slots or None, out or None) -> out
PyObject* delta_step(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  Call c;
  wpsgd_delta_rows r;
  at::ScalarType type;
  float* W = nullptr;
  int64_t n_slots = 0;
  const int32_t* slots = nullptr;
  if (!count(n_args, 13) || !head(args, &c) || !delta_rows(args + 4, c, &r, &type) || !models(args[10], c, r, -1, "W", &W, &n_slots)) return nullptr;
  if (args[11] != Py_None) {
    const at::Tensor* t = on_device(args[11], c, "slots");
    if (!t) return nullptr;
    if (t->scalar_type() != at::kInt || t->dim() != 1 || !t->is_contiguous()) return PyErr_Format(PyExc_TypeError, "slots: expected a contiguous int32 tensor");
    if (t->numel() != r.n_rows) return PyErr_Format(PyExc_ValueError, "slots: %lld, expected %lld", (long long)t->numel(), (long long)r.n_rows);
    slots = (const int32_t*)t->data_ptr();
  }
  Output out;
  if (args[12] == Py_None) out.take(empty(c, {r.n_rows, r.heads_v, r.dv}, {(int64_t)r.heads_v * r.dv, r.dv, 1}, type));
  else out.take(args[12]);
  Heads o;
  if (!rows_out(out.o, c, type, r, "out", &o)) return nullptr;
  const wpsgd_status st = wpsgd_delta_step(c.ctx, &r, W, slots, n_slots, (void*)o.p, o.ld);
  if (st) return PyLong_FromLong(st);
  Py_INCREF(out.o);
  return out.o;
  END_HANDLE_TH_ERRORS
}

PyMethodDef methods[] = {
    {"quantize_rows", (PyCFunction)(void*)quantize_rows, METH_FASTCALL, nullptr},
    {"margins_fp8", (PyCFunction)(void*)margins_fp8, METH_FASTCALL, nullptr},
    {"objective_grad", (PyCFunction)(void*)objective_grad, METH_FASTCALL, nullptr},
    {"objective_grad_fp8", (PyCFunction)(void*)objective_grad_fp8, METH_FASTCALL, nullptr},
    {"grad_norm", (PyCFunction)(void*)grad_norm, METH_FASTCALL, nullptr},
    {"sort_rows", (PyCFunction)(void*)sort_rows, METH_FASTCALL, nullptr},
    {"gather_rows", (PyCFunction)(void*)gather_rows, METH_FASTCALL, nullptr},
    {"combine_rows", (PyCFunction)(void*)combine_rows, METH_FASTCALL, nullptr},
    {"combine_rows_grad", (PyCFunction)(void*)combine_rows_grad, METH_FASTCALL, nullptr},
    {"delta_run", (PyCFunction)(void*)delta_run, METH_FASTCALL, nullptr},
    {"delta_grad", (PyCFunction)(void*)delta_grad, METH_FASTCALL, nullptr},
    {"delta_step", (PyCFunction)(void*)delta_step, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_rows", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__rows() {
  PyObject* m = PyModule_Create(&module);
  if (m && PyModule_AddStringConstant(m, "built_for", ROWS_BUILT_FOR) < 0) Py_CLEAR(m);
  return m;
}
