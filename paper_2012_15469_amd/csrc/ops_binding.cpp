// Python module _ops: the operators of cada_ops.h on torch tensors.  Checks and marshalling only (shapes, types, strides, outputs and workspaces from
// torch's allocator); in C++ because a call of a small layer takes the GPU a few microseconds and took Python's own checks ten.
#include <Python.h>

#include <ATen/ATen.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdarg>
#include <cstdio>

#include "cada_ops.h"

namespace {

PyObject *g_error;      // the binding's CadaError

struct Failed {};       // a Python error is set
[[noreturn]] void refuse(const char *fmt, ...) {
  char text[400];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(text, sizeof(text), fmt, ap);
  va_end(ap);
  PyErr_SetString(PyExc_ValueError, text);
  throw Failed{};
}
void check(int rc) {
  if (rc == CADA_OK) return;
  PyErr_Format(g_error, "libcada error %d: %s", rc, cada_last_error());
  throw Failed{};
}

const char *type_name(at::ScalarType t) { return at::toString(t); }
int type_of(const at::Tensor &t) { return t.scalar_type() == at::kFloat ? CADA_F32 : CADA_BF16; }

// The tensor of an argument; None gives nullptr.
const at::Tensor *tensor(PyObject *o, const char *name) {
  if (o == Py_None) return nullptr;
  if (!THPVariable_Check(o)) refuse("%s must be a tensor", name);
  return &THPVariable_Unpack(o);
}
const at::Tensor &needed(PyObject *o, const char *name) {
  const at::Tensor *t = tensor(o, name);
  if (!t) refuse("%s must be a tensor", name);
  return *t;
}
void first(const at::Tensor &t, const char *name) {
  if (!t.is_cuda() || (t.scalar_type() != at::kFloat && t.scalar_type() != at::kBFloat16) || t.dim() != 2)
    refuse("%s must be a two-dimensional float32 or bfloat16 tensor on a GPU, it is %lld-dimensional %s on %s", name, (long long)t.dim(), type_name(t.scalar_type()), t.device().str().c_str());
}
// Address of a [rows, cols] tensor like `like`, and the elements from one row to the next.
template <typename P> void table(const char *name, const at::Tensor &t, int64_t rows, int64_t cols, const at::Tensor &like, P **ptr, int64_t *ld) {
  if (t.dim() != 2 || t.size(0) != rows || t.size(1) != cols) refuse("%s must be [%lld, %lld]", name, (long long)rows, (long long)cols);
  if (t.scalar_type() != like.scalar_type() || t.device() != like.device())
    refuse("%s must be %s on %s like the other operands, it is %s on %s", name, type_name(like.scalar_type()), like.device().str().c_str(), type_name(t.scalar_type()), t.device().str().c_str());
  const int64_t s0 = t.stride(0), s1 = t.stride(1);
  if ((cols > 1 && s1 != 1) || (rows > 1 && s0 < cols)) refuse("%s must have contiguous rows that do not overlap (strides %lld, %lld)", name, (long long)s0, (long long)s1);
  *ptr = t.data_ptr();
  *ld = rows > 1 ? s0 : std::max(s0, cols);
}
template <typename P> void vector(const char *name, const at::Tensor &t, int64_t n, const at::Tensor &like, P **ptr) {
  if (t.dim() != 1 || t.size(0) != n || t.scalar_type() != like.scalar_type() || t.device() != like.device() || (n > 1 && t.stride(0) != 1))
    refuse("%s must be a contiguous %s [%lld] on %s", name, type_name(like.scalar_type()), (long long)n, like.device().str().c_str());
  *ptr = t.data_ptr();
}
at::Tensor fresh(at::IntArrayRef size, const at::Tensor &like) { return at::empty(size, like.options()); }

// Workspace of a call: the one handed in, or one of the size that it asks for (torch's blocks start on 512 bytes).
template <typename A> at::Tensor workspace(A *a, PyObject *given, int (*size_of)(A *), const at::Tensor &like) {
  at::Tensor ws;
  if (const at::Tensor *t = tensor(given, "workspace")) {
    if (t->device() != like.device() || t->scalar_type() != at::kByte || !t->is_contiguous()) refuse("workspace must be a contiguous uint8 tensor on %s", like.device().str().c_str());
    ws = *t;
    a->workspace_bytes = (size_t)t->numel();
  } else {
    check(size_of(a));
    if (a->workspace_bytes == 0) return ws;
    ws = at::empty({(int64_t)a->workspace_bytes}, like.options().dtype(at::kByte));
  }
  a->workspace = ws.data_ptr();
  return ws;
}

PyObject *wrap(const at::Tensor &t) {
  if (!t.defined()) Py_RETURN_NONE;
  return THPVariable_Wrap(t);
}
PyObject *triple(const at::Tensor &a, const at::Tensor &b, const at::Tensor &c) {
  PyObject *x = wrap(a), *y = wrap(b), *z = wrap(c);
  return Py_BuildValue("(NNN)", x, y, z);
}
template <typename F> PyObject *guarded(F f) {
  try {
    return f();
  } catch (const Failed &) {
    return nullptr;
  } catch (...) {
    torch::translate_exception_to_python(std::current_exception());      // (torch's own: out of memory among them)
    return nullptr;
  }
}
void *stream_of(PyObject *o) { return PyLong_AsVoidPtr(o); }

// (x, w, bias, residual, act, keep_pre, out, pre, workspace, stream) -> (y, pre)
PyObject *linear_forward(PyObject *, PyObject *const *args, Py_ssize_t n_args) {
  return guarded([&]() -> PyObject * {
    if (n_args != 10) refuse("linear_forward takes 10 arguments");
    const at::Tensor &x = needed(args[0], "x"), &w = needed(args[1], "w");
    first(x, "x");
    if (w.dim() != 2) refuse("w must be [in, out]");
    cada_linear a{};
    a.rows = x.size(0); a.in = x.size(1); a.out = w.size(1); a.type = type_of(x); a.act = (int)PyLong_AsLong(args[4]);
    void *p;
    table("x", x, a.rows, a.in, x, &p, &a.ldx); a.x = p;
    table("w", w, a.in, a.out, x, &p, &a.ldw); a.w = p;
    if (const at::Tensor *b = tensor(args[2], "bias")) { vector("bias", *b, a.out, x, &p); a.bias = p; }
    if (const at::Tensor *r = tensor(args[3], "residual")) { table("residual", *r, a.rows, a.out, x, &p, &a.ldr); a.residual = p; }
    const at::Tensor *given = tensor(args[6], "out"), *given_pre = tensor(args[7], "pre");
    const at::Tensor y = given ? *given : fresh({a.rows, a.out}, x);
    table("out", y, a.rows, a.out, x, &a.y, &a.ldy);
    at::Tensor pre;
    if (given_pre || args[5] == Py_True) {
      pre = given_pre ? *given_pre : fresh({a.rows, a.out}, x);
      table("pre", pre, a.rows, a.out, x, &a.pre, &a.ldpre);
    }
    const at::Tensor ws = workspace(&a, args[8], cada_linear_forward_workspace, x);
    a.stream = stream_of(args[9]);
    check(cada_linear_forward(&a));
    PyObject *py = wrap(y), *pp = wrap(pre);
    return Py_BuildValue("(NN)", py, pp);
  });
}

// (dy, x, w, pre, act, need_dx, need_dw, need_db, dx, dw, db, workspace, stream) -> (dx, dw, db)
PyObject *linear_backward(PyObject *, PyObject *const *args, Py_ssize_t n_args) {
  return guarded([&]() -> PyObject * {
    if (n_args != 13) refuse("linear_backward takes 13 arguments");
    const at::Tensor &dy = needed(args[0], "dy"), &x = needed(args[1], "x"), &w = needed(args[2], "w");
    first(dy, "dy");
    if (x.dim() != 2 || w.dim() != 2) refuse("x must be [rows, in] and w [in, out]");
    cada_linear_grad a{};
    a.rows = dy.size(0); a.in = x.size(1); a.out = dy.size(1); a.type = type_of(dy); a.act = (int)PyLong_AsLong(args[4]);
    void *p;
    table("dy", dy, a.rows, a.out, dy, &p, &a.lddy); a.dy = p;
    table("x", x, a.rows, a.in, dy, &p, &a.ldx); a.x = p;
    table("w", w, a.in, a.out, dy, &p, &a.ldw); a.w = p;
    if (a.act != CADA_ACT_NONE) {
      const at::Tensor *pre = tensor(args[3], "pre");
      if (!pre) refuse("an activation's gradient needs pre");
      table("pre", *pre, a.rows, a.out, dy, &p, &a.ldpre); a.pre = p;
    }
    at::Tensor dx, dw, db;
    if (args[5] == Py_True) {
      const at::Tensor *t = tensor(args[8], "dx");
      dx = t ? *t : fresh({a.rows, a.in}, dy);
      table("dx", dx, a.rows, a.in, dy, &a.dx, &a.lddx);
    }
    if (args[6] == Py_True) {
      const at::Tensor *t = tensor(args[9], "dw");
      dw = t ? *t : fresh({a.in, a.out}, dy);
      table("dw", dw, a.in, a.out, dy, &a.dw, &a.lddw);
    }
    if (args[7] == Py_True) {
      const at::Tensor *t = tensor(args[10], "db");
      db = t ? *t : fresh({a.out}, dy);
      vector("db", db, a.out, dy, &a.db);
    }
    const at::Tensor ws = workspace(&a, args[11], cada_linear_backward_workspace, dy);
    a.stream = stream_of(args[12]);
    check(cada_linear_backward(&a));
    return triple(dx, dw, db);
  });
}

// (logits, labels, smoothing, ignore_index, scale, need_grad, grad, workspace, stream) -> (mean, losses, grad)
PyObject *cross_entropy(PyObject *, PyObject *const *args, Py_ssize_t n_args) {
  return guarded([&]() -> PyObject * {
    if (n_args != 9) refuse("cross_entropy takes 9 arguments");
    const at::Tensor &z = needed(args[0], "logits"), &labels = needed(args[1], "labels");
    first(z, "logits");
    cada_xent a{};
    a.rows = z.size(0); a.classes = z.size(1); a.type = type_of(z);
    void *p;
    table("logits", z, a.rows, a.classes, z, &p, &a.ldz); a.logits = p;
    if ((labels.scalar_type() != at::kInt && labels.scalar_type() != at::kLong) || labels.dim() != 1 || labels.size(0) != a.rows || labels.device() != z.device() || (a.rows > 1 && labels.stride(0) != 1))
      refuse("labels must be a contiguous int32 or int64 [%lld] on %s", (long long)a.rows, z.device().str().c_str());
    a.labels = labels.data_ptr(); a.label_bytes = (int)labels.element_size();
    a.smoothing = PyFloat_AsDouble(args[2]); a.ignore_index = PyLong_AsLongLong(args[3]); a.scale = PyFloat_AsDouble(args[4]);
    if (PyErr_Occurred()) throw Failed{};
    const at::Tensor loss = at::empty({a.rows}, z.options().dtype(at::kFloat)), mean = at::empty({}, z.options().dtype(at::kFloat));
    a.loss = loss.data_ptr<float>(); a.mean = mean.data_ptr<float>();
    const at::Tensor *given = tensor(args[6], "grad");
    at::Tensor grad;
    if (given || args[5] == Py_True) {
      grad = given ? *given : fresh({a.rows, a.classes}, z);
      table("grad", grad, a.rows, a.classes, z, &a.grad, &a.ldg);
    }
    const at::Tensor ws = workspace(&a, args[7], cada_xent_workspace, z);
    a.stream = stream_of(args[8]);
    check(cada_cross_entropy(&a));
    return triple(mean, loss, grad);
  });
}

PyObject *set_error_class(PyObject *, PyObject *o) {
  Py_INCREF(o);
  Py_XDECREF(g_error);
  g_error = o;
  Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"linear_forward", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(linear_forward)), METH_FASTCALL, nullptr},
    {"linear_backward", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(linear_backward)), METH_FASTCALL, nullptr},
    {"cross_entropy", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(cross_entropy)), METH_FASTCALL, nullptr},
    {"set_error_class", set_error_class, METH_O, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_ops", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__ops() {
  g_error = PyExc_RuntimeError;
  Py_INCREF(g_error);
  return PyModule_Create(&module);
}
