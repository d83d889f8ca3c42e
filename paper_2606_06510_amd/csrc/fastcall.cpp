// Small calls of the model operators, where the host's share is the larger one: the checks that
// nearly every call passes, its outputs and the call, in one step from Python.  Anything else
// (another layout, a stream or outputs that are given, an argument that is wrong) is answered
// with None, or a status, and the binding's own path takes it, with the errors that name the
// fault.  One token's layer norm through ctypes 7.4 us, of which its kernel 3.1, the launch 2.5.
#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/ozaki2/model.h"

namespace {

// set by bind()
decltype(&ozaki2_layer_norm) norm;
decltype(&ozaki2_expert_route) route;
decltype(&ozaki2_expert_route_backward) route_backward;
PyObject *raw_stream, *current_device;

// a dense tensor on a GPU, and not of a class of its own
const at::Tensor* plain(PyObject* o) {
  if (!THPVariable_CheckExact(o)) return nullptr;
  const at::Tensor& t = THPVariable_Unpack(o);
  return t.defined() && t.is_cuda() && t.layout() == at::kStrided && t.is_contiguous() ? &t : nullptr;
}

int code_of(const at::Tensor& t) {
  switch (t.scalar_type()) {
    case at::kFloat: return OZ2_F32;
    case at::kHalf: return OZ2_F16;
    case at::kBFloat16: return OZ2_BF16;
    default: return -1;
  }
}

// rows and columns that the C ABI takes, of one of its types
bool matrix(const at::Tensor* t) {
  return t && t->dim() == 2 && t->size(0) < 1 << 30 && t->size(1) < 1 << 30 && code_of(*t) >= 0;
}

// None, or a plain vector of n entries on the device of `like`
bool vector(PyObject* o, const at::Tensor& like, int64_t n, at::ScalarType type, const void*& p) {
  p = nullptr;
  if (o == Py_None) return true;
  const at::Tensor* t = plain(o);
  if (!t || t->dim() != 1 || t->size(0) != n || t->scalar_type() != type || t->device() != like.device()) return false;
  p = t->const_data_ptr();
  return true;
}

// the tensor's device is the current one: its stream's handle
bool here(const at::Tensor& t, void*& stream) {
  PyObject* d = PyObject_CallNoArgs(current_device);
  if (!d) return false;
  const long current = PyLong_AsLong(d);
  if (current != t.device().index()) {
    Py_DECREF(d);
    return false;
  }
  PyObject* s = PyObject_CallOneArg(raw_stream, d);
  Py_DECREF(d);
  if (!s) return false;
  stream = PyLong_AsVoidPtr(s);
  Py_DECREF(s);
  return !PyErr_Occurred();
}

bool whole(PyObject* o, int& v) {
  if (!PyLong_Check(o)) return false;
  int overflow;
  const long n = PyLong_AsLongAndOverflow(o, &overflow);
  v = (int)n;
  return !overflow && n >= -(1l << 30) && n <= 1l << 30;
}
bool number(PyObject* o, float& v) {
  if (!PyFloat_Check(o) && !PyLong_Check(o)) return false;
  v = (float)PyFloat_AsDouble(o);
  return !PyErr_Occurred();
}

bool truth(PyObject* o, bool& v) {
  const int t = PyObject_IsTrue(o);
  v = t == 1;
  return t >= 0;
}

PyObject* other_path() {
  PyErr_Clear();
  Py_RETURN_NONE;
}

PyObject* pair(at::Tensor&& a, at::Tensor&& b) {
  PyObject *x = THPVariable_Wrap(std::move(a)), *y = x ? THPVariable_Wrap(std::move(b)) : nullptr;
  PyObject* r = y ? PyTuple_New(2) : nullptr;
  if (!r) {
    Py_XDECREF(x);
    Py_XDECREF(y);
    return nullptr;
  }
  PyTuple_SET_ITEM(r, 0, x);
  PyTuple_SET_ITEM(r, 1, y);
  return r;
}

// layer_norm(x, weight, bias, eps, save_stats)
PyObject* layer_norm(PyObject*, PyObject* const* a, Py_ssize_t n) try {
  const at::Tensor* x = n == 5 ? plain(a[0]) : nullptr;
  const void *w, *b;
  float eps;
  void* stream;
  if (!matrix(x) || !number(a[3], eps)) return other_path();
  const int64_t T = x->size(0), K = x->size(1);
  if (!vector(a[1], *x, K, x->scalar_type(), w) || !vector(a[2], *x, K, x->scalar_type(), b) || !here(*x, stream))
    return other_path();
  const bool save = a[4] == Py_True;
  at::Tensor y = at::empty({T, K}, x->options()), stats;
  if (save) stats = at::empty({T, 2}, x->options().dtype(at::kFloat));
  const void* px = x->const_data_ptr();
  void* py = y.mutable_data_ptr();
  float* ps = save ? (float*)stats.mutable_data_ptr() : nullptr;
  const int code = code_of(*x);
  int status;
  Py_BEGIN_ALLOW_THREADS
  status = norm(code, (int)T, (int)K, px, K ? K : 1, w, b, eps, py, K ? K : 1, ps, stream);
  Py_END_ALLOW_THREADS
  if (status != 0) return other_path();
  return save ? pair(std::move(y), std::move(stats)) : THPVariable_Wrap(std::move(y));
} catch (...) {
  return other_path();
}

// expert_route(logits, top_k, bias, score, groups, top_groups, group_best, renormalize, scale)
PyObject* expert_route(PyObject*, PyObject* const* a, Py_ssize_t n) try {
  const at::Tensor* l = n == 9 ? plain(a[0]) : nullptr;
  const void* bias;
  int k, score, groups, top, best;
  bool renormalize;
  float scale;
  void* stream;
  if (!matrix(l) || !whole(a[1], k) || !whole(a[3], score) || !whole(a[4], groups) || !whole(a[5], top) ||
      !whole(a[6], best) || !truth(a[7], renormalize) || !number(a[8], scale) || k < 1 || k > OZ2_MAX_TOPK)
    return other_path();
  const int64_t T = l->size(0), E = l->size(1);
  if (!vector(a[2], *l, E, at::kFloat, bias) || !here(*l, stream)) return other_path();
  at::Tensor ids = at::empty({T, k}, l->options().dtype(at::kInt));
  at::Tensor weights = at::empty({T, k}, l->options().dtype(at::kFloat));
  const void* pl = l->const_data_ptr();
  int* pi = (int*)ids.mutable_data_ptr();
  float* pw = (float*)weights.mutable_data_ptr();
  const int code = code_of(*l);
  int status;
  Py_BEGIN_ALLOW_THREADS
  status = route(code, (int)T, (int)E, k, pl, E, (const float*)bias, score, groups, top, best, renormalize, scale, pi,
                 pw, stream);
  Py_END_ALLOW_THREADS
  return status != 0 ? other_path() : pair(std::move(ids), std::move(weights));
} catch (...) {
  return other_path();
}

// expert_route_backward(dweights, logits, ids, score, renormalize, scale)
PyObject* expert_route_backward(PyObject*, PyObject* const* a, Py_ssize_t n) try {
  const at::Tensor *d = n == 6 ? plain(a[0]) : nullptr, *l = d ? plain(a[1]) : nullptr,
                   *i = l ? plain(a[2]) : nullptr;
  int score;
  bool renormalize;
  float scale;
  void* stream;
  if (!i || !matrix(l) || !whole(a[3], score) || !truth(a[4], renormalize) || !number(a[5], scale))
    return other_path();
  const int64_t T = l->size(0), E = l->size(1);
  if (i->dim() != 2 || i->size(0) != T || i->size(1) < 1 || i->size(1) > OZ2_MAX_TOPK || d->sizes() != i->sizes() ||
      i->scalar_type() != at::kInt || d->scalar_type() != at::kFloat || i->device() != l->device() ||
      d->device() != l->device() || !here(*l, stream))
    return other_path();
  const int k = (int)i->size(1);
  at::Tensor out = at::empty({T, E}, l->options());
  const float* pd = (const float*)d->const_data_ptr();
  const void* pl = l->const_data_ptr();
  const int* pi = (const int*)i->const_data_ptr();
  void* po = out.mutable_data_ptr();
  const int code = code_of(*l);
  int status;
  Py_BEGIN_ALLOW_THREADS
  status = route_backward(code, (int)T, (int)E, k, pd, pl, E, pi, score, renormalize, scale, po, E, stream);
  Py_END_ALLOW_THREADS
  return status != 0 ? other_path() : THPVariable_Wrap(std::move(out));
} catch (...) {
  return other_path();
}

// bind(addresses of the three entry points, raw_stream, current_device)
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 5) {
    PyErr_SetString(PyExc_TypeError, "bind takes 5 arguments");
    return nullptr;
  }
  void* p[3];
  for (int i = 0; i < 3; ++i) {
    p[i] = PyLong_AsVoidPtr(a[i]);
    if (!p[i]) {
      if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "null entry point");
      return nullptr;
    }
  }
  norm = (decltype(norm))p[0];
  route = (decltype(route))p[1];
  route_backward = (decltype(route_backward))p[2];
  Py_INCREF(a[3]);
  Py_INCREF(a[4]);
  raw_stream = a[3];
  current_device = a[4];
  Py_RETURN_NONE;
}

PyMethodDef methods[] = {{"bind", (PyCFunction)(void*)bind, METH_FASTCALL, nullptr},
                         {"layer_norm", (PyCFunction)(void*)layer_norm, METH_FASTCALL, nullptr},
                         {"expert_route", (PyCFunction)(void*)expert_route, METH_FASTCALL, nullptr},
                         {"expert_route_backward", (PyCFunction)(void*)expert_route_backward, METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_fastcall", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__fastcall() { return PyModule_Create(&module); }
