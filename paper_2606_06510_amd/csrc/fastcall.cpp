// Small calls of the model operators, where the host's share is the larger one: the checks that
// nearly every call passes, its outputs and the call, in one step from Python.  Anything else
// (another layout, a stream or outputs that are given, an argument that is wrong) is answered
// with None, or a status, and the binding's own path takes it, with the errors that name the
// fault.  One token's layer norm 4.7 us a call, through ctypes 7.4 (its kernel takes 3.1).
#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/ozaki2/model.h"

namespace {

// set by bind()
decltype(&ozaki2_layer_norm) norm;
decltype(&ozaki2_layer_norm_backward) norm_backward;
decltype(&ozaki2_layer_norm_backward_workspace_bytes) norm_backward_bytes;
decltype(&ozaki2_expert_route) route;
decltype(&ozaki2_expert_route_backward) route_backward;
decltype(&ozaki2_linear_cross_entropy) loss;
decltype(&ozaki2_linear_cross_entropy_workspace_bytes) loss_bytes;
decltype(&ozaki2_linear_cross_entropy_backward) loss_backward;
decltype(&ozaki2_linear_cross_entropy_backward_workspace_bytes) loss_backward_bytes;
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

// a plain matrix of this shape, of the type and on the device of `like`
const at::Tensor* same(PyObject* o, const at::Tensor& like, int64_t rows, int64_t cols) {
  const at::Tensor* t = plain(o);
  return t && t->dim() == 2 && t->size(0) == rows && t->size(1) == cols && t->scalar_type() == like.scalar_type() &&
                 t->device() == like.device()
             ? t
             : nullptr;
}

at::Tensor bytes(size_t n, const at::Tensor& like) {
  return at::empty({(int64_t)n}, like.options().dtype(at::kByte));
}
void* at_or_null(at::Tensor& t) { return t.defined() ? t.mutable_data_ptr() : nullptr; }
int64_t ld(int64_t cols) { return cols ? cols : 1; }

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

// a tuple of N tensors, None where there is none
template <size_t N>
PyObject* tuple(at::Tensor (&&t)[N]) {
  PyObject* r = PyTuple_New(N);
  for (size_t i = 0; r && i < N; ++i) {
    PyObject* o;
    if (t[i].defined()) {
      o = THPVariable_Wrap(std::move(t[i]));
    } else {
      Py_INCREF(Py_None);
      o = Py_None;
    }
    if (o)
      PyTuple_SET_ITEM(r, i, o);
    else
      Py_CLEAR(r);
  }
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
  if (save && K == 0) return other_path();   // (statistics of nothing)
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
  return save ? tuple<2>({std::move(y), std::move(stats)}) : THPVariable_Wrap(std::move(y));
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
  return status != 0 ? other_path() : tuple<2>({std::move(ids), std::move(weights)});
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

// layer_norm_backward(dy, x, stats, weight, residual, need_dx, need_dweight, need_dbias)
PyObject* layer_norm_backward(PyObject*, PyObject* const* a, Py_ssize_t n) try {
  const at::Tensor* dy = n == 8 ? plain(a[0]) : nullptr;
  if (!matrix(dy)) return other_path();
  const int64_t T = dy->size(0), K = dy->size(1);
  const at::Tensor *x = same(a[1], *dy, T, K), *stats = plain(a[2]), *res = nullptr;
  const void* w;
  bool need[3];
  void* stream;
  if (!x || !stats || stats->dim() != 2 || stats->size(0) != T || stats->size(1) != 2 ||
      stats->scalar_type() != at::kFloat || stats->device() != dy->device() ||
      !vector(a[3], *dy, K, dy->scalar_type(), w) || (a[4] != Py_None && !(res = same(a[4], *dy, T, K))) ||
      !truth(a[5], need[0]) || !truth(a[6], need[1]) || !truth(a[7], need[2]) || !here(*dy, stream))
    return other_path();
  const int code = code_of(*dy);
  const size_t bytes_needed = need[1] || need[2] ? norm_backward_bytes(code, (int)T, (int)K) : 0;
  at::Tensor dx, dw, db, ws;
  if (need[0]) dx = at::empty({T, K}, dy->options());
  if (need[1]) dw = at::empty({K}, dy->options());
  if (need[2]) db = at::empty({K}, dy->options());
  if (bytes_needed) ws = bytes(bytes_needed, *dy);
  const void *pd = dy->const_data_ptr(), *px = x->const_data_ptr(), *pr = res ? res->const_data_ptr() : nullptr;
  const float* ps = (const float*)stats->const_data_ptr();
  void *gx = at_or_null(dx), *gw = at_or_null(dw), *gb = at_or_null(db), *pw = at_or_null(ws);
  int status;
  Py_BEGIN_ALLOW_THREADS
  status = norm_backward(code, (int)T, (int)K, pd, ld(K), px, ld(K), ps, w, pr, ld(K), gx, ld(K), gw, gb, pw,
                         bytes_needed, stream);
  Py_END_ALLOW_THREADS
  return status != 0 ? other_path() : tuple<3>({std::move(dx), std::move(dw), std::move(db)});
} catch (...) {
  return other_path();
}

// x, w and targets of the loss
struct LossArgs {
  const at::Tensor *x, *w, *targets;
  int64_t T, V, K;
  int code, wide;
  bool read(PyObject* ox, PyObject* ow, PyObject* ot) {
    x = plain(ox);
    w = plain(ow);
    targets = plain(ot);
    if (!matrix(x) || !matrix(w) || !targets) return false;
    T = x->size(0);
    K = x->size(1);
    V = w->size(0);
    code = code_of(*x);
    wide = targets->scalar_type() == at::kLong;
    return w->size(1) == K && w->scalar_type() == x->scalar_type() && w->device() == x->device() &&
           targets->dim() == 1 && targets->size(0) == T && (wide || targets->scalar_type() == at::kInt) &&
           targets->device() == x->device();
  }
};

// linear_cross_entropy(x, w, targets)
PyObject* linear_cross_entropy(PyObject*, PyObject* const* a, Py_ssize_t n) try {
  LossArgs q;
  void* stream;
  if (n != 3 || !q.read(a[0], a[1], a[2]) || !here(*q.x, stream)) return other_path();
  const int T = (int)q.T, V = (int)q.V, K = (int)q.K;
  const size_t need = loss_bytes(q.code, T, V, K);
  const auto f32 = q.x->options().dtype(at::kFloat);
  at::Tensor l = at::empty({q.T}, f32), e = at::empty({q.T}, f32), ws;
  if (need) ws = bytes(need, *q.x);
  const void *px = q.x->const_data_ptr(), *pw = q.w->const_data_ptr(), *pt = q.targets->const_data_ptr();
  float *pl = (float*)l.mutable_data_ptr(), *pe = (float*)e.mutable_data_ptr();
  void* space = at_or_null(ws);
  int status;
  Py_BEGIN_ALLOW_THREADS
  status = loss(q.code, T, V, K, px, ld(K), pw, ld(K), pt, q.wide, pl, pe, space, need, stream);
  Py_END_ALLOW_THREADS
  return status != 0 ? other_path() : tuple<2>({std::move(l), std::move(e)});
} catch (...) {
  return other_path();
}

// linear_cross_entropy_backward(dloss, x, w, targets, lse, need_dx, need_dw)
PyObject* linear_cross_entropy_backward(PyObject*, PyObject* const* a, Py_ssize_t n) try {
  LossArgs q;
  void* stream;
  const void *d, *e;
  bool need_dx, need_dw;
  if (n != 7 || !q.read(a[1], a[2], a[3]) || a[0] == Py_None || a[4] == Py_None ||
      !vector(a[0], *q.x, q.T, at::kFloat, d) || !vector(a[4], *q.x, q.T, at::kFloat, e) || !truth(a[5], need_dx) ||
      !truth(a[6], need_dw) || !here(*q.x, stream))
    return other_path();
  const int T = (int)q.T, V = (int)q.V, K = (int)q.K;
  const size_t need = loss_backward_bytes(q.code, T, V, K);
  at::Tensor dx, dw, ws;
  if (need_dx) dx = at::empty({q.T, q.K}, q.x->options());
  if (need_dw) dw = at::empty({q.V, q.K}, q.x->options());
  if (need) ws = bytes(need, *q.x);
  const void *px = q.x->const_data_ptr(), *pw = q.w->const_data_ptr(), *pt = q.targets->const_data_ptr();
  void *gx = at_or_null(dx), *gw = at_or_null(dw), *space = at_or_null(ws);
  int status;
  Py_BEGIN_ALLOW_THREADS
  status = loss_backward(q.code, T, V, K, (const float*)d, px, ld(K), pw, ld(K), pt, q.wide, (const float*)e, gx,
                         ld(K), gw, ld(K), space, need, stream);
  Py_END_ALLOW_THREADS
  return status != 0 ? other_path() : tuple<2>({std::move(dx), std::move(dw)});
} catch (...) {
  return other_path();
}

// bind(addresses of the entry points, raw_stream, current_device)
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
  constexpr int N = 9;
  if (n != N + 2) {
    PyErr_Format(PyExc_TypeError, "bind takes %d arguments", N + 2);
    return nullptr;
  }
  void* p[N];
  for (int i = 0; i < N; ++i) {
    p[i] = PyLong_AsVoidPtr(a[i]);
    if (!p[i]) {
      if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "null entry point");
      return nullptr;
    }
  }
  norm = (decltype(norm))p[0];
  norm_backward = (decltype(norm_backward))p[1];
  norm_backward_bytes = (decltype(norm_backward_bytes))p[2];
  route = (decltype(route))p[3];
  route_backward = (decltype(route_backward))p[4];
  loss = (decltype(loss))p[5];
  loss_bytes = (decltype(loss_bytes))p[6];
  loss_backward = (decltype(loss_backward))p[7];
  loss_backward_bytes = (decltype(loss_backward_bytes))p[8];
  Py_INCREF(a[N]);
  Py_INCREF(a[N + 1]);
  raw_stream = a[N];
  current_device = a[N + 1];
  Py_RETURN_NONE;
}

#define OZ2_METHOD(name) {#name, (PyCFunction)(void*)name, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {OZ2_METHOD(bind), OZ2_METHOD(layer_norm), OZ2_METHOD(layer_norm_backward),
                         OZ2_METHOD(expert_route), OZ2_METHOD(expert_route_backward),
                         OZ2_METHOD(linear_cross_entropy), OZ2_METHOD(linear_cross_entropy_backward),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_fastcall", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__fastcall() { return PyModule_Create(&module); }
