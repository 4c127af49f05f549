// The common calls of binding.py in one native step: checks, output tensors and the library call.
//
// A call on 64 x 16 scores takes 2.5 us on the GPU and took 7.8 in Python: a dozen attribute reads of tensors, the
// allocation of the outputs and the foreign call, each of which costs more than what it does.  Every function here takes
// the arguments of its namesakes in binding.py and returns their result, or None where anything is not as in the common
// case (another type, layout or device, overlapping arrays, an explicit stream, a workspace to be made, a mode that
// watches tensor calls): the Python code then makes the call itself, with its own checks and errors.  Errors of the library
// are raised from here, by the same function.
//   64 x 16 JVP into given arrays 8.3 -> 4.3 us a call, 16384 x 64 VJP 8.3 -> 6.0 (5.2 on the GPU), compact
//   output 10.3 -> 6.4, the last two within a tenth from run to run.  What is left of 4.3: 2.7 the launch, 0.7 the Python
//   function, the rest the checks and the stream.
// The operators behind a router take the same way: routing one token 9.8 -> 5.6 us a call, the map of 128 pairs 14.0 -> 7.2.
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/PythonTorchFunctionTLS.h>
#include <ATen/TracerMode.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <c10/core/impl/VirtualGuardImpl.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>
#include <initializer_list>

namespace {

// entry points of the library, by the numbers that binding.py passes
using FwdFn = int (*)(const void*, int64_t, int64_t, int64_t, double, double, void*, void*);
using JvpFn = int (*)(const void*, const void*, int64_t, int64_t, int64_t, double, double, void*, void*, void*);
using SparseFn = int (*)(const void*, int64_t, int64_t, int64_t, double, double, int64_t, void*, void*, void*, void*);
using LossFn = JvpFn;

constexpr int kMaxEntries = 32;
void* g_entry[kMaxEntries] = {};
PyObject* g_names[kMaxEntries] = {};
PyObject* g_raw_stream = nullptr;   // torch._C._cuda_getCurrentRawStream
PyObject* g_check = nullptr;        // binding._check
int g_ws_device = -1;               // of the registered workspace, -1: none
constexpr int kErrWorkspace = -4;

// a plain tensor object without anything that watches or replaces tensor calls
bool plain_mode() {
  return !at::impl::torch_function_mode_enabled() && !c10::impl::TorchDispatchModeTLS::any_modes_set() &&
         !at::tracer::impl::is_dispatch_enabled();
}

const at::Tensor* matrix(PyObject* o) {
  if (!THPVariable_CheckExact(o)) return nullptr;
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.defined() || !t.is_cuda() || t.layout() != at::kStrided || t.scalar_type() != at::kFloat || t.dim() != 2 ||
      !t.unsafeGetTensorImpl()->has_storage() || !t.is_contiguous() || (t.numel() > 0 && t.data_ptr() == nullptr))
    return nullptr;
  return &t;
}
const at::Tensor* like(PyObject* o, const at::Tensor& ref) {
  const at::Tensor* t = matrix(o);
  if (t == nullptr || t->sizes() != ref.sizes() || t->get_device() != ref.get_device()) return nullptr;
  return t;
}
bool overlap(const at::Tensor& a, const at::Tensor& b) {
  const char *pa = static_cast<const char*>(a.data_ptr()), *pb = static_cast<const char*>(b.data_ptr());
  const char *ea = pa + a.nbytes(), *eb = pb + b.nbytes();
  return pa < eb && pb < ea;
}

bool number(PyObject* o, double* v) {
  if (PyFloat_CheckExact(o)) *v = PyFloat_AS_DOUBLE(o);
  else if (PyLong_CheckExact(o)) *v = PyLong_AsDouble(o);
  else return false;
  if (PyErr_Occurred()) {
    PyErr_Clear();
    return false;
  }
  return true;
}
bool integer(PyObject* o, int64_t* v) {
  if (!PyLong_CheckExact(o)) return false;
  *v = PyLong_AsLongLong(o);
  if (PyErr_Occurred()) {
    PyErr_Clear();
    return false;
  }
  return true;
}

// the raw handle of torch.cuda.current_stream(), and the current device
bool current_stream(void** st, int* device = nullptr) {
  const c10::impl::VirtualGuardImpl impl(c10::DeviceType::CUDA);
  const int current = impl.getDevice().index();
  if (device != nullptr) *device = current;
  PyObject* index = PyLong_FromLong(current);
  if (index == nullptr) return false;
  PyObject* h = PyObject_CallOneArg(g_raw_stream, index);
  Py_DECREF(index);
  if (h == nullptr) return false;
  *st = PyLong_AsVoidPtr(h);
  Py_DECREF(h);
  return !PyErr_Occurred();
}

// 1: done, 0: the Python code is to make the call, -1: an error is set
int outcome(int rc, int entry) {
  if (rc == 0) return 1;
  if (rc == kErrWorkspace) return 0;
  PyObject* r = PyObject_CallFunction(g_check, "iO", rc, g_names[entry]);
  Py_XDECREF(r);
  return r == nullptr ? -1 : 0;
}

// a tuple of new references (all of them taken over; null where one is)
PyObject* tuple_of(std::initializer_list<PyObject*> items) {
  bool whole = true;
  for (PyObject* o : items) whole = whole && o != nullptr;
  PyObject* r = whole ? PyTuple_New(Py_ssize_t(items.size())) : nullptr;
  Py_ssize_t i = 0;
  for (PyObject* o : items) {
    if (r != nullptr) PyTuple_SET_ITEM(r, i++, o);
    else Py_XDECREF(o);
  }
  return r;
}

struct Common {
  const at::Tensor* x;
  int64_t rows, n, k;
  double p, lam;
  void* stream;
};
// entry, x, .., k, p, lam and a stream that is None; false: not the common case (or an error is set)
bool common(PyObject* entry, PyObject* x, PyObject* k, PyObject* p, PyObject* lam, PyObject* stream, int* e, Common* c) {
  int64_t ev;
  if (stream != Py_None || !integer(entry, &ev) || ev < 0 || ev >= kMaxEntries || g_entry[ev] == nullptr ||
      !plain_mode() || !integer(k, &c->k) || !number(p, &c->p) || !number(lam, &c->lam))
    return false;
  *e = int(ev);
  c->x = matrix(x);
  if (c->x == nullptr || (g_ws_device >= 0 && g_ws_device != c->x->get_device())) return false;
  c->rows = c->x->size(0);
  c->n = c->x->size(1);
  return current_stream(&c->stream);
}

#define TOPK_NONE                       \
  do {                                  \
    if (PyErr_Occurred()) return nullptr; \
    Py_RETURN_NONE;                     \
  } while (0)

// fwd(entry, x, k, p, lam, out, stream) -> out
PyObject* fwd(PyObject*, PyObject* const* a, Py_ssize_t count) {
  HANDLE_TH_ERRORS
  int e;
  Common c;
  if (count != 7 || !common(a[0], a[1], a[2], a[3], a[4], a[6], &e, &c)) TOPK_NONE;
  at::Tensor fresh;
  const at::Tensor* out = &fresh;
  if (a[5] == Py_None) {
    fresh = at::empty_like(*c.x);
  } else {
    out = like(a[5], *c.x);
    if (out == nullptr || overlap(*out, *c.x)) TOPK_NONE;
  }
  const void* x = c.x->data_ptr();
  void* o = out->data_ptr();
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = reinterpret_cast<FwdFn>(g_entry[e])(x, c.rows, c.n, c.k, c.p, c.lam, o, c.stream);
  Py_END_ALLOW_THREADS
  if (outcome(rc, e) != 1) TOPK_NONE;
  if (a[5] == Py_None) return THPVariable_Wrap(fresh);
  Py_INCREF(a[5]);
  return a[5];
  END_HANDLE_TH_ERRORS
}

// jvp(entry, x, tangent, k, p, lam, out, jvp_out, want_out, stream) -> (out or None, jvp_out)
PyObject* jvp(PyObject*, PyObject* const* a, Py_ssize_t count) {
  HANDLE_TH_ERRORS
  int e;
  Common c;
  if (count != 10 || !PyBool_Check(a[8]) || !common(a[0], a[1], a[3], a[4], a[5], a[9], &e, &c)) TOPK_NONE;
  const at::Tensor* t = like(a[2], *c.x);
  if (t == nullptr) TOPK_NONE;
  at::Tensor fresh_out, fresh_jvp;
  const at::Tensor *out = nullptr, *d = &fresh_jvp;
  if (a[6] != Py_None) {
    out = like(a[6], *c.x);
    if (out == nullptr || overlap(*out, *c.x) || overlap(*out, *t)) TOPK_NONE;
  }
  if (a[7] != Py_None) {
    d = like(a[7], *c.x);
    if (d == nullptr || overlap(*d, *c.x) || overlap(*d, *t) || (out != nullptr && overlap(*out, *d))) TOPK_NONE;
  }
  if (out == nullptr && a[8] == Py_True) {
    fresh_out = at::empty_like(*c.x);
    out = &fresh_out;
  }
  if (a[7] == Py_None) fresh_jvp = at::empty_like(*c.x);
  const void *x = c.x->data_ptr(), *tp = t->data_ptr();
  void *o = out != nullptr ? out->data_ptr() : nullptr, *dp = d->data_ptr();
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = reinterpret_cast<JvpFn>(g_entry[e])(x, tp, c.rows, c.n, c.k, c.p, c.lam, o, dp, c.stream);
  Py_END_ALLOW_THREADS
  if (outcome(rc, e) != 1) TOPK_NONE;
  PyObject* ro = a[6];
  PyObject* rd = a[7];
  if (ro == Py_None && out != nullptr) ro = THPVariable_Wrap(fresh_out);
  else Py_INCREF(ro);
  if (rd == Py_None) rd = THPVariable_Wrap(fresh_jvp);
  else Py_INCREF(rd);
  return tuple_of({ro, rd});
  END_HANDLE_TH_ERRORS
}

// sparse(entry, x, k, p, lam, max_nnz, stream) -> (idx, val, nnz), all three allocated here
PyObject* sparse(PyObject*, PyObject* const* a, Py_ssize_t count) {
  HANDLE_TH_ERRORS
  int e;
  Common c;
  int64_t width;
  if (count != 7 || !integer(a[5], &width) || width < 1 || !common(a[0], a[1], a[2], a[3], a[4], a[6], &e, &c) ||
      width > c.n)
    TOPK_NONE;
  const auto words = at::TensorOptions().dtype(at::kInt).device(c.x->device());
  at::Tensor idx = at::empty({c.rows, width}, words), val = at::empty({c.rows, width}, words.dtype(at::kFloat)),
             nnz = at::empty({c.rows}, words);
  const void* x = c.x->data_ptr();
  void *ip = idx.data_ptr(), *vp = val.data_ptr(), *np = nnz.data_ptr();
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = reinterpret_cast<SparseFn>(g_entry[e])(x, c.rows, c.n, c.k, c.p, c.lam, width, ip, vp, np, c.stream);
  Py_END_ALLOW_THREADS
  if (outcome(rc, e) != 1) TOPK_NONE;
  return tuple_of({THPVariable_Wrap(idx), THPVariable_Wrap(val), THPVariable_Wrap(nnz)});
  END_HANDLE_TH_ERRORS
}

// loss(entry, x, target, k, p, lam, stream) -> (loss, grad), both allocated here
PyObject* loss(PyObject*, PyObject* const* a, Py_ssize_t count) {
  HANDLE_TH_ERRORS
  int e;
  Common c;
  if (count != 7 || !common(a[0], a[1], a[3], a[4], a[5], a[6], &e, &c)) TOPK_NONE;
  const at::Tensor* t = like(a[2], *c.x);
  if (t == nullptr) TOPK_NONE;
  at::Tensor l = at::empty({c.rows}, c.x->options().requires_grad(false)), g = at::empty_like(*c.x);
  const void *x = c.x->data_ptr(), *tp = t->data_ptr();
  void *lp = l.data_ptr(), *gp = g.data_ptr();
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = reinterpret_cast<LossFn>(g_entry[e])(x, tp, c.rows, c.n, c.k, c.p, c.lam, lp, gp, c.stream);
  Py_END_ALLOW_THREADS
  if (outcome(rc, e) != 1) TOPK_NONE;
  return tuple_of({THPVariable_Wrap(l), THPVariable_Wrap(g)});
  END_HANDLE_TH_ERRORS
}

// ---- behind a router -------------------------------------------------------------------------------------------------
using RouteFn = int (*)(const void*, int, int64_t, const void*, int64_t, int64_t, int64_t, int, int64_t, int64_t, int, int, double,
                        void*, void*, void*);
using RouteVjpFn = int (*)(const void*, int, int64_t, const void*, const void*, int64_t, int64_t, int64_t, int, int, double, void*,
                           void*);
using MapFn = int (*)(const void*, int64_t, int64_t, int64_t, int64_t, void*, void*, void*, void*, void*, size_t, void*);
using MapBytesFn = size_t (*)(int64_t, int64_t, int64_t);
using ProductFn = int (*)(const void*, int64_t, int64_t, const void*, int64_t, int64_t, int64_t, const void*, const void*, int64_t,
                          int64_t, int64_t, int64_t, int64_t, int, void*, void*);
using ProductVjpFn = int (*)(const void*, int64_t, int64_t, const void*, int64_t, int64_t, int64_t, const void*, const void*,
                             int64_t, int64_t, int64_t, int64_t, int64_t, int, const void*, int64_t, void*, void*, void*);
using CombineFn = int (*)(const void*, int64_t, const void*, const void*, int64_t, int64_t, int64_t, int64_t, int, void*, void*);
using CombineVjpFn = int (*)(const void*, int64_t, const void*, const void*, const void*, int64_t, int64_t, int64_t, int64_t,
                             int64_t, int, void*, void*, void*);

// the entry, the current stream and device; false: not the common case (or an error is set)
struct Here {
  int entry, device;
  void* stream;
};
bool here(PyObject* entry, PyObject* first, PyObject* stream, Here* h) {
  int64_t e;
  if (stream != Py_None || !integer(entry, &e) || e < 0 || e >= kMaxEntries || g_entry[e] == nullptr || !plain_mode())
    return false;
  // (a tensor of the host is refused by the Python code, also where there is no GPU to ask)
  if (!THPVariable_CheckExact(first) || !THPVariable_Unpack(first).defined() || !THPVariable_Unpack(first).is_cuda()) return false;
  h->entry = int(e);
  return current_stream(&h->stream, &h->device);
}
// a plain tensor on this device
const at::Tensor* plain(PyObject* o, int device) {
  if (!THPVariable_CheckExact(o)) return nullptr;
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.defined() || !t.is_cuda() || t.layout() != at::kStrided || t.get_device() != device ||
      !t.unsafeGetTensorImpl()->has_storage() || (t.numel() > 0 && t.data_ptr() == nullptr))
    return nullptr;
  return &t;
}
int type_code(const at::Tensor& t) {
  const at::ScalarType s = t.scalar_type();
  return s == at::kFloat ? 0 : s == at::kBFloat16 ? 1 : s == at::kHalf ? 2 : -1;
}
// a matrix of values with contiguous rows
const at::Tensor* rows_of(PyObject* o, int device) {
  const at::Tensor* t = plain(o, device);
  if (t == nullptr || t->dim() != 2 || type_code(*t) < 0 || (t->size(1) > 1 && t->stride(1) != 1)) return nullptr;
  return t;
}
const at::Tensor* whole(PyObject* o, int device, at::ScalarType type, at::IntArrayRef shape) {
  const at::Tensor* t = plain(o, device);
  if (t == nullptr || t->scalar_type() != type || t->sizes() != shape || !t->is_contiguous()) return nullptr;
  return t;
}
const at::Tensor* words_matrix(PyObject* o, int device) {
  const at::Tensor* t = plain(o, device);
  if (t == nullptr || t->dim() != 2 || t->scalar_type() != at::kInt || !t->is_contiguous()) return nullptr;
  return t;
}
bool flag(PyObject* o, bool* v) {
  if (!PyBool_Check(o)) return false;
  *v = o == Py_True;
  return true;
}
const void* data(const at::Tensor* t) { return t == nullptr ? nullptr : t->data_ptr(); }
// bytes that the tensor reaches
bool apart(const at::Tensor& out, const at::Tensor* in) {
  if (in == nullptr || out.numel() == 0 || in->numel() == 0) return true;
  const char *po = static_cast<const char*>(out.data_ptr()), *pi = static_cast<const char*>(in->data_ptr());
  int64_t last = 0;
  for (int64_t d = 0; d < in->dim(); ++d) last += (in->size(d) - 1) * in->stride(d);
  const char *eo = po + out.nbytes(), *ei = pi + (last + 1) * int64_t(in->element_size());
  return !(po < ei && pi < eo);
}

// route_fwd(entry, logits, k, score, bias, groups, keep_groups, group_top, renormalise, scale, stream) -> (idx, val)
PyObject* route_fwd(PyObject*, PyObject* const* a, Py_ssize_t count) {
  HANDLE_TH_ERRORS
  Here h;
  int64_t k, score, groups, keep, top;
  bool renorm;
  double scale;
  if (count != 11 || !here(a[0], a[1], a[10], &h) || !integer(a[2], &k) || !integer(a[3], &score) || !integer(a[5], &groups) ||
      !integer(a[6], &keep) || !integer(a[7], &top) || !flag(a[8], &renorm) || !number(a[9], &scale) || k < 0 || k > 64 ||
      score < 0 || score > 1 || top < 1 || top > 2)
    TOPK_NONE;
  const at::Tensor* x = rows_of(a[1], h.device);
  if (x == nullptr) TOPK_NONE;
  const int64_t rows = x->size(0), n = x->size(1);
  const at::Tensor* bias = a[4] == Py_None ? nullptr : whole(a[4], h.device, at::kFloat, {n});
  if (a[4] != Py_None && bias == nullptr) TOPK_NONE;
  const auto words = at::TensorOptions().dtype(at::kInt).device(x->device());
  at::Tensor idx = at::empty({rows, k}, words), val = at::empty({rows, k}, words.dtype(at::kFloat));
  const void *xp = x->data_ptr(), *bp = data(bias);
  void *ip = idx.data_ptr(), *vp = val.data_ptr();
  const int type = type_code(*x);
  const int64_t stride = x->stride(0);
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = reinterpret_cast<RouteFn>(g_entry[h.entry])(xp, type, stride, bp, rows, n, k, int(score), groups, keep, int(top), renorm,
                                                   scale, ip, vp, h.stream);
  Py_END_ALLOW_THREADS
  if (outcome(rc, h.entry) != 1) TOPK_NONE;
  return tuple_of({THPVariable_Wrap(idx), THPVariable_Wrap(val)});
  END_HANDLE_TH_ERRORS
}

// route_vjp(entry, logits, idx, cotangent, score, renormalise, scale, stream) -> grad
PyObject* route_vjp(PyObject*, PyObject* const* a, Py_ssize_t count) {
  HANDLE_TH_ERRORS
  Here h;
  int64_t score;
  bool renorm;
  double scale;
  if (count != 8 || !here(a[0], a[1], a[7], &h) || !integer(a[4], &score) || !flag(a[5], &renorm) || !number(a[6], &scale) ||
      score < 0 || score > 1)
    TOPK_NONE;
  const at::Tensor *x = rows_of(a[1], h.device), *idx = words_matrix(a[2], h.device);
  if (x == nullptr || idx == nullptr || idx->size(0) != x->size(0)) TOPK_NONE;
  const int64_t rows = x->size(0), n = x->size(1), k = idx->size(1);
  const at::Tensor* t = whole(a[3], h.device, at::kFloat, {rows, k});
  if (t == nullptr) TOPK_NONE;
  at::Tensor grad = at::empty({rows, n}, at::TensorOptions().dtype(x->scalar_type()).device(x->device()));
  const void *xp = x->data_ptr(), *ip = idx->data_ptr(), *tp = t->data_ptr();
  void* gp = grad.data_ptr();
  const int type = type_code(*x);
  const int64_t stride = x->stride(0);
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = reinterpret_cast<RouteVjpFn>(g_entry[h.entry])(xp, type, stride, ip, tp, rows, n, k, int(score), renorm, scale, gp,
                                                      h.stream);
  Py_END_ALLOW_THREADS
  if (outcome(rc, h.entry) != 1) TOPK_NONE;
  return THPVariable_Wrap(grad);
  END_HANDLE_TH_ERRORS
}

// expert_map(entry, bytes_entry, idx, n, capacity, stream) -> (slot, source, offset, load)
PyObject* expert_map(PyObject*, PyObject* const* a, Py_ssize_t count) {
  HANDLE_TH_ERRORS
  Here h;
  int64_t bytes_entry, n, capacity;
  if (count != 6 || !here(a[0], a[2], a[5], &h) || !integer(a[1], &bytes_entry) || bytes_entry < 0 || bytes_entry >= kMaxEntries ||
      g_entry[bytes_entry] == nullptr || !integer(a[3], &n) || !integer(a[4], &capacity) || n < 1 || n > 1024)
    TOPK_NONE;
  const at::Tensor* idx = words_matrix(a[2], h.device);
  if (idx == nullptr || idx->size(1) < 1) TOPK_NONE;
  const int64_t rows = idx->size(0), k = idx->size(1);
  const auto words = at::TensorOptions().dtype(at::kInt).device(idx->device());
  at::Tensor slot = at::empty({rows, k}, words), source = at::empty({rows * k}, words), offset = at::empty({n + 1}, words),
             load = at::empty({n}, words), scratch;
  const size_t need = reinterpret_cast<MapBytesFn>(g_entry[bytes_entry])(rows, k, n);
  if (need > 0) scratch = at::empty({int64_t(need)}, words.dtype(at::kByte));
  const void* ip = idx->data_ptr();
  void *sp = slot.data_ptr(), *op = source.data_ptr(), *fp = offset.data_ptr(), *lp = load.data_ptr(),
       *cp = need > 0 ? scratch.data_ptr() : nullptr;
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = reinterpret_cast<MapFn>(g_entry[h.entry])(ip, rows, k, n, capacity, sp, op, fp, lp, cp, need, h.stream);
  Py_END_ALLOW_THREADS
  if (outcome(rc, h.entry) != 1) TOPK_NONE;
  return tuple_of({THPVariable_Wrap(slot), THPVariable_Wrap(source), THPVariable_Wrap(offset), THPVariable_Wrap(load)});
  END_HANDLE_TH_ERRORS
}

struct Product {
  const at::Tensor *x, *w, *offset, *source;
  int64_t k, slots, n, ho, hi, w_expert, w_out, w_in;
};
// x, w, offset, source, k as binding.py's _product takes them
bool product_args(PyObject* const* a, int device, Product* p) {
  p->x = rows_of(a[0], device);
  p->w = plain(a[1], device);
  if (p->x == nullptr || p->w == nullptr || p->w->dim() != 3 || p->w->scalar_type() != p->x->scalar_type() ||
      p->w->size(2) != p->x->size(1) || !integer(a[4], &p->k))
    return false;
  p->n = p->w->size(0), p->ho = p->w->size(1), p->hi = p->w->size(2);
  p->w_expert = p->w->stride(0), p->w_out = p->w->stride(1), p->w_in = p->w->stride(2);
  if (p->hi <= 1 || p->ho <= 1 || (p->w_in != 1 && p->w_out != 1)) return false;
  p->offset = whole(a[2], device, at::kInt, {p->n + 1});
  if (p->offset == nullptr) return false;
  p->source = nullptr;
  p->slots = p->x->size(0);
  if (a[3] != Py_None) {
    const at::Tensor* s = plain(a[3], device);
    if (s == nullptr || s->dim() != 1 || s->scalar_type() != at::kInt || !s->is_contiguous()) return false;
    p->source = s;
    p->slots = s->size(0);
  }
  return true;
}

// product_fwd(entry, x, w, offset, source, k, stream) -> out
PyObject* product_fwd(PyObject*, PyObject* const* a, Py_ssize_t count) {
  HANDLE_TH_ERRORS
  Here h;
  Product p;
  if (count != 7 || !here(a[0], a[1], a[6], &h) || !product_args(a + 1, h.device, &p)) TOPK_NONE;
  at::Tensor out = at::empty({p.slots, p.ho}, at::TensorOptions().dtype(p.x->scalar_type()).device(p.x->device()));
  const void *xp = data(p.x), *wp = data(p.w), *fp = data(p.offset), *sp = data(p.source);
  const int64_t stride = p.x->stride(0), m = p.x->size(0);
  const int type = type_code(*p.x);
  void* op = out.data_ptr();
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = reinterpret_cast<ProductFn>(g_entry[h.entry])(xp, stride, m, wp, p.w_expert, p.w_out, p.w_in, fp, sp, p.k, p.slots, p.n,
                                                     p.hi, p.ho, type, op, h.stream);
  Py_END_ALLOW_THREADS
  if (outcome(rc, h.entry) != 1) TOPK_NONE;
  return THPVariable_Wrap(out);
  END_HANDLE_TH_ERRORS
}

// product_vjp(entry, x, w, offset, source, k, cotangent, want_x, want_w, stream) -> (dx or None, dw or None)
PyObject* product_vjp(PyObject*, PyObject* const* a, Py_ssize_t count) {
  HANDLE_TH_ERRORS
  Here h;
  Product p;
  bool want_x, want_w;
  if (count != 10 || !here(a[0], a[1], a[9], &h) || !product_args(a + 1, h.device, &p) || !flag(a[7], &want_x) || !flag(a[8], &want_w) ||
      !(want_x || want_w))
    TOPK_NONE;
  const at::Tensor* t = rows_of(a[6], h.device);
  if (t == nullptr || t->scalar_type() != p.x->scalar_type() || t->size(0) != p.slots || t->size(1) != p.ho) TOPK_NONE;
  const auto values = at::TensorOptions().dtype(p.x->scalar_type()).device(p.x->device());
  at::Tensor dx, dw;
  if (want_x) dx = at::empty({p.slots, p.hi}, values);
  if (want_w) dw = p.w_in == 1 ? at::empty({p.n, p.ho, p.hi}, values) : at::empty({p.n, p.hi, p.ho}, values).transpose(1, 2);
  const void *xp = data(p.x), *wp = data(p.w), *fp = data(p.offset), *sp = data(p.source), *tp = data(t);
  const int64_t stride = p.x->stride(0), m = p.x->size(0), t_stride = t->stride(0);
  const int type = type_code(*p.x);
  void *dxp = want_x ? dx.data_ptr() : nullptr, *dwp = want_w ? dw.data_ptr() : nullptr;
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = reinterpret_cast<ProductVjpFn>(g_entry[h.entry])(xp, stride, m, wp, p.w_expert, p.w_out, p.w_in, fp, sp, p.k, p.slots, p.n,
                                                        p.hi, p.ho, type, tp, t_stride, dxp, dwp, h.stream);
  Py_END_ALLOW_THREADS
  if (outcome(rc, h.entry) != 1) TOPK_NONE;
  if (!(want_x && want_w)) Py_INCREF(Py_None);       // (the one that is not wanted)
  return tuple_of({want_x ? THPVariable_Wrap(dx) : Py_None, want_w ? THPVariable_Wrap(dw) : Py_None});
  END_HANDLE_TH_ERRORS
}

struct Combine {
  const at::Tensor *y, *slot, *val;
  int64_t rows, k, slots, width;
};
bool combine_args(PyObject* const* a, int device, Combine* c) {
  c->y = rows_of(a[0], device);
  c->slot = words_matrix(a[1], device);
  if (c->y == nullptr || c->slot == nullptr) return false;
  c->rows = c->slot->size(0), c->k = c->slot->size(1), c->slots = c->y->size(0), c->width = c->y->size(1);
  c->val = a[2] == Py_None ? nullptr : whole(a[2], device, at::kFloat, c->slot->sizes());
  return a[2] == Py_None || c->val != nullptr;
}

// combine_fwd(entry, y, slot, val, stream) -> out
PyObject* combine_fwd(PyObject*, PyObject* const* a, Py_ssize_t count) {
  HANDLE_TH_ERRORS
  Here h;
  Combine c;
  if (count != 5 || !here(a[0], a[1], a[4], &h) || !combine_args(a + 1, h.device, &c)) TOPK_NONE;
  at::Tensor out = at::empty({c.rows, c.width}, at::TensorOptions().dtype(c.y->scalar_type()).device(c.y->device()));
  const void *yp = data(c.y), *sp = data(c.slot), *vp = data(c.val);
  const int64_t stride = c.y->stride(0);
  const int type = type_code(*c.y);
  void* op = out.data_ptr();
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = reinterpret_cast<CombineFn>(g_entry[h.entry])(yp, stride, sp, vp, c.rows, c.k, c.slots, c.width, type, op, h.stream);
  Py_END_ALLOW_THREADS
  if (outcome(rc, h.entry) != 1) TOPK_NONE;
  return THPVariable_Wrap(out);
  END_HANDLE_TH_ERRORS
}

// combine_vjp(entry, y, slot, val, cotangent, dy_out, stream) -> (dy, dval or None)
PyObject* combine_vjp(PyObject*, PyObject* const* a, Py_ssize_t count) {
  HANDLE_TH_ERRORS
  Here h;
  Combine c;
  if (count != 7 || !here(a[0], a[1], a[6], &h) || !combine_args(a + 1, h.device, &c)) TOPK_NONE;
  const at::Tensor* t = rows_of(a[4], h.device);
  if (t == nullptr || t->scalar_type() != c.y->scalar_type() || t->size(0) != c.rows || t->size(1) != c.width) TOPK_NONE;
  const auto values = at::TensorOptions().dtype(c.y->scalar_type()).device(c.y->device());
  at::Tensor fresh, dval;
  const at::Tensor* dy = &fresh;
  if (a[5] != Py_None) {
    dy = whole(a[5], h.device, c.y->scalar_type(), {c.slots, c.width});
    if (dy == nullptr || !apart(*dy, c.y) || !apart(*dy, c.slot) || !apart(*dy, c.val) || !apart(*dy, t)) TOPK_NONE;
  } else {
    fresh = at::empty({c.slots, c.width}, values);
  }
  if (c.val != nullptr) dval = at::empty({c.rows, c.k}, values.dtype(at::kFloat));
  const void *yp = data(c.y), *sp = data(c.slot), *vp = data(c.val), *tp = data(t);
  const int64_t stride = c.y->stride(0), t_stride = t->stride(0);
  const int type = type_code(*c.y);
  void *dyp = dy->data_ptr(), *dvp = c.val != nullptr ? dval.data_ptr() : nullptr;
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = reinterpret_cast<CombineVjpFn>(g_entry[h.entry])(yp, stride, sp, vp, tp, t_stride, c.rows, c.k, c.slots, c.width, type, dyp,
                                                        dvp, h.stream);
  Py_END_ALLOW_THREADS
  if (outcome(rc, h.entry) != 1) TOPK_NONE;
  PyObject *first = a[5], *second = Py_None;
  if (first == Py_None) first = THPVariable_Wrap(fresh);
  else Py_INCREF(first);
  if (c.val != nullptr) second = THPVariable_Wrap(dval);
  else Py_INCREF(second);
  return tuple_of({first, second});
  END_HANDLE_TH_ERRORS
}

// setup(raw_stream, check, ((name, address), ..)): entry i is the i-th pair
PyObject* setup(PyObject*, PyObject* args) {
  PyObject *raw, *check, *entries;
  if (!PyArg_ParseTuple(args, "OOO!", &raw, &check, &PyTuple_Type, &entries)) return nullptr;
  const Py_ssize_t count = PyTuple_GET_SIZE(entries);
  if (count > kMaxEntries) {
    PyErr_SetString(PyExc_ValueError, "too many entry points");
    return nullptr;
  }
  for (Py_ssize_t i = 0; i < count; ++i) {
    PyObject *name, *address;
    if (!PyArg_ParseTuple(PyTuple_GET_ITEM(entries, i), "UO", &name, &address)) return nullptr;
    void* ptr = PyLong_AsVoidPtr(address);
    if (PyErr_Occurred()) return nullptr;
    Py_INCREF(name);
    Py_XSETREF(g_names[i], name);
    g_entry[i] = ptr;
  }
  Py_INCREF(raw);
  Py_XSETREF(g_raw_stream, raw);
  Py_INCREF(check);
  Py_XSETREF(g_check, check);
  Py_RETURN_NONE;
}

// workspace_device(index): device of the registered workspace, -1 for none
PyObject* workspace_device(PyObject*, PyObject* o) {
  const long v = PyLong_AsLong(o);
  if (v == -1 && PyErr_Occurred()) return nullptr;
  g_ws_device = int(v);
  Py_RETURN_NONE;
}

// the torch this was built against
PyObject* torch_version(PyObject*, PyObject*) { return PyUnicode_FromString(TOPK_TORCH_VERSION); }

PyMethodDef methods[] = {
    {"fwd", reinterpret_cast<PyCFunction>(fwd), METH_FASTCALL, nullptr},
    {"jvp", reinterpret_cast<PyCFunction>(jvp), METH_FASTCALL, nullptr},
    {"sparse", reinterpret_cast<PyCFunction>(sparse), METH_FASTCALL, nullptr},
    {"loss", reinterpret_cast<PyCFunction>(loss), METH_FASTCALL, nullptr},
    {"route_fwd", reinterpret_cast<PyCFunction>(route_fwd), METH_FASTCALL, nullptr},
    {"route_vjp", reinterpret_cast<PyCFunction>(route_vjp), METH_FASTCALL, nullptr},
    {"expert_map", reinterpret_cast<PyCFunction>(expert_map), METH_FASTCALL, nullptr},
    {"product_fwd", reinterpret_cast<PyCFunction>(product_fwd), METH_FASTCALL, nullptr},
    {"product_vjp", reinterpret_cast<PyCFunction>(product_vjp), METH_FASTCALL, nullptr},
    {"combine_fwd", reinterpret_cast<PyCFunction>(combine_fwd), METH_FASTCALL, nullptr},
    {"combine_vjp", reinterpret_cast<PyCFunction>(combine_vjp), METH_FASTCALL, nullptr},
    {"torch_version", torch_version, METH_NOARGS, nullptr},
    {"setup", setup, METH_VARARGS, nullptr},
    {"workspace_device", workspace_device, METH_O, nullptr},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_call", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__call(void) { return PyModule_Create(&module); }
