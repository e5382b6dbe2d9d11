// Argument marshalling of the per-operator entry points for Python: tensors -> device pointers, sizes and types, one call of the C ABI.
//
// What bounds a small layer is the host: through ctypes a convolution's nineteen arguments cost 5 us of marshalling (1.9 us of conversions,
// 0.28 us for each of nine tensors) beside 2 to 3 us of the launch itself; here 0.6 us.  The entry points are bound by address, so that the
// library is loaded in one place (wmdec.py).  Every function returns the library's status; what torch throws (a tensor without storage has no
// address) becomes a Python error at the entry.
#include <Python.h>
#include <torch/csrc/autograd/python_variable.h>

#include <exception>
#include <initializer_list>
#include <utility>

#include "../../include/wmdec.h"

namespace {

decltype(&wmdec_gn_stats) g_gn_stats;
decltype(&wmdec_gn_silu_conv3x3) g_conv3x3;
decltype(&wmdec_gn_conv1x1) g_conv1x1;
decltype(&wmdec_gn_silu_conv3x3_shortcut) g_shortcut;
decltype(&wmdec_gn_silu_conv3x3_stats) g_conv_stats;
decltype(&wmdec_upsample2x_conv3x3) g_upconv;
decltype(&wmdec_attention) g_attention;
decltype(&wmdec_adaln_fused_projection) g_adaln;
decltype(&wmdec_residual_norm) g_residual_norm;
decltype(&wmdec_rope) g_rope;
decltype(&wmdec_cross_attention) g_cross_attention;

constexpr Py_ssize_t kBind = 8;   // arguments of bind(): as many as no other function has

// Reads the arguments; the first one that is not what it should be leaves a Python error and `ok` false.
struct Reader {
  PyObject* const* args;
  bool ok;
  Reader(const char* who, PyObject* const* a, Py_ssize_t given, Py_ssize_t wanted) : args(a), ok(given == wanted) {
    if (!ok) PyErr_Format(PyExc_TypeError, "%s: %zd arguments expected, got %zd", who, wanted, given);
    else if (wanted != kBind && !g_adaln) { ok = false; PyErr_SetString(PyExc_RuntimeError, "the entry points have not been bound"); }
  }
  const at::Tensor* tensor(int i) {
    if (!ok) return nullptr;
    if (!THPVariable_Check(args[i])) { ok = false; PyErr_Format(PyExc_TypeError, "argument %d: tensor expected", i); return nullptr; }
    const at::Tensor& t = THPVariable_Unpack(args[i]);
    if (!t.is_cuda() || !t.is_contiguous()) { ok = false; PyErr_SetString(PyExc_AssertionError, "device-resident contiguous tensor expected"); return nullptr; }
    return &t;
  }
  void* ptr(int i) {   // of a tensor, null for None
    if (!ok || args[i] == Py_None) return nullptr;
    const at::Tensor* t = tensor(i);
    return t ? t->data_ptr() : nullptr;
  }
  int dtype(int i) {
    const at::Tensor* t = tensor(i);
    if (!t) return 0;
    switch (t->scalar_type()) {
      case at::kFloat: return WMDEC_F32;
      case at::kBFloat16: return WMDEC_BF16;
      case at::kHalf: return WMDEC_F16;
      default: ok = false; PyErr_SetString(PyExc_KeyError, "tensor type is none of float32, bfloat16, float16"); return 0;
    }
  }
  int size(int i, int dim, int dims, bool more = false) {   // of a tensor of `dims` dimensions, or of more
    const at::Tensor* t = tensor(i);
    if (!t) return 0;
    if (t->dim() < dims || (t->dim() > dims && !more)) { ok = false; PyErr_Format(PyExc_ValueError, "argument %d: %d dimensions expected, got %d", i, dims, (int)t->dim()); return 0; }
    return (int)t->size(dim);
  }
  size_t bytes(int i) { const at::Tensor* t = tensor(i); return t ? (size_t)t->nbytes() : 0; }
  int integer(int i) {   // the low bits of what can stand for an index, as ctypes passes it
    if (!ok) return 0;
    const unsigned long v = PyLong_AsUnsignedLongMask(args[i]);
    if (v == (unsigned long)-1 && PyErr_Occurred()) ok = false;
    return (int)v;
  }
  int flag(int i) {   // int() of the argument: None and texts that are no number are refused, 0.5 is 0
    if (!ok) return 0;
    PyObject* whole = PyNumber_Long(args[i]);
    const unsigned long v = whole ? PyLong_AsUnsignedLongMask(whole) : 0;
    Py_XDECREF(whole);
    if (PyErr_Occurred()) ok = false;
    return (int)v;
  }
  float real(int i) {
    if (!ok) return 0.f;
    const double v = PyFloat_AsDouble(args[i]);
    if (v == -1.0 && PyErr_Occurred()) ok = false;
    return (float)v;
  }
  void* address(int i) {
    if (!ok) return nullptr;
    void* v = PyLong_AsVoidPtr(args[i]);
    if (!v && PyErr_Occurred()) ok = false;
    return v;
  }
};
// The arguments of the operators whose tensors may be strided: every tensor is on the device that the stream belongs to, and sizes that have to be
// the same are.  As above, the first fault leaves a Python error.
struct StridedReader : Reader {
  int device;
  StridedReader(const char* who, PyObject* const* a, Py_ssize_t given, Py_ssize_t wanted, int at) : Reader(who, a, given, wanted), device(ok ? integer(at) : 0) {
    if (ok && !g_cross_attention) { ok = false; PyErr_SetString(PyExc_RuntimeError, "the entry points have not been bound"); }
  }
  bool none(int i) const { return args[i] == Py_None; }
  void fail(PyObject* type, const char* what, int i) { if (ok) { ok = false; PyErr_Format(type, "argument %d: %s", i, what); } }
  // a tensor of `dims` dimensions on the device, its last dimension contiguous; null for None or a fault
  const at::Tensor* get(int i, int dims) {
    if (!ok || none(i)) return nullptr;
    if (!THPVariable_Check(args[i])) { fail(PyExc_TypeError, "tensor expected", i); return nullptr; }
    const at::Tensor& t = THPVariable_Unpack(args[i]);
    if (!t.is_cuda() || t.device().index() != device) { fail(PyExc_AssertionError, "a tensor on the current device is expected", i); return nullptr; }
    if (t.dim() != dims) { fail(PyExc_ValueError, "wrong number of dimensions", i); return nullptr; }
    if (dims && t.size(dims - 1) > 1 && t.stride(dims - 1) != 1) { fail(PyExc_ValueError, "the last dimension has to be contiguous", i); return nullptr; }
    for (int64_t s : t.sizes())
      if (s > 0x7fffffff) { fail(PyExc_ValueError, "a dimension of 2^31 or more", i); return nullptr; }
    return &t;
  }
  const at::Tensor* need(int i, int dims) {
    const at::Tensor* t = get(i, dims);
    if (ok && !t) fail(PyExc_TypeError, "tensor expected", i);
    return t;
  }
  void* address_of(const at::Tensor* t) { return ok && t ? t->data_ptr() : nullptr; }
  int type_of(const at::Tensor* t, int i) {
    if (!ok || !t) return WMDEC_F32;
    switch (t->scalar_type()) {
      case at::kFloat: return WMDEC_F32;
      case at::kBFloat16: return WMDEC_BF16;
      case at::kHalf: return WMDEC_F16;
      default: fail(PyExc_KeyError, "tensor type is none of float32, bfloat16, float16", i); return WMDEC_F32;
    }
  }
  void same(const at::Tensor* t, const at::Tensor* like, int i) {   // sizes and type
    if (ok && t && (t->sizes() != like->sizes() || t->scalar_type() != like->scalar_type())) fail(PyExc_ValueError, "sizes or type do not match", i);
  }
  void dense(const at::Tensor* t, int i) { if (ok && t && !t->is_contiguous()) fail(PyExc_AssertionError, "contiguous tensor expected", i); }
  void* typed(int i, std::initializer_list<int64_t> sizes, std::initializer_list<at::ScalarType> types) {   // dense, of these sizes and one of these types; null for None
    const at::Tensor* t = get(i, (int)sizes.size());
    dense(t, i);
    if (!ok || !t) return nullptr;
    bool fits = t->sizes() == at::IntArrayRef(sizes), known = false;
    for (at::ScalarType type : types) known = known || t->scalar_type() == type;
    if (!fits || !known) fail(PyExc_ValueError, "sizes or type do not match", i);
    return address_of(t);
  }
  // strides of a [sample, token, head, channel] tensor; those of dimensions of one element are not used
  wmdec_strides strides(const at::Tensor* t) {
    if (!ok || !t) return {0, 0, 0};
    auto of = [&](int i) -> long long { return t->size(i) > 1 ? t->stride(i) : 0; };
    return {of(0), of(1), of(2)};
  }
};
// Other threads run Python until its end, also where that is an exception: the handler in entry() sets a Python error.
struct ThreadsAllowed {
  PyThreadState* state = PyEval_SaveThread();
  ~ThreadsAllowed() { PyEval_RestoreThread(state); }
};
#define WMDEC_RETURN(call_)                    \
  do {                                         \
    if (!r.ok) return nullptr;                 \
    int status;                                \
    {                                          \
      ThreadsAllowed threads;                  \
      status = call_;                          \
    }                                          \
    return PyLong_FromLong(status);            \
  } while (0)

// x, groups, eps, mean, rstd, workspace, stream
PyObject* gn_stats(PyObject*, PyObject* const* a, Py_ssize_t na) {
  Reader r("gn_stats", a, na, 7);
  const void* x = r.ptr(0);
  const int dt = r.dtype(0), n = r.size(0, 0, 4), h = r.size(0, 1, 4), w = r.size(0, 2, 4), c = r.size(0, 3, 4), groups = r.integer(1);
  const float eps = r.real(2);
  float *mean = (float*)r.ptr(3), *rstd = (float*)r.ptr(4);
  void* ws = r.ptr(5);
  const size_t bytes = r.bytes(5);
  void* stream = r.address(6);
  WMDEC_RETURN(g_gn_stats(x, dt, n, h, w, c, groups, eps, mean, rstd, ws, bytes, stream));
}

// the arguments that the convolutions share: x, mean, rstd, gamma, beta, groups, apply_silu, w_packed, bias
struct ConvHead {
  const void *x, *w;
  const float *mean, *rstd, *gamma, *beta, *bias;
  int dt, groups, silu, cin;
  ConvHead(Reader& r, int at)
      : x(r.ptr(at)), w(nullptr), dt(r.dtype(at)), cin(r.size(at, 3, 4, true)) {
    mean = (const float*)r.ptr(at + 1); rstd = (const float*)r.ptr(at + 2); gamma = (const float*)r.ptr(at + 3); beta = (const float*)r.ptr(at + 4);
    groups = r.integer(at + 5); silu = r.flag(at + 6);
    w = r.ptr(at + 7); bias = (const float*)r.ptr(at + 8);
  }
};
struct Output { void* y; int dt, n, h, w, c; Output(Reader& r, int i) : y(r.ptr(i)), dt(r.dtype(i)), n(r.size(i, 0, 4)), h(r.size(i, 1, 4)), w(r.size(i, 2, 4)), c(r.size(i, 3, 4)) {} };

// ksize, <head>, residual, y, stream
PyObject* conv(PyObject*, PyObject* const* a, Py_ssize_t na) {
  Reader r("conv", a, na, 13);
  if (!r.ok) return nullptr;
  const int k = r.integer(0);
  const ConvHead c(r, 1);
  const void* res = r.ptr(10);
  const Output y(r, 11);
  void* stream = r.address(12);
  WMDEC_RETURN((k == 3 ? g_conv3x3 : g_conv1x1)(c.x, c.dt, c.mean, c.rstd, c.gamma, c.beta, c.groups, c.silu, c.w, c.bias, res, y.y, y.dt, y.n, y.h, y.w, c.cin, y.c, stream));
}

// <head>, x2, w2_packed, bias2, y, stream
PyObject* conv_shortcut(PyObject*, PyObject* const* a, Py_ssize_t na) {
  Reader r("gn_silu_conv3x3_shortcut", a, na, 14);
  if (!r.ok) return nullptr;
  const ConvHead c(r, 0);
  const void *x2 = r.ptr(9), *w2 = r.ptr(10);
  const int cin2 = r.size(9, 3, 4, true);
  const float* bias2 = (const float*)r.ptr(11);
  const Output y(r, 12);
  void* stream = r.address(13);
  WMDEC_RETURN(g_shortcut(c.x, c.dt, c.mean, c.rstd, c.gamma, c.beta, c.groups, c.silu, c.w, c.bias, x2, cin2, w2, bias2, y.y, y.dt, y.n, y.h, y.w, c.cin, y.c, stream));
}

// <head>, residual, y, out_groups, out_eps, mean_out, rstd_out, workspace, stream
PyObject* conv_stats(PyObject*, PyObject* const* a, Py_ssize_t na) {
  Reader r("gn_silu_conv3x3_stats", a, na, 17);
  if (!r.ok) return nullptr;
  const ConvHead c(r, 0);
  const void* res = r.ptr(9);
  const Output y(r, 10);
  const int groups = r.integer(11);
  const float eps = r.real(12);
  float *mean = (float*)r.ptr(13), *rstd = (float*)r.ptr(14);
  void* ws = r.ptr(15);
  const size_t bytes = r.bytes(15);
  void* stream = r.address(16);
  WMDEC_RETURN(g_conv_stats(c.x, c.dt, c.mean, c.rstd, c.gamma, c.beta, c.groups, c.silu, c.w, c.bias, res, y.y, y.dt, y.n, y.h, y.w, c.cin, y.c, groups, eps, mean, rstd, ws,
                            bytes, stream));
}

// x, w_packed, bias, y, stream
PyObject* upconv(PyObject*, PyObject* const* a, Py_ssize_t na) {
  Reader r("upsample2x_conv3x3", a, na, 5);
  if (!r.ok) return nullptr;
  const Output x(r, 0);   // (a tensor's pointer, type and sizes)
  const void* w = r.ptr(1);
  const float* bias = (const float*)r.ptr(2);
  const Output y(r, 3);
  void* stream = r.address(4);
  WMDEC_RETURN(g_upconv(x.y, x.dt, w, bias, y.y, y.dt, x.n, x.h, x.w, x.c, y.c, stream));
}

// x, mean, rstd, gamma, beta, groups, wqkv_packed, bqkv, wo_packed, bo, y, workspace, stream
PyObject* attention(PyObject*, PyObject* const* a, Py_ssize_t na) {
  Reader r("attention", a, na, 13);
  if (!r.ok) return nullptr;
  const Output x(r, 0);
  const float *mean = (const float*)r.ptr(1), *rstd = (const float*)r.ptr(2), *gamma = (const float*)r.ptr(3), *beta = (const float*)r.ptr(4);
  const int groups = r.integer(5);
  const void* wqkv = r.ptr(6);
  const float* bqkv = (const float*)r.ptr(7);
  const void* wo = r.ptr(8);
  const float* bo = (const float*)r.ptr(9);
  void *y = r.ptr(10), *ws = r.ptr(11);
  const size_t bytes = r.bytes(11);
  void* stream = r.address(12);
  WMDEC_RETURN(g_attention(x.y, x.dt, mean, rstd, gamma, beta, groups, wqkv, bqkv, wo, bo, y, x.n, x.h, x.w, x.c, ws, bytes, stream));
}

// c, w_fused, bias, out, apply_silu, stream
PyObject* adaln(PyObject*, PyObject* const* a, Py_ssize_t na) {
  Reader r("adaln_fused_projection", a, na, 6);
  if (!r.ok) return nullptr;
  const void *c = r.ptr(0), *w = r.ptr(1);
  const int cdt = r.dtype(0), wdt = r.dtype(1), batch = r.size(0, 0, 2), d = r.size(0, 1, 2);
  const at::Tensor* wt = r.tensor(1);
  const int rows = wt && wt->dim() > 0 ? (int)wt->size(0) : 0;
  const float* bias = (const float*)r.ptr(2);
  float* out = (float*)r.ptr(3);
  const int silu = r.flag(4);
  void* stream = r.address(5);
  WMDEC_RETURN(g_adaln(c, cdt, w, wdt, bias, out, batch, d, rows, silu, stream));
}

// (kind, eps, weight, bias) of a norm over d channels; None is the norm that does nothing
wmdec_norm norm(StridedReader& r, int at, int64_t d) {
  wmdec_norm v{WMDEC_NORM_NONE, 0.f, nullptr, nullptr};
  if (!r.ok || r.none(at)) return v;
  PyObject* spec = r.args[at];
  if (!PyTuple_Check(spec) || PyTuple_GET_SIZE(spec) != 4 || !PyUnicode_Check(PyTuple_GET_ITEM(spec, 0))) { r.fail(PyExc_TypeError, "a Norm or None is expected", at); return v; }
  PyObject* kind = PyTuple_GET_ITEM(spec, 0);
  if (PyUnicode_CompareWithASCIIString(kind, "layer") == 0) v.kind = WMDEC_NORM_LAYER;
  else if (PyUnicode_CompareWithASCIIString(kind, "rms") == 0) v.kind = WMDEC_NORM_RMS;
  else if (PyUnicode_CompareWithASCIIString(kind, "none") != 0) { r.fail(PyExc_KeyError, "the kind of a norm is none of none, layer, rms", at); return v; }
  PyObject* const* outer = r.args;
  r.args = &PyTuple_GET_ITEM(spec, 0);
  v.eps = r.real(1);
  v.weight = (const float*)r.typed(2, {d}, {at::kFloat}); v.bias = (const float*)r.typed(3, {d}, {at::kFloat});
  r.args = outer;
  return v;
}

// x, h, post, gate, res_scale, x_out, pre, scale, shift, y, device, stream
PyObject* residual_norm(PyObject*, PyObject* const* a, Py_ssize_t na) {
  StridedReader r("residual_norm", a, na, 12, 10);
  const at::Tensor *x = r.need(0, 3), *h = r.ok ? r.get(1, 3) : nullptr, *x_out = r.ok ? r.get(5, 3) : nullptr, *y = r.ok ? r.get(9, 3) : nullptr;
  for (auto [t, i] : {std::pair{x, 0}, {h, 1}, {x_out, 5}, {y, 9}}) r.dense(t, i);
  if (!r.ok) return nullptr;
  const at::Tensor* act = h ? h : y ? y : x;
  const int xdt = r.type_of(x, 0), adt = r.type_of(act, 1);
  r.same(x_out, x, 5);
  if (h && y) r.same(y, h, 9);
  if (r.ok && act->sizes() != x->sizes()) r.fail(PyExc_ValueError, "sizes or type do not match", h ? 1 : 9);
  if (!r.ok) return nullptr;
  const int64_t n = x->size(0), d = x->size(2);
  const wmdec_norm post = norm(r, 2, d), pre = norm(r, 6, d);
  long long stride = -1;
  const float* mod[3];
  const int at_mod[3] = {3, 7, 8};
  for (int i = 0; i < 3; ++i) {
    const at::Tensor* m = r.get(at_mod[i], 2);
    mod[i] = (const float*)r.address_of(m);
    if (!r.ok || !m) continue;
    const long long s = n > 1 ? m->stride(0) : 0;
    if (m->size(0) != n || m->size(1) != d || m->scalar_type() != at::kFloat) r.fail(PyExc_ValueError, "sizes or type do not match", at_mod[i]);
    else if (stride >= 0 && s != stride) r.fail(PyExc_ValueError, "gate, scale and shift have the same stride", at_mod[i]);
    stride = s;
  }
  const float res_scale = r.real(4);
  void *px = r.address_of(x), *ph = r.address_of(h), *pxo = r.address_of(x_out), *py = r.address_of(y);
  void* stream = r.address(11);
  WMDEC_RETURN(g_residual_norm(px, xdt, ph, adt, &post, mod[0], res_scale, pxo, &pre, mod[1], mod[2], stride < 0 ? 0 : stride, py, (int)n, (int)x->size(1), (int)d, stream));
}

// q, k, positions, freq, axes, dim0, dim1, dim2, q_out, k_out, interleaved, inverse, magnitude, device, stream
PyObject* rope(PyObject*, PyObject* const* a, Py_ssize_t na) {
  StridedReader r("rope", a, na, 15, 13);
  const at::Tensor *q = r.need(0, 4), *q_out = r.ok ? r.need(8, 4) : nullptr, *k = r.ok ? r.get(1, 4) : nullptr, *k_out = r.ok && k ? r.need(9, 4) : nullptr;
  if (!r.ok) return nullptr;
  if (!k && !r.none(9)) r.fail(PyExc_ValueError, "k_out without k", 9);
  const int dt = r.type_of(q, 0);
  r.same(q_out, q, 8);
  if (k) r.same(k_out, k, 9);
  const int64_t n = q->size(0), t = q->size(1), d = q->size(3);
  if (r.ok && k && (k->size(0) != n || k->size(1) != t || k->size(3) != d || k->scalar_type() != q->scalar_type())) r.fail(PyExc_ValueError, "sizes or type do not match", 1);
  wmdec_rope_layout lay;
  lay.axes = r.integer(4);
  for (int i = 0; i < 3; ++i) lay.axis_dim[i] = r.integer(5 + i);
  lay.interleaved = r.flag(10); lay.inverse = r.flag(11); lay.magnitude = r.real(12);
  if (!r.ok) return nullptr;
  if (r.none(2) || r.none(3)) { r.fail(PyExc_TypeError, "tensor expected", r.none(2) ? 2 : 3); return nullptr; }
  const bool shared = THPVariable_Check(a[2]) && THPVariable_Unpack(a[2]).dim() == 2;
  const int* pos = (const int*)(shared ? r.typed(2, {t, lay.axes}, {at::kInt}) : r.typed(2, {n, t, lay.axes}, {at::kInt}));
  int64_t pairs = 0;
  for (int i = 0; i < lay.axes && i < 3; ++i) pairs += lay.axis_dim[i] / 2;
  const double* freq = (const double*)r.typed(3, {pairs}, {at::kDouble});
  const wmdec_strides qs = r.strides(q), qos = r.strides(q_out), ks = r.strides(k), kos = r.strides(k_out);
  void *pq = r.address_of(q), *pqo = r.address_of(q_out), *pk = r.address_of(k), *pko = r.address_of(k_out);
  void* stream = r.address(14);
  WMDEC_RETURN(g_rope(pq, &qs, pqo, &qos, (int)q->size(2), pk, &ks, pko, &kos, k ? (int)k->size(2) : 0, dt, pos, shared ? 0 : t * lay.axes, freq, &lay, (int)n, (int)t, (int)d, stream));
}

// q, k, v, o, scale, key_lens, key_mask, workspace, device, stream
PyObject* cross_attention(PyObject*, PyObject* const* a, Py_ssize_t na) {
  StridedReader r("cross_attention", a, na, 10, 8);
  const at::Tensor *q = r.need(0, 4), *k = r.ok ? r.need(1, 4) : nullptr, *v = r.ok ? r.need(2, 4) : nullptr, *o = r.ok ? r.need(3, 4) : nullptr;
  if (!r.ok) return nullptr;
  const int dt = r.type_of(q, 0);
  r.same(v, k, 2);
  r.same(o, q, 3);
  const int64_t n = q->size(0), tk = k->size(1);
  if (r.ok && (k->size(0) != n || k->size(3) != q->size(3) || k->scalar_type() != q->scalar_type())) r.fail(PyExc_ValueError, "sizes or type do not match", 1);
  const float scale = r.real(4);
  const int* lens = (const int*)r.typed(5, {n}, {at::kInt});
  const unsigned char* mask = (const unsigned char*)r.typed(6, {n, tk}, {at::kBool, at::kByte});
  const at::Tensor* ws = r.get(7, 1);
  r.dense(ws, 7);
  const wmdec_strides qs = r.strides(q), ks = r.strides(k), vs = r.strides(v), os = r.strides(o);
  void *pq = r.address_of(q), *pk = r.address_of(k), *pv = r.address_of(v), *po = r.address_of(o), *pw = r.address_of(ws);
  const size_t bytes = ws ? (size_t)ws->nbytes() : 0;
  void* stream = r.address(9);
  WMDEC_RETURN(g_cross_attention(pq, &qs, pk, &ks, pv, &vs, po, &os, dt, scale, lens, mask, (int)n, (int)q->size(1), (int)tk, (int)q->size(2), (int)k->size(2), (int)q->size(3), pw,
                                 bytes, stream));
}

// the addresses of these three, in the order of wmdec.py
PyObject* bind_block(PyObject*, PyObject* const* a, Py_ssize_t na) {
  Reader r("bind_block", a, na, 3);
  void* f[3];
  for (int i = 0; i < 3; ++i) f[i] = r.address(i);
  if (!r.ok) return nullptr;
  g_residual_norm = (decltype(g_residual_norm))f[0]; g_rope = (decltype(g_rope))f[1]; g_cross_attention = (decltype(g_cross_attention))f[2];
  Py_RETURN_NONE;
}

// the addresses of the entry points, in the order of wmdec.py
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t na) {
  Reader r("bind", a, na, kBind);
  void* f[kBind];
  for (int i = 0; i < kBind; ++i) f[i] = r.address(i);
  if (!r.ok) return nullptr;
  g_gn_stats = (decltype(g_gn_stats))f[0]; g_conv3x3 = (decltype(g_conv3x3))f[1]; g_conv1x1 = (decltype(g_conv1x1))f[2];
  g_shortcut = (decltype(g_shortcut))f[3]; g_conv_stats = (decltype(g_conv_stats))f[4]; g_upconv = (decltype(g_upconv))f[5];
  g_attention = (decltype(g_attention))f[6]; g_adaln = (decltype(g_adaln))f[7];
  Py_RETURN_NONE;
}

template <PyObject* (*F)(PyObject*, PyObject* const*, Py_ssize_t)> PyObject* entry(PyObject* self, PyObject* const* a, Py_ssize_t na) {
  try {
    return F(self, a, na);
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}
#define WMDEC_METHOD(name_) {#name_, (PyCFunction)(void (*)())entry<name_>, METH_FASTCALL, nullptr}
PyMethodDef g_methods[] = {WMDEC_METHOD(gn_stats), WMDEC_METHOD(conv), WMDEC_METHOD(conv_shortcut), WMDEC_METHOD(conv_stats), WMDEC_METHOD(upconv),
                           WMDEC_METHOD(attention), WMDEC_METHOD(adaln), WMDEC_METHOD(residual_norm), WMDEC_METHOD(rope), WMDEC_METHOD(cross_attention),
                           WMDEC_METHOD(bind), WMDEC_METHOD(bind_block), {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding(void) { return PyModule_Create(&g_module); }
