// The repeated calls of the Python classes on torch tensors without the interpreter's detour: a call asks each
// tensor what it is and starts the product in native code.  A product over a few thousand rows takes the GPU 3.4 to
// 4.5 us; asked one attribute at a time and called through ctypes it took the host 4.7 to 5.2 us, of which the launch
// itself is 2.4.
//
// Every function returns 1 where it has called the library and that has accepted, the library's error code (negative)
// where it has not, and 0 where the arguments are anything but the plain case: dense float32 tensors of the
// right sizes on the handle's device.  The caller then goes the general way, which allocates, asserts and reports.
//
// The calls on sequences (attention, embedding) return their results instead, the error code, or None for the general way.
#include <Python.h>
#include <ATen/Context.h>
#include <ATen/hip/EmptyTensor.h>
#include <ATen/ops/empty.h>
#include <ATen/record_function.h>
#include <c10/core/impl/LocalDispatchKeySet.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "arrow_attention.h"
#include "arrow_embedding.h"
#include "arrow_logprobs.h"
#include "arrow_packed.h"
#include "arrow_pages.h"
#include "arrow_rotation.h"

namespace {

// The tensor where it is a dense, contiguous float32 one on the device, else null.
const at::Tensor* plain(PyObject* o, int64_t device) {
  if (!THPVariable_CheckExact(o)) return nullptr;
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.defined() || !t.has_storage() || t.scalar_type() != at::kFloat || !t.is_cuda() || t.get_device() != device || !t.is_contiguous())
    return nullptr;
  return &t;
}

const at::Tensor* matrix(PyObject* o, int64_t device, int64_t rows) {
  const at::Tensor* t = plain(o, device);
  return t && t->dim() == 2 && t->size(0) == rows ? t : nullptr;
}

bool integers(PyObject* const* args, int count, int64_t* out) {
  for (int i = 0; i < count; ++i) {
    out[i] = PyLong_AsLongLong(args[i]);
    if (out[i] == -1 && PyErr_Occurred()) return false;
  }
  return true;
}

float* at_data(const at::Tensor* t) { return static_cast<float*>(t->data_ptr()); }
void* stream_of(int64_t device) { return c10::hip::getCurrentHIPStream((c10::DeviceIndex)device).stream(); }

template <typename F>
PyObject* guarded(F&& call) {
  try {
    return PyLong_FromLong(call());
  } catch (...) {             // (a tensor without data: the general way says what is wrong with it)
    return PyLong_FromLong(0);
  }
}

template <typename F>
long started(F&& call) {
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = call();
  Py_END_ALLOW_THREADS
  return rc == 0 ? 1 : rc;
}

bool arguments(Py_ssize_t have, Py_ssize_t want) {
  if (have != want) PyErr_Format(PyExc_TypeError, "%zd arguments expected, got %zd", want, have);
  return have == want;
}

// spmm(function, handle, device, n, most columns, X, Y)
PyObject* spmm(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
  int64_t v[5];
  if (!arguments(n_args, 7) || !integers(args, 5, v)) return nullptr;
  return guarded([&]() -> long {
    const at::Tensor *X = matrix(args[5], v[2], v[3]), *Y = matrix(args[6], v[2], v[3]);
    if (!X || !Y || X->size(1) != Y->size(1) || X->size(1) < 1 || X->size(1) > v[4]) return 0;
    auto call = reinterpret_cast<int (*)(void*, const float*, float*, int32_t, void*)>(v[0]);
    float *x = at_data(X), *y = at_data(Y);
    const int32_t k = (int32_t)X->size(1);
    void* stream = stream_of(v[2]);
    return started([&] { return call(reinterpret_cast<void*>(v[1]), x, y, k, stream); });
  });
}

// sddmm(function, handle, device, n, most columns, entries, U, V, S)
PyObject* sddmm(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
  int64_t v[6];
  if (!arguments(n_args, 9) || !integers(args, 6, v)) return nullptr;
  return guarded([&]() -> long {
    const at::Tensor *U = matrix(args[6], v[2], v[3]), *V = matrix(args[7], v[2], v[3]), *S = plain(args[8], v[2]);
    if (!U || !V || !S || U->size(1) != V->size(1) || U->size(1) < 1 || U->size(1) > v[4] || S->numel() != v[5]) return 0;
    auto call = reinterpret_cast<int (*)(void*, const float*, const float*, float*, int32_t, void*)>(v[0]);
    float *u = at_data(U), *w = at_data(V), *s = at_data(S);
    const int32_t k = (int32_t)U->size(1);
    void* stream = stream_of(v[2]);
    return started([&] { return call(reinterpret_cast<void*>(v[1]), u, w, s, k, stream); });
  });
}

// mttkrp(function, handle, device, I, J, K, most columns, B, C, A)
PyObject* mttkrp(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
  int64_t v[7];
  if (!arguments(n_args, 10) || !integers(args, 7, v)) return nullptr;
  return guarded([&]() -> long {
    const at::Tensor *B = matrix(args[7], v[2], v[4]), *C = matrix(args[8], v[2], v[5]), *A = matrix(args[9], v[2], v[3]);
    if (!A || !B || !C || B->size(1) != A->size(1) || C->size(1) != A->size(1) || A->size(1) < 1 || A->size(1) > v[6]) return 0;
    auto call = reinterpret_cast<int (*)(void*, const float*, const float*, float*, int32_t, void*)>(v[0]);
    float *a = at_data(A), *b = at_data(B), *c = at_data(C);
    const int32_t R = (int32_t)A->size(1);
    void* stream = stream_of(v[2]);
    return started([&] { return call(reinterpret_cast<void*>(v[1]), b, c, a, R, stream); });
  });
}

// ---- sequences ----

PyObject* none() { Py_RETURN_NONE; }

// Of a call's arguments: the tensor, or null for None; `ok` becomes false for anything else, and for tensors elsewhere.
struct Tensors {
  int64_t device;
  bool ok = true;
  const at::Tensor* operator()(PyObject* o) {
    if (o == Py_None) return nullptr;
    if (!THPVariable_CheckExact(o)) { ok = false; return nullptr; }
    const at::Tensor& t = THPVariable_Unpack(o);
    ok = ok && t.defined() && t.has_storage() && t.is_cuda() && t.get_device() == device;
    return &t;
  }
};

int half_type(const at::Tensor& t) { return t.scalar_type() == at::kBFloat16 ? ARROW_BF16 : t.scalar_type() == at::kHalf ? ARROW_F16 : -1; }
bool rows_whole(const at::Tensor& t) { return t.size(-1) <= 1 || t.stride(-1) == 1; }
bool like(const at::Tensor& t, const at::Tensor& other) { return t.scalar_type() == other.scalar_type() && t.sizes() == other.sizes() && rows_whole(t); }
// Whether someone looks at allocations, or wants them filled: dispatch modes and the like, profilers, deterministic algorithms.
bool watched() {
  if (!(c10::impl::tls_local_dispatch_key_set().included_ - c10::default_included_set).empty() || at::hasCallbacks()) return true;
  const at::Context& context = at::globalContext();
  return context.deterministicAlgorithms() && context.deterministicFillUninitializedMemory();
}
// (without torch's dispatcher where nobody does: 0.47 us instead of 0.70, which a call takes up to seven times)
at::Tensor made(at::IntArrayRef sizes, const at::Tensor& on, at::ScalarType type) {
  return watched() ? at::empty(sizes, on.options().dtype(type)) : at::detail::empty_cuda(sizes, type, on.device(), std::nullopt);
}
void* data(const at::Tensor& t) { return t.data_ptr(); }

// Steps between sequences, tokens and heads of (sequences, tokens, heads, dim) or (tokens, heads, dim); one that is never taken counts as none.
arrow_strides_t steps(const at::Tensor& t) {
  const int64_t n = t.dim();
  auto step = [&](int64_t d) { return t.size(d) > 1 ? t.stride(d) : 0; };
  return {n == 4 ? step(0) : 0, step(n - 3), step(n - 2)};
}

bool small(int64_t x) { return x >= 0 && x <= 0x7fffffff; }

// Mask, scale, operands and offsets of a call on whole sequences; false for the general way.
bool describe(arrow_attention_t& a, int64_t window, int64_t sinks, double scale, const at::Tensor* q, const at::Tensor* k, const at::Tensor* v,
              const at::Tensor* q_offsets, const at::Tensor* k_offsets, int64_t q_len, int64_t k_len) {
  if (!q || !k || !v || !q_offsets != !k_offsets) return false;
  const bool ragged = q_offsets;
  const int64_t n = ragged ? 3 : 4;
  if (q->dim() != n || k->dim() != n || half_type(*q) < 0 || k->scalar_type() != q->scalar_type() || !like(*v, *k)) return false;
  if (k->size(-1) != q->size(-1) || !rows_whole(*q) || !rows_whole(*k)) return false;
  for (int64_t d = 0; d < n; ++d)
    if (!small(q->size(d)) || !small(k->size(d))) return false;
  a.dtype = half_type(*q);
  a.q_heads = (int32_t)q->size(-2); a.kv_heads = (int32_t)k->size(-2); a.dim = (int32_t)q->size(-1);
  a.window = (int32_t)window; a.sinks = (int32_t)sinks;
  a.scale = (float)(scale >= 0 ? scale : 1.0 / std::sqrt((double)std::max<int64_t>(1, a.dim)));
  if (ragged) {
    for (auto* t : {q_offsets, k_offsets})
      if (t->scalar_type() != at::kInt || t->dim() != 1 || !t->is_contiguous() || t->numel() < 1 || t->numel() != q_offsets->numel()) return false;
    a.batch = (int32_t)(q_offsets->numel() - 1);
    a.q_tokens = q->size(0); a.k_tokens = k->size(0);
    a.q_len = (int32_t)(q_len >= 0 ? std::min(q_len, a.q_tokens) : a.q_tokens);
    a.k_len = (int32_t)(k_len >= 0 ? std::min(k_len, a.k_tokens) : a.k_tokens);
    a.q_offsets = q_offsets->const_data_ptr<int32_t>(); a.k_offsets = k_offsets->const_data_ptr<int32_t>();
  } else {
    if (q_len >= 0 || k_len >= 0 || q->size(0) != k->size(0)) return false;
    a.batch = (int32_t)q->size(0); a.q_len = (int32_t)q->size(1); a.k_len = (int32_t)k->size(1);
  }
  a.q = steps(*q); a.k = steps(*k); a.v = steps(*v);
  return true;
}

bool is_lse(const at::Tensor& t, const arrow_attention_t& a) {
  if (t.scalar_type() != at::kFloat || !t.is_contiguous()) return false;
  return a.q_offsets ? t.dim() == 2 && t.size(0) == a.q_heads && t.size(1) == a.q_tokens
                     : t.dim() == 3 && t.size(0) == a.batch && t.size(1) == a.q_heads && t.size(2) == a.q_len;
}

// One value of a call's arguments each, None as -1.
bool lengths(PyObject* const* args, int count, int64_t* out) {
  for (int i = 0; i < count; ++i) {
    out[i] = -1;
    if (args[i] == Py_None) continue;
    out[i] = PyLong_AsLongLong(args[i]);
    if (out[i] < 0) { PyErr_Clear(); return false; }
  }
  return true;
}

// What the functions below have in common: None where `call` says so or throws, its error code, or the results.
template <typename F>
PyObject* results(int64_t device, F&& call) {
  at::Tensor out[6];
  int rc = 0, n = 0;
  try {
    if (c10::hip::current_device() != (c10::DeviceIndex)device) return none();
    n = call(out, rc);
  } catch (...) {             // (a tensor without data, or no memory left: the general way says what is wrong)
    return none();
  }
  if (n == 0) return none();
  if (rc != 0) return PyLong_FromLong(rc);
  if (n == 1) return THPVariable_Wrap(out[0]);
  PyObject* tuple = PyTuple_New(n);
  for (int i = 0; tuple && i < n; ++i) PyTuple_SET_ITEM(tuple, i, THPVariable_Wrap(out[i]));
  return tuple;
}

template <typename F>
int quietly(F&& call) {
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = call();
  Py_END_ALLOW_THREADS
  return rc;
}

// attention_forward(function, of the workspace's size, device, window, sinks, scale or -1, q, k, v, o, lse, q_offsets, k_offsets, q_len, k_len)
PyObject* attention_forward(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
  int64_t x[5], len[2];
  if (!arguments(n_args, 15) || !integers(args, 5, x)) return nullptr;
  const double scale = PyFloat_AsDouble(args[5]);
  if (PyErr_Occurred()) return nullptr;
  if (!lengths(args + 13, 2, len)) return none();
  return results(x[2], [&](at::Tensor* out, int& rc) {
    Tensors tensor{x[2]};
    const at::Tensor *q = tensor(args[6]), *k = tensor(args[7]), *v = tensor(args[8]), *o = tensor(args[9]), *lse = tensor(args[10]);
    const at::Tensor *q_offsets = tensor(args[11]), *k_offsets = tensor(args[12]);
    arrow_attention_t a{};
    if (!tensor.ok || !describe(a, x[3], x[4], scale, q, k, v, q_offsets, k_offsets, len[0], len[1])) return 0;
    if ((o && !like(*o, *q)) || (lse && !is_lse(*lse, a))) return 0;
    out[0] = o ? *o : made(q->sizes(), *q, q->scalar_type());
    out[1] = lse ? *lse : a.q_offsets ? made({a.q_heads, a.q_tokens}, *q, at::kFloat) : made({a.batch, a.q_heads, a.q_len}, *q, at::kFloat);
    a.o = steps(out[0]);
    const size_t bytes = reinterpret_cast<decltype(&arrow_attention_forward_split_bytes)>(x[1])(&a);
    const at::Tensor ws = bytes ? made({(int64_t)bytes}, *q, at::kByte) : at::Tensor();
    void *qp = data(*q), *kp = data(*k), *vp = data(*v), *op = data(out[0]), *lp = data(out[1]), *wp = bytes ? data(ws) : nullptr, *stream = stream_of(x[2]);
    rc = quietly([&] { return reinterpret_cast<decltype(&arrow_attention_forward_split)>(x[0])(&a, qp, kp, vp, op, (float*)lp, wp, bytes, stream); });
    return 2;
  });
}

// attention_backward(function, of the workspace's size, device, window, sinks, scale or -1, d_o, q, k, v, o, lse, dq, dk, dv, q_offsets, k_offsets,
// q_len, k_len)
PyObject* attention_backward(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
  int64_t x[5], len[2];
  if (!arguments(n_args, 19) || !integers(args, 5, x)) return nullptr;
  const double scale = PyFloat_AsDouble(args[5]);
  if (PyErr_Occurred()) return nullptr;
  if (!lengths(args + 17, 2, len)) return none();
  return results(x[2], [&](at::Tensor* out, int& rc) {
    Tensors tensor{x[2]};
    const at::Tensor *d_o = tensor(args[6]), *q = tensor(args[7]), *k = tensor(args[8]), *v = tensor(args[9]), *o = tensor(args[10]);
    const at::Tensor *lse = tensor(args[11]), *dq = tensor(args[12]), *dk = tensor(args[13]), *dv = tensor(args[14]);
    const at::Tensor *q_offsets = tensor(args[15]), *k_offsets = tensor(args[16]);
    arrow_attention_t a{};
    if (!tensor.ok || !describe(a, x[3], x[4], scale, q, k, v, q_offsets, k_offsets, len[0], len[1])) return 0;
    if (!d_o || !o || !lse || !like(*d_o, *q) || !like(*o, *q) || !is_lse(*lse, a)) return 0;
    if ((dq && !like(*dq, *q)) || (dk && !like(*dk, *k)) || (dv && !like(*dv, *v))) return 0;
    out[0] = dq ? *dq : made(q->sizes(), *q, q->scalar_type());
    out[1] = dk ? *dk : made(k->sizes(), *k, q->scalar_type());
    out[2] = dv ? *dv : made(v->sizes(), *v, q->scalar_type());
    a.d_o = steps(*d_o); a.o = steps(*o); a.dq = steps(out[0]); a.dk = steps(out[1]); a.dv = steps(out[2]);
    const at::Tensor ws = made({(int64_t)reinterpret_cast<decltype(&arrow_attention_workspace_bytes)>(x[1])(&a)}, *q, at::kByte);
    void *qp = data(*q), *kp = data(*k), *vp = data(*v), *op = data(*o), *lp = data(*lse), *gp = data(*d_o);
    void *dqp = data(out[0]), *dkp = data(out[1]), *dvp = data(out[2]), *wp = data(ws), *stream = stream_of(x[2]);
    const size_t bytes = (size_t)ws.numel();
    rc = quietly([&] {
      return reinterpret_cast<decltype(&arrow_attention_backward)>(x[0])(&a, qp, kp, vp, op, (const float*)lp, gp, dqp, dkp, dvp, wp, bytes, stream);
    });
    return 3;
  });
}

// attention_decode(function, of the workspace's size, device, window, sinks, scale or -1, q, k_cache, v_cache, table, lengths, max_len, k, v, o)
PyObject* attention_decode(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
  int64_t x[5], max_len;
  if (!arguments(n_args, 15) || !integers(args, 5, x)) return nullptr;
  const double scale = PyFloat_AsDouble(args[5]);
  if (PyErr_Occurred()) return nullptr;
  if (!lengths(args + 11, 1, &max_len)) return none();
  return results(x[2], [&](at::Tensor* out, int& rc) {
    Tensors tensor{x[2]};
    const at::Tensor *q = tensor(args[6]), *kc = tensor(args[7]), *vc = tensor(args[8]), *table = tensor(args[9]), *n = tensor(args[10]);
    const at::Tensor *k = tensor(args[12]), *v = tensor(args[13]), *o = tensor(args[14]);
    if (!tensor.ok || !q || !kc || !vc || !table || !n || !k != !v || q->dim() != 3 || kc->dim() != 4 || half_type(*kc) < 0) return 0;
    if (q->scalar_type() != kc->scalar_type() || !like(*vc, *kc) || !rows_whole(*kc) || !rows_whole(*q) || q->size(2) != kc->size(3)) return 0;
    if (table->scalar_type() != at::kInt || n->scalar_type() != at::kInt || table->dim() != 2 || n->dim() != 1 || !table->is_contiguous() ||
        !n->is_contiguous() || table->size(0) != n->size(0) || q->size(0) != n->size(0))
      return 0;
    for (auto* t : {k, v})
      if (t && (t->scalar_type() != q->scalar_type() || t->dim() != 3 || t->size(0) != n->size(0) || t->size(1) != kc->size(2) || t->size(2) != kc->size(3) ||
                !rows_whole(*t)))
        return 0;
    if (o && !like(*o, *q)) return 0;
    for (int64_t s : {table->size(0), table->size(1), kc->size(1), kc->size(2), q->size(1)})
      if (!small(s)) return 0;
    arrow_cache_t c{};
    c.dtype = half_type(*kc);
    c.batch = (int32_t)table->size(0); c.columns = (int32_t)table->size(1);
    c.pages = kc->size(0); c.page = (int32_t)kc->size(1); c.kv_heads = (int32_t)kc->size(2); c.dim = (int32_t)std::min<int64_t>(kc->size(3), 1 << 20);
    c.q_heads = (int32_t)q->size(1);
    c.window = (int32_t)x[3]; c.sinks = (int32_t)x[4];
    c.scale = (float)(scale >= 0 ? scale : 1.0 / std::sqrt((double)std::max(1, c.dim)));
    c.max_len = max_len >= 0 ? max_len : (int64_t)c.columns * c.page;
    auto step = [](const at::Tensor& t, int64_t d) { return t.size(d) > 1 ? t.stride(d) : 0; };
    c.k_page = step(*kc, 0); c.k_token = step(*kc, 1); c.k_head = step(*kc, 2);
    c.v_page = step(*vc, 0); c.v_token = step(*vc, 1); c.v_head = step(*vc, 2);
    c.table = table->const_data_ptr<int32_t>(); c.lengths = n->const_data_ptr<int32_t>();
    out[0] = o ? *o : made(q->sizes(), *q, q->scalar_type());
    auto token = [&](const at::Tensor* t) { return t ? arrow_strides_t{step(*t, 0), 0, step(*t, 1)} : arrow_strides_t{}; };
    const arrow_strides_t qs = token(q), ks = token(k), vs = token(v), os = token(&out[0]);
    const at::Tensor ws = made({(int64_t)reinterpret_cast<decltype(&arrow_attention_decode_workspace_bytes)>(x[1])(&c)}, *q, at::kByte);
    void *qp = data(*q), *kp = k ? data(*k) : nullptr, *vp = v ? data(*v) : nullptr, *kcp = data(*kc), *vcp = data(*vc), *op = data(out[0]);
    void *wp = data(ws), *stream = stream_of(x[2]);
    const size_t bytes = (size_t)ws.numel();
    rc = quietly([&] {
      return reinterpret_cast<decltype(&arrow_attention_decode)>(x[0])(&c, qp, qs, kp, vp, ks, vs, kcp, vcp, op, os, wp, bytes, stream);
    });
    return 1;
  });
}

int any_type(const at::Tensor& t) { return t.scalar_type() == at::kFloat ? ARROW_F32 : half_type(t); }

// Ids, the table (W or dW) and what belongs to the tokens (Y or dY); false for the general way.
bool describe(arrow_embedding_t& e, int64_t rows, double scale, const at::Tensor* table, const at::Tensor* ids, const at::Tensor* tokens) {
  if (!table || !ids || !tokens || any_type(*tokens) < 0 || any_type(*table) < 0) return false;
  if ((ids->scalar_type() != at::kLong && ids->scalar_type() != at::kInt) || !ids->is_contiguous()) return false;
  if (table->dim() != 2 || table->size(0) != rows || table->size(1) < 1 || table->size(1) > (1 << 24) || !rows_whole(*table)) return false;
  if (tokens->dim() != ids->dim() + 1 || tokens->size(-1) != table->size(1) || tokens->sizes().slice(0, ids->dim()) != ids->sizes()) return false;
  const int64_t columns = table->size(1), n = ids->numel();
  if (tokens->dim() == 2 ? !rows_whole(*tokens) : !tokens->is_contiguous()) return false;
  e.dtype = any_type(*tokens); e.grad_dtype = any_type(*table);
  e.id_bytes = ids->scalar_type() == at::kLong ? 8 : 4;
  e.columns = (int32_t)columns; e.rows = rows; e.tokens = n; e.scale = (float)scale;
  e.w_stride = rows > 1 ? table->stride(0) : columns;
  e.y_stride = tokens->dim() == 2 && n > 1 ? tokens->stride(0) : columns;
  return true;
}

at::DimVector with(at::IntArrayRef sizes, int64_t last) {
  at::DimVector r(sizes.begin(), sizes.end());
  r.push_back(last);
  return r;
}

// embedding_forward(function, device, rows, scale, W, ids, Y)
PyObject* embedding_forward(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
  int64_t x[3];
  if (!arguments(n_args, 7) || !integers(args, 3, x)) return nullptr;
  const double scale = PyFloat_AsDouble(args[3]);
  if (PyErr_Occurred()) return nullptr;
  return results(x[1], [&](at::Tensor* out, int& rc) {
    Tensors tensor{x[1]};
    const at::Tensor *W = tensor(args[4]), *ids = tensor(args[5]), *Y = tensor(args[6]);
    if (!tensor.ok || !W || !ids || W->dim() != 2) return 0;
    out[0] = Y ? *Y : made(with(ids->sizes(), W->size(1)), *W, W->scalar_type());
    arrow_embedding_t e{};
    if (out[0].scalar_type() != W->scalar_type() || !describe(e, x[2], scale, W, ids, &out[0])) return 0;
    void *wp = data(*W), *ip = data(*ids), *yp = data(out[0]), *stream = stream_of(x[1]);
    rc = quietly([&] { return reinterpret_cast<decltype(&arrow_embedding_forward)>(x[0])(&e, wp, ip, yp, stream); });
    return 1;
  });
}

// embedding_backward(function, of the workspace's size, device, rows, scale, dY, ids, dW)
PyObject* embedding_backward(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
  int64_t x[4];
  if (!arguments(n_args, 8) || !integers(args, 4, x)) return nullptr;
  const double scale = PyFloat_AsDouble(args[4]);
  if (PyErr_Occurred()) return nullptr;
  return results(x[2], [&](at::Tensor* out, int& rc) {
    Tensors tensor{x[2]};
    const at::Tensor *dY = tensor(args[5]), *ids = tensor(args[6]), *dW = tensor(args[7]);
    if (!tensor.ok || !dY || !ids || dY->dim() < 1) return 0;
    out[0] = dW ? *dW : made({x[3], dY->size(-1)}, *dY, dY->scalar_type());
    arrow_embedding_t e{};
    if ((out[0].scalar_type() != dY->scalar_type() && out[0].scalar_type() != at::kFloat) || !describe(e, x[3], scale, &out[0], ids, dY)) return 0;
    const at::Tensor ws = made({(int64_t)reinterpret_cast<decltype(&arrow_embedding_workspace_bytes)>(x[1])(&e)}, *dY, at::kByte);
    void *gp = data(*dY), *ip = data(*ids), *wp = data(out[0]), *sp = data(ws), *stream = stream_of(x[2]);
    const size_t bytes = (size_t)ws.numel();
    rc = quietly([&] { return reinterpret_cast<decltype(&arrow_embedding_backward)>(x[0])(&e, gp, ip, wp, sp, bytes, stream); });
    return 1;
  });
}

// ---- rotation ----

bool steps_fit(const at::Tensor& t) {
  for (int64_t d = 0; d < t.dim(); ++d)
    if (!small(t.size(d))) return false;
  return true;
}

// q, k, their weights and positions; false for the general way.  values: dim, rotary, interleaved, address of the turns.
bool describe(arrow_rotation_t& a, const int64_t* values, double eps, const at::Tensor* q, const at::Tensor* k, const at::Tensor* wq, const at::Tensor* wk,
              const at::Tensor* positions, int64_t shift) {
  if (!q || !k || !wq != !wk || (q->dim() != 3 && q->dim() != 4) || k->dim() != q->dim() || any_type(*q) < 0 || k->scalar_type() != q->scalar_type()) return false;
  const int64_t n = q->dim();
  if (q->size(-1) != values[0] || k->size(-1) != values[0] || k->sizes().slice(0, n - 2) != q->sizes().slice(0, n - 2) || !rows_whole(*q) || !rows_whole(*k)) return false;
  if (!steps_fit(*q) || !steps_fit(*k)) return false;
  a.dtype = a.weight_dtype = any_type(*q);
  for (auto* t : {wq, wk})
    if (t) {
      if (t->dim() != 1 || t->size(0) != values[0] || !rows_whole(*t) || t->scalar_type() != wq->scalar_type()) return false;
      if (t->scalar_type() != q->scalar_type() && t->scalar_type() != at::kFloat) return false;
      a.weight_dtype = any_type(*t);
    }
  if (positions) {
    if ((positions->scalar_type() != at::kInt && positions->scalar_type() != at::kLong) || positions->sizes() != q->sizes().slice(0, n - 2) || !positions->is_contiguous())
      return false;
    a.positions = positions->const_data_ptr();
    a.position_bytes = positions->scalar_type() == at::kLong ? 8 : 4;
  }
  a.batch = (int32_t)(n == 4 ? q->size(0) : 1);
  a.tokens = (int32_t)q->size(n - 3);
  a.q_heads = (int32_t)q->size(-2); a.kv_heads = (int32_t)k->size(-2);
  a.dim = (int32_t)values[0]; a.rotary = (int32_t)values[1]; a.interleaved = (int32_t)values[2];
  a.eps = (float)eps; a.shift = shift;
  a.turns = a.rotary ? reinterpret_cast<const double*>(values[3]) : nullptr;
  a.q = steps(*q); a.k = steps(*k);
  return true;
}

// rotation_forward(function, device, dim, rotary, interleaved, turns, eps, q, k, q_weight, k_weight, positions, shift, q_out, k_out)
PyObject* rotation_forward(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
  int64_t x[6], shift;
  if (!arguments(n_args, 15) || !integers(args, 6, x)) return nullptr;
  const double eps = PyFloat_AsDouble(args[6]);
  if (PyErr_Occurred()) return nullptr;
  if (!integers(args + 12, 1, &shift)) { PyErr_Clear(); return none(); }
  return results(x[1], [&](at::Tensor* out, int& rc) {
    Tensors tensor{x[1]};
    const at::Tensor *q = tensor(args[7]), *k = tensor(args[8]), *wq = tensor(args[9]), *wk = tensor(args[10]), *positions = tensor(args[11]);
    const at::Tensor *qo = tensor(args[13]), *ko = tensor(args[14]);
    arrow_rotation_t a{};
    if (!tensor.ok || !describe(a, x + 2, eps, q, k, wq, wk, positions, shift) || (qo && !like(*qo, *q)) || (ko && !like(*ko, *k))) return 0;
    out[0] = qo ? *qo : made(q->sizes(), *q, q->scalar_type());
    out[1] = ko ? *ko : made(k->sizes(), *k, q->scalar_type());
    a.q_out = steps(out[0]); a.k_out = steps(out[1]);
    void *qp = data(*q), *kp = data(*k), *wqp = wq ? data(*wq) : nullptr, *wkp = wk ? data(*wk) : nullptr, *op = data(out[0]), *okp = data(out[1]);
    void* stream = stream_of(x[1]);
    rc = quietly([&] { return reinterpret_cast<decltype(&arrow_rotation_forward)>(x[0])(&a, qp, kp, wqp, wkp, op, okp, stream); });
    return 2;
  });
}

// rotation_backward(function, of the workspace's size, device, dim, rotary, interleaved, turns, eps, d_q, d_k, q, k, q_weight, k_weight, positions, shift, dq, dk)
PyObject* rotation_backward(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
  int64_t x[7], shift;
  if (!arguments(n_args, 18) || !integers(args, 7, x)) return nullptr;
  const double eps = PyFloat_AsDouble(args[7]);
  if (PyErr_Occurred()) return nullptr;
  if (!integers(args + 15, 1, &shift)) { PyErr_Clear(); return none(); }
  return results(x[2], [&](at::Tensor* out, int& rc) {
    Tensors tensor{x[2]};
    const at::Tensor *gq = tensor(args[8]), *gk = tensor(args[9]), *q = tensor(args[10]), *k = tensor(args[11]), *wq = tensor(args[12]), *wk = tensor(args[13]);
    const at::Tensor *positions = tensor(args[14]), *dq = tensor(args[16]), *dk = tensor(args[17]);
    arrow_rotation_t a{};
    if (!tensor.ok || !describe(a, x + 3, eps, q, k, wq, wk, positions, shift) || !gq || !gk || !like(*gq, *q) || !like(*gk, *k)) return 0;
    if ((dq && !like(*dq, *q)) || (dk && !like(*dk, *k))) return 0;
    out[0] = dq ? *dq : made(q->sizes(), *q, q->scalar_type());
    out[1] = dk ? *dk : made(k->sizes(), *k, q->scalar_type());
    a.q_out = steps(*gq); a.k_out = steps(*gk); a.dq = steps(out[0]); a.dk = steps(out[1]);
    at::Tensor ws;
    size_t bytes = 0;
    if (wq) {
      out[2] = made(wq->sizes(), *wq, wq->scalar_type());
      out[3] = made(wk->sizes(), *wk, wk->scalar_type());
      bytes = reinterpret_cast<decltype(&arrow_rotation_workspace_bytes)>(x[1])(&a);
      ws = made({(int64_t)bytes}, *q, at::kByte);
    }
    void *gqp = data(*gq), *gkp = data(*gk), *qp = data(*q), *kp = data(*k), *dqp = data(out[0]), *dkp = data(out[1]);
    void *wqp = wq ? data(*wq) : nullptr, *wkp = wk ? data(*wk) : nullptr, *dwqp = wq ? data(out[2]) : nullptr, *dwkp = wq ? data(out[3]) : nullptr;
    void *wp = bytes ? data(ws) : nullptr, *stream = stream_of(x[2]);
    rc = quietly([&] {
      return reinterpret_cast<decltype(&arrow_rotation_backward)>(x[0])(&a, gqp, gkp, qp, kp, wqp, wkp, dqp, dkp, dwqp, dwkp, wp, bytes, stream);
    });
    return wq ? 4 : 2;
  });
}

// ---- pages ----

bool ints(const at::Tensor* t, at::ScalarType type, at::IntArrayRef shape) {
  return t && t->scalar_type() == type && t->sizes() == shape && t->is_contiguous();
}

// pages_step(function, of the workspace's size, device, pages, page, window, sinks, table, held, free, lengths, tokens, offsets, slots)
PyObject* pages_step(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
  int64_t x[7], tokens;
  if (!arguments(n_args, 14) || !integers(args, 7, x)) return nullptr;
  if (!integers(args + 11, 1, &tokens)) { PyErr_Clear(); return none(); }
  return results(x[2], [&](at::Tensor* out, int& rc) {
    Tensors tensor{x[2]};
    const at::Tensor *table = tensor(args[7]), *held = tensor(args[8]), *list = tensor(args[9]), *lengths = tensor(args[10]), *offsets = tensor(args[12]);
    const at::Tensor* slots = tensor(args[13]);
    if (!tensor.ok || !small(tokens) || !table || table->dim() != 2 || !ints(table, at::kInt, table->sizes()) || !steps_fit(*table)) return 0;
    const int64_t batch = table->size(0);
    if (!ints(held, at::kInt, {batch}) || !ints(list, at::kInt, {1 + x[3]}) || !ints(lengths, at::kInt, {batch}) || (offsets && !ints(offsets, at::kInt, {batch + 1})))
      return 0;
    const at::DimVector shape = offsets ? at::DimVector{tokens} : at::DimVector{batch, tokens};
    if (slots && !ints(slots, at::kLong, shape)) return 0;
    out[0] = slots ? *slots : made(shape, *table, at::kLong);
    arrow_pages_t a{};
    a.batch = (int32_t)batch; a.columns = (int32_t)table->size(1); a.page = (int32_t)std::min<int64_t>(x[4], 0x7fffffff); a.pages = x[3];
    a.window = (int32_t)x[5]; a.sinks = (int32_t)x[6];
    if (offsets) { a.offsets = offsets->const_data_ptr<int32_t>(); a.rows = tokens; }
    else a.tokens = (int32_t)tokens;
    const size_t bytes = reinterpret_cast<decltype(&arrow_pages_workspace_bytes)>(x[1])(&a);
    const at::Tensor ws = bytes ? made({(int64_t)bytes}, *table, at::kByte) : at::Tensor();
    auto address = [](const at::Tensor* t) { return static_cast<int32_t*>(data(*t)); };
    int32_t *tp = address(table), *hp = address(held), *fp = address(list), *lp = address(lengths);
    void *sp = data(out[0]), *wp = bytes ? data(ws) : nullptr, *stream = stream_of(x[2]);
    rc = quietly([&] { return reinterpret_cast<decltype(&arrow_pages_step)>(x[0])(&a, lp, hp, tp, fp, static_cast<int64_t*>(sp), wp, bytes, stream); });
    return 1;
  });
}

// ---- the cache in 4 bits ----

bool describe(arrow_packed_t& c, const at::Tensor* pool, int64_t dim, at::ScalarType type) {
  if (!pool || (dim != 32 && dim != 64 && dim != 128) || (type != at::kBFloat16 && type != at::kHalf)) return false;
  const int64_t size = dim + dim / 16;
  if (pool->scalar_type() != at::kByte || pool->dim() != 3 || pool->size(2) % size || !rows_whole(*pool) || !steps_fit(*pool)) return false;
  auto step = [&](int64_t d) { return pool->size(d) > 1 ? pool->stride(d) : 0; };
  c.dtype = type == at::kBFloat16 ? ARROW_BF16 : ARROW_F16;
  c.pages = pool->size(0); c.kv_heads = (int32_t)pool->size(1); c.page = (int32_t)(pool->size(2) / size); c.dim = (int32_t)dim;
  c.page_step = step(0); c.head_step = step(1);
  return true;
}

// Steps of (rows, heads, dim).
arrow_strides_t row_steps(const at::Tensor* t) {
  if (!t) return {};
  const int64_t row = t->size(0) > 1 ? t->stride(0) : 0;
  return {row, row, t->size(1) > 1 ? t->stride(1) : 0};
}

bool is_rows(const at::Tensor* t, at::IntArrayRef shape, at::ScalarType type) {
  return t && t->scalar_type() == type && t->sizes() == shape && (t->stride(-1) == 1 || t->numel() == 0);
}

// packed_append(function, device, k, v, pool, slots): the pool
PyObject* packed_append(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
  int64_t x[2];
  if (!arguments(n_args, 6) || !integers(args, 2, x)) return nullptr;
  return results(x[1], [&](at::Tensor* out, int& rc) {
    Tensors tensor{x[1]};
    const at::Tensor *k = tensor(args[2]), *v = tensor(args[3]), *pool = tensor(args[4]), *slots = tensor(args[5]);
    arrow_packed_t c{};
    if (!tensor.ok || !k || !v || k->dim() != 3 || !describe(c, pool, k->size(2), k->scalar_type())) return 0;
    if (!slots || slots->dim() != 1 || !ints(slots, at::kLong, slots->sizes())) return 0;
    const int64_t shape[] = {slots->size(0), c.kv_heads, c.dim};
    if (!is_rows(k, shape, k->scalar_type()) || !is_rows(v, shape, k->scalar_type())) return 0;
    out[0] = *pool;
    const arrow_strides_t ks = row_steps(k), vs = row_steps(v);
    void *kp = data(*k), *vp = data(*v), *pp = data(*pool), *sp = data(*slots), *stream = stream_of(x[1]);
    rc = quietly([&] { return reinterpret_cast<decltype(&arrow_packed_append)>(x[0])(&c, shape[0], kp, vp, ks, vs, (const int64_t*)sp, pp, stream); });
    return 1;
  });
}

// packed_read(function, device, pool, slots, dim, dtype, k, v)
PyObject* packed_read(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
  int64_t x[2], dim;
  if (!arguments(n_args, 8) || !integers(args, 2, x)) return nullptr;
  if (!integers(args + 4, 1, &dim)) { PyErr_Clear(); return none(); }
  if (!THPDtype_Check(args[5])) return none();
  const at::ScalarType type = reinterpret_cast<THPDtype*>(args[5])->scalar_type;
  return results(x[1], [&](at::Tensor* out, int& rc) {
    Tensors tensor{x[1]};
    const at::Tensor *pool = tensor(args[2]), *slots = tensor(args[3]), *k = tensor(args[6]), *v = tensor(args[7]);
    arrow_packed_t c{};
    if (!tensor.ok || !describe(c, pool, dim, type) || !slots || slots->dim() != 1 || !ints(slots, at::kLong, slots->sizes())) return 0;
    const int64_t shape[] = {slots->size(0), c.kv_heads, c.dim};
    if ((k && !is_rows(k, shape, type)) || (v && !is_rows(v, shape, type))) return 0;
    out[0] = k ? *k : made(shape, *pool, type);
    out[1] = v ? *v : made(shape, *pool, type);
    const arrow_strides_t ks = row_steps(&out[0]), vs = row_steps(&out[1]);
    void *kp = data(out[0]), *vp = data(out[1]), *pp = data(*pool), *sp = data(*slots), *stream = stream_of(x[1]);
    rc = quietly([&] { return reinterpret_cast<decltype(&arrow_packed_read)>(x[0])(&c, shape[0], (const int64_t*)sp, pp, kp, vp, ks, vs, stream); });
    return 2;
  });
}

// packed_decode(function, of the workspace's size, device, window, sinks, scale or -1, q, pool, table, lengths, max_len, k, v, o)
PyObject* packed_decode(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
  int64_t x[5], max_len;
  if (!arguments(n_args, 14) || !integers(args, 5, x)) return nullptr;
  const double scale = PyFloat_AsDouble(args[5]);
  if (PyErr_Occurred()) return nullptr;
  if (!lengths(args + 10, 1, &max_len)) return none();
  return results(x[2], [&](at::Tensor* out, int& rc) {
    Tensors tensor{x[2]};
    const at::Tensor *q = tensor(args[6]), *pool = tensor(args[7]), *table = tensor(args[8]), *n = tensor(args[9]);
    const at::Tensor *k = tensor(args[11]), *v = tensor(args[12]), *o = tensor(args[13]);
    arrow_packed_t c{};
    if (!tensor.ok || !q || !table || !n || !k != !v || q->dim() != 3 || !describe(c, pool, q->size(2), q->scalar_type())) return 0;
    if (table->dim() != 2 || !ints(table, at::kInt, table->sizes()) || !ints(n, at::kInt, {q->size(0)}) || table->size(0) != q->size(0)) return 0;
    const int64_t own[] = {q->size(0), c.kv_heads, c.dim};
    if (!is_rows(q, q->sizes(), q->scalar_type()) || (o && !is_rows(o, q->sizes(), q->scalar_type()))) return 0;
    if ((k && !is_rows(k, own, q->scalar_type())) || (v && !is_rows(v, own, q->scalar_type())) || !steps_fit(*table) || !steps_fit(*q)) return 0;
    c.batch = (int32_t)table->size(0); c.columns = (int32_t)table->size(1);
    c.q_heads = (int32_t)q->size(1);
    c.window = (int32_t)x[3]; c.sinks = (int32_t)x[4];
    c.scale = (float)(scale >= 0 ? scale : 1.0 / std::sqrt((double)c.dim));
    c.max_len = max_len >= 0 ? max_len : (int64_t)c.columns * c.page;
    c.table = table->const_data_ptr<int32_t>(); c.lengths = n->const_data_ptr<int32_t>();
    out[0] = o ? *o : made(q->sizes(), *q, q->scalar_type());
    const arrow_strides_t qs = row_steps(q), ks = row_steps(k), vs = row_steps(v), os = row_steps(&out[0]);
    const size_t bytes = reinterpret_cast<decltype(&arrow_packed_decode_workspace_bytes)>(x[1])(&c);
    const at::Tensor ws = bytes ? made({(int64_t)bytes}, *q, at::kByte) : at::Tensor();
    void *qp = data(*q), *kp = k ? data(*k) : nullptr, *vp = v ? data(*v) : nullptr, *pp = data(*pool), *op = data(out[0]);
    void *wp = bytes ? data(ws) : nullptr, *stream = stream_of(x[2]);
    rc = quietly([&] { return reinterpret_cast<decltype(&arrow_packed_decode)>(x[0])(&c, qp, qs, kp, vp, ks, vs, pp, op, os, wp, bytes, stream); });
    return 1;
  });
}

// ---- log probabilities ----

// Logits (or their gradient) as rows that lie evenly apart; 0: not so.
int64_t row_step(const at::Tensor& t, int64_t rows) {
  const int64_t n = t.size(-1);
  if (!rows_whole(t)) return 0;
  if (rows <= 1) return n;
  if (t.dim() == 2) return t.stride(0);
  return t.is_contiguous() ? n : 0;
}

bool describe(arrow_logprobs_t& a, const at::Tensor* logits, const at::Tensor* targets, double scale) {
  if (!logits || !targets || any_type(*logits) < 0 || logits->dim() < 1 || logits->dim() != targets->dim() + 1) return false;
  if ((targets->scalar_type() != at::kInt && targets->scalar_type() != at::kLong) || !targets->is_contiguous()) return false;
  if (logits->sizes().slice(0, targets->dim()) != targets->sizes() || logits->size(-1) < 1 || logits->size(-1) > (1 << 30)) return false;
  a.dtype = any_type(*logits);
  a.target_bytes = targets->scalar_type() == at::kLong ? 8 : 4;
  a.vocabulary = (int32_t)logits->size(-1);
  a.rows = targets->numel();
  a.stride = row_step(*logits, a.rows);
  a.scale = (float)scale;
  return a.stride != 0;
}

// logprobs_forward(function, of the workspace's size, device, scale, logits, targets, top): logp, entropy, lse, stats and, with top, top_logp, top_ids
PyObject* logprobs_forward(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
  int64_t x[3], top;
  if (!arguments(n_args, 7) || !integers(args, 3, x)) return nullptr;
  const double scale = PyFloat_AsDouble(args[3]);
  if (PyErr_Occurred()) return nullptr;
  if (!integers(args + 6, 1, &top)) { PyErr_Clear(); return none(); }
  return results(x[2], [&](at::Tensor* out, int& rc) {
    Tensors tensor{x[2]};
    const at::Tensor *logits = tensor(args[4]), *targets = tensor(args[5]);
    arrow_logprobs_t a{};
    if (!tensor.ok || !describe(a, logits, targets, scale) || top < 0 || top > 32 || top > a.vocabulary) return 0;
    a.top = (int32_t)top;
    for (int i = 0; i < 3; ++i) out[i] = made(targets->sizes(), *logits, at::kFloat);
    out[3] = made(with(targets->sizes(), 2), *logits, at::kFloat);
    if (top) {
      out[4] = made(with(targets->sizes(), top), *logits, at::kFloat);
      out[5] = made(with(targets->sizes(), top), *logits, at::kLong);
    }
    const size_t bytes = reinterpret_cast<decltype(&arrow_logprobs_workspace_bytes)>(x[1])(&a);
    const at::Tensor ws = bytes ? made({(int64_t)bytes}, *logits, at::kByte) : at::Tensor();
    float* p[5] = {};
    for (int i = 0; i < (top ? 5 : 4); ++i) p[i] = static_cast<float*>(data(out[i]));
    void *xp = data(*logits), *tp = data(*targets), *ip = top ? data(out[5]) : nullptr, *wp = bytes ? data(ws) : nullptr, *stream = stream_of(x[2]);
    rc = quietly([&] {
      return reinterpret_cast<decltype(&arrow_logprobs_forward)>(x[0])(&a, xp, tp, p[0], p[1], p[2], p[3], p[4], static_cast<int64_t*>(ip), wp, bytes, stream);
    });
    return top ? 6 : 4;
  });
}

// logprobs_backward(function, device, scale, d_logp, d_entropy, logits, targets, stats, entropy, d_logits)
PyObject* logprobs_backward(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
  int64_t x[2];
  if (!arguments(n_args, 10) || !integers(args, 2, x)) return nullptr;
  const double scale = PyFloat_AsDouble(args[2]);
  if (PyErr_Occurred()) return nullptr;
  return results(x[1], [&](at::Tensor* out, int& rc) {
    Tensors tensor{x[1]};
    const at::Tensor *d_logp = tensor(args[3]), *d_entropy = tensor(args[4]), *logits = tensor(args[5]), *targets = tensor(args[6]), *stats = tensor(args[7]);
    const at::Tensor *entropy = tensor(args[8]), *to = tensor(args[9]);
    arrow_logprobs_t a{};
    if (!tensor.ok || !describe(a, logits, targets, scale) || (d_entropy && !entropy) || !ints(stats, at::kFloat, with(targets->sizes(), 2))) return 0;
    for (auto* t : {d_logp, d_entropy, entropy})
      if (t && !ints(t, at::kFloat, targets->sizes())) return 0;
    if (to && (to->scalar_type() != logits->scalar_type() || to->sizes() != logits->sizes())) return 0;
    out[0] = to ? *to : made(logits->sizes(), *logits, logits->scalar_type());
    a.d_stride = row_step(out[0], a.rows);
    if (a.d_stride == 0) return 0;
    auto address = [](const at::Tensor* t) { return t ? static_cast<const float*>(t->const_data_ptr()) : nullptr; };
    const float *gp = address(d_logp), *hp = address(d_entropy), *sp = address(stats), *ep = address(entropy);
    void *xp = data(*logits), *tp = data(*targets), *op = data(out[0]), *stream = stream_of(x[1]);
    rc = quietly([&] { return reinterpret_cast<decltype(&arrow_logprobs_backward)>(x[0])(&a, gp, hp, xp, tp, sp, ep, op, stream); });
    return 1;
  });
}

template <PyObject* (*F)(PyObject*, PyObject* const*, Py_ssize_t)>
PyMethodDef method(const char* name) {
  return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(F)), METH_FASTCALL, nullptr};
}

PyMethodDef methods[] = {method<spmm>("spmm"), method<sddmm>("sddmm"), method<mttkrp>("mttkrp"),
                         method<attention_forward>("attention_forward"), method<attention_backward>("attention_backward"),
                         method<attention_decode>("attention_decode"), method<embedding_forward>("embedding_forward"),
                         method<embedding_backward>("embedding_backward"),
                         method<rotation_forward>("rotation_forward"), method<rotation_backward>("rotation_backward"),
                         method<pages_step>("pages_step"), method<packed_append>("packed_append"), method<packed_read>("packed_read"),
                         method<packed_decode>("packed_decode"), method<logprobs_forward>("logprobs_forward"),
                         method<logprobs_backward>("logprobs_backward"), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "tensor_call", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit_tensor_call() { return PyModule_Create(&module); }
