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
#include <ATen/ops/empty.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "arrow_attention.h"
#include "arrow_embedding.h"

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
at::Tensor made(at::IntArrayRef sizes, const at::Tensor& on, at::ScalarType type) { return at::empty(sizes, on.options().dtype(type)); }
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
  at::Tensor out[3];
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

template <PyObject* (*F)(PyObject*, PyObject* const*, Py_ssize_t)>
PyMethodDef method(const char* name) {
  return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(F)), METH_FASTCALL, nullptr};
}

PyMethodDef methods[] = {method<spmm>("spmm"), method<sddmm>("sddmm"), method<mttkrp>("mttkrp"),
                         method<attention_forward>("attention_forward"), method<attention_backward>("attention_backward"),
                         method<attention_decode>("attention_decode"), method<embedding_forward>("embedding_forward"),
                         method<embedding_backward>("embedding_backward"), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "tensor_call", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit_tensor_call() { return PyModule_Create(&module); }
