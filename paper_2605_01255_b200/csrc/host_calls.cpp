// Argument checks and marshalling of the row operators, the vocabulary cross entropy, attention, the embedding table and gradient
// clipping for Python: torch tensors in, one C
// call of libacx out.  The small calls (decoding, short batches) are bound by the host: checked in Python and called through
// ctypes the norm join of 16 x 896 with seven tensors took 8.2 us (0.41 us per tensor checked, 1.4 us to convert the
// arguments), through this file 3.3 us, launch included; the gated activation of 8 x 4864 5.7 and 2.6 us.  The library
// itself stays free of Python and torch: its entry points are handed in by address.
#include <Python.h>
#include <ATen/core/Tensor.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <array>
#include <cstring>
#include <exception>

#include "../../include/acx.h"

namespace {

struct PythonError {};   // the Python exception is set

struct Entries {
  decltype(&acx_q8_store) q8_store;
  decltype(&acx_q8_load) q8_load;
  decltype(&acx_swiglu_fwd) swiglu_fwd;
  decltype(&acx_swiglu_bwd) swiglu_bwd;
  decltype(&acx_norm_join_fwd) norm_join_fwd;
  decltype(&acx_norm_join_bwd) norm_join_bwd;
  decltype(&acx_linear_ce_fwd) linear_ce_fwd;
  decltype(&acx_linear_ce_bwd_loss) linear_ce_bwd;
  decltype(&acx_attn_plan) attn_plan;
  decltype(&acx_attn_fwd) attn_fwd;
  decltype(&acx_attn_bwd) attn_bwd;
  decltype(&acx_embed_fwd) embed_fwd;
  decltype(&acx_embed_bwd) embed_bwd;
  decltype(&acx_grad_clip) grad_clip;
} entries;
constexpr int kEntries = sizeof(Entries) / sizeof(void*);

const at::Tensor* tensor(PyObject* o, const char* name) {
  if (o == Py_None) return nullptr;
  if (!THPVariable_Check(o)) {
    PyErr_Format(PyExc_ValueError, "%s must be a CUDA tensor (got %s)", name, Py_TYPE(o)->tp_name);
    throw PythonError();
  }
  return &THPVariable_Unpack(o);
}

[[noreturn]] void refuse(PyObject* o, const char* name, const char* what, at::IntArrayRef shape, at::ScalarType type) {
  PyObject* const want = PyTuple_New(Py_ssize_t(shape.size()));
  for (size_t i = 0; want && i < shape.size(); ++i) PyTuple_SET_ITEM(want, Py_ssize_t(i), PyLong_FromLongLong(shape[i]));
  PyObject* const got[3] = {PyObject_GetAttrString(o, "shape"), PyObject_GetAttrString(o, "dtype"), PyObject_GetAttrString(o, "device")};
  if (want && got[0] && got[1] && got[2])
    PyErr_Format(PyExc_ValueError, "%s must be a %s of shape %R and dtype %s (got %S %S on %S)", name, what, want, c10::toString(type), got[0],
                 got[1], got[2]);
  Py_XDECREF(want);
  for (PyObject* g : got) Py_XDECREF(g);
  throw PythonError();
}

bool fits(const at::Tensor& t, at::IntArrayRef shape, at::ScalarType type) {
  return t.is_cuda() && t.layout() == at::kStrided && t.scalar_type() == type && t.sizes() == shape;
}

struct Matrix {
  void* p;
  int64_t ld;
};
struct Workspace {
  void* p;
  size_t bytes;
};

// What the arguments of one call have in common: the device of its tensors, which has to be the current one (the library
// launches there) and the stream's.
class Call {
 public:
  template <typename P = void>
  P* dense(PyObject* o, const char* name, at::IntArrayRef shape, at::ScalarType type) {
    const at::Tensor* t = tensor(o, name);
    if (!t) return nullptr;
    if (!fits(*t, shape, type) || !t->is_contiguous()) refuse(o, name, "contiguous CUDA tensor", shape, type);
    same_device(*t, name);
    return static_cast<P*>(t->data_ptr());
  }

  // A matrix whose rows are dense: a column slice of a wider one is fine.
  Matrix strided(PyObject* o, const char* name, at::IntArrayRef shape, at::ScalarType type) {
    const at::Tensor* t = tensor(o, name);
    if (!t) {
      PyErr_Format(PyExc_ValueError, "%s must be a CUDA matrix (got None)", name);
      throw PythonError();
    }
    if (!fits(*t, shape, type) || t->stride(1) != 1) refuse(o, name, "CUDA matrix with unit column stride", shape, type);
    same_device(*t, name);
    return Matrix{t->data_ptr(), shape[0] > 1 ? t->stride(0) : shape[1]};
  }

  // [tokens][heads][columns] whose heads lie one behind the other: a column slice of a wider matrix of tokens is fine.
  Matrix heads(PyObject* o, const char* name, at::IntArrayRef shape, at::ScalarType type) {
    const at::Tensor* t = tensor(o, name);
    if (!t) {
      PyErr_Format(PyExc_ValueError, "%s must be a CUDA tensor (got None)", name);
      throw PythonError();
    }
    if (!fits(*t, shape, type) || t->stride(2) != 1 || (shape[1] > 1 && t->stride(1) != shape[2]))
      refuse(o, name, "CUDA tensor with dense heads", shape, type);
    same_device(*t, name);
    return Matrix{t->data_ptr(), shape[0] > 1 ? t->stride(0) : shape[1] * shape[2]};
  }

  Workspace workspace(PyObject* o, const char* name = "workspace") {
    const at::Tensor* t = tensor(o, name);
    if (!t) return Workspace{nullptr, 0};
    if (!t->is_cuda() || !t->is_contiguous()) {
      PyErr_Format(PyExc_ValueError, "%s must be a contiguous CUDA tensor", name);
      throw PythonError();
    }
    same_device(*t, name);
    return Workspace{t->data_ptr(), t->nbytes()};
  }

  // None: torch's current stream of the current device.  Taken last, when the tensors' device is known.
  void* stream(PyObject* o) const {
    if (o == Py_None) {
      const c10::cuda::CUDAStream s = c10::cuda::getCurrentCUDAStream();
      current_is(s.device_index());
      return s.stream();
    }
    PyObject* h = PyObject_GetAttrString(o, "cuda_stream");
    if (!h) throw PythonError();
    void* p = PyLong_AsVoidPtr(h);
    Py_DECREF(h);
    if (!p && PyErr_Occurred()) throw PythonError();
    if (PyObject* d = PyObject_GetAttrString(o, "device_index")) {
      const long index = PyLong_AsLong(d);
      Py_DECREF(d);
      if (index == -1 && PyErr_Occurred()) throw PythonError();
      if (device_ >= 0 && index != device_) {
        PyErr_Format(PyExc_ValueError, "the stream is on cuda:%ld, the tensors on cuda:%d", index, device_);
        throw PythonError();
      }
    } else {
      PyErr_Clear();   // a handle without a device
    }
    current_is(c10::cuda::current_device());
    return p;
  }

 private:
  int device_ = -1;

  void same_device(const at::Tensor& t, const char* name) {
    const int index = t.device().index();
    if (device_ < 0) device_ = index;
    if (index == device_) return;
    PyErr_Format(PyExc_ValueError, "%s is on cuda:%d, the tensors before it on cuda:%d", name, index, device_);
    throw PythonError();
  }
  void current_is(int device) const {
    if (device_ < 0 || device == device_) return;
    PyErr_Format(PyExc_ValueError, "the tensors are on cuda:%d, the current device is cuda:%d", device_, device);
    throw PythonError();
  }
};

float number(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw PythonError();
  return float(v);
}

// A copy of a descriptor: a ctypes structure of the same layout.
template <typename D>
D descriptor(PyObject* o) {
  Py_buffer b;
  if (PyObject_GetBuffer(o, &b, PyBUF_SIMPLE) != 0) throw PythonError();
  const bool same = b.len == Py_ssize_t(sizeof(D));
  D d{};
  if (same) memcpy(&d, b.buf, sizeof d);
  PyBuffer_Release(&b);
  if (!same) {
    PyErr_SetString(PyExc_TypeError, "descriptor of another operator");
    throw PythonError();
  }
  return d;
}

at::ScalarType io_type(const acx_rows_desc& d) { return d.io_dtype == ACX_BF16 ? at::kBFloat16 : at::kFloat; }

struct RowArgs : Call {
  acx_rows_desc d;
  at::ScalarType io;
  std::array<int64_t, 2> shape, groups;
  std::array<int64_t, 1> row, vec;
  explicit RowArgs(PyObject* o) : d(descriptor<acx_rows_desc>(o)), io(io_type(d)) {
    shape = {d.rows, d.cols};
    groups = {d.rows, (d.cols + ACX_Q8_GROUP - 1) / ACX_Q8_GROUP};
    row = {d.rows};
    vec = {d.cols};
  }
  int8_t* codes(PyObject* o, const char* name) { return dense<int8_t>(o, name, shape, at::kChar); }
  float* scales(PyObject* o, const char* name) { return dense<float>(o, name, groups, at::kFloat); }
  void* matrix(PyObject* o, const char* name) { return dense(o, name, shape, io); }
  void* vector(PyObject* o, const char* name) { return dense(o, name, vec, io); }
  float* row_f32(PyObject* o, const char* name) { return dense<float>(o, name, row, at::kFloat); }
  float* vec_f32(PyObject* o, const char* name) { return dense<float>(o, name, vec, at::kFloat); }
  Matrix rows_of(PyObject* o, const char* name) { return strided(o, name, shape, io); }
};

struct CeArgs : Call {
  acx_ce_desc d;
  std::array<int64_t, 2> x, w;
  std::array<int64_t, 1> row;
  explicit CeArgs(PyObject* o) : d(descriptor<acx_ce_desc>(o)) {
    x = {d.tokens, d.d};
    w = {d.vocab, d.d};
    row = {d.tokens};
  }
  float* row_f32(PyObject* o, const char* name) { return dense<float>(o, name, row, at::kFloat); }
};

struct AttnArgs : Call {
  acx_attn_desc d;
  std::array<int64_t, 3> q, kv;
  std::array<int64_t, 2> row;
  std::array<int64_t, 1> per_head;
  explicit AttnArgs(PyObject* o) : d(descriptor<acx_attn_desc>(o)) {
    q = {d.tokens, d.heads, d.head_dim};
    kv = {d.tokens, d.kv_heads, d.head_dim};
    row = {d.heads, d.tokens};
    per_head = {d.heads};
  }
  Matrix queries(PyObject* o, const char* name) { return heads(o, name, q, at::kBFloat16); }
  Matrix keys(PyObject* o, const char* name) { return heads(o, name, kv, at::kBFloat16); }
};

struct EmbedArgs : Call {
  acx_embed_desc d;
  std::array<int64_t, 2> rows, table;
  std::array<int64_t, 1> row;
  explicit EmbedArgs(PyObject* o) : d(descriptor<acx_embed_desc>(o)) {
    rows = {d.tokens, d.d};
    table = {d.vocab, d.d};
    row = {d.tokens};
  }
  static at::ScalarType type(int32_t t) { return t == ACX_BF16 ? at::kBFloat16 : at::kFloat; }
  const int64_t* ids(PyObject* o) { return dense<int64_t>(o, "ids", row, at::kLong); }
};

template <typename F>
acx_status without_gil(F&& f) {
  PyThreadState* const s = PyEval_SaveThread();
  const acx_status r = f();
  PyEval_RestoreThread(s);
  return r;
}

acx_status q8_store(PyObject* const* a) {
  RowArgs r(a[0]);
  const Matrix X = r.rows_of(a[1], "X");
  int8_t* const q = r.codes(a[2], "codes of X");
  float* const s = r.scales(a[3], "scales of X");
  void* const st = r.stream(a[4]);
  return without_gil([&] { return entries.q8_store(&r.d, X.p, X.ld, q, s, st); });
}

acx_status q8_load(PyObject* const* a) {
  RowArgs r(a[0]);
  const int8_t* const q = r.codes(a[1], "codes of X");
  const float* const s = r.scales(a[2], "scales of X");
  const Matrix X = r.rows_of(a[3], "X");
  void* const st = r.stream(a[4]);
  return without_gil([&] { return entries.q8_load(&r.d, q, s, X.p, X.ld, st); });
}

acx_status swiglu_fwd(PyObject* const* a) {
  RowArgs r(a[0]);
  const Matrix G = r.rows_of(a[1], "G"), U = r.rows_of(a[2], "U");
  void* const H = r.matrix(a[3], "H");
  int8_t* const Gq = r.codes(a[4], "Gq");
  float* const Gs = r.scales(a[5], "Gs");
  int8_t* const Uq = r.codes(a[6], "Uq");
  float* const Us = r.scales(a[7], "Us");
  void* const st = r.stream(a[8]);
  return without_gil([&] { return entries.swiglu_fwd(&r.d, G.p, G.ld, U.p, U.ld, H, Gq, Gs, Uq, Us, st); });
}

acx_status swiglu_bwd(PyObject* const* a) {
  RowArgs r(a[0]);
  const void* const dH = r.matrix(a[1], "dH");
  const int8_t* const Gq = r.codes(a[2], "Gq");
  const float* const Gs = r.scales(a[3], "Gs");
  const int8_t* const Uq = r.codes(a[4], "Uq");
  const float* const Us = r.scales(a[5], "Us");
  const Matrix dG = r.rows_of(a[6], "dG"), dU = r.rows_of(a[7], "dU");
  void* const st = r.stream(a[8]);
  return without_gil([&] { return entries.swiglu_bwd(&r.d, dH, Gq, Gs, Uq, Us, dG.p, dG.ld, dU.p, dU.ld, st); });
}

acx_status norm_join_fwd(PyObject* const* a) {
  RowArgs r(a[0]);
  const void *const h = r.matrix(a[1], "h"), *const b = r.matrix(a[2], "b");
  const void *const w_post = r.vector(a[3], "w_post"), *const gate = r.vector(a[4], "gate"), *const w_pre = r.vector(a[5], "w_pre");
  void *const h_out = r.matrix(a[6], "h_out"), *const y = r.matrix(a[7], "y");
  int8_t* const Hq = r.codes(a[8], "Hq");
  float* const Hs = r.scales(a[9], "Hs");
  int8_t* const Bq = r.codes(a[10], "Bq");
  float* const Bs = r.scales(a[11], "Bs");
  float *const rstd_post = r.row_f32(a[12], "rstd_post"), *const rstd_pre = r.row_f32(a[13], "rstd_pre");
  const float eps = number(a[14]), alpha = number(a[15]);
  void* const st = r.stream(a[16]);
  return without_gil([&] {
    return entries.norm_join_fwd(&r.d, h, b, w_post, gate, w_pre, h_out, y, Hq, Hs, Bq, Bs, rstd_post, rstd_pre, eps, alpha, st);
  });
}

acx_status norm_join_bwd(PyObject* const* a) {
  RowArgs r(a[0]);
  const void *const dy = r.matrix(a[1], "dy"), *const dh_next = r.matrix(a[2], "dh_next");
  const void *const w_post = r.vector(a[3], "w_post"), *const gate = r.vector(a[4], "gate"), *const w_pre = r.vector(a[5], "w_pre");
  const int8_t* const Hq = r.codes(a[6], "Hq");
  const float* const Hs = r.scales(a[7], "Hs");
  const int8_t* const Bq = r.codes(a[8], "Bq");
  const float* const Bs = r.scales(a[9], "Bs");
  const float *const rstd_post = r.row_f32(a[10], "rstd_post"), *const rstd_pre = r.row_f32(a[11], "rstd_pre");
  void *const dh = r.matrix(a[12], "dh"), *const db = r.matrix(a[13], "db");
  float *const dw_post = r.vec_f32(a[14], "dw_post"), *const dgate = r.vec_f32(a[15], "dgate"), *const dw_pre = r.vec_f32(a[16], "dw_pre");
  const float alpha = number(a[17]);
  const Workspace ws = r.workspace(a[18]);
  void* const st = r.stream(a[19]);
  return without_gil([&] {
    return entries.norm_join_bwd(&r.d, dy, dh_next, w_post, gate, w_pre, Hq, Hs, Bq, Bs, rstd_post, rstd_pre, dh, db, dw_post, dgate, dw_pre,
                                 alpha, ws.p, ws.bytes, st);
  });
}

acx_status linear_ce_fwd(PyObject* const* a) {
  CeArgs c(a[0]);
  const std::array<int64_t, 1> two{2};
  const void *const X = c.dense(a[1], "X", c.x, at::kBFloat16), *const W = c.dense(a[2], "W", c.w, at::kBFloat16);
  const int64_t* const targets = c.dense<int64_t>(a[3], "targets", c.row, at::kLong);
  const float* const weight = c.row_f32(a[4], "weight");
  float *const loss = c.row_f32(a[5], "loss"), *const lse = c.row_f32(a[6], "lse");
  float* const total = c.dense<float>(a[7], "total", two, at::kFloat);
  const Workspace ws = c.workspace(a[8]);
  void* const st = c.stream(a[9]);
  return without_gil([&] { return entries.linear_ce_fwd(&c.d, X, W, targets, weight, loss, lse, total, ws.p, ws.bytes, st); });
}

acx_status linear_ce_bwd(PyObject* const* a) {
  CeArgs c(a[0]);
  const std::array<int64_t, 1> one{1};
  const void *const X = c.dense(a[1], "X", c.x, at::kBFloat16), *const W = c.dense(a[2], "W", c.w, at::kBFloat16);
  const int64_t* const targets = c.dense<int64_t>(a[3], "targets", c.row, at::kLong);
  const float* const weight = c.row_f32(a[4], "weight");
  const float* const lse = c.row_f32(a[5], "lse");
  const float* const loss = c.row_f32(a[6], "loss");
  const float* const denom = c.dense<float>(a[7], "denom", one, at::kFloat);
  const float scale = number(a[8]);
  void *const dX = c.dense(a[9], "dX", c.x, at::kBFloat16), *const dW = c.dense(a[10], "dW", c.w, at::kBFloat16);
  const Workspace ws = c.workspace(a[11]);
  void* const st = c.stream(a[12]);
  return without_gil([&] { return entries.linear_ce_bwd(&c.d, X, W, targets, weight, lse, loss, denom, scale, dX, dW, ws.p, ws.bytes, st); });
}

acx_status attn_plan(PyObject* const* a) {
  AttnArgs c(a[0]);
  const std::array<int64_t, 1> ends{c.d.docs + 1}, docs{c.d.docs};
  const int32_t* const offsets = c.dense<int32_t>(a[1], "offsets", ends, at::kInt);
  const int32_t* const prefix = c.dense<int32_t>(a[2], "prefix", docs, at::kInt);
  const Workspace plan = c.workspace(a[3], "plan");
  void* const st = c.stream(a[4]);
  return without_gil([&] { return entries.attn_plan(&c.d, offsets, prefix, plan.p, plan.bytes, st); });
}

acx_status attn_fwd(PyObject* const* a) {
  AttnArgs c(a[0]);
  const Matrix Q = c.queries(a[1], "Q"), K = c.keys(a[2], "K"), V = c.keys(a[3], "V");
  const float* const slopes = c.dense<float>(a[4], "slopes", c.per_head, at::kFloat);
  const Workspace plan = c.workspace(a[5], "plan");
  const Matrix O = c.queries(a[6], "O");
  float* const lse = c.dense<float>(a[7], "lse", c.row, at::kFloat);
  void* const st = c.stream(a[8]);
  return without_gil([&] { return entries.attn_fwd(&c.d, Q.p, Q.ld, K.p, K.ld, V.p, V.ld, slopes, plan.p, plan.bytes, O.p, O.ld, lse, st); });
}

acx_status attn_bwd(PyObject* const* a) {
  AttnArgs c(a[0]);
  const Matrix Q = c.queries(a[1], "Q"), K = c.keys(a[2], "K"), V = c.keys(a[3], "V");
  const float* const slopes = c.dense<float>(a[4], "slopes", c.per_head, at::kFloat);
  const Workspace plan = c.workspace(a[5], "plan");
  const Matrix O = c.queries(a[6], "O"), dO = c.queries(a[7], "dO");
  const float* const lse = c.dense<float>(a[8], "lse", c.row, at::kFloat);
  const Matrix dQ = c.queries(a[9], "dQ"), dK = c.keys(a[10], "dK"), dV = c.keys(a[11], "dV");
  const Workspace ws = c.workspace(a[12]);
  void* const st = c.stream(a[13]);
  return without_gil([&] {
    return entries.attn_bwd(&c.d, Q.p, Q.ld, K.p, K.ld, V.p, V.ld, slopes, plan.p, plan.bytes, O.p, O.ld, dO.p, dO.ld, lse, dQ.p, dQ.ld, dK.p,
                            dK.ld, dV.p, dV.ld, ws.p, ws.bytes, st);
  });
}

acx_status embed_fwd(PyObject* const* a) {
  EmbedArgs c(a[0]);
  const int64_t* const ids = c.ids(a[1]);
  const void* const E = c.dense(a[2], "E", c.table, c.type(c.d.io_dtype));
  void* const Y = c.dense(a[3], "Y", c.rows, c.type(c.d.io_dtype));
  void* const st = c.stream(a[4]);
  return without_gil([&] { return entries.embed_fwd(&c.d, ids, E, Y, st); });
}

acx_status embed_bwd(PyObject* const* a) {
  EmbedArgs c(a[0]);
  const int64_t* const ids = c.ids(a[1]);
  const void* const dY = c.dense(a[2], "dY", c.rows, c.type(c.d.io_dtype));
  void* const dE = c.dense(a[3], "dE", c.table, c.type(c.d.grad_dtype));
  const float beta = number(a[4]);
  const Workspace ws = c.workspace(a[5]);
  void* const st = c.stream(a[6]);
  return without_gil([&] { return entries.embed_bwd(&c.d, ids, dY, dE, beta, ws.p, ws.bytes, st); });
}

acx_status grad_clip(PyObject* const* a) {
  Call c;
  const acx_grad_desc d = descriptor<acx_grad_desc>(a[0]);
  const std::array<int64_t, 1> two{2};
  const Workspace plan = c.workspace(a[1], "plan");
  const float max_norm = number(a[2]);
  float* const total = c.dense<float>(a[3], "total", two, at::kFloat);
  const Workspace ws = c.workspace(a[4]);
  void* const st = c.stream(a[5]);
  return without_gil([&] { return entries.grad_clip(&d, plan.p, plan.bytes, max_norm, total, ws.p, ws.bytes, st); });
}

// Python entry of an operator of COUNT arguments: its acx_status as an int.
template <acx_status (*OP)(PyObject* const*), int COUNT>
PyObject* entry(PyObject*, PyObject* const* args, Py_ssize_t count) {
  try {
    if (count != COUNT) {
      PyErr_Format(PyExc_TypeError, "%d arguments expected, %zd given", COUNT, count);
      return nullptr;
    }
    if (!entries.q8_store) {
      PyErr_SetString(PyExc_RuntimeError, "bind() has not been called");
      return nullptr;
    }
    return PyLong_FromLong(OP(args));
  } catch (const PythonError&) {
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  }
  return nullptr;
}

// bind(addresses): the library's entry points, in the order of Entries.
PyObject* bind(PyObject*, PyObject* addresses) {
  if (!PyTuple_Check(addresses) || PyTuple_GET_SIZE(addresses) != kEntries) {
    PyErr_Format(PyExc_TypeError, "a tuple of %d addresses expected", kEntries);
    return nullptr;
  }
  void* p[kEntries];
  for (int i = 0; i < kEntries; ++i) {
    p[i] = PyLong_AsVoidPtr(PyTuple_GET_ITEM(addresses, i));
    if (!p[i]) {
      if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "null address");
      return nullptr;
    }
  }
  memcpy(&entries, p, sizeof entries);
  Py_RETURN_NONE;
}

#define ACX_ENTRY(name, count) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&entry<name, count>)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {
    {"bind", bind, METH_O, nullptr},
    ACX_ENTRY(q8_store, 5),       ACX_ENTRY(q8_load, 5),        ACX_ENTRY(swiglu_fwd, 9),     ACX_ENTRY(swiglu_bwd, 9),
    ACX_ENTRY(norm_join_fwd, 17), ACX_ENTRY(norm_join_bwd, 20), ACX_ENTRY(linear_ce_fwd, 10), ACX_ENTRY(linear_ce_bwd, 13),
    ACX_ENTRY(attn_plan, 5),      ACX_ENTRY(attn_fwd, 9),       ACX_ENTRY(attn_bwd, 14),      ACX_ENTRY(embed_fwd, 5),
    ACX_ENTRY(embed_bwd, 7),      ACX_ENTRY(grad_clip, 6),
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module_def = {PyModuleDef_HEAD_INIT, "_acx_host", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__acx_host(void) { return PyModule_Create(&module_def); }
