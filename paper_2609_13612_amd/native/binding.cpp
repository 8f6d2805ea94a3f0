// Native half of the Python binding (api.py): argument checks, output and
// scratch allocation, and the call into the library, for the ordinary form of
// every entry point.
//
// A call's host work is what bounds the smallest calls: marshalled in Python
// through ctypes, a B1 H2 S128 D64 forward kept the host busy for 17.7 us and a
// backward for 27.2; here 5.4 and 9.2 (one library call is 4 of them), and a
// differentiable forward and backward went from 196 to 99, of which 52 are
// torch's own for an empty function.
//
// Each function takes positional arguments and returns
//   * the call's outputs,
//   * the library's return code, when that is not 0, or
//   * None for anything but plain arguments: a tensor of another type, shape,
//     device or layout than the call needs, a tensor subclass, a transform's
//     or a mode's wrapper, a table not built yet, a value that does not
//     convert.  The caller then marshals the call itself, which raises what
//     there is to raise.
// Nothing is kept between calls.
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <ATen/ops/empty_like.h>
#include <c10/core/DeviceGuard.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/custom_function.h>
#include <torch/csrc/autograd/functions/basic_ops.h>
#include <torch/csrc/autograd/functions/utils.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>

#include "attnfuse.h"
#include "attnfuse_llm.h"
#include "binding.h"

namespace {

using at::Tensor;

struct NotPlain {};   // thrown inside, never past an entry function

// ---------------------------------------------------------------- arguments
struct Args {
  PyObject* const* v;
  Py_ssize_t n, i = 0;
  PyObject* next() {
    if (i >= n) throw NotPlain{};
    return v[i++];
  }
  // A tensor whose memory is its own: exactly torch.Tensor (or Parameter),
  // strided, not wrapped by a transform or a mode.  None: an empty optional.
  const Tensor* tensor() {
    PyObject* o = next();
    if (o == Py_None) return nullptr;
    if (!THPVariable_CheckExact(o)) throw NotPlain{};
    const Tensor& t = THPVariable_Unpack(o);
    if (!t.defined() || t.layout() != at::kStrided || !t.has_storage()) throw NotPlain{};
    constexpr c10::DispatchKeySet wrapped({c10::DispatchKey::FuncTorchBatched, c10::DispatchKey::FuncTorchGradWrapper,
                                           c10::DispatchKey::Functionalize, c10::DispatchKey::Python,
                                           c10::DispatchKey::Conjugate, c10::DispatchKey::Negative,
                                           c10::DispatchKey::ZeroTensor});
    if (t.key_set().has_any(wrapped)) throw NotPlain{};
    return &t;
  }
  const Tensor& need() {
    const Tensor* t = tensor();
    if (!t) throw NotPlain{};
    return *t;
  }
  double number() {
    PyObject* o = next();
    if (!PyFloat_CheckExact(o) && !PyLong_CheckExact(o)) throw NotPlain{};
    const double x = PyFloat_AsDouble(o);
    if (x == -1.0 && PyErr_Occurred()) {
      PyErr_Clear();
      throw NotPlain{};
    }
    return x;
  }
  long long whole() {
    PyObject* o = next();
    if (o == Py_None) return 0;
    if (!PyLong_CheckExact(o)) throw NotPlain{};
    const long long x = PyLong_AsLongLong(o);
    if (x == -1 && PyErr_Occurred()) {
      PyErr_Clear();
      throw NotPlain{};
    }
    return x;
  }
  long long positive() {   // 0 for None
    if (i < n && v[i] == Py_None) return whole();
    const long long x = whole();
    if (x < 1) throw NotPlain{};
    return x;
  }
  int index() {   // an enum's value, or -1 for an unknown name
    const long long x = whole();
    if (x < 0 || x > 2) throw NotPlain{};
    return (int)x;
  }
  int size() {
    const long long x = whole();
    if (x < INT_MIN || x > INT_MAX) throw NotPlain{};
    return (int)x;
  }
  template <class T>
  const T* pointer() {
    return reinterpret_cast<const T*>(static_cast<uintptr_t>(whole()));
  }
  float scale(int64_t D) {
    if (i < n && v[i] == Py_None) {
      ++i;
      return (float)(1.0 / std::sqrt((double)D));
    }
    return (float)number();
  }
};

void same(const Tensor& t, at::IntArrayRef shape, at::ScalarType type, c10::Device dev) {
  if (t.device() != dev || t.scalar_type() != type || t.sizes() != shape || !t.is_contiguous()) throw NotPlain{};
}

Tensor out_or(const Tensor* given, at::IntArrayRef shape, at::ScalarType type, c10::Device dev) {
  if (given) {
    same(*given, shape, type, dev);
    return *given;
  }
  return at::empty(shape, at::TensorOptions().dtype(type).device(dev));
}

int dtype_of(const Tensor& q) {
  if (!q.is_cuda()) throw NotPlain{};
  if (q.scalar_type() == at::kBFloat16) return AF_DTYPE_BF16;
  if (q.scalar_type() == at::kFloat) return AF_DTYPE_FP32;
  throw NotPlain{};
}

// ---------------------------------------------------------------- RoPE table
// The call's cos/sin table: the caller's, or one of the binding's (api._TABLES:
// a dict of (device index, D, theta) -> list of tables; own: of (device index, D, theta,
// sections, section_order), where every axis has its own frequencies).
struct Table {
  const float* ptr = nullptr;
  int rows = 0;
  Tensor own;   // the tensor itself: a differentiable call keeps it for its backward
};

struct OwnKey {
  PyObject *sections, *order;
};

Table table_of(Args& a, int rope, double theta, int64_t D, int64_t S, c10::Device dev, const OwnKey* own = nullptr) {
  const Tensor* given = a.tensor();
  PyObject* tables = a.next();
  Table r;
  if (rope == AF_ROPE_NONE) return r;
  auto take = [&](const Tensor& t) {
    r.ptr = static_cast<const float*>(t.const_data_ptr());
    r.rows = (int)t.size(0);
    r.own = t;
  };
  if (given) {
    if (given->dim() != 3 || given->size(0) < S || given->size(0) > INT_MAX) throw NotPlain{};
    same(*given, {given->size(0), D / 2, 2}, at::kFloat, dev);
    take(*given);
    return r;
  }
  if (!PyDict_CheckExact(tables)) throw NotPlain{};
  PyObject* key = own ? Py_BuildValue("(iidOO)", (int)dev.index(), (int)D, (double)(float)theta, own->sections, own->order)
                      : Py_BuildValue("(iid)", (int)dev.index(), (int)D, (double)(float)theta);
  if (!key) {
    PyErr_Clear();
    throw NotPlain{};
  }
  PyObject* list = PyDict_GetItemWithError(tables, key);   // borrowed
  Py_DECREF(key);
  if (!list || !PyList_CheckExact(list)) {
    PyErr_Clear();
    throw NotPlain{};
  }
  for (Py_ssize_t i = 0; i < PyList_GET_SIZE(list); ++i) {
    PyObject* o = PyList_GET_ITEM(list, i);
    if (!THPVariable_CheckExact(o)) throw NotPlain{};
    const Tensor& t = THPVariable_Unpack(o);
    if (t.size(0) >= S) {
      take(t);
      return r;
    }
  }
  throw NotPlain{};
}

// ---------------------------------------------------------------- calls
struct NoGil {   // (a backward runs in a thread of the engine, which does not hold the lock)
  PyThreadState* s = PyGILState_Check() ? PyEval_SaveThread() : nullptr;
  ~NoGil() {
    if (s) PyEval_RestoreThread(s);
  }
};

// f(stream) on dev's current stream, without the interpreter's lock.
template <class F>
int enqueue(c10::Device dev, F f) {
  const c10::DeviceGuard guard(dev);
  void* st = c10::hip::getCurrentHIPStream(dev.index()).stream();
  NoGil unlocked;
  return f(st);
}

const float* slopes_of(const Tensor* s, int64_t H, c10::Device dev) {
  if (!s) return nullptr;
  same(*s, {H}, at::kFloat, dev);
  return static_cast<const float*>(s->const_data_ptr());
}

const void* in(const Tensor& t) { return t.const_data_ptr(); }
void* out(const Tensor& t) { return t.mutable_data_ptr(); }

PyObject* tuple_of(std::initializer_list<const Tensor*> ts) {
  PyObject* r = PyTuple_New((Py_ssize_t)ts.size());
  if (!r) return nullptr;
  Py_ssize_t i = 0;
  for (const Tensor* t : ts) {
    PyObject* o = t && t->defined() ? THPVariable_Wrap(*t) : (Py_INCREF(Py_None), Py_None);
    if (!o) {
      Py_DECREF(r);
      return nullptr;
    }
    PyTuple_SET_ITEM(r, i++, o);
  }
  return r;
}

// q [B, H, S, D], k and v [B, H_kv, S, D], one device, one dtype.
struct Qkv {
  const Tensor &q, &k, &v;
  c10::Device dev;
  int dtype;
  int64_t B, H, Hkv, S, D;
  at::ScalarType type;
  explicit Qkv(Args& a) : Qkv(a.need(), a) {}
  Qkv(const Tensor& q_, Args& a) : Qkv(q_, a.need(), a) {}   // (in the arguments' order)
  Qkv(const Tensor& q_, const Tensor& k_, Args& a) : Qkv(q_, k_, a.need()) {}
  Qkv(const Tensor& q_, const Tensor& k_, const Tensor& v_)
      : q(q_), k(k_), v(v_), dev(q.device()), dtype(dtype_of(q)), type(q.scalar_type()) {
    if (q.dim() != 4 || k.dim() != 4) throw NotPlain{};
    B = q.size(0); H = q.size(1); S = q.size(2); D = q.size(3); Hkv = k.size(1);
    for (int64_t x : {B, H, S, D, Hkv}) if (x > INT_MAX) throw NotPlain{};
    same(q, q.sizes(), type, dev);
    same(k, {B, Hkv, S, D}, type, dev);
    same(v, {B, Hkv, S, D}, type, dev);
  }
};

// bias pointer and strides, normalisation (zeros for the plain calls)
struct Bias {
  const float* p;
  long long sb, sh, sq;
  int norm;
  explicit Bias(Args& a) : p(a.pointer<float>()), sb(a.whole()), sh(a.whole()), sq(a.whole()), norm(a.index()) {}
};

// fwd(q, k, v, out, lse, slopes, table, tables, rope, theta, mask, window, scale,
//     bias, sb, sh, sq, norm, q_block_ptr, k_block_idx, blocks) -> (O, LSE)
PyObject* fwd(Args a) {
  Qkv x(a);
  const Tensor *out_ = a.tensor(), *lse = a.tensor(), *slopes = a.tensor();
  Args late = a;            // the table needs the variant, which follows it
  a.i += 2;
  const int rope = a.index();
  const double theta = a.number();
  const int mask = a.index(), window = a.size();
  const float scale = a.scale(x.D);
  const Bias bias(a);
  const int *qp = a.pointer<int>(), *ki = a.pointer<int>();
  const long long blocks = a.whole();
  const Table tab = table_of(late, rope, theta, x.D, x.S, x.dev);
  const float* sl = slopes_of(slopes, x.H, x.dev);
  const bool relu = bias.norm == AF_NORM_RELU;
  const Tensor o = out_or(out_, x.q.sizes(), x.type, x.dev);
  Tensor l;
  if (!relu || lse) l = out_or(lse, {x.B, x.H, x.S}, at::kFloat, x.dev);
  float* lp = l.defined() ? static_cast<float*>(out(l)) : nullptr;
  const int B = (int)x.B, H = (int)x.H, Hkv = (int)x.Hkv, S = (int)x.S, D = (int)x.D;
  Tensor ws;                // keys rotated once, where that is faster
  if (const size_t n = af_fwd_workspace_bytes(B, H, Hkv, S, D, x.dtype, rope, mask, window, bias.norm,
                                              sl || bias.p, blocks)) {
    try {
      ws = at::empty({(int64_t)n}, at::TensorOptions().dtype(at::kByte).device(x.dev));
    } catch (const c10::OutOfMemoryError&) {   // rotated in the loop instead
    }
  }
  const int rc = enqueue(x.dev, [&](void* st) {
    if (ws.defined())
      return af_fwd_ws(in(x.q), in(x.k), in(x.v), out(o), lp, qp, ki, bias.p, bias.sb, bias.sh, bias.sq,
                       bias.norm, out(ws), (size_t)ws.numel(), B, H, Hkv, S, D, x.dtype, rope, (float)theta, tab.ptr,
                       tab.rows, mask, window, sl, scale, st);
    if (qp)
      return attnfuse_fwd_blocksparse(in(x.q), in(x.k), in(x.v), out(o), lp, qp, ki, B, H, Hkv, S, D, x.dtype,
                                      rope, (float)theta, tab.ptr, tab.rows, mask, window, sl, scale, st);
    return attnfuse_fwd_bias_norm(in(x.q), in(x.k), in(x.v), out(o), lp, bias.p, bias.sb, bias.sh, bias.sq,
                                  bias.norm, B, H, Hkv, S, D, x.dtype, rope, (float)theta, tab.ptr, tab.rows, mask,
                                  window, sl, scale, st);
  });
  return rc ? PyLong_FromLong(rc) : tuple_of({&o, &l});
}

// bwd(q, k, v, o, do, lse, dq, dk, dv, workspace, slopes, table, tables, rope, theta, mask, window, scale,
//     bias, sb, sh, sq, norm, q_block_ptr, k_block_idx, k_block_ptr, q_block_idx, longest, tiles) -> (dQ, dK, dV)
PyObject* bwd(Args a) {
  Qkv x(a);
  const Tensor &o = a.need(), &dout = a.need();
  const Tensor *lse = a.tensor(), *dq_ = a.tensor(), *dk_ = a.tensor(), *dv_ = a.tensor(), *ws_ = a.tensor(),
               *slopes = a.tensor();
  Args late = a;
  a.i += 2;
  const int rope = a.index();
  const double theta = a.number();
  const int mask = a.index(), window = a.size();
  const float scale = a.scale(x.D);
  const Bias bias(a);
  const int *qp = a.pointer<int>(), *ki = a.pointer<int>(), *kp = a.pointer<int>(), *qi = a.pointer<int>();
  const int longest = a.size();
  const long long tiles = a.whole();
  const Table tab = table_of(late, rope, theta, x.D, x.S, x.dev);
  const float* sl = slopes_of(slopes, x.H, x.dev);
  same(o, x.q.sizes(), x.type, x.dev);
  same(dout, x.q.sizes(), x.type, x.dev);
  if (lse) same(*lse, {x.B, x.H, x.S}, at::kFloat, x.dev);
  else if (bias.norm != AF_NORM_RELU) throw NotPlain{};
  const float* lp = lse ? static_cast<const float*>(lse->const_data_ptr()) : nullptr;
  const Tensor dq = out_or(dq_, x.q.sizes(), x.type, x.dev), dk = out_or(dk_, x.k.sizes(), x.type, x.dev),
               dv = out_or(dv_, x.k.sizes(), x.type, x.dev);
  const int B = (int)x.B, H = (int)x.H, Hkv = (int)x.Hkv, S = (int)x.S, D = (int)x.D;
  Tensor ws;
  if (ws_) {
    if (ws_->device() != x.dev || !ws_->is_contiguous()) throw NotPlain{};
    ws = *ws_;
  } else {
    ws = at::empty({(int64_t)attnfuse_bwd_workspace_bytes(B, H, Hkv, S, D, rope)},
                   at::TensorOptions().dtype(at::kByte).device(x.dev));
  }
  const size_t n = (size_t)ws.numel() * ws.element_size();
  const int rc = enqueue(x.dev, [&](void* st) {
    if (qp)
      return af_bwd_blocksparse(in(x.q), in(x.k), in(x.v), in(o), in(dout), lp, out(dq), out(dk), out(dv), qp, ki,
                                kp, qi, longest, tiles, out(ws), n, B, H, Hkv, S, D, x.dtype, rope, (float)theta,
                                tab.ptr, tab.rows, mask, window, sl, scale, st);
    return attnfuse_bwd_bias_norm(in(x.q), in(x.k), in(x.v), in(o), in(dout), lp, out(dq), out(dk),
                                  out(dv), bias.p, bias.sb, bias.sh, bias.sq, bias.norm, out(ws), n, B, H, Hkv, S,
                                  D, x.dtype, rope, (float)theta, tab.ptr, tab.rows, mask, window, sl, scale, st);
  });
  return rc ? PyLong_FromLong(rc) : tuple_of({&dq, &dk, &dv});
}

// decode(q, k, v, lens, out, lse, workspace, slopes, table, tables, rope, theta, mask, window, scale, noalloc) -> (O, LSE)
PyObject* decode(Args a) {
  const Tensor &q = a.need(), &k = a.need(), &v = a.need();
  const Tensor *lens = a.tensor(), *out_ = a.tensor(), *lse = a.tensor(), *ws_ = a.tensor(), *slopes = a.tensor();
  Args late = a;
  a.i += 2;
  const int rope = a.index();
  const double theta = a.number();
  const int mask = a.index(), window = a.size();
  const int dtype = dtype_of(q);
  const c10::Device dev = q.device();
  const at::ScalarType type = q.scalar_type();
  if (q.dim() != 3 || k.dim() != 4) throw NotPlain{};
  const int64_t B = q.size(0), H = q.size(1), D = q.size(2), Hkv = k.size(1), S = k.size(2);
  for (int64_t n : {B, H, D, Hkv, S}) if (n > INT_MAX) throw NotPlain{};
  const float scale = a.scale(D);
  const bool noalloc = a.whole() != 0;
  same(q, q.sizes(), type, dev);
  same(k, {B, Hkv, S, D}, type, dev);
  same(v, {B, Hkv, S, D}, type, dev);
  if (lens) same(*lens, {B}, at::kInt, dev);
  const Table tab = table_of(late, rope, theta, D, S, dev);
  const float* sl = slopes_of(slopes, H, dev);
  const Tensor o = out_or(out_, q.sizes(), type, dev), l = out_or(lse, {B, H}, at::kFloat, dev);
  float* lp = static_cast<float*>(out(l));
  const int* ln = lens ? static_cast<const int*>(lens->const_data_ptr()) : nullptr;
  Tensor ws;
  if (!noalloc) {
    if (ws_) {
      if (ws_->device() != dev || !ws_->is_contiguous()) throw NotPlain{};
      ws = *ws_;
    } else {
      ws = at::empty({(int64_t)attnfuse_decode_workspace_bytes((int)B, (int)H, (int)Hkv, (int)S, (int)D)},
                     at::TensorOptions().dtype(at::kByte).device(dev));
    }
  }
  const int rc = enqueue(dev, [&](void* st) {
    if (noalloc)
      return attnfuse_decode_noalloc(in(q), in(k), in(v), ln, out(o), lp, (int)B, (int)H, (int)Hkv, (int)S,
                                     (int)D, dtype, rope, (float)theta, tab.ptr, tab.rows, mask, window, sl, scale, st);
    return attnfuse_decode(in(q), in(k), in(v), ln, out(o), lp, out(ws),
                           (size_t)ws.numel() * ws.element_size(), (int)B, (int)H, (int)Hkv, (int)S, (int)D, dtype,
                           rope, (float)theta, tab.ptr, tab.rows, mask, window, sl, scale, st);
  });
  return rc ? PyLong_FromLong(rc) : tuple_of({&o, &l});
}

// rope(q, k, out_q, out_k, table, tables, rope, theta, inverse) -> (Qr, Kr)
PyObject* rope(Args a) {
  const Tensor& x0 = a.need();
  const Tensor *x1 = a.tensor(), *y0_ = a.tensor(), *y1_ = a.tensor();
  Args late = a;
  a.i += 2;
  const int kind = a.index();
  const double theta = a.number();
  const bool inverse = a.whole() != 0;
  const int dtype = dtype_of(x0);
  const c10::Device dev = x0.device();
  const at::ScalarType type = x0.scalar_type();
  if (x0.dim() != 4 || (!x1 && y1_)) throw NotPlain{};
  const int64_t B = x0.size(0), H = x0.size(1), S = x0.size(2), D = x0.size(3);
  const int64_t Hkv = x1 ? (x1->dim() == 4 ? x1->size(1) : -1) : 1;
  for (int64_t n : {B, H, S, D, Hkv}) if (n > INT_MAX || n < 0) throw NotPlain{};
  same(x0, x0.sizes(), type, dev);
  if (x1) same(*x1, {B, Hkv, S, D}, type, dev);
  const Table tab = table_of(late, kind, theta, D, S, dev);
  const Tensor y0 = out_or(y0_, x0.sizes(), type, dev);
  Tensor y1;
  if (x1) y1 = out_or(y1_, x1->sizes(), type, dev);
  const void* p1 = x1 ? in(*x1) : nullptr;
  void* r1 = x1 ? out(y1) : nullptr;
  const int rc = enqueue(dev, [&](void* st) {
    return (inverse ? attnfuse_rope_bwd : attnfuse_rope)(in(x0), p1, out(y0), r1, (int)B, (int)H, (int)Hkv, (int)S,
                                                         (int)D, dtype, kind, (float)theta, tab.ptr, tab.rows, st);
  });
  return rc ? PyLong_FromLong(rc) : tuple_of({&y0, &y1});
}

// ---------------------------------------------------------------- include/attnfuse_llm.h
// A tensor of rows that may lie apart: exactly that shape, type and device, each
// row contiguous and 16-byte aligned; s: the strides of its other dimensions in
// elements, 0 for one of a single row.
struct Rows {
  long long s[3] = {0, 0, 0};
  Rows(const Tensor& t, at::IntArrayRef shape, at::ScalarType type, c10::Device dev) {
    if (t.device() != dev || t.scalar_type() != type || t.sizes() != shape) throw NotPlain{};
    const int64_t last = t.dim() - 1;
    if ((t.stride(last) != 1 && t.size(last) > 1) || reinterpret_cast<uintptr_t>(t.const_data_ptr()) % 16) throw NotPlain{};
    for (int64_t i = 0; i < last; ++i) {
      s[i] = t.size(i) > 1 ? t.stride(i) : 0;
      if (s[i] * (long long)t.element_size() % 16) throw NotPlain{};
    }
  }
  Rows() = default;
};

// The norm weights: both [D], fp32 or the rows' type, the same for both.
struct Weights {
  const void *q = nullptr, *k = nullptr;
  int type = AF_DTYPE_FP32;
  at::ScalarType scalar = at::kFloat;
  Weights(const Tensor* qw, const Tensor* kw, int64_t D, at::ScalarType rows, c10::Device dev) {
    if (const Tensor* w = qw ? qw : kw) scalar = w->scalar_type();
    if (scalar != at::kFloat && scalar != rows) throw NotPlain{};
    type = scalar == at::kFloat ? AF_DTYPE_FP32 : AF_DTYPE_BF16;
    for (const Tensor* w : {qw, kw}) {
      if (!w) continue;
      same(*w, {D}, scalar, dev);
      if (reinterpret_cast<uintptr_t>(w->const_data_ptr()) % 16) throw NotPlain{};
    }
    q = qw ? qw->const_data_ptr() : nullptr;
    k = kw ? kw->const_data_ptr() : nullptr;
  }
};

// Positions and the table of their angles (of its rows the first max_positions, where
// that is given: not 0); args: positions, then (at `late`) the table and the binding's
// tables; n rows at 0..n-1 without positions.
struct Placed {
  const int* positions = nullptr;
  Table table;
  Placed(const Tensor* pos, Args late, int rope, double theta, int64_t D, int64_t n, at::IntArrayRef shape,
         long long max_positions, c10::Device dev) {
    if (rope == AF_ROPE_NONE) return;
    if (pos) {
      same(*pos, shape, at::kInt, dev);
      positions = static_cast<const int*>(pos->const_data_ptr());
      Args peek = late;
      if (max_positions <= 0 && !peek.tensor()) throw NotPlain{};
      n = max_positions > 0 ? max_positions : 1;
    }
    table = table_of(late, rope, theta, D, n, dev);
    if (pos && max_positions > 0) table.rows = (int)max_positions;
  }
};

Tensor workspace_or(const Tensor* given, size_t bytes, c10::Device dev) {
  if (given) {
    if (given->device() != dev || !given->is_contiguous()) throw NotPlain{};
    return *given;
  }
  return at::empty({(int64_t)bytes}, at::TensorOptions().dtype(at::kByte).device(dev));
}

size_t bytes_of(const Tensor& t) { return (size_t)t.numel() * t.element_size(); }

// q [B, H, S, D] and k [B, H_kv, S, D] or None, rows apart.
struct Qk {
  const Tensor& q;
  const Tensor* k;
  c10::Device dev;
  int dtype;
  at::ScalarType type;
  int64_t B, H, S, D, Hkv = 0;
  Rows qs, ks;
  Qk(const Tensor& q_, const Tensor* k_) : q(q_), k(k_), dev(q.device()), dtype(dtype_of(q)), type(q.scalar_type()) {
    if (q.dim() != 4 || (k && k->dim() != 4)) throw NotPlain{};
    B = q.size(0); H = q.size(1); S = q.size(2); D = q.size(3);
    if (k) Hkv = k->size(1);
    for (int64_t x : {B, H, S, D, Hkv}) if (x > INT_MAX) throw NotPlain{};
    qs = Rows(q, q.sizes(), type, dev);
    if (k) ks = Rows(*k, {B, Hkv, S, D}, type, dev);
  }
};

// A norm call's variant; positions of several axes: their sections (n 0: one axis).
struct Norm {
  float eps;
  int rope;
  double theta;
  bool norm = true;
  int n = 0, sections[4] = {0, 0, 0, 0}, order = 0;
  explicit Norm(Args& a) : eps((float)a.number()), rope(a.index()), theta(a.number()) {}
  Norm(float e, int r, double t) : eps(e), rope(r), theta(t) {}
  bool own = false;   // every axis has its own frequencies
  OwnKey key = {nullptr, nullptr};
  void take_axes(Args& a) {   // norm, sections, section_order's name and value, frequencies
    norm = a.whole() != 0;
    PyObject* s = a.next();
    if (!PyTuple_CheckExact(s) || PyTuple_GET_SIZE(s) < 1 || PyTuple_GET_SIZE(s) > 4) throw NotPlain{};
    n = (int)PyTuple_GET_SIZE(s);
    for (int i = 0; i < n; ++i) {
      PyObject* x = PyTuple_GET_ITEM(s, i);
      Args one{&x, 1};
      sections[i] = one.size();
    }
    key = {s, a.next()};
    order = a.index();
    own = a.index() == AF_FREQUENCIES_OWN;
  }
};

int norm_fwd(const Qk& x, const Weights& w, const Norm& n, const Table& table, const int* positions, const Tensor& oq,
             const Tensor& ok) {
  return enqueue(x.dev, [&](void* st) {
    if (n.n)
      return attnfuse_qknorm_axes(in(x.q), x.k ? in(*x.k) : nullptr, out(oq), x.k ? out(ok) : nullptr, w.q, w.k, w.type,
                                  n.norm, n.eps, x.qs.s[0], x.qs.s[1], x.qs.s[2], x.ks.s[0], x.ks.s[1], x.ks.s[2], (int)x.B,
                                  (int)x.H, (int)x.Hkv, (int)x.S, (int)x.D, x.dtype, n.rope, (float)n.theta, table.ptr,
                                  table.rows, positions, n.n, n.sections, n.order, st);
    return attnfuse_qknorm_rope(in(x.q), x.k ? in(*x.k) : nullptr, out(oq), x.k ? out(ok) : nullptr, w.q, w.k, w.type, n.eps,
                                x.qs.s[0], x.qs.s[1], x.qs.s[2], x.ks.s[0], x.ks.s[1], x.ks.s[2], (int)x.B, (int)x.H,
                                (int)x.Hkv, (int)x.S, (int)x.D, x.dtype, n.rope, (float)n.theta, table.ptr, table.rows,
                                positions, st);
  });
}

int norm_bwd(const Qk& x, const Weights& w, const Norm& n, const Table& table, const int* positions, const Tensor& dqr,
             const Tensor* dkr, const Tensor& dq, const Tensor& dk, Tensor& dqw, Tensor& dkw, const Tensor* ws_, bool grads) {
  same(dqr, x.q.sizes(), x.type, x.dev);
  if (dkr) same(*dkr, x.k->sizes(), x.type, x.dev);
  const Rows dqs(dq, x.q.sizes(), x.type, x.dev);
  Rows dks;
  if (x.k) dks = Rows(dk, x.k->sizes(), x.type, x.dev);
  Tensor ws;
  if (grads) {
    const auto options = at::TensorOptions().dtype(w.scalar).device(x.dev);
    dqw = at::empty({x.D}, options);
    if (x.k) dkw = at::empty({x.D}, options);
    ws = workspace_or(ws_, attnfuse_qknorm_rope_bwd_workspace_bytes((int)x.B, (int)x.H, (int)x.Hkv, (int)x.S, (int)x.D,
                                                                    x.dtype), x.dev);
  }
  return enqueue(x.dev, [&](void* st) {
    if (n.n)
      return attnfuse_qknorm_axes_bwd(
          in(x.q), x.k ? in(*x.k) : nullptr, in(dqr), dkr ? in(*dkr) : nullptr, out(dq), x.k ? out(dk) : nullptr,
          grads ? out(dqw) : nullptr, grads && x.k ? out(dkw) : nullptr, w.q, w.k, w.type, 1, n.eps, x.qs.s[0], x.qs.s[1],
          x.qs.s[2], x.ks.s[0], x.ks.s[1], x.ks.s[2], dqs.s[0], dqs.s[1], dqs.s[2], dks.s[0], dks.s[1], dks.s[2],
          grads ? out(ws) : nullptr, grads ? bytes_of(ws) : 0, (int)x.B, (int)x.H, (int)x.Hkv, (int)x.S, (int)x.D, x.dtype,
          n.rope, (float)n.theta, table.ptr, table.rows, positions, n.n, n.sections, n.order, st);
    return attnfuse_qknorm_rope_bwd(
        in(x.q), x.k ? in(*x.k) : nullptr, in(dqr), dkr ? in(*dkr) : nullptr, out(dq), x.k ? out(dk) : nullptr,
        grads ? out(dqw) : nullptr, grads && x.k ? out(dkw) : nullptr, w.q, w.k, w.type, n.eps, x.qs.s[0], x.qs.s[1],
        x.qs.s[2], x.ks.s[0], x.ks.s[1], x.ks.s[2], dqs.s[0], dqs.s[1], dqs.s[2], dks.s[0], dks.s[1], dks.s[2],
        grads ? out(ws) : nullptr, grads ? bytes_of(ws) : 0, (int)x.B, (int)x.H, (int)x.Hkv, (int)x.S, (int)x.D, x.dtype,
        n.rope, (float)n.theta, table.ptr, table.rows, positions, st);
  });
}

// qknorm(q, k, q_weight, k_weight, out_q, out_k, positions, table, tables, eps, rope, theta, max_positions) -> (Qr, Kr)
PyObject* qknorm(Args a) {
  const Tensor &q = a.need(), *k = a.tensor();
  const Qk x(q, k);
  const Tensor *qw = a.tensor(), *kw = a.tensor(), *oq_ = a.tensor(), *ok_ = a.tensor(), *pos = a.tensor();
  Args late = a;
  a.i += 2;
  const Norm n(a);
  const long long most = a.positive();
  if (!x.k && (kw || ok_)) throw NotPlain{};
  const Weights w(qw, kw, x.D, x.type, x.dev);
  const Placed at_(pos, late, n.rope, n.theta, x.D, x.S, {x.B, x.S}, most, x.dev);
  const Tensor oq = out_or(oq_, x.q.sizes(), x.type, x.dev);
  Tensor ok;
  if (x.k) ok = out_or(ok_, x.k->sizes(), x.type, x.dev);
  const int rc = norm_fwd(x, w, n, at_.table, at_.positions, oq, ok);
  return rc ? PyLong_FromLong(rc) : tuple_of({&oq, &ok});
}

// qknorm_bwd(q, k, dqr, dkr, q_weight, k_weight, dq, dk, workspace, positions, table, tables, eps, rope, theta,
//            max_positions, weight_grads) -> (dQ, dK, dq_weight, dk_weight)
PyObject* qknorm_bwd(Args a) {
  const Tensor &q = a.need(), *k = a.tensor();
  const Qk x(q, k);
  const Tensor& dqr = a.need();
  const Tensor *dkr = a.tensor(), *qw = a.tensor(), *kw = a.tensor(), *dq_ = a.tensor(), *dk_ = a.tensor(), *ws_ = a.tensor(),
               *pos = a.tensor();
  Args late = a;
  a.i += 2;
  const Norm n(a);
  const long long most = a.positive();
  const bool grads = a.whole() != 0;
  if (!x.k != !dkr || (!x.k && (kw || dk_))) throw NotPlain{};
  const Weights w(qw, kw, x.D, x.type, x.dev);
  const Placed at_(pos, late, n.rope, n.theta, x.D, x.S, {x.B, x.S}, most, x.dev);
  const Tensor dq = dq_ ? *dq_ : at::empty_like(x.q);
  Tensor dk, dqw, dkw;
  if (x.k) dk = dk_ ? *dk_ : at::empty_like(*x.k);
  const int rc = norm_bwd(x, w, n, at_.table, at_.positions, dqr, dkr, dq, dk, dqw, dkw, ws_, grads);
  return rc ? PyLong_FromLong(rc) : tuple_of({&dq, &dk, &dqw, &dkw});
}

// Positions of several axes [axes, lead...] and the table of their angles, of its rows the
// first max_positions (0: all of the given one); late: the table and the binding's tables.
struct AxesPlaced {
  const int* positions;
  Table table;
  AxesPlaced(const Tensor& pos, Args late, const Norm& n, int64_t D, at::IntArrayRef shape, long long most, c10::Device dev) {
    int64_t pairs = 0;
    for (int s : n.sections) pairs += s;
    if (n.rope == AF_ROPE_NONE || 2 * pairs != D) throw NotPlain{};
    same(pos, shape, at::kInt, dev);
    positions = static_cast<const int*>(pos.const_data_ptr());
    Args peek = late;
    if (most <= 0 && !peek.tensor()) throw NotPlain{};
    table = table_of(late, n.rope, n.theta, D, most > 0 ? most : 1, dev, n.own ? &n.key : nullptr);
    if (most > 0) table.rows = (int)most;
  }
};

// dX = R^T dXr of a rotation without norm; dq, dk: given, or undefined and then made.
int unturn(const Tensor& dqr, const Tensor* dkr, Tensor& dq, Tensor& dk, const Norm& n, const Table& table,
           const int* positions) {
  const int dtype = dtype_of(dqr);
  const c10::Device dev = dqr.device();
  const at::ScalarType type = dqr.scalar_type();
  const int64_t B = dqr.size(0), H = dqr.size(1), S = dqr.size(2), D = dqr.size(3), Hkv = dkr ? dkr->size(1) : 0;
  for (int64_t x : {B, H, S, D, Hkv}) if (x > INT_MAX) throw NotPlain{};
  same(dqr, dqr.sizes(), type, dev);
  if (dkr) same(*dkr, {B, Hkv, S, D}, type, dev);
  if (!dq.defined()) dq = at::empty_like(dqr);
  if (dkr && !dk.defined()) dk = at::empty_like(*dkr);
  const Rows qs(dq, dqr.sizes(), type, dev);
  Rows ks;
  if (dkr) ks = Rows(dk, dkr->sizes(), type, dev);
  return enqueue(dev, [&](void* st) {
    return attnfuse_qknorm_axes_bwd(nullptr, nullptr, in(dqr), dkr ? in(*dkr) : nullptr, out(dq), dkr ? out(dk) : nullptr,
                                    nullptr, nullptr, nullptr, nullptr, AF_DTYPE_FP32, 0, 0.f, 0, 0, 0, 0, 0, 0, qs.s[0],
                                    qs.s[1], qs.s[2], ks.s[0], ks.s[1], ks.s[2], nullptr, 0, (int)B, (int)H, (int)Hkv, (int)S,
                                    (int)D, dtype, n.rope, (float)n.theta, table.ptr, table.rows, positions, n.n, n.sections,
                                    n.order, st);
  });
}

// axes(q, k, q_weight, k_weight, out_q, out_k, positions, table, tables, eps, rope, theta, max_positions, norm, sections,
//      section_order, its value, frequencies) -> (Qr, Kr)
PyObject* axes(Args a) {
  const Tensor &q = a.need(), *k = a.tensor();
  const Qk x(q, k);
  const Tensor *qw = a.tensor(), *kw = a.tensor(), *oq_ = a.tensor(), *ok_ = a.tensor();
  const Tensor& pos = a.need();
  Args late = a;
  a.i += 2;
  Norm n(a);
  const long long most = a.positive();
  n.take_axes(a);
  if ((!x.k && (kw || ok_)) || (!n.norm && (qw || kw))) throw NotPlain{};
  const Weights w(qw, kw, x.D, x.type, x.dev);
  const AxesPlaced at_(pos, late, n, x.D, {n.n, x.B, x.S}, most, x.dev);
  const Tensor oq = out_or(oq_, x.q.sizes(), x.type, x.dev);
  Tensor ok;
  if (x.k) ok = out_or(ok_, x.k->sizes(), x.type, x.dev);
  const int rc = norm_fwd(x, w, n, at_.table, at_.positions, oq, ok);
  return rc ? PyLong_FromLong(rc) : tuple_of({&oq, &ok});
}

// axes_bwd(q, k, dqr, dkr, q_weight, k_weight, dq, dk, workspace, positions, table, tables, eps, rope, theta,
//          max_positions, weight_grads, norm, sections, section_order, its value, frequencies)
//     -> (dQ, dK, dq_weight, dk_weight); without norm q and k are None
PyObject* axes_bwd(Args a) {
  const Tensor *q = a.tensor(), *k = a.tensor(), &dqr = a.need();
  const Tensor *dkr = a.tensor(), *qw = a.tensor(), *kw = a.tensor(), *dq_ = a.tensor(), *dk_ = a.tensor(), *ws_ = a.tensor();
  const Tensor& pos = a.need();
  Args late = a;
  a.i += 2;
  Norm n(a);
  const long long most = a.positive();
  const bool grads = a.whole() != 0;
  n.take_axes(a);
  Tensor dq, dk, dqw, dkw;
  if (dq_) dq = *dq_;
  if (dk_) dk = *dk_;
  int rc;
  if (!n.norm) {
    if (q || k || qw || kw || grads || (!dkr && dk_) || dqr.dim() != 4 || (dkr && dkr->dim() != 4)) throw NotPlain{};
    const AxesPlaced at_(pos, late, n, dqr.size(3), {n.n, dqr.size(0), dqr.size(2)}, most, dqr.device());
    rc = unturn(dqr, dkr, dq, dk, n, at_.table, at_.positions);
  } else {
    if (!q || !k != !dkr || (!k && (kw || dk_))) throw NotPlain{};
    const Qk x(*q, k);
    const Weights w(qw, kw, x.D, x.type, x.dev);
    const AxesPlaced at_(pos, late, n, x.D, {n.n, x.B, x.S}, most, x.dev);
    if (!dq_) dq = at::empty_like(x.q);
    if (k && !dk_) dk = at::empty_like(*k);
    rc = norm_bwd(x, w, n, at_.table, at_.positions, dqr, dkr, dq, dk, dqw, dkw, ws_, grads);
  }
  return rc ? PyLong_FromLong(rc) : tuple_of({&dq, &dk, &dqw, &dkw});
}

// append(q, k, v, k_cache, v_cache, slots, q_weight, k_weight, out_q, positions, table, tables, norm, eps, rope, theta,
//        max_positions) -> (Qr,)
// axes_append(q, k, v, k_cache, v_cache, slots, q_weight, k_weight, out_q, positions, table, tables, eps, rope, theta,
//             max_positions, norm, sections, section_order, its value, frequencies) -> (Qr,)
template <bool AXES>
PyObject* append(Args a) {
  const Tensor &q = a.need(), &k = a.need(), &v = a.need(), &kc = a.need(), &vc = a.need(), &slots = a.need();
  const Tensor *qw = a.tensor(), *kw = a.tensor(), *oq_ = a.tensor(), *pos = a.tensor();
  Args late = a;
  a.i += 2;
  bool norm = true;
  if constexpr (!AXES) norm = a.whole() != 0;
  Norm n(a);
  const float eps = n.eps;
  const int rope = n.rope;
  const double theta = n.theta;
  const long long most = a.positive();
  if constexpr (AXES) {
    n.take_axes(a);
    norm = n.norm;
    if (!pos) throw NotPlain{};
  }
  const int dtype = dtype_of(q);
  const c10::Device dev = q.device();
  const at::ScalarType type = q.scalar_type();
  if (q.dim() != 3 || k.dim() != 3 || kc.dim() != 4 || (rope != AF_ROPE_NONE && !pos)) throw NotPlain{};
  const int64_t T = q.size(0), H = q.size(1), D = q.size(2), Hkv = k.size(1), pages = kc.size(0), page = kc.size(2);
  for (int64_t m : {T, H, D, Hkv, pages, page}) if (m > INT_MAX) throw NotPlain{};
  const Rows qs(q, {T, H, D}, type, dev), ks(k, {T, Hkv, D}, type, dev), vs(v, {T, Hkv, D}, type, dev),
      kcs(kc, {pages, Hkv, page, D}, type, dev), vcs(vc, {pages, Hkv, page, D}, type, dev);
  same(slots, {T}, at::kLong, dev);
  const Weights w(qw, kw, D, type, dev);
  if constexpr (AXES) {
    if (!norm && (qw || kw)) throw NotPlain{};
    const AxesPlaced at_(*pos, late, n, D, {n.n, T}, most, dev);
    const Tensor oq = out_or(oq_, q.sizes(), type, dev);
    const int rc = enqueue(dev, [&](void* st) {
      return attnfuse_qknorm_axes_append(
          in(q), in(k), in(v), out(oq), out(kc), out(vc), reinterpret_cast<const long long*>(slots.const_data_ptr()), w.q,
          w.k, w.type, norm, eps, qs.s[0], qs.s[1], ks.s[0], ks.s[1], vs.s[0], vs.s[1], kcs.s[0], kcs.s[1], kcs.s[2],
          vcs.s[0], vcs.s[1], vcs.s[2], (int)T, (int)H, (int)Hkv, (int)D, (int)pages, (int)page, dtype, rope, (float)theta,
          at_.table.ptr, at_.table.rows, at_.positions, n.n, n.sections, n.order, st);
    });
    return rc ? PyLong_FromLong(rc) : tuple_of({&oq});
  }
  const Placed at_(pos, late, rope, theta, D, 1, {T}, most, dev);
  const Tensor oq = out_or(oq_, q.sizes(), type, dev);
  const int rc = enqueue(dev, [&](void* st) {
    return attnfuse_qknorm_rope_append(
        in(q), in(k), in(v), out(oq), out(kc), out(vc), reinterpret_cast<const long long*>(slots.const_data_ptr()), w.q, w.k,
        w.type, norm, eps, qs.s[0], qs.s[1], ks.s[0], ks.s[1], vs.s[0], vs.s[1], kcs.s[0], kcs.s[1], kcs.s[2], vcs.s[0],
        vcs.s[1], vcs.s[2], (int)T, (int)H, (int)Hkv, (int)D, (int)pages, (int)page, dtype, rope, (float)theta,
        at_.table.ptr, at_.table.rows, at_.positions, st);
  });
  return rc ? PyLong_FromLong(rc) : tuple_of({&oq});
}

// decode_paged(q, k_cache, v_cache, block_table, lens, out, lse, workspace, slopes, table, tables, rope, theta, mask, window,
//              sinks, scale) -> (O, LSE)
PyObject* decode_paged(Args a) {
  const Tensor &q = a.need(), &kc = a.need(), &vc = a.need(), &table = a.need();
  const Tensor *lens = a.tensor(), *out_ = a.tensor(), *lse = a.tensor(), *ws_ = a.tensor(), *slopes = a.tensor();
  Args late = a;
  a.i += 2;
  const int rope = a.index();
  const double theta = a.number();
  const int mask = a.index(), window = a.size(), sinks = a.size();
  const c10::Device dev = q.device();
  const at::ScalarType type = q.scalar_type();
  if (dtype_of(q) != AF_DTYPE_BF16 || q.dim() != 3 || kc.dim() != 4 || table.dim() != 2) throw NotPlain{};
  const int64_t B = q.size(0), H = q.size(1), D = q.size(2), pages = kc.size(0), Hkv = kc.size(1), page = kc.size(2),
                most = table.size(1);
  for (int64_t n : {B, H, D, Hkv, pages, page, most}) if (n > (1 << 28)) throw NotPlain{};
  const int64_t S = most * page;
  if (S > INT_MAX) throw NotPlain{};
  const float scale = a.scale(D);
  same(q, q.sizes(), type, dev);
  const Rows ks(kc, {pages, Hkv, page, D}, type, dev), vs(vc, {pages, Hkv, page, D}, type, dev);
  same(table, {B, most}, at::kInt, dev);
  if (lens) same(*lens, {B}, at::kInt, dev);
  const Table tab = table_of(late, rope, theta, D, S, dev);
  const float* sl = slopes_of(slopes, H, dev);
  const Tensor o = out_or(out_, q.sizes(), type, dev), l = out_or(lse, {B, H}, at::kFloat, dev);
  const Tensor ws = workspace_or(ws_, attnfuse_decode_paged_workspace_bytes((int)B, (int)H, (int)Hkv, (int)S, (int)D,
                                                                            mask == AF_MASK_SLIDING_WINDOW ? window : 0,
                                                                            sinks), dev);
  const int rc = enqueue(dev, [&](void* st) {
    return attnfuse_decode_paged(in(q), in(kc), in(vc), static_cast<const int*>(table.const_data_ptr()),
                                 lens ? static_cast<const int*>(lens->const_data_ptr()) : nullptr, out(o),
                                 static_cast<float*>(out(l)), out(ws), bytes_of(ws), ks.s[0], ks.s[1], ks.s[2], vs.s[0],
                                 vs.s[1], vs.s[2], (int)B, (int)H, (int)Hkv, (int)D, (int)pages, (int)page, (int)most, rope,
                                 (float)theta, tab.ptr, tab.rows, mask, window, sinks, sl, scale, st);
  });
  return rc ? PyLong_FromLong(rc) : tuple_of({&o, &l});
}

// fwd_paged(q, k_cache, v_cache, block_table, q_starts, lens, prefix_table, prefix_len, out, lse, workspace, scale) -> (O, LSE)
PyObject* fwd_paged(Args a) {
  const Tensor &q = a.need(), &kc = a.need(), &vc = a.need(), &table = a.need();
  const Tensor *starts = a.tensor(), *lens = a.tensor(), *prefix = a.tensor(), *plen = a.tensor(), *out_ = a.tensor(),
               *lse = a.tensor(), *ws_ = a.tensor();
  const c10::Device dev = q.device();
  const at::ScalarType type = q.scalar_type();
  if (dtype_of(q) != AF_DTYPE_BF16 || q.dim() != 3 || kc.dim() != 4 || table.dim() != 2) throw NotPlain{};
  const int64_t T = q.size(0), H = q.size(1), D = q.size(2), pages = kc.size(0), Hkv = kc.size(1), page = kc.size(2),
                B = table.size(0), most = table.size(1);
  if (prefix && (prefix->dim() != 1 || prefix->size(0) < 1)) throw NotPlain{};
  const int64_t ahead = prefix ? prefix->size(0) : 0;
  for (int64_t n : {T, B, H, D, Hkv, pages, page, most, ahead}) if (n > (1 << 28)) throw NotPlain{};
  if (most * page > INT_MAX || ahead * page > INT_MAX || (!starts && B != T) || (!prefix && plen)) throw NotPlain{};
  const float scale = a.scale(D);
  same(q, q.sizes(), type, dev);
  const Rows ks(kc, {pages, Hkv, page, D}, type, dev), vs(vc, {pages, Hkv, page, D}, type, dev);
  same(table, {B, most}, at::kInt, dev);
  if (starts) same(*starts, {B + 1}, at::kInt, dev);
  if (lens) same(*lens, {B}, at::kInt, dev);
  if (prefix) same(*prefix, {ahead}, at::kInt, dev);
  if (plen) same(*plen, {1}, at::kInt, dev);
  const auto whole = [](const Tensor* t) { return t ? static_cast<const int*>(t->const_data_ptr()) : nullptr; };
  const Tensor o = out_or(out_, q.sizes(), type, dev), l = out_or(lse, {T, H}, at::kFloat, dev);
  const Tensor ws = workspace_or(ws_, attnfuse_fwd_paged_workspace_bytes((int)T, (int)B, (int)H, (int)Hkv, (int)D,
                                                                         (int)(most * page), (int)(ahead * page)), dev);
  const size_t bytes = bytes_of(ws);
  const int rc = enqueue(dev, [&](void* st) {
    return attnfuse_fwd_paged(in(q), in(kc), in(vc), whole(&table), whole(starts), whole(lens), whole(prefix), whole(plen),
                              out(o), static_cast<float*>(out(l)), bytes ? out(ws) : nullptr, bytes, ks.s[0], ks.s[1], ks.s[2],
                              vs.s[0], vs.s[1], vs.s[2], (int)T, (int)B, (int)H, (int)Hkv, (int)D, (int)pages, (int)page,
                              (int)most, (int)ahead, scale, st);
  });
  return rc ? PyLong_FromLong(rc) : tuple_of({&o, &l});
}

// decode_sinks(q, k, v, lens, out, lse, workspace, table, tables, rope, theta, window, sinks, scale) -> (O, LSE)
PyObject* decode_sinks(Args a) {
  const Tensor &q = a.need(), &k = a.need(), &v = a.need();
  const Tensor *lens = a.tensor(), *out_ = a.tensor(), *lse = a.tensor(), *ws_ = a.tensor();
  Args late = a;
  a.i += 2;
  const int rope = a.index();
  const double theta = a.number();
  const int window = a.size(), sinks = a.size();
  const c10::Device dev = q.device();
  const at::ScalarType type = q.scalar_type();
  if (dtype_of(q) != AF_DTYPE_BF16 || q.dim() != 3 || k.dim() != 4) throw NotPlain{};
  const int64_t B = q.size(0), H = q.size(1), D = q.size(2), Hkv = k.size(1), S = k.size(2);
  for (int64_t n : {B, H, D, Hkv, S}) if (n > INT_MAX) throw NotPlain{};
  const float scale = a.scale(D);
  same(q, q.sizes(), type, dev);
  same(k, {B, Hkv, S, D}, type, dev);
  same(v, {B, Hkv, S, D}, type, dev);
  if (lens) same(*lens, {B}, at::kInt, dev);
  const Table tab = table_of(late, rope, theta, D, S, dev);
  const Tensor o = out_or(out_, q.sizes(), type, dev), l = out_or(lse, {B, H}, at::kFloat, dev);
  const Tensor ws = workspace_or(ws_, attnfuse_decode_paged_workspace_bytes((int)B, (int)H, (int)Hkv, (int)S, (int)D, window,
                                                                            sinks), dev);
  const int rc = enqueue(dev, [&](void* st) {
    return attnfuse_decode_sinks(in(q), in(k), in(v), lens ? static_cast<const int*>(lens->const_data_ptr()) : nullptr,
                                 out(o), static_cast<float*>(out(l)), out(ws), bytes_of(ws), (int)B, (int)H, (int)Hkv, (int)S,
                                 (int)D, rope, (float)theta, tab.ptr, tab.rows, window, sinks, scale, st);
  });
  return rc ? PyLong_FromLong(rc) : tuple_of({&o, &l});
}

// A call under a window with sinks.
struct Sinks {
  int rope;
  double theta;
  int window, sinks;
  float scale;
};

int sinks_fwd(const Qkv& x, const Sinks& c, const Table& tab, const Tensor& o, const Tensor& l) {
  const int B = (int)x.B, H = (int)x.H, Hkv = (int)x.Hkv, S = (int)x.S, D = (int)x.D;
  Tensor ws;
  const size_t n = attnfuse_fwd_sinks_workspace_bytes(B, Hkv, S, D, x.dtype, c.rope);
  if (n) ws = workspace_or(nullptr, n, x.dev);
  return enqueue(x.dev, [&](void* st) {
    return attnfuse_fwd_sinks(in(x.q), in(x.k), in(x.v), out(o), static_cast<float*>(out(l)), n ? out(ws) : nullptr, n, B, H,
                              Hkv, S, D, x.dtype, c.rope, (float)c.theta, tab.ptr, tab.rows, c.window, c.sinks, c.scale, st);
  });
}

int sinks_bwd(const Qkv& x, const Sinks& c, const Table& tab, const Tensor& o, const Tensor& dout, const Tensor& lse,
              const Tensor& dq, const Tensor& dk, const Tensor& dv, const Tensor* ws_) {
  same(o, x.q.sizes(), x.type, x.dev);
  same(dout, x.q.sizes(), x.type, x.dev);
  same(lse, {x.B, x.H, x.S}, at::kFloat, x.dev);
  const int B = (int)x.B, H = (int)x.H, Hkv = (int)x.Hkv, S = (int)x.S, D = (int)x.D;
  const Tensor ws = workspace_or(ws_, attnfuse_bwd_sinks_workspace_bytes(B, H, Hkv, S, D, c.rope, c.window, c.sinks), x.dev);
  return enqueue(x.dev, [&](void* st) {
    return attnfuse_bwd_sinks(in(x.q), in(x.k), in(x.v), in(o), in(dout), static_cast<const float*>(lse.const_data_ptr()),
                              out(dq), out(dk), out(dv), out(ws), bytes_of(ws), B, H, Hkv, S, D, x.dtype, c.rope,
                              (float)c.theta, tab.ptr, tab.rows, c.window, c.sinks, c.scale, st);
  });
}

Sinks sinks_of(Args& a, int64_t D) {
  Sinks c;
  c.rope = a.index();
  c.theta = a.number();
  c.window = a.size();
  c.sinks = a.size();
  c.scale = a.scale(D);
  return c;
}

// fwd_sinks(q, k, v, out, lse, table, tables, rope, theta, window, sinks, scale) -> (O, LSE)
PyObject* fwd_sinks(Args a) {
  Qkv x(a);
  const Tensor *out_ = a.tensor(), *lse = a.tensor();
  Args late = a;
  a.i += 2;
  const Sinks c = sinks_of(a, x.D);
  const Table tab = table_of(late, c.rope, c.theta, x.D, x.S, x.dev);
  const Tensor o = out_or(out_, x.q.sizes(), x.type, x.dev), l = out_or(lse, {x.B, x.H, x.S}, at::kFloat, x.dev);
  const int rc = sinks_fwd(x, c, tab, o, l);
  return rc ? PyLong_FromLong(rc) : tuple_of({&o, &l});
}

// bwd_sinks(q, k, v, o, do, lse, dq, dk, dv, workspace, table, tables, rope, theta, window, sinks, scale) -> (dQ, dK, dV)
PyObject* bwd_sinks(Args a) {
  Qkv x(a);
  const Tensor &o = a.need(), &dout = a.need(), &lse = a.need();
  const Tensor *dq_ = a.tensor(), *dk_ = a.tensor(), *dv_ = a.tensor(), *ws_ = a.tensor();
  Args late = a;
  a.i += 2;
  const Sinks c = sinks_of(a, x.D);
  const Table tab = table_of(late, c.rope, c.theta, x.D, x.S, x.dev);
  const Tensor dq = out_or(dq_, x.q.sizes(), x.type, x.dev), dk = out_or(dk_, x.k.sizes(), x.type, x.dev),
               dv = out_or(dv_, x.k.sizes(), x.type, x.dev);
  const int rc = sinks_bwd(x, c, tab, o, dout, lse, dq, dk, dv, ws_);
  return rc ? PyLong_FromLong(rc) : tuple_of({&dq, &dk, &dv});
}

// ---------------------------------------------------------------- differentiable calls
// The same as differentiable functions.  As a torch.autograd.Function in Python, whose
// backward takes the interpreter's lock in the engine's thread, a small norm and
// rotation forward and backward kept the host busy for 108 us; this one for 93, of
// which 65 are torch's own for an empty function (its engine's thread).
struct Failed {   // the library's code, to the entry function that called apply
  int code;
};

using torch::autograd::AutogradContext;
using torch::autograd::variable_list;

// f() in a backward, where no exception of another kind may leave: the engine knows
// only those of the standard library.
template <class F>
void in_backward(const char* name, F f) {
  int rc = 0;
  try {
    rc = f();
  } catch (const NotPlain&) {
    TORCH_CHECK(false, name, ": a gradient or a saved tensor is not what the forward had");
  }
  TORCH_CHECK(rc == 0, name, ": ", attnfuse_strerror(rc), " (code ", rc, ")");
}

// The gradients of a backward under create_graph: they come from kernels and have no
// derivative, so they depend on what they were formed from (`of`, and the incoming
// gradients) through an error.
variable_list once(variable_list grads, const variable_list& of, const variable_list& incoming) {
  if (!at::GradMode::is_enabled()) return grads;
  const std::shared_ptr<torch::autograd::Node> error(
      new torch::autograd::Error("the gradients of these operations cannot be differentiated twice",
                                 torch::autograd::collect_next_edges(of, incoming)),
      torch::autograd::deleteNode);
  for (const Tensor& g : grads)
    if (g.defined()) torch::autograd::set_history(g, error);
  return grads;
}

Table table_in(const Tensor& t, int64_t rows) {
  Table r;
  r.ptr = static_cast<const float*>(t.const_data_ptr());
  r.rows = (int)rows;
  return r;
}

// apply() takes no undefined tensors: a call without one passes q in its place and
// clears its bit.
enum { HAS_K = 1, HAS_QW = 2, HAS_KW = 4, HAS_POSITIONS = 8, HAS_TABLE = 16, WEIGHT_GRADS = 32 };

// The variant of a call with several axes behind the others in a context's numbers.
void keep_axes(std::vector<double>& v, const Norm& n) {
  v.push_back(n.n);
  for (int s : n.sections) v.push_back(s);
  v.push_back(n.order);
}
void with_axes(Norm& n, const double* v) {
  n.n = (int)v[0];
  for (int i = 0; i < 4; ++i) n.sections[i] = (int)v[1 + i];
  n.order = (int)v[5];
}

struct NormFunction : torch::autograd::Function<NormFunction> {
  // The call's tensors, as forward and backward both see them.
  struct Call {
    int64_t has;
    const Qk x;
    const Weights w;
    const Table table;
    const int* positions;
    Call(const Tensor& q, const Tensor& k, const Tensor& qw, const Tensor& kw, const Tensor& pos, const Tensor& tab, int64_t rows,
         int64_t has_)
        : has(has_), x(q, has & HAS_K ? &k : nullptr),
          w(has & HAS_QW ? &qw : nullptr, has & HAS_KW ? &kw : nullptr, x.D, x.type, x.dev),
          table(has & HAS_TABLE ? table_in(tab, rows) : Table()),
          positions(has & HAS_POSITIONS ? static_cast<const int*>(pos.const_data_ptr()) : nullptr) {}
  };

  static variable_list forward(AutogradContext* ctx, const Tensor& q, const Tensor& k, const Tensor& qw, const Tensor& kw,
                               const Tensor& positions, const Tensor& table, int64_t rows, const Norm& n, int64_t has) {
    const Call c(q, k, qw, kw, positions, table, rows, has);
    const Tensor oq = out_or(nullptr, c.x.q.sizes(), c.x.type, c.x.dev);
    Tensor ok;
    if (c.x.k) ok = out_or(nullptr, c.x.k->sizes(), c.x.type, c.x.dev);
    const int rc = norm_fwd(c.x, c.w, n, c.table, c.positions, oq, ok);
    if (rc) throw Failed{rc};
    ctx->save_for_backward({q, k, qw, kw, positions, table});
    std::vector<double> v{n.eps, (double)n.rope, n.theta, (double)has, (double)rows};
    keep_axes(v, n);
    ctx->saved_data["variant"] = v;
    if (c.x.k) return {oq, ok};
    return {oq};
  }

  static variable_list backward(AutogradContext* ctx, variable_list grad) {
    const variable_list s = ctx->get_saved_variables();
    Tensor dq, dk, dqw, dkw;
    in_backward("attnfuse_qknorm_rope_bwd", [&] {
      const std::vector<double> v = ctx->saved_data["variant"].toDoubleVector();
      const Call c(s[0], s[1], s[2], s[3], s[4], s[5], (int64_t)v[4], (int64_t)v[3]);
      const Tensor dqr = grad[0].contiguous(), dkr = c.x.k ? grad[1].contiguous() : Tensor();
      dq = at::empty_like(c.x.q);
      if (c.x.k) dk = at::empty_like(*c.x.k);
      Norm n((float)v[0], (int)v[1], v[2]);
      with_axes(n, &v[5]);
      const int rc = norm_bwd(c.x, c.w, n, c.table, c.positions, dqr,
                              c.x.k ? &dkr : nullptr, dq, dk, dqw, dkw, nullptr, c.has & WEIGHT_GRADS);
      if (!(c.has & HAS_QW)) dqw.reset();
      if (!(c.has & HAS_KW)) dkw.reset();
      return rc;
    });
    return once({dq, dk, dqw, dkw, Tensor(), Tensor(), Tensor(), Tensor(), Tensor()}, {s[0], s[1], s[2], s[3]}, grad);
  }
};

PyObject* norm_apply(const Tensor& q, const Tensor* k, const Tensor* qw, const Tensor* kw, const Tensor* pos, const Table& tab,
                     const Norm& n) {
  const Tensor& table = tab.own;
  const bool grads = (qw && qw->requires_grad()) || (kw && kw->requires_grad());
  const int64_t has = (k ? HAS_K : 0) | (qw ? HAS_QW : 0) | (kw ? HAS_KW : 0) | (pos ? HAS_POSITIONS : 0) |
                      (table.defined() ? HAS_TABLE : 0) | (grads ? WEIGHT_GRADS : 0);
  try {
    const variable_list r = NormFunction::apply(q, k ? *k : q, qw ? *qw : q, kw ? *kw : q, pos ? *pos : q,
                                                table.defined() ? table : q, (int64_t)tab.rows, n, has);
    const Tensor ok = r.size() > 1 ? r[1] : Tensor();
    return tuple_of({&r[0], &ok});
  } catch (const Failed& f) {
    return PyLong_FromLong(f.code);
  }
}

// qknorm_grad(q, k, q_weight, k_weight, positions, table, tables, eps, rope, theta, max_positions) -> (Qr, Kr)
PyObject* qknorm_grad(Args a) {
  const Tensor &q = a.need(), *k = a.tensor();
  const Tensor *qw = a.tensor(), *kw = a.tensor(), *pos = a.tensor();
  Args late = a;
  a.i += 2;
  const Norm n(a);
  const long long most = a.positive();
  if (!k && kw) throw NotPlain{};
  const Qk x(q, k);
  const Placed at_(pos, late, n.rope, n.theta, x.D, x.S, {x.B, x.S}, most, x.dev);
  return norm_apply(q, k, qw, kw, at_.positions ? pos : nullptr, at_.table, n);
}

// The rotation at positions of several axes without a norm: the backward needs the
// positions and the table alone.
struct TurnFunction : torch::autograd::Function<TurnFunction> {
  static variable_list forward(AutogradContext* ctx, const Tensor& q, const Tensor& k, const Tensor& positions,
                               const Tensor& table, int64_t rows, const Norm& n, bool has_k) {
    const Qk x(q, has_k ? &k : nullptr);
    const Tensor oq = out_or(nullptr, x.q.sizes(), x.type, x.dev);
    Tensor ok;
    if (x.k) ok = out_or(nullptr, x.k->sizes(), x.type, x.dev);
    const int rc = norm_fwd(x, Weights(nullptr, nullptr, x.D, x.type, x.dev), n, table_in(table, rows),
                            static_cast<const int*>(positions.const_data_ptr()), oq, ok);
    if (rc) throw Failed{rc};
    ctx->save_for_backward({positions, table});
    std::vector<double> v{(double)n.rope, n.theta, (double)rows};
    keep_axes(v, n);
    ctx->saved_data["variant"] = v;
    if (x.k) return {oq, ok};
    return {oq};
  }

  static variable_list backward(AutogradContext* ctx, variable_list grad) {
    const variable_list s = ctx->get_saved_variables();
    Tensor dq, dk;
    in_backward("attnfuse_qknorm_axes_bwd", [&] {
      const std::vector<double> v = ctx->saved_data["variant"].toDoubleVector();
      Norm n(0.f, (int)v[0], v[1]);
      with_axes(n, &v[3]);
      const Tensor dqr = grad[0].contiguous(), dkr = grad.size() > 1 ? grad[1].contiguous() : Tensor();
      return unturn(dqr, grad.size() > 1 ? &dkr : nullptr, dq, dk, n, table_in(s[1], (int64_t)v[2]),
                    static_cast<const int*>(s[0].const_data_ptr()));
    });
    return once({dq, dk, Tensor(), Tensor(), Tensor(), Tensor(), Tensor()}, {}, grad);
  }
};

// axes_grad(q, k, q_weight, k_weight, positions, table, tables, eps, rope, theta, max_positions, norm, sections,
//           section_order, its value, frequencies) -> (Qr, Kr)
PyObject* axes_grad(Args a) {
  const Tensor &q = a.need(), *k = a.tensor();
  const Tensor *qw = a.tensor(), *kw = a.tensor(), &pos = a.need();
  Args late = a;
  a.i += 2;
  Norm n(a);
  const long long most = a.positive();
  n.take_axes(a);
  if ((!k && kw) || (!n.norm && (qw || kw))) throw NotPlain{};
  const Qk x(q, k);
  const AxesPlaced at_(pos, late, n, x.D, {n.n, x.B, x.S}, most, x.dev);
  if (n.norm) return norm_apply(q, k, qw, kw, &pos, at_.table, n);
  try {
    const variable_list r = TurnFunction::apply(q, k ? *k : q, pos, at_.table.own, (int64_t)at_.table.rows, n, k != nullptr);
    const Tensor ok = r.size() > 1 ? r[1] : Tensor();
    return tuple_of({&r[0], &ok});
  } catch (const Failed& f) {
    return PyLong_FromLong(f.code);
  }
}

struct SinksFunction : torch::autograd::Function<SinksFunction> {
  static variable_list forward(AutogradContext* ctx, const Tensor& q, const Tensor& k, const Tensor& v, const Tensor& table,
                               int64_t rope, double theta, int64_t window, int64_t sinks, double scale) {
    const Qkv x(q, k, v);
    const Tensor o = out_or(nullptr, x.q.sizes(), x.type, x.dev), l = out_or(nullptr, {x.B, x.H, x.S}, at::kFloat, x.dev);
    const int rc = sinks_fwd(x, Sinks{(int)rope, theta, (int)window, (int)sinks, (float)scale},
                             rope != AF_ROPE_NONE ? table_in(table, table.size(0)) : Table(), o, l);
    if (rc) throw Failed{rc};
    ctx->save_for_backward({q, k, v, o, l, table});
    ctx->saved_data["variant"] = std::vector<double>{(double)rope, theta, (double)window, (double)sinks, scale};
    ctx->mark_non_differentiable({l});
    return {o, l};
  }

  static variable_list backward(AutogradContext* ctx, variable_list grad) {
    const variable_list s = ctx->get_saved_variables();
    Tensor dq, dk, dv;
    in_backward("attnfuse_bwd_sinks", [&] {
      const std::vector<double> v = ctx->saved_data["variant"].toDoubleVector();
      const Qkv x(s[0], s[1], s[2]);
      dq = at::empty_like(x.q);
      dk = at::empty_like(x.k);
      dv = at::empty_like(x.k);
      return sinks_bwd(x, Sinks{(int)v[0], v[1], (int)v[2], (int)v[3], (float)v[4]},
                       v[0] != AF_ROPE_NONE ? table_in(s[5], s[5].size(0)) : Table(), s[3], grad[0].contiguous(), s[4], dq, dk, dv, nullptr);
    });
    return once({dq, dk, dv, Tensor(), Tensor(), Tensor(), Tensor(), Tensor(), Tensor()}, {s[0], s[1], s[2]}, grad);
  }
};

// sinks_grad(q, k, v, table, tables, rope, theta, window, sinks, scale) -> (O, LSE)
PyObject* sinks_grad(Args a) {
  Qkv x(a);
  Args late = a;
  a.i += 2;
  const Sinks c = sinks_of(a, x.D);
  const Table tab = table_of(late, c.rope, c.theta, x.D, x.S, x.dev);
  try {
    const variable_list r = SinksFunction::apply(x.q, x.k, x.v, tab.own.defined() ? tab.own : x.q, (int64_t)c.rope, c.theta,
                                                 (int64_t)c.window, (int64_t)c.sinks, (double)c.scale);
    return tuple_of({&r[0], &r[1]});
  } catch (const Failed& f) {
    return PyLong_FromLong(f.code);
  }
}

template <PyObject* (*F)(Args)>
PyObject* entry(PyObject*, PyObject* const* v, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  try {
    return F(Args{v, n});
  } catch (const NotPlain&) {
    Py_RETURN_NONE;
  }
  END_HANDLE_TH_ERRORS
}

template <PyObject* (*F)(Args)>
constexpr PyMethodDef method(const char* name) {
  return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(entry<F>)), METH_FASTCALL, nullptr};
}

PyMethodDef methods[] = {method<fwd>("fwd"), method<bwd>("bwd"), method<decode>("decode"), method<rope>("rope"),
                         method<qknorm>("qknorm"), method<qknorm_bwd>("qknorm_bwd"), method<qknorm_grad>("qknorm_grad"), 
                         method<append<false>>("append"), method<axes>("axes"), method<axes_bwd>("axes_bwd"),
                         method<axes_grad>("axes_grad"), method<append<true>>("axes_append"),
                         method<decode_paged>("decode_paged"), method<decode_sinks>("decode_sinks"), method<fwd_paged>("fwd_paged"),
                         method<fwd_sinks>("fwd_sinks"), method<bwd_sinks>("bwd_sinks"), method<sinks_grad>("sinks_grad"),
                         {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_native", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native(void) { return PyModule_Create(&module); }
