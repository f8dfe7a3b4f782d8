// Python boundary of the sequence operators: torch tensors in, one C-ABI call out.  As in per_binding.cpp, a tensor taken apart
// here costs nanoseconds; an actor's step is a few microseconds of kernel, and results are allocated here too.
#include <Python.h>

#include <ATen/Functions.h>
#include <c10/core/DeviceGuard.h>
#include <c10/core/GradMode.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <cmath>
#include <initializer_list>
#include <stdexcept>
#include <string>

#include "../../include/per_seq.h"

namespace {

struct Raised {};   // a Python exception is set

[[noreturn]] void raise_value(const std::string& what) {
  PyErr_SetString(PyExc_ValueError, what.c_str());
  throw Raised{};
}

const at::Tensor* maybe(PyObject* o, const char* name) {
  if (o == Py_None) return nullptr;
  if (!THPVariable_Check(o)) {
    PyErr_Format(PyExc_TypeError, "%s: expected a tensor, got %.100s", name, Py_TYPE(o)->tp_name);
    throw Raised{};
  }
  return &THPVariable_Unpack(o);
}
const at::Tensor& tensor(PyObject* o, const char* name) {
  const at::Tensor* t = maybe(o, name);
  if (!t) {
    PyErr_Format(PyExc_TypeError, "%s: expected a tensor, got None", name);
    throw Raised{};
  }
  return *t;
}
double real(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw Raised{};
  return v;
}
bool truth(PyObject* o) {
  const int v = PyObject_IsTrue(o);
  if (v < 0) throw Raised{};
  return v != 0;
}

struct Need {   // what the tensors of a call have in common
  c10::Device device;
  at::ScalarType type;
};

std::string shape_of(const at::Tensor& t) {
  std::string s = "[";
  for (int64_t i = 0; i < t.dim(); ++i) s += (i ? ", " : "") + std::to_string(t.size(i));
  return s + "]";
}
void check(const at::Tensor& t, const char* name, const Need& n, at::ScalarType type, std::initializer_list<int64_t> shape) {
  if (t.device() != n.device) raise_value(std::string(name) + ": expected a tensor on " + n.device.str() + ", got one on " + t.device().str());
  if (t.scalar_type() != type) raise_value(std::string(name) + ": expected type " + c10::toString(type) + ", got " + c10::toString(t.scalar_type()));
  bool fits = t.dim() == (int64_t)shape.size();
  int64_t i = 0;
  for (int64_t d : shape) fits = fits && t.size(i++) == d;
  if (!fits) {
    std::string want = "[";
    for (int64_t d : shape) want += (want.size() > 1 ? ", " : "") + std::to_string(d);
    raise_value(std::string(name) + ": expected shape " + want + "], got " + shape_of(t));
  }
}

Need need_of(const at::Tensor& t, const char* name) {
  if (!t.is_cuda()) raise_value(std::string(name) + ": expected a device tensor");
  if (t.scalar_type() != at::kBFloat16 && t.scalar_type() != at::kFloat)
    raise_value(std::string(name) + ": expected bfloat16 or float32, got " + c10::toString(t.scalar_type()));
  return Need{t.device(), t.scalar_type()};
}
uint32_t dtype_of(const Need& n) { return n.type == at::kBFloat16 ? PER_SEQ_BF16 : PER_SEQ_F32; }

uint32_t count(int64_t n, const char* name) {
  if (n < 0 || n > 0xFFFFFFFFll) raise_value(std::string(name) + ": too large");
  return (uint32_t)n;
}

// A dimension of size 1 has no stride that counts.
int64_t step_of(const at::Tensor& t, int64_t d) { return t.size(d) == 1 ? 0 : t.stride(d); }

per_seq_rows rows(const at::Tensor& t, const char* name) {
  if (t.numel() && t.size(3) > 1 && t.stride(3) != 1) raise_value(std::string(name) + ": the last dimension must be contiguous");
  return per_seq_rows{t.data_ptr(), step_of(t, 0), step_of(t, 1), step_of(t, 2)};
}
per_seq_states states(const at::Tensor& t, const char* name) {
  if (t.numel() && ((t.size(3) > 1 && t.stride(3) != 1) || (t.size(2) > 1 && t.stride(2) != t.size(3))))
    raise_value(std::string(name) + ": the last two dimensions must be contiguous");
  return per_seq_states{static_cast<float*>(t.data_ptr()), step_of(t, 0), step_of(t, 1)};
}
template <typename V>
V* vector(const at::Tensor* t, const char* name, const Need& n, at::ScalarType type, int64_t size) {
  if (!t) return nullptr;
  check(*t, name, n, type, {size});
  if (size > 1 && t->stride(0) != 1) raise_value(std::string(name) + ": expected a contiguous tensor");
  return static_cast<V*>(t->data_ptr());
}

at::Tensor make(const Need& n, at::ScalarType type, at::IntArrayRef shape) {
  return at::empty(shape, at::TensorOptions().dtype(type).device(n.device));
}

void* stream_of(const Need& n) { return c10::hip::getCurrentHIPStream(n.device.index()).stream(); }

template <typename F>
int unlocked(F call) {
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = call();
  Py_END_ALLOW_THREADS
  return rc;
}

// (code, result, ...): the code of the C-ABI call and the tensors it filled (None where there is none).
PyObject* answer(int rc, std::initializer_list<const at::Tensor*> results) {
  PyObject* tuple = PyTuple_New(1 + (Py_ssize_t)results.size());
  if (!tuple) throw Raised{};
  PyTuple_SET_ITEM(tuple, 0, PyLong_FromLong(rc));
  Py_ssize_t i = 1;
  for (const at::Tensor* t : results) {
    PyObject* o = t && t->defined() ? THPVariable_Wrap(*t) : Py_NewRef(Py_None);
    PyTuple_SET_ITEM(tuple, i++, o);
  }
  return tuple;
}

using Args = PyObject* const*;

bool asks(std::initializer_list<PyObject*> tensors) {
  for (PyObject* o : tensors)
    if (THPVariable_Check(o) && THPVariable_Unpack(o).requires_grad()) return true;
  return false;
}
// Whether a gradient of the inputs is asked for: the call has to be made as a node of torch's graph then (its caller is told by None),
// and results that are given, which may hold what another node has kept, have no place in it.
bool differentiated(std::initializer_list<PyObject*> inputs, std::initializer_list<PyObject*> given) {
  if (!c10::GradMode::is_enabled()) return false;
  bool any = false;
  for (PyObject* o : given) any = any || o != Py_None;
  if (!asks(inputs) && !(any && asks(given))) return false;
  if (!any) return true;
  PyErr_SetString(PyExc_RuntimeError, "no gradient is formed where results are written over given tensors: call it under no_grad, or without them");
  throw Raised{};
}

void expect(Py_ssize_t n, Py_ssize_t want) {
  if (n == want) return;
  PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", want, n);
  throw Raised{};
}

// The tensor given for a result, or a new one.
at::Tensor result(PyObject* given, const char* name, const Need& n, at::ScalarType type, std::initializer_list<int64_t> shape) {
  const at::Tensor* t = maybe(given, name);
  if (!t) return make(n, type, at::IntArrayRef(shape.begin(), shape.size()));
  check(*t, name, n, type, shape);
  return *t;
}

// The caller's tensors (or None) that a call has written: if torch has kept one of them for a gradient, it finds out by its version.
void written(int rc, std::initializer_list<PyObject*> given) {
  if (rc) return;
  for (PyObject* o : given) {
    if (!THPVariable_Check(o)) continue;
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
  }
}

struct Attention {
  per_attention_config c{};
  Need n;
  int64_t B, L, H, G, dk, dv;
  per_seq_rows q, k, v;
  const float* decay;
  const int32_t* lengths;
  // (q, k, v, log_decay, lengths, scale); scale None: 1 / sqrt(dk)
  Attention(PyObject* oq, PyObject* ok, PyObject* ov, PyObject* odecay, PyObject* olengths, PyObject* oscale, const char* lengths_name = "lengths")
      : n(need_of(tensor(oq, "q"), "q")) {
    const at::Tensor &tq = tensor(oq, "q"), &tk = tensor(ok, "k"), &tv = tensor(ov, "v");
    if (tq.dim() != 4 || tk.dim() != 4 || tv.dim() != 4) raise_value("q, k and v must be [batch, length, heads, width]");
    B = tq.size(0);
    L = tq.size(1);
    H = tq.size(2);
    G = tk.size(2);
    dk = tq.size(3);
    dv = tv.size(3);
    check(tk, "k", n, n.type, {B, L, G, dk});
    check(tv, "v", n, n.type, {B, L, G, dv});
    if (H && (!G || H % G)) raise_value("the heads of k and v must divide those of q");
    c.struct_size = sizeof(c);
    c.dtype = dtype_of(n);
    c.batch = count(B, "batch");
    c.length = count(L, "length");
    c.heads = count(H, "heads");
    c.kv_heads = count(G, "heads");
    c.dk = count(dk, "dk");
    c.dv = count(dv, "dv");
    c.scale = oscale == Py_None ? 1.0f / sqrtf((float)(dk ? dk : 1)) : (float)real(oscale);
    q = rows(tq, "q");
    k = rows(tk, "k");
    v = rows(tv, "v");
    decay = vector<float>(&tensor(odecay, "log_decay"), "log_decay", n, at::kFloat, H);
    lengths = vector<int32_t>(maybe(olengths, lengths_name), lengths_name, n, at::kInt, B);
  }
  per_seq_rows rows_of(const at::Tensor& t, const char* name, int64_t heads, int64_t width) const {
    check(t, name, n, n.type, {B, L, heads, width});
    return rows(t, name);
  }
  per_seq_states states_of(const at::Tensor& t, const char* name) const {
    check(t, name, n, at::kFloat, {B, H, dk, dv});
    return states(t, name);
  }
  at::Tensor work(int backward, size_t* bytes, int* rc) const {
    *bytes = 0;
    *rc = per_linear_attention_workspace(&c, backward, bytes);
    return *rc == 0 && *bytes ? make(n, at::kByte, {(int64_t)*bytes}) : at::Tensor();
  }
};

void* data(const at::Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; }

// (q, k, v, log_decay, state, lengths, scale, out, out_state, want_state) -> (code, out, out_state), or None
PyObject* do_attention(Args a, Py_ssize_t n_args) {
  expect(n_args, 10);
  if (differentiated({a[0], a[1], a[2], a[3], a[4]}, {a[7], a[8]})) Py_RETURN_NONE;
  const Attention p(a[0], a[1], a[2], a[3], a[5], a[6]);
  const c10::DeviceGuard guard(p.n.device);
  const at::Tensor* in = maybe(a[4], "state");
  per_seq_states si{}, so{};
  if (in) si = p.states_of(*in, "state");
  at::Tensor out = result(a[7], "out", p.n, p.n.type, {p.B, p.L, p.H, p.dv}), last;
  const per_seq_rows ro = p.rows_of(out, "out", p.H, p.dv);
  if (truth(a[9])) {
    last = result(a[8], "out_state", p.n, at::kFloat, {p.B, p.H, p.dk, p.dv});
    so = p.states_of(last, "out_state");
  }
  size_t bytes;
  int rc;
  const at::Tensor work = p.work(0, &bytes, &rc);
  void* s = stream_of(p.n);
  if (rc == 0)
    rc = unlocked([&] {
      return per_linear_attention(&p.c, &p.q, &p.k, &p.v, p.decay, p.lengths, in ? &si : nullptr, &ro, last.defined() ? &so : nullptr, data(work), bytes, s);
    });
  written(rc, {a[7], last.defined() ? a[8] : Py_None});
  return answer(rc, {&out, &last});
}

// (dout, q, k, v, log_decay, state, dstate, lengths, scale, dq, dk, dv, dstate0, want_dstate) -> (code, dq, dk, dv, dstate0)
PyObject* do_attention_backward(Args a, Py_ssize_t n_args) {
  expect(n_args, 14);
  const Attention p(a[1], a[2], a[3], a[4], a[7], a[8]);
  const c10::DeviceGuard guard(p.n.device);
  const per_seq_rows dout = p.rows_of(tensor(a[0], "dout"), "dout", p.H, p.dv);
  const at::Tensor *in = maybe(a[5], "state"), *din = maybe(a[6], "dstate");
  per_seq_states si{}, sd{}, so{};
  if (in) si = p.states_of(*in, "state");
  if (din) sd = p.states_of(*din, "dstate");
  at::Tensor dq = result(a[9], "dq", p.n, p.n.type, {p.B, p.L, p.H, p.dk}), dk = result(a[10], "dk", p.n, p.n.type, {p.B, p.L, p.G, p.dk}),
             dv = result(a[11], "dv", p.n, p.n.type, {p.B, p.L, p.G, p.dv}), first;
  const per_seq_rows rq = p.rows_of(dq, "dq", p.H, p.dk), rk = p.rows_of(dk, "dk", p.G, p.dk), rv = p.rows_of(dv, "dv", p.G, p.dv);
  if (truth(a[13])) {
    first = result(a[12], "dstate0", p.n, at::kFloat, {p.B, p.H, p.dk, p.dv});
    so = p.states_of(first, "dstate0");
  }
  size_t bytes;
  int rc;
  const at::Tensor work = p.work(1, &bytes, &rc);
  void* s = stream_of(p.n);
  if (rc == 0)
    rc = unlocked([&] {
      return per_linear_attention_backward(&p.c, &dout, &p.q, &p.k, &p.v, p.decay, p.lengths, in ? &si : nullptr, din ? &sd : nullptr, &rq, &rk, &rv,
                                           first.defined() ? &so : nullptr, data(work), bytes, s);
    });
  written(rc, {a[9], a[10], a[11], first.defined() ? a[12] : Py_None});
  return answer(rc, {&dq, &dk, &dv, &first});
}

// (q, k, v, log_decay, state, active, scale, out) -> (code, out)
PyObject* do_attention_step(Args a, Py_ssize_t n_args) {
  expect(n_args, 8);
  differentiated({a[0], a[1], a[2], a[3]}, {a[4], a[7]});   // (the state is a given result)
  const Attention p(a[0], a[1], a[2], a[3], a[5], a[6], "active");
  const c10::DeviceGuard guard(p.n.device);
  const per_seq_states st = p.states_of(tensor(a[4], "state"), "state");
  at::Tensor out = result(a[7], "out", p.n, p.n.type, {p.B, p.L, p.H, p.dv});
  const per_seq_rows ro = p.rows_of(out, "out", p.H, p.dv);
  void* s = stream_of(p.n);
  const int rc = unlocked([&] { return per_linear_attention_step(&p.c, &p.q, &p.k, &p.v, p.decay, p.lengths, &st, &ro, s); });
  written(rc, {a[4], a[7]});
  return answer(rc, {&out});
}

struct Rotary {
  per_rotary_config c{};
  Need n;
  int64_t B, L, D;
  per_seq_positions at{};
  const float* freqs;
  // (x, positions, freqs, layout, magnitude): layout 0 or 1
  Rotary(PyObject* ox, PyObject* opos, PyObject* ofreqs, PyObject* olayout, PyObject* omagnitude, const char* name) : n(need_of(tensor(ox, name), name)) {
    const at::Tensor& x = tensor(ox, name);
    if (x.dim() != 4) raise_value(std::string(name) + ": expected [batch, length, heads, width], got " + shape_of(x));
    B = x.size(0);
    L = x.size(1);
    D = x.size(3);
    const at::Tensor& f = tensor(ofreqs, "freqs");
    freqs = vector<float>(&f, "freqs", n, at::kFloat, f.dim() == 1 ? f.size(0) : -1);
    if (const at::Tensor* pos = maybe(opos, "positions")) {
      check(*pos, "positions", n, at::kInt, {B, L});
      at = per_seq_positions{static_cast<const int32_t*>(pos->data_ptr()), step_of(*pos, 0), step_of(*pos, 1)};
    }
    c.struct_size = sizeof(c);
    c.dtype = dtype_of(n);
    c.batch = count(B, "batch");
    c.length = count(L, "length");
    c.heads = count(x.size(2), "heads");
    c.dim = count(D, "width");
    c.rot = count(2 * f.size(0), "freqs");
    if (c.rot > c.dim) raise_value("freqs: there are more pairs than a head holds");
    c.layout = truth(olayout) ? PER_SEQ_INTERLEAVED : PER_SEQ_HALF;
    c.magnitude = (float)real(omagnitude);
  }
};

// (x, positions, freqs, layout, magnitude, inverse, out) -> (code, out), or None
PyObject* do_rotate(Args a, Py_ssize_t n_args) {
  expect(n_args, 7);
  if (differentiated({a[0], a[2]}, {a[6]})) Py_RETURN_NONE;
  Rotary p(a[0], a[1], a[2], a[3], a[4], "x");
  const c10::DeviceGuard guard(p.n.device);
  p.c.inverse = truth(a[5]);
  const at::Tensor& x = tensor(a[0], "x");
  at::Tensor out = result(a[6], "out", p.n, p.n.type, {p.B, p.L, x.size(2), p.D});
  const per_seq_rows rx = rows(x, "x"), ro = rows(out, "out");
  void* s = stream_of(p.n);
  const int rc = unlocked([&] { return per_rotate(&p.c, &rx, &p.at, p.freqs, &ro, s); });
  written(rc, {a[6]});
  return answer(rc, {&out});
}

// (q, k, q_weight, k_weight, positions, freqs, layout, magnitude, eps, q_out, k_out) -> (code, q_out, k_out), or None
PyObject* do_norm_rotate(Args a, Py_ssize_t n_args) {
  expect(n_args, 11);
  if (differentiated({a[0], a[1], a[2], a[3], a[5]}, {a[9], a[10]})) Py_RETURN_NONE;
  Rotary p(a[0], a[4], a[5], a[6], a[7], "q");
  const c10::DeviceGuard guard(p.n.device);
  const at::Tensor &q = tensor(a[0], "q"), &k = tensor(a[1], "k");
  if (k.dim() != 4) raise_value("k: expected [batch, length, heads, width], got " + shape_of(k));
  check(k, "k", p.n, p.n.type, {p.B, p.L, k.size(2), p.D});
  p.c.kv_heads = count(k.size(2), "heads");
  p.c.eps = (float)real(a[8]);
  const float *qw = vector<float>(maybe(a[2], "q_weight"), "q_weight", p.n, at::kFloat, p.D), *kw = vector<float>(maybe(a[3], "k_weight"), "k_weight", p.n, at::kFloat, p.D);
  at::Tensor qo = result(a[9], "q_out", p.n, p.n.type, {p.B, p.L, q.size(2), p.D}), ko = result(a[10], "k_out", p.n, p.n.type, {p.B, p.L, k.size(2), p.D});
  const per_seq_rows rq = rows(q, "q"), rk = rows(k, "k"), oq = rows(qo, "q_out"), ok = rows(ko, "k_out");
  void* s = stream_of(p.n);
  const int rc = unlocked([&] { return per_norm_rotate(&p.c, &rq, &rk, qw, kw, &p.at, p.freqs, &oq, &ok, s); });
  written(rc, {a[9], a[10]});
  return answer(rc, {&qo, &ko});
}

// (dq_out, dk_out, q, k, q_weight, k_weight, positions, freqs, layout, magnitude, eps, dq, dk, want_weights)
//   -> (code, dq, dk, dq_weight, dk_weight)
PyObject* do_norm_rotate_backward(Args a, Py_ssize_t n_args) {
  expect(n_args, 14);
  Rotary p(a[2], a[6], a[7], a[8], a[9], "q");
  const c10::DeviceGuard guard(p.n.device);
  const at::Tensor &q = tensor(a[2], "q"), &k = tensor(a[3], "k"), &gq = tensor(a[0], "dq_out"), &gk = tensor(a[1], "dk_out");
  if (k.dim() != 4) raise_value("k: expected [batch, length, heads, width], got " + shape_of(k));
  check(k, "k", p.n, p.n.type, {p.B, p.L, k.size(2), p.D});
  check(gq, "dq_out", p.n, p.n.type, {p.B, p.L, q.size(2), p.D});
  check(gk, "dk_out", p.n, p.n.type, {p.B, p.L, k.size(2), p.D});
  p.c.kv_heads = count(k.size(2), "heads");
  p.c.eps = (float)real(a[10]);
  const float *qw = vector<float>(maybe(a[4], "q_weight"), "q_weight", p.n, at::kFloat, p.D), *kw = vector<float>(maybe(a[5], "k_weight"), "k_weight", p.n, at::kFloat, p.D);
  at::Tensor dq = result(a[11], "dq", p.n, p.n.type, {p.B, p.L, q.size(2), p.D}), dk = result(a[12], "dk", p.n, p.n.type, {p.B, p.L, k.size(2), p.D}), wq, wk;
  if (truth(a[13])) {
    wq = make(p.n, at::kFloat, {p.D});
    wk = make(p.n, at::kFloat, {p.D});
  }
  size_t bytes = 0;
  int rc = per_norm_rotate_workspace(&p.c, &bytes);
  const at::Tensor work = rc == 0 && bytes ? make(p.n, at::kByte, {(int64_t)bytes}) : at::Tensor();
  const per_seq_rows rgq = rows(gq, "dq_out"), rgk = rows(gk, "dk_out"), rq = rows(q, "q"), rk = rows(k, "k"), oq = rows(dq, "dq"), ok = rows(dk, "dk");
  void* s = stream_of(p.n);
  if (rc == 0)
    rc = unlocked([&] {
      return per_norm_rotate_backward(&p.c, &rgq, &rgk, &rq, &rk, qw, kw, &p.at, p.freqs, &oq, &ok, static_cast<float*>(data(wq)),
                                      static_cast<float*>(data(wk)), data(work), bytes, s);
    });
  written(rc, {a[11], a[12]});
  return answer(rc, {&dq, &dk, &wq, &wk});
}

struct Delta {
  per_delta_config c{};
  Need n;
  int64_t B, L, H, Q, K, V, dk, dv;
  per_seq_rows q, k, v;
  per_seq_gates decay, beta;
  const int32_t* lengths;
  // (q, k, v, log_decay, beta, lengths, scale); scale None: 1 / sqrt(dk)
  Delta(PyObject* oq, PyObject* ok, PyObject* ov, PyObject* odecay, PyObject* obeta, PyObject* olengths, PyObject* oscale, const char* lengths_name = "lengths")
      : n(need_of(tensor(oq, "q"), "q")) {
    const at::Tensor &tq = tensor(oq, "q"), &tk = tensor(ok, "k"), &tv = tensor(ov, "v"), &tg = tensor(odecay, "log_decay"), &tb = tensor(obeta, "beta");
    if (tq.dim() != 4 || tk.dim() != 4 || tv.dim() != 4) raise_value("q, k and v must be [batch, length, heads, width]");
    if (tg.dim() != 3) raise_value("log_decay: expected [batch, length, heads], got " + shape_of(tg));
    B = tq.size(0);
    L = tq.size(1);
    H = tg.size(2);
    Q = tq.size(2);
    K = tk.size(2);
    V = tv.size(2);
    dk = tq.size(3);
    dv = tv.size(3);
    check(tk, "k", n, n.type, {B, L, K, dk});
    check(tv, "v", n, n.type, {B, L, V, dv});
    decay = gates_of(tg, "log_decay");
    beta = gates_of(tb, "beta");
    for (int64_t heads : {Q, K, V})
      if (H ? !heads || H % heads : heads != 0) raise_value("the heads of q, k and v must divide those of log_decay");
    c.struct_size = sizeof(c);
    c.dtype = dtype_of(n);
    c.batch = count(B, "batch");
    c.length = count(L, "length");
    c.heads = count(H, "heads");
    c.q_heads = count(Q, "heads");
    c.k_heads = count(K, "heads");
    c.v_heads = count(V, "heads");
    c.dk = count(dk, "dk");
    c.dv = count(dv, "dv");
    c.scale = oscale == Py_None ? 1.0f / sqrtf((float)(dk ? dk : 1)) : (float)real(oscale);
    q = rows(tq, "q");
    k = rows(tk, "k");
    v = rows(tv, "v");
    lengths = vector<int32_t>(maybe(olengths, lengths_name), lengths_name, n, at::kInt, B);
  }
  per_seq_gates gates_of(const at::Tensor& t, const char* name) const {
    check(t, name, n, at::kFloat, {B, L, H});
    return per_seq_gates{static_cast<float*>(t.data_ptr()), step_of(t, 0), step_of(t, 1), step_of(t, 2)};
  }
  per_seq_rows rows_of(const at::Tensor& t, const char* name, int64_t heads, int64_t width) const {
    check(t, name, n, n.type, {B, L, heads, width});
    return rows(t, name);
  }
  per_seq_states states_of(const at::Tensor& t, const char* name) const {
    check(t, name, n, at::kFloat, {B, H, dk, dv});
    return states(t, name);
  }
  at::Tensor work(int backward, size_t* bytes, int* rc) const {
    *bytes = 0;
    *rc = per_gated_delta_workspace(&c, backward, bytes);
    return *rc == 0 && *bytes ? make(n, at::kByte, {(int64_t)*bytes}) : at::Tensor();
  }
};

// (q, k, v, log_decay, beta, state, lengths, scale, out, out_state, want_state) -> (code, out, out_state), or None
PyObject* do_delta(Args a, Py_ssize_t n_args) {
  expect(n_args, 11);
  if (differentiated({a[0], a[1], a[2], a[3], a[4], a[5]}, {a[8], a[9]})) Py_RETURN_NONE;
  const Delta p(a[0], a[1], a[2], a[3], a[4], a[6], a[7]);
  const c10::DeviceGuard guard(p.n.device);
  const at::Tensor* in = maybe(a[5], "state");
  per_seq_states si{}, so{};
  if (in) si = p.states_of(*in, "state");
  at::Tensor out = result(a[8], "out", p.n, p.n.type, {p.B, p.L, p.H, p.dv}), last;
  const per_seq_rows ro = p.rows_of(out, "out", p.H, p.dv);
  if (truth(a[10])) {
    last = result(a[9], "out_state", p.n, at::kFloat, {p.B, p.H, p.dk, p.dv});
    so = p.states_of(last, "out_state");
  }
  size_t bytes;
  int rc;
  const at::Tensor work = p.work(0, &bytes, &rc);
  void* s = stream_of(p.n);
  if (rc == 0)
    rc = unlocked([&] {
      return per_gated_delta(&p.c, &p.q, &p.k, &p.v, &p.decay, &p.beta, p.lengths, in ? &si : nullptr, &ro, last.defined() ? &so : nullptr, data(work), bytes, s);
    });
  written(rc, {a[8], last.defined() ? a[9] : Py_None});
  return answer(rc, {&out, &last});
}

// (dout, q, k, v, log_decay, beta, state, dstate, lengths, scale, dq, dk, dv, dlog_decay, dbeta, dstate0, want_dstate)
//   -> (code, dq, dk, dv, dlog_decay, dbeta, dstate0)
PyObject* do_delta_backward(Args a, Py_ssize_t n_args) {
  expect(n_args, 17);
  const Delta p(a[1], a[2], a[3], a[4], a[5], a[8], a[9]);
  const c10::DeviceGuard guard(p.n.device);
  const per_seq_rows dout = p.rows_of(tensor(a[0], "dout"), "dout", p.H, p.dv);
  const at::Tensor *in = maybe(a[6], "state"), *din = maybe(a[7], "dstate");
  per_seq_states si{}, sd{}, so{};
  if (in) si = p.states_of(*in, "state");
  if (din) sd = p.states_of(*din, "dstate");
  at::Tensor dq = result(a[10], "dq", p.n, p.n.type, {p.B, p.L, p.Q, p.dk}), dk = result(a[11], "dk", p.n, p.n.type, {p.B, p.L, p.K, p.dk}),
             dv = result(a[12], "dv", p.n, p.n.type, {p.B, p.L, p.V, p.dv}), dg = result(a[13], "dlog_decay", p.n, at::kFloat, {p.B, p.L, p.H}),
             db = result(a[14], "dbeta", p.n, at::kFloat, {p.B, p.L, p.H}), first;
  const per_seq_rows rq = p.rows_of(dq, "dq", p.Q, p.dk), rk = p.rows_of(dk, "dk", p.K, p.dk), rv = p.rows_of(dv, "dv", p.V, p.dv);
  const per_seq_gates gg = p.gates_of(dg, "dlog_decay"), gb = p.gates_of(db, "dbeta");
  if (truth(a[16])) {
    first = result(a[15], "dstate0", p.n, at::kFloat, {p.B, p.H, p.dk, p.dv});
    so = p.states_of(first, "dstate0");
  }
  size_t bytes;
  int rc;
  const at::Tensor work = p.work(1, &bytes, &rc);
  void* s = stream_of(p.n);
  if (rc == 0)
    rc = unlocked([&] {
      return per_gated_delta_backward(&p.c, &dout, &p.q, &p.k, &p.v, &p.decay, &p.beta, p.lengths, in ? &si : nullptr, din ? &sd : nullptr, &rq, &rk, &rv,
                                      &gg, &gb, first.defined() ? &so : nullptr, data(work), bytes, s);
    });
  written(rc, {a[10], a[11], a[12], a[13], a[14], first.defined() ? a[15] : Py_None});
  return answer(rc, {&dq, &dk, &dv, &dg, &db, &first});
}

// (q, k, v, log_decay, beta, state, active, scale, out) -> (code, out)
PyObject* do_delta_step(Args a, Py_ssize_t n_args) {
  expect(n_args, 9);
  differentiated({a[0], a[1], a[2], a[3], a[4]}, {a[5], a[8]});   // (the state is a given result)
  const Delta p(a[0], a[1], a[2], a[3], a[4], a[6], a[7], "active");
  const c10::DeviceGuard guard(p.n.device);
  const per_seq_states st = p.states_of(tensor(a[5], "state"), "state");
  at::Tensor out = result(a[8], "out", p.n, p.n.type, {p.B, p.L, p.H, p.dv});
  const per_seq_rows ro = p.rows_of(out, "out", p.H, p.dv);
  void* s = stream_of(p.n);
  const int rc = unlocked([&] { return per_gated_delta_step(&p.c, &p.q, &p.k, &p.v, &p.decay, &p.beta, p.lengths, &st, &ro, s); });
  written(rc, {a[5], a[8]});
  return answer(rc, {&out});
}

// Rows [..., dim] of up to four dimensions.
struct Block {
  per_block_config c{};
  Need n;
  at::IntArrayRef shape;
  Block(const at::Tensor& x) : n(need_of(x, "x")), shape(x.sizes()) {
    if (x.dim() < 1 || x.dim() > 4) raise_value("x: expected one to four dimensions, got " + shape_of(x));
    const int64_t d = x.dim();
    c.struct_size = sizeof(c);
    c.dtype = dtype_of(n);
    c.batch = d > 3 ? count(x.size(d - 4), "x") : 1;
    c.length = d > 2 ? count(x.size(d - 3), "x") : 1;
    c.heads = d > 1 ? count(x.size(d - 2), "x") : 1;
    c.dim = count(x.size(d - 1), "x");
  }
  per_seq_rows rows_of(const at::Tensor& t, const char* name) const {
    if (t.device() != n.device) raise_value(std::string(name) + ": expected a tensor on " + n.device.str() + ", got one on " + t.device().str());
    if (t.scalar_type() != n.type) raise_value(std::string(name) + ": expected type " + c10::toString(n.type) + ", got " + c10::toString(t.scalar_type()));
    if (t.sizes() != shape) raise_value(std::string(name) + ": its shape is " + shape_of(t) + ", not that of x");
    const int64_t d = t.dim();
    if (t.numel() && t.size(d - 1) > 1 && t.stride(d - 1) != 1) raise_value(std::string(name) + ": the last dimension must be contiguous");
    return per_seq_rows{t.data_ptr(), d > 3 ? step_of(t, d - 4) : 0, d > 2 ? step_of(t, d - 3) : 0, d > 1 ? step_of(t, d - 2) : 0};
  }
  at::Tensor result_of(PyObject* given, const char* name) const {
    const at::Tensor* t = maybe(given, name);
    return t ? *t : make(n, n.type, shape);
  }
};

// (x, weight, bias, eps, out) -> (code, out), or None
PyObject* do_layer_norm(Args a, Py_ssize_t n_args) {
  expect(n_args, 5);
  if (differentiated({a[0], a[1], a[2]}, {a[4]})) Py_RETURN_NONE;
  const at::Tensor& x = tensor(a[0], "x");
  Block p(x);
  const c10::DeviceGuard guard(p.n.device);
  p.c.eps = (float)real(a[3]);
  const float *w = vector<float>(maybe(a[1], "weight"), "weight", p.n, at::kFloat, p.c.dim), *b = vector<float>(maybe(a[2], "bias"), "bias", p.n, at::kFloat, p.c.dim);
  at::Tensor out = p.result_of(a[4], "out");
  const per_seq_rows rx = p.rows_of(x, "x"), ro = p.rows_of(out, "out");
  void* s = stream_of(p.n);
  const int rc = unlocked([&] { return per_layer_norm(&p.c, &rx, w, b, &ro, s); });
  written(rc, {a[4]});
  return answer(rc, {&out});
}

// (dout, x, weight, eps, dx, want_weights) -> (code, dx, dweight, dbias)
PyObject* do_layer_norm_backward(Args a, Py_ssize_t n_args) {
  expect(n_args, 6);
  const at::Tensor &dout = tensor(a[0], "dout"), &x = tensor(a[1], "x");
  Block p(x);
  const c10::DeviceGuard guard(p.n.device);
  p.c.eps = (float)real(a[3]);
  const float* w = vector<float>(maybe(a[2], "weight"), "weight", p.n, at::kFloat, p.c.dim);
  at::Tensor dx = p.result_of(a[4], "dx"), dw, db;
  const per_seq_rows rd = p.rows_of(dout, "dout"), rx = p.rows_of(x, "x"), ro = p.rows_of(dx, "dx");
  if (truth(a[5])) {
    dw = make(p.n, at::kFloat, {(int64_t)p.c.dim});
    db = make(p.n, at::kFloat, {(int64_t)p.c.dim});
  }
  size_t bytes = 0;
  int rc = per_layer_norm_workspace(&p.c, &bytes);
  const at::Tensor work = rc == 0 && bytes ? make(p.n, at::kByte, {(int64_t)bytes}) : at::Tensor();
  void* s = stream_of(p.n);
  if (rc == 0)
    rc = unlocked([&] {
      return per_layer_norm_backward(&p.c, &rd, &rx, w, &ro, static_cast<float*>(data(dw)), static_cast<float*>(data(db)), data(work), bytes, s);
    });
  written(rc, {a[4]});
  return answer(rc, {&dx, &dw, &db});
}

uint64_t whole(PyObject* o, const char* name) {
  if (!PyLong_Check(o)) {
    PyErr_Format(PyExc_TypeError, "%s: expected a whole number, got %.100s", name, Py_TYPE(o)->tp_name);
    throw Raised{};
  }
  const unsigned long long v = PyLong_AsUnsignedLongLong(o);
  if (PyErr_Occurred()) {
    PyErr_Clear();
    raise_value(std::string(name) + ": expected 0 <= " + name + " < 2^64");
  }
  return v;
}

// (x, p, seed, offset, residual, out) -> (code, out), or None.  offset: a number, or an int64 tensor of one value on the device
PyObject* do_dropout(Args a, Py_ssize_t n_args) {
  expect(n_args, 6);
  if (differentiated({a[0], a[4]}, {a[5]})) Py_RETURN_NONE;
  const at::Tensor& x = tensor(a[0], "x");
  Block p(x);
  const c10::DeviceGuard guard(p.n.device);
  const double share = real(a[1]);
  if (!(share >= 0.0 && share < 1.0)) raise_value("p: expected 0 <= p < 1");
  p.c.p = (float)(std::min(65535.0, std::floor(share * 65536.0 + 0.5)) / 65536.0);   // (a whole number of 1/65536, which a float has)
  p.c.seed = whole(a[2], "seed");
  const int64_t* at_offset = nullptr;
  if (THPVariable_Check(a[3])) {
    const at::Tensor& o = THPVariable_Unpack(a[3]);
    if (o.device() != p.n.device || o.scalar_type() != at::kLong || o.numel() != 1) raise_value("offset: expected a number, or an int64 tensor of one value on " + p.n.device.str());
    at_offset = static_cast<const int64_t*>(o.data_ptr());
  } else {
    p.c.offset = whole(a[3], "offset");
  }
  const at::Tensor* residual = maybe(a[4], "residual");
  per_seq_rows rr{};
  if (residual) rr = p.rows_of(*residual, "residual");
  at::Tensor out = p.result_of(a[5], "out");
  const per_seq_rows rx = p.rows_of(x, "x"), ro = p.rows_of(out, "out");
  void* s = stream_of(p.n);
  const int rc = unlocked([&] { return per_dropout(&p.c, &rx, residual ? &rr : nullptr, at_offset, &ro, s); });
  written(rc, {a[5]});
  return answer(rc, {&out});
}

// What a tensor has besides its memory.  No call forms derivatives along its inputs: a tangent would be lost without a word.  A view that
// torch negates when it reads it (the imaginary part of a conjugate) would be read with the other sign.
void refuse_unseen(Args a, Py_ssize_t n) {
  for (Py_ssize_t i = 0; i < n; ++i) {
    if (!THPVariable_Check(a[i])) continue;
    const at::Tensor& t = THPVariable_Unpack(a[i]);
    if (t._fw_grad(0).defined()) {
      PyErr_SetString(PyExc_RuntimeError, "a tensor carries a forward-mode derivative, which is not formed here: take its primal (torch.autograd.forward_ad.unpack_dual)");
      throw Raised{};
    }
    if (t.is_neg()) raise_value("a tensor is a view that stands for its negative: call resolve_neg() on it first");
  }
}

// Every function: C++ and library errors become Python exceptions, nothing is thrown past the interpreter.
template <PyObject* (*F)(Args, Py_ssize_t)>
PyObject* function(PyObject*, Args a, Py_ssize_t n) {
  try {
    refuse_unseen(a, n);
    return F(a, n);
  } catch (const Raised&) {
  } catch (const std::exception& e) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, e.what());
  }
  return nullptr;
}
template <PyObject* (*F)(Args, Py_ssize_t)>
constexpr PyMethodDef entry(const char* name) {
  return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&function<F>)), METH_FASTCALL, nullptr};
}
PyMethodDef functions[] = {entry<do_attention>("linear_attention"), entry<do_attention_backward>("linear_attention_backward"),
                           entry<do_attention_step>("linear_attention_step"), entry<do_rotate>("rotate"), entry<do_norm_rotate>("norm_rotate"),
                           entry<do_norm_rotate_backward>("norm_rotate_backward"), entry<do_delta>("gated_delta"),
                           entry<do_delta_backward>("gated_delta_backward"), entry<do_delta_step>("gated_delta_step"),
                           entry<do_layer_norm>("layer_norm"), entry<do_layer_norm_backward>("layer_norm_backward"),
                           entry<do_dropout>("dropout"), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_seq_binding", "The sequence operators, tensors in, C-ABI calls out.", -1, functions};

}  // namespace

PyMODINIT_FUNC PyInit__seq_binding() { return PyModule_Create(&module); }
