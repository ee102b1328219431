// Python's way into the C ABI for the calls that a training step or a decode loop makes: tensors are taken apart, results
// and workspaces allocated and the library called without passing through ctypes and torch's Python functions (forward of
// two heads of 512 rows: 8.8 us of host time, of which the launch 3; 13.7 for the backward).  Argument marshalling only.
//
// Every function takes its arguments by position, None for a tensor to be allocated, and returns its results, or the
// library's status as an int where that is not RSA_OK.  What is allocated here are plain tensors.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ops/empty.h>
#include <ATen/ops/empty_like.h>
#include <ATen/ops/zeros_like.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <array>

#include "rsa.h"

namespace {

struct Refused {};  // a Python error is set

// The arguments of one call.
struct Call {
  PyObject *const *args;
  rsa_desc *d = nullptr;
  const rsa_cache_desc *cd = nullptr;  // ... or this one, of the calls on the cache
  Py_buffer view{};

  Call(PyObject *const *args_, Py_ssize_t n, Py_ssize_t want, bool cache) : args(args_) {
    if (n != want) {
      PyErr_Format(PyExc_TypeError, "%zd arguments expected, %zd given", want, n);
      throw Refused{};
    }
    // the descriptor is a ctypes structure, which exports its memory
    if (PyObject_GetBuffer(args[0], &view, PyBUF_SIMPLE) != 0) throw Refused{};
    if (view.len != (Py_ssize_t)(cache ? sizeof(rsa_cache_desc) : sizeof(rsa_desc))) {
      PyErr_SetString(PyExc_TypeError, "not a descriptor");
      PyBuffer_Release(&view);
      throw Refused{};
    }
    if (cache) cd = static_cast<const rsa_cache_desc *>(view.buf);
    else d = static_cast<rsa_desc *>(view.buf);
  }
  ~Call() { PyBuffer_Release(&view); }
  Call(const Call &) = delete;

  bool given(int i) const { return args[i] != Py_None; }
  const at::Tensor &tensor(int i) const {
    if (!THPVariable_Check(args[i])) {
      PyErr_Format(PyExc_TypeError, "argument %d: a tensor expected, not %s", i, Py_TYPE(args[i])->tp_name);
      throw Refused{};
    }
    return THPVariable_Unpack(args[i]);
  }
  // ... of the GPU with a contiguous last index; other strides travel in the descriptor
  const at::Tensor &input(int i) const {
    const at::Tensor &t = tensor(i);
    if (!t.is_cuda() || t.dim() == 0 || t.stride(-1) != 1) {
      PyErr_Format(PyExc_AssertionError, "argument %d: a tensor of the GPU with a contiguous last index expected", i);
      throw Refused{};
    }
    return t;
  }
  template <class F> at::Tensor tensor_or(int i, F make) const { return given(i) ? tensor(i) : make(); }
};

void *ptr(const at::Tensor &t) { return t.defined() ? t.data_ptr() : nullptr; }

at::Tensor bytes(size_t n, const at::Tensor &like) { return at::empty({(int64_t)n}, like.options().dtype(at::kByte)); }

PyObject *wrapped(std::initializer_list<at::Tensor> ts) {
  if (ts.size() == 1) return THPVariable_Wrap(*ts.begin());
  PyObject *r = PyTuple_New((Py_ssize_t)ts.size());
  if (!r) return nullptr;
  Py_ssize_t i = 0;
  for (const at::Tensor &t : ts) {
    PyObject *o = THPVariable_Wrap(t);
    if (!o) { Py_DECREF(r); return nullptr; }
    PyTuple_SET_ITEM(r, i++, o);
  }
  return r;
}

// The library call, on the current device's current stream and without the interpreter's lock (a launch may wait for a
// place in the queue).
template <class F> PyObject *finish(F call, std::initializer_list<at::Tensor> results) {
  void *stream = c10::hip::getCurrentHIPStream().stream();
  int status;
  Py_BEGIN_ALLOW_THREADS
  status = call(stream);
  Py_END_ALLOW_THREADS
  return status == RSA_OK ? wrapped(results) : PyLong_FromLong(status);
}

template <PyObject *(*F)(Call &), bool CACHE> struct Entry {
  template <int N> static PyObject *call(PyObject *, PyObject *const *args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    try {
      Call c(args, n, N, CACHE);
      return F(c);
    } catch (Refused) {
      return nullptr;
    }
    END_HANDLE_TH_ERRORS
  }
};

// workspace i of a pass of the attention: given, or what the descriptor asks for (nothing: none)
at::Tensor pass_workspace(const Call &c, int i, int pass, const at::Tensor &like, size_t &n) {
  if (c.given(i)) {
    const at::Tensor &t = c.tensor(i);
    n = (size_t)t.numel();
    return t;
  }
  n = rsa_workspace_bytes(c.d, pass);
  return n ? bytes(n, like) : at::Tensor();
}
at::Tensor workspace(const Call &c, int i, size_t need, const at::Tensor &like, size_t &n) {
  at::Tensor t = c.given(i) ? c.tensor(i) : bytes(need > 16 ? need : 16, like);
  n = (size_t)t.numel();
  return t;
}
at::Tensor row_terms(const at::Tensor &Q) {  // (Q may have fewer dimensions than the descriptor's four: taken as dense)
  return at::empty(Q.sizes().slice(0, Q.dim() < 3 ? Q.dim() : 3), Q.options().dtype(at::kFloat).memory_format(std::nullopt));
}
// The ranks' rows, as Python divides: a descriptor that the library will refuse gets there with any numbers in it.
int64_t rows_of(const rsa_desc *d) {
  if (d->N == 0) {
    PyErr_SetString(PyExc_ZeroDivisionError, "integer division or modulo by zero");
    throw Refused{};
  }
  int64_t chunk;
  if (d->N == -1) {
    chunk = (int64_t)(0 - (uint64_t)d->L);
  } else {
    chunk = d->L / d->N;
    if (d->L % d->N != 0 && (d->L < 0) != (d->N < 0)) --chunk;
  }
  return (int64_t)((uint64_t)((int64_t)d->rank_end - d->rank_begin) * (uint64_t)chunk);
}

// desc, Q, K, V, O, LSE, ws
PyObject *forward(Call &c) {
  const at::Tensor &Q = c.input(1), &K = c.input(2), &V = c.input(3);
  const at::Tensor O = c.tensor_or(4, [&] { return at::empty_like(Q); });
  const at::Tensor LSE = c.tensor_or(5, [&] { return row_terms(Q); });
  size_t n;
  const at::Tensor ws = pass_workspace(c, 6, 0, Q, n);
  return finish([&](void *st) {
    return rsa_forward(c.d, ptr(Q), ptr(K), ptr(V), ptr(O), static_cast<float *>(ptr(LSE)), ptr(ws), n, st); }, {O, LSE});
}

// desc, dO, Q, K, V, O, LSE, dQ, dK, dV, ws
PyObject *backward(Call &c) {
  const at::Tensor &dO = c.input(1), &Q = c.input(2), &K = c.input(3), &V = c.input(4), &O = c.input(5), &LSE = c.input(6);
  const at::Tensor dQ = c.tensor_or(7, [&] { return at::empty_like(Q); });
  const at::Tensor dK = c.tensor_or(8, [&] { return at::empty_like(K); });
  const at::Tensor dV = c.tensor_or(9, [&] { return at::empty_like(V); });
  size_t n;
  const at::Tensor ws = pass_workspace(c, 10, 1, Q, n);
  return finish([&](void *st) {
    return rsa_backward(c.d, ptr(dO), ptr(Q), ptr(K), ptr(V), ptr(O), static_cast<const float *>(ptr(LSE)), ptr(dQ), ptr(dK),
                        ptr(dV), ptr(ws), n, st); }, {dQ, dK, dV});
}

at::Tensor heads_like(const Call &c, const at::Tensor &X) {
  return at::empty({c.d->B, c.d->Z, rows_of(c.d), c.d->A}, X.options());
}
// desc, X, W, Q, K, V
PyObject *qkv_proj(Call &c) {
  const at::Tensor &X = c.tensor(1), &W = c.tensor(2);
  const int32_t H = (int32_t)X.size(-1);
  const auto make = [&] { return heads_like(c, X); };
  const at::Tensor Q = c.tensor_or(3, make), K = c.tensor_or(4, make), V = c.tensor_or(5, make);
  return finish([&](void *st) { return rsa_qkv_proj(c.d, H, ptr(X), ptr(W), ptr(Q), ptr(K), ptr(V), st); }, {Q, K, V});
}
// desc, O, Wo, Y
PyObject *out_proj(Call &c) {
  const at::Tensor &O = c.tensor(1), &Wo = c.tensor(2);
  const int32_t H = (int32_t)Wo.size(-1);
  const at::Tensor Y = c.tensor_or(3, [&] { return at::empty({O.size(0), O.size(2), H}, O.options()); });
  return finish([&](void *st) { return rsa_out_proj(c.d, H, ptr(O), ptr(Wo), ptr(Y), st); }, {Y});
}
// desc, dY, O, Wo, dO, dWo, ws
PyObject *out_proj_bwd(Call &c) {
  const at::Tensor &dY = c.tensor(1), &O = c.tensor(2), &Wo = c.tensor(3);
  const int32_t H = (int32_t)Wo.size(-1);
  const at::Tensor dO = c.tensor_or(4, [&] { return at::empty_like(O); });
  const at::Tensor dWo = c.tensor_or(5, [&] { return at::empty(Wo.sizes(), Wo.options().dtype(at::kFloat)); });
  size_t n;
  const at::Tensor ws = workspace(c, 6, rsa_proj_workspace_bytes(c.d, H), O, n);
  return finish([&](void *st) {
    return rsa_out_proj_bwd(c.d, H, ptr(dY), ptr(O), ptr(Wo), ptr(dO), static_cast<float *>(ptr(dWo)), ptr(ws), n, st); },
    {dO, dWo});
}
// desc, dQ, dK, dV, X, W, dX, dW, ws
PyObject *qkv_proj_bwd(Call &c) {
  const at::Tensor &dQ = c.tensor(1), &dK = c.tensor(2), &dV = c.tensor(3), &X = c.tensor(4), &W = c.tensor(5);
  const int32_t H = (int32_t)X.size(-1);
  const at::Tensor dX = c.tensor_or(6, [&] { return at::empty_like(X); });
  const at::Tensor dW = c.tensor_or(7, [&] { return at::empty(W.sizes(), W.options().dtype(at::kFloat)); });
  size_t n;
  const at::Tensor ws = workspace(c, 8, rsa_proj_workspace_bytes(c.d, H), X, n);
  return finish([&](void *st) {
    return rsa_qkv_proj_bwd(c.d, H, ptr(dQ), ptr(dK), ptr(dV), ptr(X), ptr(W), ptr(dX), static_cast<float *>(ptr(dW)), ptr(ws),
                            n, st); }, {dX, dW});
}
// desc, X, E, Xp, ws
PyObject *linformer_project(Call &c) {
  const at::Tensor &X = c.tensor(1), &E = c.tensor(2);
  const int32_t Kp = (int32_t)E.size(1);
  const at::Tensor Xp = c.tensor_or(3, [&] { return at::empty({X.size(0), X.size(1), Kp, X.size(3)}, X.options()); });
  size_t n;
  const at::Tensor ws = workspace(c, 4, rsa_linformer_workspace_bytes(c.d, Kp), X, n);
  return finish([&](void *st) { return rsa_linformer_project(c.d, Kp, ptr(X), ptr(E), ptr(Xp), ptr(ws), n, st); }, {Xp});
}
// desc, Q, Kp, Vp, O, LSE
PyObject *linformer_forward(Call &c) {
  const at::Tensor &Q = c.tensor(1), &Kp = c.tensor(2), &Vp = c.tensor(3);
  const at::Tensor O = c.tensor_or(4, [&] { return at::empty_like(Q); });
  const at::Tensor LSE = c.tensor_or(5, [&] { return row_terms(Q); });
  return finish([&](void *st) {
    return rsa_linformer_forward(c.d, (int32_t)Kp.size(2), ptr(Q), ptr(Kp), ptr(Vp), ptr(O), static_cast<float *>(ptr(LSE)), st); },
    {O, LSE});
}
// desc, dO, Q, Kp, Vp, O, LSE, dQ, dKp, dVp, ws
PyObject *linformer_backward(Call &c) {
  const at::Tensor &dO = c.tensor(1), &Q = c.tensor(2), &Kp = c.tensor(3), &Vp = c.tensor(4), &O = c.tensor(5), &LSE = c.tensor(6);
  const int32_t kp = (int32_t)Kp.size(2);
  const at::Tensor dQ = c.tensor_or(7, [&] { return at::empty_like(Q); });
  const at::Tensor dKp = c.tensor_or(8, [&] { return at::empty_like(Kp); });
  const at::Tensor dVp = c.tensor_or(9, [&] { return at::empty_like(Vp); });
  size_t n;
  const at::Tensor ws = workspace(c, 10, rsa_linformer_workspace_bytes(c.d, kp), Q, n);
  return finish([&](void *st) {
    return rsa_linformer_backward(c.d, kp, ptr(dO), ptr(Q), ptr(Kp), ptr(Vp), ptr(O), static_cast<const float *>(ptr(LSE)),
                                  ptr(dQ), ptr(dKp), ptr(dVp), ptr(ws), n, st); }, {dQ, dKp, dVp});
}
// desc, dXp, X, E, dX, dE: the rows of the descriptor's ranks; a new tensor is zero elsewhere (with all ranks every row is
// written: zeroing both first costs as much as a fifth of the kernels' traffic)
PyObject *linformer_project_bwd(Call &c) {
  const at::Tensor &dXp = c.tensor(1), &X = c.tensor(2), &E = c.tensor(3);
  const bool all = c.d->rank_begin == 0 && c.d->rank_end == c.d->N;
  const at::Tensor dX = c.tensor_or(4, [&] { return all ? at::empty_like(X) : at::zeros_like(X); });
  const at::Tensor dE = c.tensor_or(5, [&] {
    const auto o = E.options().dtype(at::kFloat);
    return all ? at::empty_like(E, o, at::MemoryFormat::Contiguous) : at::zeros_like(E, o, at::MemoryFormat::Contiguous);
  });
  return finish([&](void *st) {
    return rsa_linformer_project_bwd(c.d, (int32_t)E.size(1), ptr(dXp), ptr(X), ptr(E), ptr(dX), static_cast<float *>(ptr(dE)), st); },
    {dX, dE});
}

// The calls below read tables, so that a wrong shape would reach memory that is not the tensor's: every tensor is held against
// the descriptor.  Tensors on the CPU come last, so that this is the same without a GPU.
[[noreturn]] void refuse(int i, const char *what) {
  PyErr_Format(PyExc_ValueError, "argument %d: %s", i, what);
  throw Refused{};
}
// st: strides of all indices but the last; zeros: dense; nullptr: any dense
void check(int i, const at::Tensor &t, at::ScalarType type, at::IntArrayRef shape, const int64_t *st = nullptr) {
  if (t.scalar_type() != type) refuse(i, "not of the descriptor's (or the expected) dtype");
  if (t.sizes() != shape) refuse(i, "not of the descriptor's (or the other tensors') shape");
  bool dense = true;
  if (st)
    for (size_t k = 0; k + 1 < shape.size(); ++k) dense = dense && st[k] == 0;
  if (dense ? !t.is_contiguous() : t.stride(-1) != 1 && shape.back() != 1) refuse(i, "not laid out as the descriptor says");
  if (!dense)
    for (size_t k = 0; k + 1 < shape.size(); ++k)
      if (shape[k] != 1 && t.stride((int64_t)k) != st[k]) refuse(i, "not laid out as the descriptor says");
}
// ... and that they are where the work is enqueued
void check_device(const Call &c, int n) {
  int current = -1;  // (asked for once a tensor of a GPU is there)
  for (int i = 1; i < n; ++i)
    if (THPVariable_Check(c.args[i])) {
      const at::Tensor &t = THPVariable_Unpack(c.args[i]);
      if (t.is_cuda() && current < 0) current = c10::hip::getCurrentHIPStream().device_index();
      if (!t.is_cuda() || t.get_device() != current) {
        PyErr_Format(PyExc_AssertionError, "argument %d: a tensor of the current GPU expected", i);
        throw Refused{};
      }
    }
}
// a result laid out as an input is, which only an input without gaps can lend
at::Tensor laid_out_as(int i, const at::Tensor &t, bool zero) {
  if (!t.is_non_overlapping_and_dense()) refuse(i, "a result for an input with gaps has to be given");
  return zero ? at::zeros_like(t) : at::empty_like(t);
}
at::ScalarType type_of(int32_t dtype) { return dtype == RSA_F32 ? at::kFloat : at::kBFloat16; }
int32_t truth(const Call &c, int i) {
  const int v = PyObject_IsTrue(c.args[i]);
  if (v < 0) throw Refused{};
  return v;
}
// R, from the frequencies
int32_t check_frequencies(const Call &c, int i) {
  const at::Tensor &t = c.tensor(i);
  const int64_t n = t.dim() == 1 ? t.size(0) : 0;
  if (n < 1 || n > 128) refuse(i, "frequencies of 1 to A / 2 pairs expected");
  check(i, t, at::kFloat, {n});
  return (int32_t)(2 * n);
}

// desc, inv_freq, Q, K, Qr, Kr, adjacent, back
PyObject *rotate(Call &c) {
  const rsa_desc &d = *c.d;
  const int32_t R = check_frequencies(c, 1), adjacent = truth(c, 6), back = truth(c, 7);
  at::Tensor in[2], out[2];
  for (int i = 0; i < 2; ++i) {
    if (!c.given(2 + i)) {
      if (c.given(4 + i)) refuse(4 + i, "a result without its input");
      continue;
    }
    const std::array<int64_t, 4> shape{d.B, d.Z, i ? d.L : rows_of(&d), d.A};
    const int64_t *st = i ? d.kv_stride : d.q_stride;
    in[i] = c.tensor(2 + i);
    check(2 + i, in[i], type_of(d.dtype), shape, st);
    out[i] = c.tensor_or(4 + i, [&] { return laid_out_as(2 + i, in[i], false); });
    check(4 + i, out[i], type_of(d.dtype), shape, st);
  }
  check_device(c, 6);
  const auto call = back ? rsa_rotate_bwd : rsa_rotate;
  const float *freq = static_cast<const float *>(ptr(c.tensor(1)));
  void *stream = c10::hip::getCurrentHIPStream().stream();
  int status;
  Py_BEGIN_ALLOW_THREADS
  status = call(&d, R, adjacent, freq, ptr(in[0]), ptr(in[1]), ptr(out[0]), ptr(out[1]), stream);
  Py_END_ALLOW_THREADS
  if (status != RSA_OK) return PyLong_FromLong(status);
  PyObject *r = PyTuple_New(2);
  for (int i = 0; r && i < 2; ++i) {
    PyObject *o = out[i].defined() ? THPVariable_Wrap(out[i]) : (Py_INCREF(Py_None), Py_None);
    if (!o) { Py_DECREF(r); return nullptr; }
    PyTuple_SET_ITEM(r, i, o);
  }
  return r;
}

const int32_t *int32s(const Call &c, int i, at::IntArrayRef shape) {
  if (!c.given(i)) return nullptr;
  check(i, c.tensor(i), at::kInt, shape);
  return static_cast<const int32_t *>(ptr(c.tensor(i)));
}
void check_pools(const Call &c, int i) {
  const rsa_cache_desc &d = *c.cd;
  for (int k = i; k < i + 2; ++k) check(k, c.tensor(k), type_of(d.dtype), {d.pages, d.Zkv, d.page, d.A});
}

// desc, K, V, Kc, Vc, table, lengths, counts, first, inv_freq, adjacent, Q, Qr
PyObject *cache_append(Call &c) {
  const rsa_cache_desc &d = *c.cd;
  const at::Tensor &K = c.tensor(1), &V = c.tensor(2), &Kc = c.tensor(3), &Vc = c.tensor(4);
  if (K.dim() != 4 || K.size(2) < 1 || K.size(2) > INT32_MAX) refuse(1, "(B, Zkv, T, A) expected");
  const int64_t T = K.size(2);
  for (int i = 1; i < 3; ++i) check(i, c.tensor(i), type_of(d.dtype), {d.B, d.Zkv, T, d.A}, d.kv_stride);
  check_pools(c, 3);
  if (!c.given(5) || !c.given(6)) refuse(c.given(5) ? 6 : 5, "a tensor expected");
  const int32_t *table = int32s(c, 5, {d.B, d.width}), *lengths = int32s(c, 6, {d.B}), *counts = int32s(c, 7, {d.B});
  const int32_t *first = int32s(c, 8, {d.B}), R = c.given(9) ? check_frequencies(c, 9) : 0, adjacent = truth(c, 10);
  const float *freq = c.given(9) ? static_cast<const float *>(ptr(c.tensor(9))) : nullptr;
  at::Tensor Q, Qr;
  if (c.given(11)) {
    Q = c.tensor(11);
    check(11, Q, type_of(d.dtype), {d.B, d.Z, T, d.A}, d.q_stride);
    Qr = c.tensor_or(12, [&] { return laid_out_as(11, Q, counts != nullptr); });
    check(12, Qr, type_of(d.dtype), {d.B, d.Z, T, d.A}, d.q_stride);
  } else if (c.given(12)) {
    refuse(12, "a result without its input");
  }
  check_device(c, 13);
  const auto call = [&](void *st) {
    return rsa_cache_append(&d, (int32_t)T, ptr(Q), ptr(K), ptr(V), table, lengths, counts, first, R, adjacent, freq, ptr(Qr), ptr(Kc),
                            ptr(Vc), st); };
  if (Q.defined()) return finish(call, {Qr});
  PyObject *r = finish(call, {Kc});
  if (!r || PyLong_Check(r)) return r;
  Py_DECREF(r);
  Py_RETURN_NONE;
}

// desc, Q, Kc, Vc, table, lengths, O, LSE, ws
PyObject *cache_attend(Call &c) {
  const rsa_cache_desc &d = *c.cd;
  const at::Tensor &Q = c.tensor(1), &Kc = c.tensor(2), &Vc = c.tensor(3);
  const std::array<int64_t, 4> shape{d.B, d.Z, 1, d.A};
  check(1, Q, type_of(d.dtype), shape, d.q_stride);
  check_pools(c, 2);
  if (!c.given(4) || !c.given(5)) refuse(c.given(4) ? 5 : 4, "a tensor expected");
  const int32_t *table = int32s(c, 4, {d.B, d.width}), *lengths = int32s(c, 5, {d.B});
  const at::Tensor O = c.tensor_or(6, [&] { return at::empty(shape, Q.options()); });
  check(6, O, type_of(d.dtype), shape, d.o_stride);
  const at::Tensor LSE = c.tensor_or(7, [&] { return at::empty({d.B, d.Z, 1}, Q.options().dtype(at::kFloat)); });
  check(7, LSE, at::kFloat, {d.B, d.Z, 1});
  check_device(c, 9);
  size_t n = 0;
  at::Tensor ws;
  if (c.given(8)) {
    ws = c.tensor(8);
    if (!ws.is_contiguous()) refuse(8, "a workspace without gaps expected");
    n = ws.nbytes();
  } else if ((n = rsa_cache_workspace_bytes(&d)) > 0) {
    ws = bytes(n, Q);
  }
  return finish([&](void *st) {
    return rsa_cache_attend(&d, ptr(Q), ptr(Kc), ptr(Vc), table, lengths, ptr(O), static_cast<float *>(ptr(LSE)), ptr(ws), n, st); },
    {O, LSE});
}

// desc, Op, LSEp, O, LSE
PyObject *cache_join(Call &c) {
  const rsa_cache_desc &d = *c.cd;
  const at::Tensor &Op = c.tensor(1), &LSEp = c.tensor(2);
  if (Op.dim() != 5 || Op.size(0) < 1 || Op.size(0) > INT32_MAX) refuse(1, "(N, B, Z, 1, A) expected");
  const int64_t N = Op.size(0);
  check(1, Op, type_of(d.dtype), {N, d.B, d.Z, 1, d.A});
  check(2, LSEp, at::kFloat, {N, d.B, d.Z, 1});
  const std::array<int64_t, 4> shape{d.B, d.Z, 1, d.A};
  const at::Tensor O = c.tensor_or(3, [&] { return at::empty(shape, Op.options()); });
  check(3, O, type_of(d.dtype), shape, d.o_stride);
  const at::Tensor LSE = c.tensor_or(4, [&] { return at::empty({d.B, d.Z, 1}, LSEp.options()); });
  check(4, LSE, at::kFloat, {d.B, d.Z, 1});
  check_device(c, 5);
  return finish([&](void *st) {
    return rsa_cache_join(&d, (int32_t)N, ptr(Op), static_cast<const float *>(ptr(LSEp)), ptr(O), static_cast<float *>(ptr(LSE)), st); },
    {O, LSE});
}

template <PyObject *(*F)(Call &), int N, bool CACHE = false> PyMethodDef method(const char *name) {
  return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&Entry<F, CACHE>::template call<N>)), METH_FASTCALL, nullptr};
}

}  // namespace

PyMODINIT_FUNC PyInit__binding(void);
PyMODINIT_FUNC PyInit__binding(void) {
  static PyMethodDef table[] = {
      method<forward, 7>("forward"), method<backward, 11>("backward"), method<qkv_proj, 6>("qkv_proj"),
      method<out_proj, 4>("out_proj"), method<out_proj_bwd, 7>("out_proj_bwd"), method<qkv_proj_bwd, 9>("qkv_proj_bwd"),
      method<linformer_project, 5>("linformer_project"), method<linformer_forward, 6>("linformer_forward"),
      method<linformer_backward, 11>("linformer_backward"), method<linformer_project_bwd, 6>("linformer_project_bwd"),
      method<rotate, 8>("rotate"), method<cache_append, 13, true>("cache_append"),
      method<cache_attend, 9, true>("cache_attend"), method<cache_join, 5, true>("cache_join"),
      {nullptr, nullptr, 0, nullptr}};
  static PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, table, nullptr, nullptr, nullptr, nullptr};
  return PyModule_Create(&module);
}
