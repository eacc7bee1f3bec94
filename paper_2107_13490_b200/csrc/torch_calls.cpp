// The training-step operators' calls from torch tensors: checks, outputs, the current stream, and the entry
// point of adapt.h.  Same checks and calls as ctypes would make, in C++ because a small call is bound by
// the host: see binding.py for what it measured.
//
// The entry points' addresses come from the library that binding.py has loaded (bind), so that there is one
// library in the process whichever build of it that is.
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>
#include <initializer_list>
#include <optional>

#include "../../include/adapt.h"

namespace {

decltype(&adapt_dropout) g_dropout;
decltype(&adapt_token_logprobs) g_logprobs;
decltype(&adapt_token_logprobs_backward) g_logprobs_backward;
decltype(&adapt_gated_scan) g_scan;
decltype(&adapt_gated_scan_backward) g_scan_backward;
decltype(&adapt_gated_scan_workspace_bytes) g_scan_workspace;
PyObject* g_error;   // called with (status, entry point): the exception to raise

// An argument that does not fit (AssertionError); the Python error is set already where there is no text.
struct Refused { const char* why; };
void need(bool ok, const char* why) {
  if (!ok) throw Refused{why};
}

const at::Tensor& tensor(PyObject* o) {
  need(THPVariable_Check(o), "needs a tensor");
  return THPVariable_Unpack(o);
}
const at::Tensor* maybe(PyObject* o) { return o == Py_None ? nullptr : &tensor(o); }

double real(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw Refused{nullptr};
  return v;
}
uint64_t bits(PyObject* o) {
  const uint64_t v = PyLong_AsUnsignedLongLongMask(o);
  if (v == ~0ull && PyErr_Occurred()) throw Refused{nullptr};
  return v;
}
int32_t whole(PyObject* o) { return static_cast<int32_t>(bits(o)); }   // modulo 2^32
// A number that has to be meant as it stands.
int32_t between(PyObject* o, int32_t least, int32_t most, const char* why) {
  int beyond = 0;
  const long long v = PyLong_AsLongLongAndOverflow(o, &beyond);
  if (v == -1 && !beyond && PyErr_Occurred()) throw Refused{nullptr};
  need(!beyond && v >= least && v <= most, why);
  return static_cast<int32_t>(v);
}
bool truth(PyObject* o) {
  const int v = PyObject_IsTrue(o);
  if (v < 0) throw Refused{nullptr};
  return v != 0;
}

// The element type of a tensor on the current device.
int elem(const at::Tensor& t) {
  const auto d = t.scalar_type();
  need(t.is_cuda() && (d == at::kFloat || d == at::kHalf || d == at::kBFloat16),
       "needs a CUDA tensor of float32, float16 or bfloat16");
  need(t.get_device() == c10::cuda::current_device(), "the tensors are not on the current device");
  return d == at::kFloat ? ADAPT_DTYPE_F32 : d == at::kHalf ? ADAPT_DTYPE_F16 : ADAPT_DTYPE_BF16;
}
bool like(const at::Tensor& t, const at::Tensor& x) {
  return t.scalar_type() == x.scalar_type() && t.device() == x.device() && t.sizes() == x.sizes();
}
void need_like(const at::Tensor& t, const at::Tensor& x) {
  need(like(t, x), "a tensor's shape, type or device differs from its partner's");
}
at::Tensor make(const at::Tensor& x, at::IntArrayRef sizes, at::ScalarType type) {
  return at::empty(sizes, at::TensorOptions().dtype(type).device(x.device()));
}
at::Tensor make_like(const at::Tensor& x) { return make(x, x.sizes(), x.scalar_type()); }
// `given`, which has to be as x is, or a new tensor.
at::Tensor out_like(const at::Tensor* given, const at::Tensor& x) {
  if (!given) return make_like(x);
  need_like(*given, x);
  return *given;
}

void* stream_of(const at::Tensor& x) { return c10::cuda::getCurrentCUDAStream(x.get_device()).stream(); }

// Makes the call without the interpreter's lock; raises what the status says.
template <typename F>
void call(const char* name, F f) {
  int status;
  Py_BEGIN_ALLOW_THREADS
  status = f();
  Py_END_ALLOW_THREADS
  if (status == ADAPT_OK) return;
  PyObject* e = PyObject_CallFunction(g_error, "is", status, name);
  if (e) {
    PyErr_SetObject(reinterpret_cast<PyObject*>(Py_TYPE(e)), e);
    Py_DECREF(e);
  }
  throw Refused{nullptr};
}

PyObject* wrap(const at::Tensor& t) { return t.defined() ? THPVariable_Wrap(t) : Py_NewRef(Py_None); }
PyObject* wrap(std::initializer_list<const at::Tensor*> all) {
  PyObject* r = PyTuple_New(static_cast<Py_ssize_t>(all.size()));
  Py_ssize_t i = 0;
  if (r)
    for (const at::Tensor* t : all) PyTuple_SET_ITEM(r, i++, wrap(*t));
  return r;
}

// f() with its refusals and torch's exceptions turned into Python's.
template <typename F>
PyObject* guarded(Py_ssize_t n, Py_ssize_t want, F f) {
  HANDLE_TH_ERRORS
  try {
    need(n == want, "wrong number of arguments");
    return f();
  } catch (const Refused& r) {
    if (r.why) PyErr_SetString(PyExc_AssertionError, r.why);
    return nullptr;
  }
  END_HANDLE_TH_ERRORS
}

// (x, p, seed, layer, index_base, residual, out) -> out
PyObject* dropout(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 7, [&] {
    const at::Tensor& x = tensor(a[0]);
    const int dtype = elem(x);
    const double p = real(a[1]);
    const uint64_t seed = bits(a[2]), base = bits(a[4]);
    const int32_t layer = whole(a[3]);
    const at::Tensor* r = maybe(a[5]);
    bool flat = x.is_contiguous();
    if (r) { need_like(*r, x); flat = flat && r->is_contiguous(); }
    const at::Tensor* given = maybe(a[6]);
    const at::Tensor out = out_like(given, x);
    flat = flat && (!given || out.is_contiguous());
    int64_t rows = 1, cols = x.numel(), ldx = cols, ldy = cols, ldr = cols;   // elements in order: one long row
    if (!flat) {
      need(x.dim() == 2, "needs contiguous tensors, or matrices with unit inner stride");
      rows = x.size(0); cols = x.size(1);
      auto line = [&](const at::Tensor& t) {
        need(cols <= 1 || t.stride(1) == 1, "needs contiguous tensors, or matrices with unit inner stride");
        return rows > 1 ? t.stride(0) : cols;
      };
      ldx = line(x); ldy = line(out);
      ldr = r ? line(*r) : ldy;
    }
    const void *px = x.const_data_ptr(), *pr = r ? r->const_data_ptr() : nullptr;
    void *py = out.mutable_data_ptr(), *stream = stream_of(x);
    call("adapt_dropout", [&] { return g_dropout(px, pr, py, rows, cols, ldx, ldr, ldy, dtype, p, seed, layer, base, stream); });
    return wrap(out);
  });
}

struct Matrix { int64_t rows, cols, ld; };
Matrix matrix(const at::Tensor& t) {
  need(t.dim() == 2, "needs a matrix");
  const int64_t rows = t.size(0), cols = t.size(1);
  need(cols <= 1 || t.stride(1) == 1, "needs a matrix with unit inner stride");
  return {rows, cols, rows > 1 ? t.stride(0) : cols};
}
// What goes with the rows of x: on its device, an element a row.
const void* per_row(const at::Tensor* t, const at::Tensor& x, at::ScalarType type) {
  if (!t) return nullptr;
  need(t->device() == x.device() && t->scalar_type() == type && t->numel() == x.size(0) && t->is_contiguous(),
       "needs a contiguous tensor on the logits' device with an element a row (targets int64, others float32)");
  return t->const_data_ptr();
}
const float* floats(const at::Tensor* t, const at::Tensor& x) { return static_cast<const float*>(per_row(t, x, at::kFloat)); }
const int64_t* numbers(const at::Tensor* t, const at::Tensor& x) { return static_cast<const int64_t*>(per_row(t, x, at::kLong)); }
template <typename T>
T* out_data(const at::Tensor& t) { return t.defined() ? static_cast<T*>(t.mutable_data_ptr()) : nullptr; }

// (logits, targets, scale, n_top, want_entropy, d_logprob, d_entropy, dlogits)
// -> (logprob, entropy, lse, top_ids, top_logprobs, dlogits)
PyObject* logprobs(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 8, [&] {
    const at::Tensor& x = tensor(a[0]);
    const int dtype = elem(x);
    const Matrix m = matrix(x);
    const float scale = static_cast<float>(real(a[2]));
    const int32_t k = between(a[3], 0, ADAPT_MAX_TOP, "between 0 and 32 alternatives");
    const int64_t* pt = numbers(maybe(a[1]), x);
    const float *pdl = floats(maybe(a[5]), x), *pdh = floats(maybe(a[6]), x);
    const at::Tensor* given = maybe(a[7]);
    at::Tensor logprob, entropy, lse = make(x, {m.rows}, at::kFloat), ids, tops, dx;
    if (a[1] != Py_None) logprob = make(x, {m.rows}, at::kFloat);
    if (truth(a[4])) entropy = make(x, {m.rows}, at::kFloat);
    if (k) {
      ids = make(x, {m.rows, k}, at::kInt);
      tops = make(x, {m.rows, k}, at::kFloat);
    }
    int64_t ldg = 0;
    if (given || a[5] != Py_None || a[6] != Py_None) {
      dx = out_like(given, x);
      ldg = matrix(dx).ld;
    }
    const void* px = x.const_data_ptr();
    void* stream = stream_of(x);
    call("adapt_token_logprobs", [&] {
      return g_logprobs(px, m.rows, m.cols, m.ld, dtype, scale, pt, k, out_data<float>(logprob), out_data<float>(entropy),
                        out_data<float>(lse), out_data<int32_t>(ids), out_data<float>(tops), pdl, pdh, out_data<void>(dx), ldg, stream);
    });
    return wrap({&logprob, &entropy, &lse, &ids, &tops, &dx});
  });
}

// (logits, targets, lse, d_logprob, entropy, d_entropy, scale, out) -> out
PyObject* logprobs_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 8, [&] {
    const at::Tensor& x = tensor(a[0]);
    const int dtype = elem(x);
    const Matrix m = matrix(x);
    const int64_t* pt = numbers(maybe(a[1]), x);
    const float *pl = floats(maybe(a[2]), x), *pdl = floats(maybe(a[3]), x), *ph = floats(maybe(a[4]), x),
                *pdh = floats(maybe(a[5]), x);
    const float scale = static_cast<float>(real(a[6]));
    const at::Tensor out = out_like(maybe(a[7]), x);
    const int64_t ldg = matrix(out).ld;
    const void* px = x.const_data_ptr();
    void *po = out.mutable_data_ptr(), *stream = stream_of(x);
    call("adapt_token_logprobs_backward", [&] {
      return g_logprobs_backward(px, m.rows, m.cols, m.ld, dtype, scale, pt, pl, ph, pdl, pdh, po, ldg, stream);
    });
    return wrap(out);
  });
}

// What the forward and the backward call of the recurrence share.
struct ScanCall {
  const at::Tensor &x, &gate;
  int dtype;
  int64_t batch, steps, channels;
  int group;
  const int32_t* lengths;
  const uint8_t* reset;
  ScanCall(PyObject* x_, PyObject* gate_, PyObject* lengths_, PyObject* reset_)
      : x(tensor(x_)), gate(tensor(gate_)), dtype(elem(x)), lengths(nullptr), reset(nullptr) {
    need(x.dim() == 3 && gate.dim() == 3 && gate.scalar_type() == x.scalar_type() && gate.device() == x.device(),
         "x and the gate have three dimensions, one type and one device");
    batch = x.size(0); steps = x.size(1); channels = x.size(2);
    const int64_t gates = gate.size(2);
    need(gate.size(0) == batch && gate.size(1) == steps, "x and the gate have the same sequences and steps");
    need(channels == 0 || (gates > 0 && channels % gates == 0), "the gates have to divide the channels");
    group = static_cast<int>(gates ? channels / gates : 1);
    if (const at::Tensor* t = maybe(lengths_)) {
      need(t->device() == x.device() && t->scalar_type() == at::kInt && t->dim() == 1 && t->size(0) == batch && t->is_contiguous(),
           "lengths: int32 [batch], on the device of x");
      lengths = static_cast<const int32_t*>(t->const_data_ptr());
    }
    if (const at::Tensor* t = maybe(reset_)) {
      need(t->device() == x.device() && (t->scalar_type() == at::kByte || t->scalar_type() == at::kBool) && t->dim() == 2 &&
               t->size(0) == batch && t->size(1) == steps && t->is_contiguous(), "reset: uint8 or bool [batch, steps], on the device of x");
      reset = static_cast<const uint8_t*>(t->const_data_ptr());
    }
  }
  void need_state(const at::Tensor& t) const {
    need(t.device() == x.device() && t.scalar_type() == at::kFloat && t.dim() == 2 && t.size(0) == batch &&
             t.size(1) == channels && t.is_contiguous(), "states: float32 [batch, channels], on the device of x");
  }
  const float* state(const at::Tensor* t) const {
    if (!t) return nullptr;
    need_state(*t);
    return static_cast<const float*>(t->const_data_ptr());
  }
  int64_t kept() const { return (steps + ADAPT_SCAN_TILE - 1) / ADAPT_SCAN_TILE; }
};

// {batch, step} strides of the tensors, or null where all are contiguous.
struct Strides {
  int64_t v[10];
  bool plain = true;
  Strides(std::initializer_list<const at::Tensor*> all) {
    for (const at::Tensor* t : all) plain = plain && t->is_contiguous();
    if (plain) return;
    int i = 0;
    for (const at::Tensor* t : all) {
      need(t->size(2) <= 1 || t->stride(2) == 1, "the channels need unit stride");
      v[i++] = t->stride(0); v[i++] = t->stride(1);
    }
  }
  const int64_t* get() const { return plain ? nullptr : v; }
};

// (x, gate, h0, lengths, reset, mode, want_carry, y, h_last) -> (y, h_last, carry)
PyObject* scan(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 9, [&] {
    const ScanCall c(a[0], a[1], a[3], a[4]);
    const float* h0 = c.state(maybe(a[2]));
    const int mode = between(a[5], INT32_MIN, INT32_MAX, "no such gate");
    const at::Tensor y = out_like(maybe(a[7]), c.x);
    const at::Tensor* given = maybe(a[8]);
    const at::Tensor h = given ? *given : make(c.x, {c.batch, c.channels}, at::kFloat);
    c.need_state(h);
    at::Tensor carry;
    if (truth(a[6])) carry = make(c.x, {c.batch, c.kept(), c.channels}, at::kFloat);
    const Strides s{&c.x, &c.gate, &y};
    const void *px = c.x.const_data_ptr(), *pg = c.gate.const_data_ptr();
    void* stream = stream_of(c.x);
    call("adapt_gated_scan", [&] {   // (the forward pass needs no workspace)
      return g_scan(px, pg, h0, c.lengths, c.reset, c.batch, c.steps, c.channels, c.group, c.dtype, mode, s.get(),
                    out_data<void>(y), out_data<float>(h), out_data<float>(carry), nullptr, 0, stream);
    });
    return wrap({&y, &h, &carry});
  });
}

// (x, gate, dy, carry, dh_last, lengths, reset, mode, want_dh0, dx, dgate) -> (dx, dgate, dh0)
PyObject* scan_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 11, [&] {
    const ScanCall c(a[0], a[1], a[5], a[6]);
    const at::Tensor &dy = tensor(a[2]), &carry = tensor(a[3]);
    need_like(dy, c.x);
    need(carry.device() == c.x.device() && carry.scalar_type() == at::kFloat && carry.is_contiguous() && carry.dim() == 3 &&
             carry.size(0) == c.batch && carry.size(1) == c.kept() && carry.size(2) == c.channels,
         "carry: as adapt_gated_scan made it");
    const float* dh = c.state(maybe(a[4]));
    const int mode = between(a[7], INT32_MIN, INT32_MAX, "no such gate");
    const at::Tensor dx = out_like(maybe(a[9]), c.x), dgate = out_like(maybe(a[10]), c.gate);
    at::Tensor dh0, workspace;
    if (truth(a[8])) dh0 = make(c.x, {c.batch, c.channels}, at::kFloat);
    size_t bytes = 0;
    if (c.group > 1) {
      bytes = g_scan_workspace(c.batch, c.steps, c.channels, c.group, c.dtype, 1);
      if (bytes) workspace = make(c.x, {static_cast<int64_t>(bytes)}, at::kByte);
    }
    const Strides s{&c.x, &c.gate, &dy, &dx, &dgate};
    const void *px = c.x.const_data_ptr(), *pg = c.gate.const_data_ptr(), *pdy = dy.const_data_ptr();
    const float* pc = static_cast<const float*>(carry.const_data_ptr());
    void* stream = stream_of(c.x);
    call("adapt_gated_scan_backward", [&] {
      return g_scan_backward(px, pg, pdy, pc, dh, c.lengths, c.reset, c.batch, c.steps, c.channels, c.group, c.dtype, mode,
                             s.get(), out_data<void>(dx), out_data<void>(dgate), out_data<float>(dh0), out_data<void>(workspace),
                             bytes, stream);
    });
    return wrap({&dx, &dgate, &dh0});
  });
}

// (addresses of the six entry points, error)
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 7, [&] {
    void* at[6];
    for (int i = 0; i < 6; ++i) at[i] = reinterpret_cast<void*>(static_cast<uintptr_t>(bits(a[i])));
    g_dropout = reinterpret_cast<decltype(g_dropout)>(at[0]);
    g_logprobs = reinterpret_cast<decltype(g_logprobs)>(at[1]);
    g_logprobs_backward = reinterpret_cast<decltype(g_logprobs_backward)>(at[2]);
    g_scan = reinterpret_cast<decltype(g_scan)>(at[3]);
    g_scan_backward = reinterpret_cast<decltype(g_scan_backward)>(at[4]);
    g_scan_workspace = reinterpret_cast<decltype(g_scan_workspace)>(at[5]);
    Py_XDECREF(g_error);
    g_error = Py_NewRef(a[6]);
    return Py_NewRef(Py_None);
  });
}

#define ADAPT_CALL(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(name)), METH_FASTCALL, nullptr}
PyMethodDef g_methods[] = {ADAPT_CALL(dropout), ADAPT_CALL(logprobs), ADAPT_CALL(logprobs_backward), ADAPT_CALL(scan),
                           ADAPT_CALL(scan_backward), ADAPT_CALL(bind), {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_adapt_torch", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__adapt_torch() { return PyModule_Create(&g_module); }
