// The language-model operators' calls from torch tensors: checks, outputs, the current stream, and the entry
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
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>
#include <initializer_list>
#include <optional>
#include <type_traits>

#include "../../include/adapt.h"

namespace {

decltype(&adapt_dropout) g_dropout;
decltype(&adapt_token_logprobs) g_logprobs;
decltype(&adapt_token_logprobs_backward) g_logprobs_backward;
decltype(&adapt_gated_scan) g_scan;
decltype(&adapt_gated_scan_backward) g_scan_backward;
decltype(&adapt_gated_scan_workspace_bytes) g_scan_workspace;
decltype(&adapt_embedding) g_embedding;
decltype(&adapt_embedding_backward) g_embedding_backward;
decltype(&adapt_embedding_workspace_bytes) g_embedding_workspace;
decltype(&adapt_block_norm) g_norm;
decltype(&adapt_block_norm_backward) g_norm_backward;
decltype(&adapt_block_norm_workspace_bytes) g_norm_workspace;
decltype(&adapt_int8_rows) g_int8_rows;
decltype(&adapt_int8_linear) g_int8_linear;
decltype(&adapt_int8_linear_workspace_bytes) g_int8_workspace;
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
// Scratch for a call, undefined where none is needed.
at::Tensor scratch(const at::Tensor& x, size_t bytes) {
  return bytes ? make(x, {static_cast<int64_t>(bytes)}, at::kByte) : at::Tensor();
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

at::ScalarType floating(PyObject* o) {   // a torch.dtype that the operators know
  need(THPDtype_Check(o), "needs a torch.dtype");
  const at::ScalarType t = reinterpret_cast<THPDtype*>(o)->scalar_type;
  need(t == at::kFloat || t == at::kHalf || t == at::kBFloat16, "needs float32, float16 or bfloat16");
  return t;
}
int elem_of(at::ScalarType t) { return t == at::kFloat ? ADAPT_DTYPE_F32 : t == at::kHalf ? ADAPT_DTYPE_F16 : ADAPT_DTYPE_BF16; }
int64_t count(PyObject* o, const char* why) {
  int beyond = 0;
  const long long v = PyLong_AsLongLongAndOverflow(o, &beyond);
  if (v == -1 && !beyond && PyErr_Occurred()) throw Refused{nullptr};
  need(!beyond && v >= 0, why);
  return v;
}
// Tokens in order (copied where they do not lie so: a column of a batch).
at::Tensor tokens(const at::Tensor& ids, const at::Tensor& x) {
  need(ids.device() == x.device() && ids.scalar_type() == at::kLong, "tokens: an int64 tensor on the device of its partner");
  return ids.contiguous();
}
// [tokens..., dim] as rows: contiguous, or a matrix with unit inner stride.
Matrix rows_of(const at::Tensor& t, int64_t n, int64_t dim) {
  need(t.dim() >= 1 && t.size(t.dim() - 1) == dim && t.numel() == n * dim, "a row for each token");
  if (t.is_contiguous()) return {n, dim, dim};
  need(t.dim() == 2 && (dim <= 1 || t.stride(1) == 1), "needs contiguous rows, or a matrix with unit inner stride");
  return {n, dim, n > 1 ? t.stride(0) : dim};
}

// (table, ids, scale, out) -> out
PyObject* embedding(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 4, [&] {
    const at::Tensor& table = tensor(a[0]);
    const int dtype = elem(table);
    const Matrix m = matrix(table);
    const at::Tensor ids = tokens(tensor(a[1]), table);
    const int64_t* pi = static_cast<const int64_t*>(ids.const_data_ptr());
    const float scale = static_cast<float>(real(a[2]));
    at::Tensor out;
    if (const at::Tensor* given = maybe(a[3])) {
      out = *given;
      need(out.scalar_type() == table.scalar_type() && out.device() == table.device(), "out: of the table's type, on its device");
    } else {
      c10::SmallVector<int64_t, 6> sizes(ids.sizes().begin(), ids.sizes().end());
      sizes.push_back(m.cols);
      out = make(table, sizes, table.scalar_type());
    }
    const Matrix r = rows_of(out, ids.numel(), m.cols);
    const void* pt = table.const_data_ptr();
    void* stream = stream_of(table);
    call("adapt_embedding", [&] { return g_embedding(pt, m.rows, m.cols, m.ld, dtype, pi, r.rows, scale, out_data<void>(out), r.ld, stream); });
    return wrap(out);
  });
}

// (dy, ids, vocab, scale, dtype, dtable, accumulate) -> dtable
PyObject* embedding_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 7, [&] {
    const at::Tensor& dy = tensor(a[0]);
    const int dtype = elem(dy);
    need(dy.dim() >= 1, "a row for each token");
    const at::Tensor ids = tokens(tensor(a[1]), dy);
    const int64_t* pi = static_cast<const int64_t*>(ids.const_data_ptr());
    const Matrix m = rows_of(dy, ids.numel(), dy.size(dy.dim() - 1));
    const int64_t vocab = count(a[2], "the vocabulary is a whole number");
    const float scale = static_cast<float>(real(a[3]));
    const bool accumulate = truth(a[6]);
    at::Tensor grad;
    if (const at::Tensor* given = maybe(a[5])) {
      grad = *given;
      need(grad.device() == dy.device() && (grad.scalar_type() == dy.scalar_type() || grad.scalar_type() == at::kFloat),
           "dtable: of the type of dy or float32, on its device");
      need(a[4] == Py_None || floating(a[4]) == grad.scalar_type(), "dtable is of another type than asked for");
      need(grad.dim() == 2 && grad.size(0) == vocab && grad.size(1) == m.cols, "dtable: [vocab, dim]");
    } else {
      need(!accumulate, "accumulation needs a dtable");
      const at::ScalarType t = a[4] == Py_None ? dy.scalar_type() : floating(a[4]);
      grad = make(dy, {vocab, m.cols}, t);
    }
    const Matrix g = matrix(grad);
    const size_t bytes = g_embedding_workspace(m.rows, m.cols, vocab);
    const at::Tensor workspace = scratch(dy, bytes);
    const void* pd = dy.const_data_ptr();
    void* stream = stream_of(dy);
    call("adapt_embedding_backward", [&] {
      return g_embedding_backward(pd, m.rows, m.cols, m.ld, dtype, pi, vocab, scale, accumulate, out_data<void>(grad), g.ld,
                                  elem_of(grad.scalar_type()), out_data<void>(workspace), bytes, stream);
    });
    return wrap(grad);
  });
}

// What the forward and the backward call of the norms share.  The rows are the first tensor's without its last
// dimension; all are contiguous, or all are matrices with unit inner stride.
struct NormCall {
  const at::Tensor& x;
  const int dtype;
  int64_t rows, dim;
  adapt_norm_args args;
  const at::Tensor *residual, *gate;
  const float *weight_after, *weight_before;
  int64_t lines[8];
  // (block, residual, gate, weight_after, weight_before, after, before, gate_mode, scale, residual_scale, eps)
  explicit NormCall(PyObject* const* a) : x(tensor(a[0])), dtype(elem(x)), residual(maybe(a[1])), gate(maybe(a[2])) {
    need(x.dim() >= 1, "needs rows");
    dim = x.size(x.dim() - 1);
    rows = 1;
    for (int64_t d = 0; d + 1 < x.dim(); ++d) rows *= x.size(d);
    args.after = between(a[5], INT32_MIN, INT32_MAX, "no such norm");
    args.before = between(a[6], INT32_MIN, INT32_MAX, "no such norm");
    args.gate_mode = between(a[7], INT32_MIN, INT32_MAX, "no such gate");
    args.scale = static_cast<float>(real(a[8]));
    args.residual_scale = static_cast<float>(real(a[9]));
    args.eps = static_cast<float>(real(a[10]));
    args.gate_shared = gate && gate->dim() == 1 && x.dim() != 1;
    weight_after = parameter(maybe(a[3]));
    weight_before = parameter(maybe(a[4]));
    for (int64_t& v : lines) v = dim;
    lines[0] = line(x);
    if (residual) { need_like(*residual, x); lines[1] = line(*residual); }
    if (gate) {
      if (args.gate_shared) parameter(gate);
      else { need_like(*gate, x); lines[2] = line(*gate); }
    }
  }
  const float* parameter(const at::Tensor* t) const {
    if (!t) return nullptr;
    need(t->device() == x.device() && t->scalar_type() == at::kFloat && t->dim() == 1 && t->size(0) == dim && t->is_contiguous(),
         "weights and shared gates: float32 [dim], on the device of the rows");
    return static_cast<const float*>(t->const_data_ptr());
  }
  int64_t line(const at::Tensor& t) const {
    if (t.is_contiguous() || rows == 1) {
      need(dim <= 1 || t.stride(t.dim() - 1) == 1, "needs unit inner stride");
      return dim;
    }
    need(t.dim() == 2 && (dim <= 1 || t.stride(1) == 1), "needs contiguous tensors, or matrices with unit inner stride");
    return t.stride(0);
  }
  static const void* data(const at::Tensor* t) { return t ? t->const_data_ptr() : nullptr; }
};

// (..., want_y, want_normed, want_stats, y, normed) -> (y, normed, stats)
PyObject* block_norm(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 16, [&] {
    NormCall c(a);
    at::Tensor y, normed, stats;
    if (truth(a[11])) { y = out_like(maybe(a[14]), c.x); c.lines[3] = c.line(y); }
    else need(a[14] == Py_None, "y is given but not wanted");
    if (truth(a[12])) { normed = out_like(maybe(a[15]), c.x); c.lines[4] = c.line(normed); }
    else need(a[15] == Py_None, "normed is given but not wanted");
    if (truth(a[13])) stats = make(c.x, {c.rows, 4}, at::kFloat);
    const void* px = c.x.const_data_ptr();
    void* stream = stream_of(c.x);
    call("adapt_block_norm", [&] {
      return g_norm(px, NormCall::data(c.residual), NormCall::data(c.gate), c.weight_after, c.weight_before, c.rows, c.dim, c.dtype,
                    &c.args, c.lines, out_data<void>(y), out_data<void>(normed), out_data<float>(stats), stream);
    });
    return wrap({&y, &normed, &stats});
  });
}

// (..., stats, d_y, d_normed, want_block, want_residual, want_gate, want_weights, d_residual)
// -> (d_block, d_residual, d_gate, d_weight_after, d_weight_before)
PyObject* block_norm_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 19, [&] {
    NormCall c(a);
    const at::Tensor &stats = tensor(a[11]), *d_y = maybe(a[12]), *d_normed = maybe(a[13]);
    need(stats.device() == c.x.device() && stats.scalar_type() == at::kFloat && stats.is_contiguous() && stats.dim() == 2 &&
             stats.size(0) == c.rows && stats.size(1) == 4, "stats: as adapt_block_norm made them");
    if (d_y) { need_like(*d_y, c.x); c.lines[3] = c.line(*d_y); }
    if (d_normed) { need_like(*d_normed, c.x); c.lines[4] = c.line(*d_normed); }
    at::Tensor d_block, d_residual, d_gate, d_after, d_before;
    if (truth(a[14])) d_block = make_like(c.x);
    if (truth(a[15]) && c.residual) { d_residual = out_like(maybe(a[18]), c.x); c.lines[6] = c.line(d_residual); }
    else need(a[18] == Py_None, "d_residual is given but there is none");
    if (truth(a[16]) && c.gate) d_gate = c.args.gate_shared ? make(c.x, {c.dim}, at::kFloat) : make_like(c.x);
    const bool weights = truth(a[17]);
    if (weights && c.weight_after) d_after = make(c.x, {c.dim}, at::kFloat);
    if (weights && c.weight_before && d_normed) d_before = make(c.x, {c.dim}, at::kFloat);
    size_t bytes = 0;
    if (d_after.defined() || d_before.defined() || (d_gate.defined() && c.args.gate_shared)) bytes = g_norm_workspace(c.rows, c.dim);
    const at::Tensor workspace = scratch(c.x, bytes);
    const void* px = c.x.const_data_ptr();
    const float* ps = static_cast<const float*>(stats.const_data_ptr());
    void* stream = stream_of(c.x);
    call("adapt_block_norm_backward", [&] {
      return g_norm_backward(px, NormCall::data(c.residual), NormCall::data(c.gate), c.weight_after, c.weight_before, ps,
                             NormCall::data(d_y), NormCall::data(d_normed), c.rows, c.dim, c.dtype, &c.args, c.lines,
                             out_data<void>(d_block), out_data<void>(d_residual), out_data<void>(d_gate), out_data<float>(d_after),
                             out_data<float>(d_before), out_data<void>(workspace), bytes, stream);
    });
    return wrap({&d_block, &d_residual, &d_gate, &d_after, &d_before});
  });
}

// (x, codes, scales) -> (codes, scales)
PyObject* int8_rows(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 3, [&] {
    const at::Tensor& x = tensor(a[0]);
    const int dtype = elem(x);
    const Matrix m = matrix(x);
    const at::Tensor *given = maybe(a[1]), *given_scales = maybe(a[2]);
    const at::Tensor codes = given ? *given : make(x, x.sizes(), at::kChar);
    need(codes.scalar_type() == at::kChar && codes.device() == x.device() && codes.sizes() == x.sizes(), "codes: int8, of the shape of x, on its device");
    const at::Tensor scales = given_scales ? *given_scales : make(x, {m.rows}, at::kFloat);
    per_row(&scales, x, at::kFloat);
    const Matrix c = matrix(codes);
    const void* px = x.const_data_ptr();
    void* stream = stream_of(x);
    call("adapt_int8_rows", [&] {
      return g_int8_rows(px, m.rows, m.cols, m.ld, dtype, out_data<int8_t>(codes), c.ld, out_data<float>(scales), stream);
    });
    return wrap({&codes, &scales});
  });
}

// (x, weight, weight_scales, x_scales, bias, dtype, out) -> out
PyObject* int8_linear(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 7, [&] {
    const at::Tensor &x = tensor(a[0]), &w = tensor(a[1]), &ws = tensor(a[2]);
    const at::Tensor *xs = maybe(a[3]), *bias = maybe(a[4]), *given = maybe(a[6]);
    const bool coded = x.scalar_type() == at::kChar;
    need(x.is_cuda() && (!coded || x.get_device() == c10::cuda::current_device()), "needs CUDA tensors on the current device");
    const int x_dtype = coded ? ADAPT_DTYPE_I8 : elem(x);
    need(w.device() == x.device() && w.scalar_type() == at::kChar, "the weights are int8, on the device of x");
    const Matrix m = matrix(x), mw = matrix(w);
    need(mw.cols == m.cols, "x and the weights have the same number of columns");
    auto scales = [&](const at::Tensor& t, int64_t most) {
      need(t.device() == x.device() && t.scalar_type() == at::kFloat && t.is_contiguous() && t.dim() <= 1 && (t.numel() == 1 || t.numel() == most),
           "scales: contiguous float32, one for all or one for each row, on the device of x");
      return static_cast<const float*>(t.const_data_ptr());
    };
    need(coded == (xs != nullptr), "codes come with their scales, other types without");
    const float *pws = scales(ws, mw.rows), *pxs = xs ? scales(*xs, m.rows) : nullptr;
    const float* pb = nullptr;
    if (bias) {
      need(bias->device() == x.device() && bias->scalar_type() == at::kFloat && bias->is_contiguous() && bias->dim() == 1 && bias->size(0) == mw.rows,
           "bias: float32, one for each row of the weights, on the device of x");
      pb = static_cast<const float*>(bias->const_data_ptr());
    }
    at::Tensor out;
    if (given) {
      out = *given;
      need(out.device() == x.device() && out.dim() == 2 && out.size(0) == m.rows && out.size(1) == mw.rows, "out: [rows, channels], on the device of x");
      need(a[5] == Py_None || floating(a[5]) == out.scalar_type(), "out is of another type than asked for");
    } else {
      const at::ScalarType t = a[5] != Py_None ? floating(a[5]) : coded ? at::kFloat : x.scalar_type();
      out = make(x, {m.rows, mw.rows}, t);
    }
    const int dtype = elem(out);
    const Matrix o = matrix(out);
    const void *px = x.const_data_ptr();
    const int8_t* pw = static_cast<const int8_t*>(w.const_data_ptr());
    const size_t bytes = g_int8_workspace(px, x_dtype, pw, m.rows, mw.rows, m.cols, m.ld, mw.ld);
    const at::Tensor workspace = scratch(x, bytes);
    const int64_t xn = xs ? xs->numel() : 0, wn = ws.numel();
    void* stream = stream_of(x);
    call("adapt_int8_linear", [&] {
      return g_int8_linear(px, x_dtype, pxs, xn, pw, pws, wn, pb, m.rows, mw.rows, m.cols, m.ld, mw.ld, out_data<void>(out), o.ld, dtype,
                           out_data<void>(workspace), bytes, stream);
    });
    return wrap(out);
  });
}

// Entry points' addresses in the order of binding.py, then the error.
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 16, [&] {
    int i = 0;
    auto take = [&](auto& f) { f = reinterpret_cast<std::remove_reference_t<decltype(f)>>(static_cast<uintptr_t>(bits(a[i++]))); };
    take(g_dropout); take(g_logprobs); take(g_logprobs_backward); take(g_scan); take(g_scan_backward); take(g_scan_workspace);
    take(g_embedding); take(g_embedding_backward); take(g_embedding_workspace);
    take(g_norm); take(g_norm_backward); take(g_norm_workspace);
    take(g_int8_rows); take(g_int8_linear); take(g_int8_workspace);
    Py_XDECREF(g_error);
    g_error = Py_NewRef(a[i]);
    return Py_NewRef(Py_None);
  });
}

#define ADAPT_CALL(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(name)), METH_FASTCALL, nullptr}
PyMethodDef g_methods[] = {ADAPT_CALL(dropout), ADAPT_CALL(logprobs), ADAPT_CALL(logprobs_backward), ADAPT_CALL(scan),
                           ADAPT_CALL(scan_backward), ADAPT_CALL(embedding),
                           ADAPT_CALL(embedding_backward), ADAPT_CALL(block_norm), ADAPT_CALL(block_norm_backward),
                           ADAPT_CALL(int8_rows), ADAPT_CALL(int8_linear), ADAPT_CALL(bind), {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_adapt_torch", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__adapt_torch() { return PyModule_Create(&g_module); }
