// The operators of include/lstm_approx_ops.h on torch tensors: checks of the
// tensors, allocation of what is not passed in, the call on torch's current
// stream.  _operators.py holds the functions that users call and their
// documentation; this file is the part that every call pays for.  (Through
// ctypes a single step took 15.6 us of host time a call, from here 4.1, for a
// kernel of about 2.)
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <cmath>
#include <optional>
#include <stdexcept>
#include <string>
#include <utility>
#include <vector>

#include "../../include/lstm_approx_ops.h"

namespace {

using at::Tensor;

struct Invalid : std::runtime_error {
  using std::runtime_error::runtime_error;
};
[[noreturn]] void invalid(const std::string& text) { throw Invalid(text); }
void need(bool ok, const char* text) {
  if (!ok) invalid(text);
}

PyObject* g_error = nullptr;  // LSTMApproxError

// An error of the library as its Python exception.
struct Failed {
  int code;
  std::string text;
};

template <typename F>
PyObject* guarded(F f) {
  HANDLE_TH_ERRORS
  try {
    return f();
  } catch (const Invalid& e) {
    PyErr_SetString(PyExc_ValueError, e.what());
  } catch (const Failed& e) {
    PyObject* value = PyObject_CallFunction(g_error, "is", e.code, e.text.c_str());
    if (value) {
      PyErr_SetObject(g_error, value);
      Py_DECREF(value);
    }
  }
  return nullptr;
  END_HANDLE_TH_ERRORS
}

const Tensor& tensor(PyObject* o, const char* name) {
  if (!THPVariable_Check(o)) invalid(std::string(name) + " must be a tensor");
  return THPVariable_Unpack(o);
}
long long integer(PyObject* o) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) {
    PyErr_Clear();
    invalid("a whole number was expected");
  }
  return v;
}
float real(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) {
    PyErr_Clear();
    invalid("a number was expected");
  }
  return (float)v;
}

int float_code(at::ScalarType t) {
  return t == at::kFloat      ? LSTM_APPROX_OP_FP32
         : t == at::kBFloat16 ? LSTM_APPROX_OP_BF16
         : t == at::kHalf     ? LSTM_APPROX_OP_FP16
                              : -1;
}
int float_code(const Tensor& t, const char* name) {
  const int c = float_code(t.scalar_type());
  if (c < 0) invalid(std::string(name) + " must be float32, bfloat16 or float16, not " + toString(t.scalar_type()));
  return c;
}

// What every tensor of a call is held against.
struct Call {
  c10::Device device;
  c10::cuda::OptionalCUDAGuard guard;
  void* stream;
  char msg[256];

  explicit Call(const Tensor& first, const char* name) : device(first.device()), stream(nullptr) {
    if (!first.is_cuda()) invalid(std::string(name) + " must be a CUDA tensor");
    guard.set_device(device);
    stream = c10::cuda::getCurrentCUDAStream(device.index()).stream();
    msg[0] = '\0';
  }
  // The address of a tensor of this device, type and shape whose last axis is contiguous.
  void* rows(const Tensor& t, const char* name, at::ScalarType type, at::IntArrayRef shape) const {
    if (t.scalar_type() != type)
      invalid(std::string(name) + " must be " + toString(type) + ", not " + toString(t.scalar_type()));
    if (t.sizes() != shape) invalid(std::string(name) + " has the wrong shape");
    if (t.device() != device) invalid(std::string(name) + " must be on the CUDA device of the other tensors");
    if (t.dim() > 0 && t.size(-1) > 1 && t.stride(-1) != 1) invalid(std::string(name) + "'s last axis must be contiguous");
    return t.data_ptr();
  }
  // That of a contiguous one.
  void* dense(const Tensor& t, const char* name, at::ScalarType type, at::IntArrayRef shape) const {
    void* p = rows(t, name, type, shape);
    if (!t.is_contiguous()) invalid(std::string(name) + " must be contiguous");
    return p;
  }
  void* dense(PyObject* o, const char* name, at::ScalarType type, at::IntArrayRef shape) const {
    return o == Py_None ? nullptr : dense(tensor(o, name), name, type, shape);
  }
  // A tensor of the caller that the call writes to: torch counts its changes.
  static void written(const Tensor& t) {
    if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
  }
  // The caller's tensor, or a new one.
  Tensor out(PyObject* o, const char* name, at::ScalarType type, at::IntArrayRef shape) const {
    if (o == Py_None) return at::empty(shape, at::TensorOptions().dtype(type).device(device));
    const Tensor& t = tensor(o, name);
    dense(t, name, type, shape);
    written(t);
    return t;
  }
  // The caller's workspace (its bytes are checked by the library), or a new one.
  Tensor workspace(PyObject* o, size_t bytes) const {
    if (o == Py_None)
      return at::empty({(int64_t)std::max<size_t>(bytes, 16)}, at::TensorOptions().dtype(at::kByte).device(device));
    const Tensor& t = tensor(o, "workspace");
    if (t.device() != device || !t.is_contiguous()) invalid("workspace must be a contiguous tensor of the same device");
    return t;
  }
  void done(int rc) const {
    if (rc != LSTM_APPROX_OK) throw Failed{rc, msg};
  }
};

// The element pitch of the rows of t [..., D], which lie at one pitch (no rows: at any).
long long pitch_of(const Tensor& t, const char* name) {
  if (t.numel() == 0) return t.size(-1);
  long long pitch = -1, span = 0;
  for (int64_t k = t.dim() - 2; k >= 0; --k) {
    if (t.size(k) == 1) continue;
    if (pitch < 0) pitch = span = t.stride(k);
    else if (t.stride(k) != span) invalid(std::string(name) + "'s rows must lie at one pitch");
    span *= t.size(k);
  }
  return pitch < 0 ? t.size(-1) : pitch;
}

PyObject* wrap(const Tensor& t) { return THPVariable_Wrap(t); }
template <typename... Ts>
PyObject* wrap_all(const Ts&... ts) {
  PyObject* tuple = PyTuple_New(sizeof...(ts));
  if (!tuple) return nullptr;
  Py_ssize_t k = 0;
  bool ok = true;
  auto put = [&](const std::optional<Tensor>& t) {
    PyObject* o = t ? wrap(*t) : (Py_INCREF(Py_None), Py_None);
    ok = ok && o;
    PyTuple_SET_ITEM(tuple, k++, o);
  };
  (put(std::optional<Tensor>(ts)), ...);
  if (ok) return tuple;
  Py_DECREF(tuple);
  return nullptr;
}

// A 16-bit sum of rms_norm that a backward pass will read carries what its rounding took off as its attribute `sum_low`.
// It belongs to that one call: beside it stand the version that the sum had then and the call's rstd with its version
// (a tuple).  It counts for the backward pass of that rstd only: another norm of the same sum, without a residual, read
// the rounded values.  After a change of either in place, by torch or by an operator here, it no longer counts.  (A
// change that torch does not see does little: a low part moves a value by half a unit in the last place of the 16-bit
// type at most.)
PyObject *g_sum_low = nullptr, *g_sum_low_call = nullptr;

bool set_sum_low(PyObject* sum, const Tensor& t, const std::optional<Tensor>& low, PyObject* rstd) {
  if (!low) {  // an earlier call's
    for (PyObject* name : {g_sum_low, g_sum_low_call})
      if (PyObject_HasAttr(sum, name) && PyObject_DelAttr(sum, name) != 0) return false;
    return true;
  }
  PyObject* v = wrap(*low);
  PyObject* call = v ? Py_BuildValue("LOL", (long long)t._version(), rstd, (long long)tensor(rstd, "rstd")._version()) : nullptr;
  const bool ok = call && PyObject_SetAttr(sum, g_sum_low, v) == 0 && PyObject_SetAttr(sum, g_sum_low_call, call) == 0;
  Py_XDECREF(v);
  Py_XDECREF(call);
  return ok;
}
// Whether the call noted beside the low part left the sum t and this rstd, both unchanged since.
bool is_sum_low_call(PyObject* call, const Tensor& t, const Tensor& rstd) {
  if (!call || !PyTuple_Check(call) || PyTuple_GET_SIZE(call) != 3) return false;
  PyObject *version = PyTuple_GET_ITEM(call, 0), *of = PyTuple_GET_ITEM(call, 1), *of_version = PyTuple_GET_ITEM(call, 2);
  if (!PyLong_Check(version) || !THPVariable_Check(of) || !PyLong_Check(of_version)) return false;
  const Tensor& r = THPVariable_Unpack(of);
  return PyLong_AsLongLong(version) == (long long)t._version() && !r.is_inference() &&
         PyLong_AsLongLong(of_version) == (long long)r._version() && rstd.is_alias_of(r) && rstd.data_ptr() == r.data_ptr();
}
std::optional<Tensor> get_sum_low(PyObject* sum, const Tensor& t, const Tensor& rstd) {
  std::optional<Tensor> found;
  if (t.is_inference() || !PyObject_HasAttr(sum, g_sum_low)) return found;
  PyObject *v = PyObject_GetAttr(sum, g_sum_low), *call = PyObject_GetAttr(sum, g_sum_low_call);
  if (v && THPVariable_Check(v) && is_sum_low_call(call, t, rstd)) {
    const Tensor& low = THPVariable_Unpack(v);
    if (low.scalar_type() == at::kShort && low.sizes() == t.sizes() && low.device() == t.device() &&
        low.is_contiguous() && t.is_contiguous())
      found = low;
  }
  Py_XDECREF(v);
  Py_XDECREF(call);
  PyErr_Clear();
  return found;
}

// rms_norm(x, weight, residual, eps, group, out, scales, residual_out, rstd, sum_low) -> (out, scales, residual_out)
// (sum_low: None where it is made as needed, False, or the tensor for it)
PyObject* rms_norm(PyObject*, PyObject* const* a, Py_ssize_t) {
  return guarded([&]() -> PyObject* {
    const Tensor& x = tensor(a[0], "x");
    Call call(x, "x");
    const int code = float_code(x, "x");
    need(x.dim() >= 1 && x.size(-1) >= 1, "x must be [..., D]");
    const auto type = x.scalar_type();
    const auto shape = x.sizes(), lead = shape.slice(0, shape.size() - 1);
    const int64_t D = x.size(-1), rows = x.numel() / D;
    const long long group = integer(a[4]);
    void* px = call.rows(x, "x", type, shape);
    const long long pitch = pitch_of(x, "x");
    const void* pw = call.dense(tensor(a[1], "weight"), "weight", at::kFloat, {D});
    void* pr = nullptr;
    long long res_pitch = 0;
    std::optional<Tensor> total, scales;
    if (a[2] != Py_None) {
      const Tensor& r = tensor(a[2], "residual");
      pr = call.rows(r, "residual", type, shape);
      res_pitch = pitch_of(r, "residual");
    }
    float* rstd = static_cast<float*>(call.dense(a[8], "rstd", at::kFloat, lead));
    if (rstd) Call::written(tensor(a[8], "rstd"));
    need(D <= 0x7fffffff && group <= 0x7fffffff && group >= 0, "D and group must be 32-bit numbers");
    if (a[2] != Py_None || a[7] != Py_None) total = call.out(a[7], "residual_out", type, shape);
    if (group > 0) {
      auto sizes = lead.vec();
      sizes.push_back(group >= D ? 1 : (D + group - 1) / group);
      scales = call.out(a[6], "scales", at::kFloat, sizes);
    }
    Tensor out = call.out(a[5], "out", group > 0 ? at::kFloat8_e4m3fn : type, shape);
    std::optional<Tensor> low;
    if (a[9] == Py_None) {  // where a backward pass will follow (rstd is asked for) and s has more than 16 bits
      if (a[2] != Py_None && a[8] != Py_None && group == 0 && type != at::kFloat && !total->is_inference() &&
          !tensor(a[8], "rstd").is_inference())
        low = call.out(Py_None, "", at::kShort, shape);
    } else if (a[9] != Py_False) {
      need(total && type != at::kFloat && group == 0, "sum_low is for the 16-bit sum of x and a residual");
      low = call.out(a[9], "sum_low", at::kShort, shape);
    }
    call.done(lstm_approx_rms_norm(code, (int)group, px, pitch, pr, res_pitch, static_cast<const float*>(pw), real(a[3]),
                                   rows, (int)D, out.data_ptr(), scales ? scales->data_ptr<float>() : nullptr,
                                   total ? total->data_ptr() : nullptr, low ? low->data_ptr<int16_t>() : nullptr, rstd,
                                   call.stream, call.msg, sizeof(call.msg)));
    PyObject* result = wrap_all(out, scales, total);
    // one that the caller handed over without an rstd is the caller's alone
    if (low && (a[8] == Py_None || total->is_inference() || tensor(a[8], "rstd").is_inference())) low.reset();
    if (result && total && !set_sum_low(PyTuple_GET_ITEM(result, 2), *total, low, a[8])) Py_CLEAR(result);
    return result;
  });
}

// rms_norm_backward(dy, s, weight, rstd, dsum, dx, dweight, workspace, sum_low) -> (dx, dweight)
// (sum_low: None where s brings its own along, False, or that of the forward call)
PyObject* rms_norm_backward(PyObject*, PyObject* const* a, Py_ssize_t) {
  return guarded([&]() -> PyObject* {
    const Tensor& dy = tensor(a[0], "dy");
    Call call(dy, "dy");
    const int code = float_code(dy, "dy");
    need(dy.dim() >= 1 && dy.size(-1) >= 1, "dy must be [..., D]");
    const auto type = dy.scalar_type();
    const auto shape = dy.sizes(), lead = shape.slice(0, shape.size() - 1);
    const int64_t D = dy.size(-1), rows = dy.numel() / D;
    need(D <= 0x7fffffff, "D must be a 32-bit number");
    const Tensor& s = tensor(a[1], "s");
    void *pdy = call.rows(dy, "dy", type, shape), *ps = call.rows(s, "s", type, shape), *pd = nullptr;
    const Tensor& rs = tensor(a[3], "rstd");
    std::optional<Tensor> low;
    if (a[8] == Py_None) {
      if (type != at::kFloat) low = get_sum_low(a[1], s, rs);
    } else if (a[8] != Py_False) {
      need(type != at::kFloat, "sum_low is for 16-bit sums");
      low = tensor(a[8], "sum_low");
      call.dense(*low, "sum_low", at::kShort, shape);
    }
    if (low) low->record_stream(c10::Stream(c10::cuda::getCurrentCUDAStream(call.device.index())));
    long long d_pitch = 0;
    if (a[4] != Py_None) {
      const Tensor& d = tensor(a[4], "dsum");
      pd = call.rows(d, "dsum", type, shape);
      d_pitch = pitch_of(d, "dsum");
    }
    const float* w = static_cast<const float*>(call.dense(tensor(a[2], "weight"), "weight", at::kFloat, {D}));
    const float* rstd = static_cast<const float*>(call.dense(rs, "rstd", at::kFloat, lead));
    Tensor dx = call.out(a[5], "dx", type, shape), dw = call.out(a[6], "dweight", at::kFloat, {D});
    Tensor ws = call.workspace(a[7], lstm_approx_rms_norm_workspace_bytes(rows, (int)D));
    call.done(lstm_approx_rms_norm_backward(code, pdy, pitch_of(dy, "dy"), ps, pitch_of(s, "s"),
                                            low ? low->data_ptr<int16_t>() : nullptr, w, rstd, pd, d_pitch, rows, (int)D,
                                            dx.data_ptr(), dw.data_ptr<float>(), ws.data_ptr(), ws.nbytes(),
                                            call.stream, call.msg, sizeof(call.msg)));
    return wrap_all(dx, dw);
  });
}

// x, r, i and what goes with them in the scan's calls.
struct Sequence {
  int code;
  at::ScalarType type;
  at::IntArrayRef shape;
  int64_t T, B, D, chunks;
  const int32_t* lengths;
  const unsigned char* reset;

  Sequence(const Call& call, const Tensor& x, PyObject* lengths_, PyObject* reset_)
      : code(float_code(x, "x")), type(x.scalar_type()), shape(x.sizes()) {
    need(x.dim() == 3, "x must be [T, B, D]");
    T = x.size(0);
    B = x.size(1);
    D = x.size(2);
    need(T <= 0x7fffffff && B <= 0x7fffffff && D <= 0x7fffffff && D >= 1, "D must not be zero, sizes 32-bit numbers");
    chunks = (T + LSTM_APPROX_SCAN_CHUNK - 1) / LSTM_APPROX_SCAN_CHUNK;
    lengths = static_cast<const int32_t*>(call.dense(lengths_, "lengths", at::kInt, {B}));
    reset = resets(call, reset_, {T, B});
  }
  static const unsigned char* resets(const Call& call, PyObject* o, at::IntArrayRef shape) {
    if (o == Py_None) return nullptr;
    const Tensor& t = tensor(o, "reset");
    return static_cast<const unsigned char*>(
        call.dense(t, "reset", t.scalar_type() == at::kByte ? at::kByte : at::kBool, shape));
  }
  // A tensor of the sequence's shape with any t and b strides: its address, its strides appended.
  void* add(const Call& call, const Tensor& t, const char* name, long long* strides, int& n) const {
    void* p = call.rows(t, name, type, shape);
    strides[n++] = t.stride(0);
    strides[n++] = t.stride(1);
    return p;
  }
};
Tensor sequence_out(const Call& call, const Sequence& q, PyObject* o, const char* name) {
  if (o == Py_None) return call.out(o, name, q.type, q.shape);
  Call::written(tensor(o, name));
  return tensor(o, name);
}

// gated_scan(x, r, i, decay, h0, c, lengths, reset, y, h_last, states, workspace) -> (y, h_last)
PyObject* gated_scan(PyObject*, PyObject* const* a, Py_ssize_t) {
  return guarded([&]() -> PyObject* {
    const Tensor& x = tensor(a[0], "x");
    Call call(x, "x");
    Sequence q(call, x, a[6], a[7]);
    long long strides[8];
    int n = 0;
    void* px = q.add(call, x, "x", strides, n);
    void* pr = q.add(call, tensor(a[1], "r"), "r", strides, n);
    void* pi = q.add(call, tensor(a[2], "i"), "i", strides, n);
    const float* decay = static_cast<const float*>(call.dense(tensor(a[3], "decay"), "decay", at::kFloat, {q.D}));
    const float* h0 = static_cast<const float*>(call.dense(a[4], "h0", at::kFloat, {q.B, q.D}));
    float* states = static_cast<float*>(call.dense(a[10], "states", at::kFloat, {q.chunks, q.B, q.D}));
    if (states) Call::written(tensor(a[10], "states"));
    Tensor y = sequence_out(call, q, a[8], "y"), last = call.out(a[9], "h_last", at::kFloat, {q.B, q.D});
    void* py = q.add(call, y, "y", strides, n);
    Tensor ws = call.workspace(a[11], lstm_approx_gated_scan_workspace_bytes((int)q.T, (int)q.B, (int)q.D));
    call.done(lstm_approx_gated_scan(q.code, px, pr, pi, decay, real(a[5]), h0, q.lengths, q.reset, (int)q.T, (int)q.B,
                                     (int)q.D, py, strides, last.data_ptr<float>(), states, ws.data_ptr(), ws.nbytes(),
                                     call.stream, call.msg, sizeof(call.msg)));
    return wrap_all(y, last);
  });
}

// gated_scan_backward(dy, x, r, i, decay, states, dh_last, c, lengths, reset, dx, dr, di, ddecay, dh0, workspace)
//   -> (dx, dr, di, ddecay, dh0)
PyObject* gated_scan_backward(PyObject*, PyObject* const* a, Py_ssize_t) {
  return guarded([&]() -> PyObject* {
    const Tensor& x = tensor(a[1], "x");
    Call call(x, "x");
    Sequence q(call, x, a[8], a[9]);
    long long strides[14];
    int n = 0;
    void* pdy = q.add(call, tensor(a[0], "dy"), "dy", strides, n);
    void* px = q.add(call, x, "x", strides, n);
    void* pr = q.add(call, tensor(a[2], "r"), "r", strides, n);
    void* pi = q.add(call, tensor(a[3], "i"), "i", strides, n);
    const float* decay = static_cast<const float*>(call.dense(tensor(a[4], "decay"), "decay", at::kFloat, {q.D}));
    const float* states = static_cast<const float*>(
        call.dense(tensor(a[5], "states"), "states", at::kFloat, {q.chunks, q.B, q.D}));
    const float* dl = static_cast<const float*>(call.dense(a[6], "dh_last", at::kFloat, {q.B, q.D}));
    Tensor dx = sequence_out(call, q, a[10], "dx"), dr = sequence_out(call, q, a[11], "dr");
    Tensor di = sequence_out(call, q, a[12], "di");
    void* pdx = q.add(call, dx, "dx", strides, n);
    void* pdr = q.add(call, dr, "dr", strides, n);
    void* pdi = q.add(call, di, "di", strides, n);
    Tensor dd = call.out(a[13], "ddecay", at::kFloat, {q.D}), dh0 = call.out(a[14], "dh0", at::kFloat, {q.B, q.D});
    Tensor ws = call.workspace(a[15], lstm_approx_gated_scan_workspace_bytes((int)q.T, (int)q.B, (int)q.D));
    call.done(lstm_approx_gated_scan_backward(q.code, pdy, dl, px, pr, pi, decay, real(a[7]), states, q.lengths, q.reset,
                                              (int)q.T, (int)q.B, (int)q.D, pdx, pdr, pdi, strides, dd.data_ptr<float>(),
                                              dh0.data_ptr<float>(), ws.data_ptr(), ws.nbytes(), call.stream, call.msg,
                                              sizeof(call.msg)));
    return wrap_all(dx, dr, di, dd, dh0);
  });
}

// gated_step(x, r, i, decay, state, c, slots, reset, y) -> y
PyObject* gated_step(PyObject*, PyObject* const* a, Py_ssize_t) {
  return guarded([&]() -> PyObject* {
    const Tensor &x = tensor(a[0], "x"), &r = tensor(a[1], "r"), &i = tensor(a[2], "i"), &state = tensor(a[4], "state");
    Call call(x, "x");
    const int code = float_code(x, "x");
    need(x.dim() == 2 && state.dim() == 2 && x.size(1) >= 1, "x must be [B, D] and state [n_slots, D]");
    const auto type = x.scalar_type();
    const auto shape = x.sizes();
    const int64_t B = x.size(0), D = x.size(1), slots = state.size(0);
    need(B <= 0x7fffffff && D <= 0x7fffffff && slots <= 0x7fffffff, "sizes must be 32-bit numbers");
    void *px = call.rows(x, "x", type, shape), *pr = call.rows(r, "r", type, shape), *pi = call.rows(i, "i", type, shape);
    const float* decay = static_cast<const float*>(call.dense(tensor(a[3], "decay"), "decay", at::kFloat, {D}));
    float* ps = static_cast<float*>(call.dense(state, "state", at::kFloat, {slots, D}));
    Call::written(state);
    const int32_t* at_slots = static_cast<const int32_t*>(call.dense(a[6], "slots", at::kInt, {B}));
    const unsigned char* reset = Sequence::resets(call, a[7], {B});
    Tensor y = call.out(a[8], "y", type, shape);
    call.done(lstm_approx_gated_step(code, px, x.stride(0), pr, r.stride(0), pi, i.stride(0), decay, real(a[5]), ps,
                                     (int)slots, at_slots, reset, (int)B, (int)D, y.data_ptr(), call.stream, call.msg,
                                     sizeof(call.msg)));
    return wrap(y);
  });
}

// w4_quantize(w, group, q, scale, zero): fills the last three
PyObject* w4_quantize(PyObject*, PyObject* const* a, Py_ssize_t) {
  return guarded([&]() -> PyObject* {
    const Tensor &w = tensor(a[0], "w"), &q = tensor(a[2], "q"), &scale = tensor(a[3], "scale"), &zero = tensor(a[4], "zero");
    Call call(w, "w");
    const int code = float_code(w, "w");
    void* pw = call.rows(w, "w", w.scalar_type(), w.sizes());
    need(w.size(0) <= 0x7fffffff && w.size(1) <= 0x7fffffff, "sizes must be 32-bit numbers");
    call.done(lstm_approx_w4_quantize(code, pw, w.stride(0), (int)w.size(0), (int)w.size(1), (int)integer(a[1]),
                                      q.data_ptr<uint8_t>(), q.size(1), scale.data_ptr(), float_code(scale, "scale"),
                                      zero.data_ptr<uint8_t>(), call.stream, call.msg, sizeof(call.msg)));
    Py_RETURN_NONE;
  });
}

// w4_matvec(x, q, scale, zero, K, group, pitch, x_scale, bias, out, out_dtype, workspace) -> out  (out_dtype: an operator code or -1;
// q, scale and zero have been checked against one another)
PyObject* w4_matvec(PyObject*, PyObject* const* a, Py_ssize_t) {
  return guarded([&]() -> PyObject* {
    const Tensor &x = tensor(a[0], "x"), &q = tensor(a[1], "q"), &scale = tensor(a[2], "scale");
    Call call(x, "x");
    need(q.device() == call.device, "x must be on w's device");
    const int64_t K = integer(a[4]), N = q.size(0);
    const auto type = x.scalar_type();
    const bool x8 = type == at::kFloat8_e4m3fn;
    const int code = x8 ? LSTM_APPROX_OP_E4M3 : float_code(x, "x");
    need(x.dim() >= 1 && x.size(-1) == K, "x must be [..., K]");
    const int64_t M = x.numel() / K;
    need(M <= 0x7fffffff && N <= 0x7fffffff, "sizes must be 32-bit numbers");
    void* px = call.rows(x, "x", type, x.sizes());
    auto sizes = x.sizes().vec();
    const float* x_scale = nullptr;
    int x_group = 0;
    if (x8) {
      need(a[7] != Py_None, "8-bit x needs x_scale");
      const Tensor& s = tensor(a[7], "x_scale");
      const int64_t groups = s.dim() >= 1 ? s.size(-1) : 0;
      need(groups == 1 || groups == (K + 127) / 128, "x_scale must be [..., 1] or [..., ceil(K / 128)]");
      x_group = groups == 1 ? (int)K : 128;
      sizes.back() = groups;
      x_scale = static_cast<const float*>(call.dense(s, "x_scale", at::kFloat, sizes));
    } else {
      need(a[7] == Py_None, "x_scale is for 8-bit x");
    }
    const float* bias = static_cast<const float*>(call.dense(a[8], "bias", at::kFloat, {N}));
    sizes.back() = N;
    const long long wanted = integer(a[10]);
    const at::ScalarType out_type = a[9] != Py_None ? tensor(a[9], "out").scalar_type()
                                    : wanted == LSTM_APPROX_OP_FP32 ? at::kFloat
                                    : wanted == LSTM_APPROX_OP_BF16 ? at::kBFloat16
                                    : wanted == LSTM_APPROX_OP_FP16 ? at::kHalf
                                    : x8                            ? at::kBFloat16
                                                                    : type;
    const int out_code = float_code(out_type);
    need(out_code >= 0, "out must be float32, bfloat16 or float16");
    Tensor out = call.out(a[9], "out", out_type, sizes);
    std::optional<Tensor> ws;
    const size_t bytes = lstm_approx_w4_workspace_bytes(code, (int)M, (int)K);
    if (bytes > 0) ws = call.workspace(a[11], bytes);
    call.done(lstm_approx_w4_matvec(code, px, pitch_of(x, "x"), x_scale, x_group, q.data_ptr<uint8_t>(), integer(a[6]),
                                    scale.data_ptr(), float_code(scale, "scale"),
                                    a[3] == Py_None ? nullptr : tensor(a[3], "zero").data_ptr<uint8_t>(), bias, (int)M,
                                    (int)N, (int)K, (int)integer(a[5]), out.data_ptr(), out_code, ws ? ws->data_ptr() : nullptr,
                                    ws ? ws->nbytes() : 0, call.stream, call.msg, sizeof(call.msg)));
    return wrap(out);
  });
}

// q, k, v, g and beta of the delta rule's calls; `lead`: the axes before the heads (T and B, or B).
struct Heads {
  int code;
  at::ScalarType type;
  std::vector<int64_t> lead;
  int64_t H, Hk, Dk, Dv;

  Heads(const Call& call, const Tensor& q, const Tensor& v, int64_t axes)
      : code(float_code(q, "q")), type(q.scalar_type()) {
    need(q.dim() == axes + 2 && v.dim() == axes + 2,
         axes == 2 ? "q must be [T, B, Hk, Dk] and v [T, B, H, Dv]" : "q must be [B, Hk, Dk] and v [B, H, Dv]");
    lead = q.sizes().slice(0, axes).vec();
    Hk = q.size(axes), Dk = q.size(axes + 1), H = v.size(axes), Dv = v.size(axes + 1);
    for (int64_t n : lead) need(n <= 0x7fffffff, "sizes must be 32-bit numbers");
    need(Hk <= 0x7fffffff && Dk <= 0x7fffffff && H <= 0x7fffffff && Dv <= 0x7fffffff, "sizes must be 32-bit numbers");
    need(Hk >= 1 && H >= 1 && H % Hk == 0, "v's heads must be a multiple of q's");
    need(Dk >= 1 && Dv >= 1, "Dk and Dv must not be zero");
  }
  std::vector<int64_t> shape(bool keys) const {
    std::vector<int64_t> s = lead;
    s.push_back(keys ? Hk : H);
    s.push_back(keys ? Dk : Dv);
    return s;
  }
  std::vector<int64_t> per_head() const {
    std::vector<int64_t> s = lead;
    s.push_back(H);
    return s;
  }
  // A tensor of q's or v's shape (any strides but the last axis's): its address, its strides appended.
  void* add(const Call& call, const Tensor& t, const char* name, bool keys, long long* strides, int& n) const {
    void* p = call.rows(t, name, type, shape(keys));
    for (size_t k = 0; k <= lead.size(); ++k) strides[n++] = t.stride(k);
    return p;
  }
  // One of g's shape.
  float* add_gate(const Call& call, const Tensor& t, const char* name, long long* strides, int& n) const {
    void* p = call.rows(t, name, at::kFloat, per_head());
    for (size_t k = 0; k < lead.size(); ++k) strides[n++] = t.stride(k);
    return static_cast<float*>(p);
  }
  // The caller's tensor of any strides, no value of it at two places, or a new one.
  static Tensor out(const Call& call, PyObject* o, const char* name, at::ScalarType type, const std::vector<int64_t>& shape) {
    if (o == Py_None) return call.out(o, name, type, shape);
    const Tensor& t = tensor(o, name);
    for (int64_t k = 0; k < t.dim(); ++k) need(t.size(k) < 2 || t.stride(k) != 0, "an output must not be an expanded tensor");
    Call::written(t);
    return t;
  }
  Tensor out(const Call& call, PyObject* o, const char* name, bool keys) const { return out(call, o, name, type, shape(keys)); }
  float scale(PyObject* o) const { return o == Py_None ? (float)(1.0 / std::sqrt((double)Dk)) : real(o); }
};

// delta_scan(q, k, v, g, beta, h0, scale, lengths, reset, o, h_last, states, workspace) -> (o, h_last)
PyObject* delta_scan(PyObject*, PyObject* const* a, Py_ssize_t) {
  return guarded([&]() -> PyObject* {
    const Tensor &q = tensor(a[0], "q"), &v = tensor(a[2], "v");
    Call call(q, "q");
    const Heads heads(call, q, v, 2);
    const int64_t T = heads.lead[0], B = heads.lead[1], H = heads.H, Dk = heads.Dk, Dv = heads.Dv;
    long long strides[16];
    int n = 0;
    void* pq = heads.add(call, q, "q", true, strides, n);
    void* pk = heads.add(call, tensor(a[1], "k"), "k", true, strides, n);
    void* pv = heads.add(call, v, "v", false, strides, n);
    n += 3;
    const float* g = heads.add_gate(call, tensor(a[3], "g"), "g", strides, n);
    const float* beta = heads.add_gate(call, tensor(a[4], "beta"), "beta", strides, n);
    const float* h0 = static_cast<const float*>(call.dense(a[5], "h0", at::kFloat, {B, H, Dk, Dv}));
    const int32_t* lengths = static_cast<const int32_t*>(call.dense(a[7], "lengths", at::kInt, {B}));
    const unsigned char* reset = Sequence::resets(call, a[8], {T, B});
    float* states = static_cast<float*>(call.dense(
        a[11], "states", at::kFloat, {(T + LSTM_APPROX_DELTA_CHUNK - 1) / LSTM_APPROX_DELTA_CHUNK, B, H, Dk + LSTM_APPROX_DELTA_CHUNK, Dv}));
    const float scale = heads.scale(a[6]);
    Tensor o = heads.out(call, a[9], "o", false);
    n = 9;
    void* po = heads.add(call, o, "o", false, strides, n);
    Tensor last = call.out(a[10], "h_last", at::kFloat, {B, H, Dk, Dv});
    if (states) Call::written(tensor(a[11], "states"));
    Tensor ws = call.workspace(a[12], lstm_approx_delta_scan_workspace_bytes(heads.code, (int)T, (int)B, (int)H, (int)heads.Hk, (int)Dk, (int)Dv, 0));
    call.done(lstm_approx_delta_scan(heads.code, pq, pk, pv, g, beta, scale, h0, lengths, reset, (int)T, (int)B, (int)H,
                                     (int)heads.Hk, (int)Dk, (int)Dv, po, strides, last.data_ptr<float>(), states,
                                     ws.data_ptr(), ws.nbytes(), call.stream, call.msg, sizeof(call.msg)));
    return wrap_all(o, last);
  });
}

// delta_scan_backward(do, q, k, v, g, beta, states, dh_last, scale, lengths, reset, dq, dk, dv, dg, dbeta, dh0, workspace)
//   -> (dq, dk, dv, dg, dbeta, dh0)
PyObject* delta_scan_backward(PyObject*, PyObject* const* a, Py_ssize_t) {
  return guarded([&]() -> PyObject* {
    const Tensor &q = tensor(a[1], "q"), &v = tensor(a[3], "v");
    Call call(q, "q");
    const Heads heads(call, q, v, 2);
    const int64_t T = heads.lead[0], B = heads.lead[1], H = heads.H, Dk = heads.Dk, Dv = heads.Dv;
    long long strides[29];
    int n = 0;
    void* pdo = heads.add(call, tensor(a[0], "do"), "do", false, strides, n);
    void* pq = heads.add(call, q, "q", true, strides, n);
    void* pk = heads.add(call, tensor(a[2], "k"), "k", true, strides, n);
    void* pv = heads.add(call, v, "v", false, strides, n);
    n = 21;
    const float* g = heads.add_gate(call, tensor(a[4], "g"), "g", strides, n);
    const float* beta = heads.add_gate(call, tensor(a[5], "beta"), "beta", strides, n);
    const float* states = static_cast<const float*>(
        call.dense(tensor(a[6], "states"), "states", at::kFloat,
                   {(T + LSTM_APPROX_DELTA_CHUNK - 1) / LSTM_APPROX_DELTA_CHUNK, B, H, Dk + LSTM_APPROX_DELTA_CHUNK, Dv}));
    const float* dl = static_cast<const float*>(call.dense(a[7], "dh_last", at::kFloat, {B, H, Dk, Dv}));
    const int32_t* lengths = static_cast<const int32_t*>(call.dense(a[9], "lengths", at::kInt, {B}));
    const unsigned char* reset = Sequence::resets(call, a[10], {T, B});
    const float scale = heads.scale(a[8]);
    Tensor dq = heads.out(call, a[11], "dq", true), dk = heads.out(call, a[12], "dk", true), dv = heads.out(call, a[13], "dv", false);
    Tensor dg = Heads::out(call, a[14], "dg", at::kFloat, heads.per_head()), dbeta = Heads::out(call, a[15], "dbeta", at::kFloat, heads.per_head());
    n = 12;
    void* pdq = heads.add(call, dq, "dq", true, strides, n);
    void* pdk = heads.add(call, dk, "dk", true, strides, n);
    void* pdv = heads.add(call, dv, "dv", false, strides, n);
    n = 25;
    float* pdg = heads.add_gate(call, dg, "dg", strides, n);
    float* pdbeta = heads.add_gate(call, dbeta, "dbeta", strides, n);
    Tensor dh0 = call.out(a[16], "dh0", at::kFloat, {B, H, Dk, Dv});
    Tensor ws = call.workspace(a[17], lstm_approx_delta_scan_workspace_bytes(heads.code, (int)T, (int)B, (int)H, (int)heads.Hk, (int)Dk, (int)Dv, 1));
    call.done(lstm_approx_delta_scan_backward(heads.code, pdo, dl, pq, pk, pv, g, beta, scale, states, lengths, reset, (int)T,
                                              (int)B, (int)H, (int)heads.Hk, (int)Dk, (int)Dv, pdq, pdk, pdv, pdg, pdbeta,
                                              dh0.data_ptr<float>(), strides, ws.data_ptr(), ws.nbytes(), call.stream, call.msg,
                                              sizeof(call.msg)));
    return wrap_all(dq, dk, dv, dg, dbeta, dh0);
  });
}

// delta_step(q, k, v, g, beta, state, scale, slots, reset, o) -> o
PyObject* delta_step(PyObject*, PyObject* const* a, Py_ssize_t) {
  return guarded([&]() -> PyObject* {
    const Tensor &q = tensor(a[0], "q"), &v = tensor(a[2], "v"), &state = tensor(a[5], "state");
    Call call(q, "q");
    const Heads heads(call, q, v, 1);
    const int64_t B = heads.lead[0], slots = state.dim() > 0 ? state.size(0) : 0;
    need(slots <= 0x7fffffff, "sizes must be 32-bit numbers");
    long long strides[10];
    int n = 0;
    void* pq = heads.add(call, q, "q", true, strides, n);
    void* pk = heads.add(call, tensor(a[1], "k"), "k", true, strides, n);
    void* pv = heads.add(call, v, "v", false, strides, n);
    const int at_o = n;
    n += 2;
    const float* g = heads.add_gate(call, tensor(a[3], "g"), "g", strides, n);
    const float* beta = heads.add_gate(call, tensor(a[4], "beta"), "beta", strides, n);
    float* ps = static_cast<float*>(call.dense(state, "state", at::kFloat, {slots, heads.H, heads.Dk, heads.Dv}));
    const int32_t* at_slots = static_cast<const int32_t*>(call.dense(a[7], "slots", at::kInt, {B}));
    const unsigned char* reset = Sequence::resets(call, a[8], {B});
    const float scale = heads.scale(a[6]);
    Tensor o = heads.out(call, a[9], "o", false);
    n = at_o;
    void* po = heads.add(call, o, "o", false, strides, n);
    Call::written(state);
    call.done(lstm_approx_delta_step(heads.code, pq, pk, pv, g, beta, scale, ps, (int)slots, at_slots, reset, (int)B,
                                     (int)heads.H, (int)heads.Hk, (int)heads.Dk, (int)heads.Dv, po, strides, call.stream,
                                     call.msg, sizeof(call.msg)));
    return wrap(o);
  });
}

// The items of a sequence of tensors.
struct Items {
  PyObject* fast;
  Items(PyObject* o, const char* name) : fast(PySequence_Fast(o, "")) {
    if (!fast) {
      PyErr_Clear();
      invalid(std::string(name) + " must be a sequence of tensors");
    }
  }
  Items(const Items&) = delete;
  ~Items() { Py_DECREF(fast); }
  Py_ssize_t size() const { return PySequence_Fast_GET_SIZE(fast); }
  PyObject* operator[](Py_ssize_t i) const { return PySequence_Fast_GET_ITEM(fast, i); }
};

// Memory that a call reads, or writes.
struct Span {
  uintptr_t at, end;
  bool written;
};
// Whether none of it that is written is written or read by another's name.
bool apart(std::vector<Span>& spans) {
  std::sort(spans.begin(), spans.end(), [](const Span& a, const Span& b) { return a.at < b.at; });
  uintptr_t end = 0, written_end = 0;  // of those before
  for (const Span& s : spans) {
    if (s.at < (s.written ? end : written_end)) return false;
    end = std::max(end, s.end);
    if (s.written) written_end = std::max(written_end, s.end);
  }
  return true;
}

// adamw_step(params, grads, exp_avg, exp_avg_sq, exp_avg_scale, exp_avg_sq_scale, copies, step, lr, beta1, beta2, eps,
// weight_decay, grad_scale, skip, seed): the averages have 8 bits where there are scales
PyObject* adamw_step(PyObject*, PyObject* const* a, Py_ssize_t) {
  return guarded([&]() -> PyObject* {
    const Items params(a[0], "params"), grads(a[1], "grads"), m(a[2], "exp_avg"), v(a[3], "exp_avg_sq");
    const Py_ssize_t count = params.size();
    need(count <= 0x7fffffff, "too many tensors");
    need(grads.size() == count && m.size() == count && v.size() == count, "params, grads and the averages must be as many");
    if (count == 0) Py_RETURN_NONE;
    const bool few_bits = a[4] != Py_None, copied = a[6] != Py_None;
    std::optional<Items> ms, vs, copies;
    if (few_bits) ms.emplace(a[4], "exp_avg_scale"), vs.emplace(a[5], "exp_avg_sq_scale");
    if (copied) copies.emplace(a[6], "copies");
    need(!few_bits || (ms->size() == count && vs->size() == count), "params and the scales must be as many");
    need(!copied || copies->size() == count, "params and copies must be as many");
    Call call(tensor(params[0], "params"), "params");
    const at::ScalarType kind = few_bits ? at::kFloat8_e4m3fn : at::kFloat;
    std::vector<lstm_approx_adamw_tensor> table((size_t)count);
    std::vector<Span> spans;
    spans.reserve((size_t)count * 7);
    auto span = [&](const void* p, size_t bytes, bool written) {
      const auto at = reinterpret_cast<uintptr_t>(p);
      if (p && bytes > 0) spans.push_back({at, at + bytes, written});
    };
    for (Py_ssize_t i = 0; i < count; ++i) {
      const Tensor& p = tensor(params[i], "params");
      lstm_approx_adamw_tensor& t = table[(size_t)i];
      t = {};
      const auto shape = p.sizes();
      t.n = p.numel();
      t.p_dtype = t.g_dtype = float_code(p, "params");
      t.p = call.dense(p, "params", p.scalar_type(), shape);
      t.m = call.dense(tensor(m[i], "exp_avg"), "exp_avg", kind, shape);
      t.v = call.dense(tensor(v[i], "exp_avg_sq"), "exp_avg_sq", kind, shape);
      if (few_bits) {
        const int64_t blocks = (t.n + 255) / 256;
        t.m_scale = static_cast<float*>(call.dense(tensor((*ms)[i], "exp_avg_scale"), "exp_avg_scale", at::kFloat, {blocks}));
        t.v_scale = static_cast<float*>(call.dense(tensor((*vs)[i], "exp_avg_sq_scale"), "exp_avg_sq_scale", at::kFloat, {blocks}));
      }
      if (copied && (*copies)[i] != Py_None) {
        const Tensor& c = tensor((*copies)[i], "copies");
        t.copy_dtype = float_code(c, "copies");
        t.copy = call.dense(c, "copies", c.scalar_type(), shape);
      }
      if (grads[i] != Py_None) {
        const Tensor& g = tensor(grads[i], "grads");
        t.g_dtype = float_code(g, "grads");
        t.g = call.dense(g, "grads", g.scalar_type(), shape);
      }
      span(t.p, p.nbytes(), true);
      if (!t.g) continue;
      const size_t average = (size_t)t.n * (few_bits ? 1 : 4), scales = (size_t)((t.n + 255) / 256) * 4;
      // (a copy or a gradient that is the parameter itself is read before, and written after, by who reads and writes that)
      if (t.g != t.p || t.g_dtype != t.p_dtype) span(t.g, tensor(grads[i], "grads").nbytes(), false);
      span(t.m, average, true), span(t.v, average, true);
      span(t.m_scale, scales, true), span(t.v_scale, scales, true);
      if (t.copy && (t.copy != t.p || t.copy_dtype != t.p_dtype)) span(t.copy, tensor((*copies)[i], "copies").nbytes(), true);
    }
    need(apart(spans), "params, averages, scales and copies must not overlap one another, nor a gradient");
    auto device_value = [&](PyObject* o, const char* name, at::ScalarType type) -> const void* {
      const Tensor& t = tensor(o, name);
      need(t.numel() == 1, "step, lr, grad_scale and skip must have one value");
      return call.dense(t, name, type, t.sizes());
    };
    const int32_t* step_at = nullptr;
    const float *lr_at = nullptr, *clip = nullptr;
    const unsigned char* skip = nullptr;
    long long step = 0;
    double lr = 0.0;
    if (THPVariable_Check(a[7])) step_at = static_cast<const int32_t*>(device_value(a[7], "step", at::kInt));
    else step = integer(a[7]);
    need(step_at || (step >= 1 && step <= 0x7fffffff), "step must be 1 or more");
    auto number = [](PyObject* o) {
      const double x = PyFloat_AsDouble(o);
      if (x == -1.0 && PyErr_Occurred()) {
        PyErr_Clear();
        invalid("a number was expected");
      }
      return x;
    };
    if (THPVariable_Check(a[8])) lr_at = static_cast<const float*>(device_value(a[8], "lr", at::kFloat));
    else lr = number(a[8]);
    if (a[13] != Py_None) clip = static_cast<const float*>(device_value(a[13], "grad_scale", at::kFloat));
    if (a[14] != Py_None)
      skip = static_cast<const unsigned char*>(device_value(
          a[14], "skip", tensor(a[14], "skip").scalar_type() == at::kByte ? at::kByte : at::kBool));
    const double beta1 = number(a[9]), beta2 = number(a[10]), eps = number(a[11]), decay = number(a[12]);
    const unsigned seed = (unsigned)(unsigned long long)integer(a[15]);
    for (Py_ssize_t i = 0; i < count; ++i) {
      if (grads[i] == Py_None) continue;
      for (const Items* list : {&params, &m, &v}) Call::written(tensor((*list)[i], ""));
      if (few_bits) Call::written(tensor((*ms)[i], "")), Call::written(tensor((*vs)[i], ""));
      if (table[(size_t)i].copy) Call::written(tensor((*copies)[i], ""));
    }
    call.done(lstm_approx_adamw_step((int)count, table.data(), few_bits ? 8 : 32, (int)step, step_at, lr, lr_at, beta1, beta2,
                                     eps, decay, clip, skip, seed, call.stream, call.msg, sizeof(call.msg)));
    Py_RETURN_NONE;
  });
}

// Each entry takes exactly the arguments that _operators.py gives it.
template <PyObject* (*kF)(PyObject*, PyObject* const*, Py_ssize_t), Py_ssize_t kN>
PyObject* counted(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  if (n != kN) {
    PyErr_Format(PyExc_TypeError, "%zd arguments expected, not %zd", kN, n);
    return nullptr;
  }
  return kF(self, a, n);
}
template <PyObject* (*kF)(PyObject*, PyObject* const*, Py_ssize_t), Py_ssize_t kN>
PyMethodDef entry(const char* name) {
  return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(&counted<kF, kN>)), METH_FASTCALL, nullptr};
}

PyMethodDef g_methods[] = {
    entry<rms_norm, 10>("rms_norm"),          entry<rms_norm_backward, 9>("rms_norm_backward"),
    entry<gated_scan, 12>("gated_scan"),      entry<gated_scan_backward, 16>("gated_scan_backward"),
    entry<gated_step, 9>("gated_step"),       entry<w4_quantize, 5>("w4_quantize"),
    entry<w4_matvec, 12>("w4_matvec"),        entry<delta_step, 10>("delta_step"),
    entry<delta_scan, 13>("delta_scan"),      entry<delta_scan_backward, 18>("delta_scan_backward"),
    entry<adamw_step, 16>("adamw_step"),      {nullptr, nullptr, 0, nullptr},
};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_torch_ops", "The operators on torch tensors (see _operators).", -1,
                        g_methods};

}  // namespace

PyMODINIT_FUNC PyInit__torch_ops() {
  PyObject* binding = PyImport_ImportModule("paper_1905_00689_gb300._binding");
  if (!binding) return nullptr;
  g_error = PyObject_GetAttrString(binding, "LSTMApproxError");
  Py_DECREF(binding);
  g_sum_low = PyUnicode_InternFromString("sum_low");
  g_sum_low_call = PyUnicode_InternFromString("_sum_low_call");
  return g_error && g_sum_low && g_sum_low_call ? PyModule_Create(&g_module) : nullptr;
}
