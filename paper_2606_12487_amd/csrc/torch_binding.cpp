// Host side of the per-call entry points of the Python binding (module
// _dptq_torch): checks the tensors, allocates the outputs the caller did not
// pass, and calls the C ABI on the current stream.  The same checks, in the
// same order and with the same errors, as the Python they replace; written
// against the CPython API and the tensor type directly because a pass of a few
// launches is bound by this work: two calls with fresh outputs took 24 us of
// host time in Python (interpreting the checks, two torch.empty, a stream
// object and the ctypes marshalling), of which the two launches are 6.6 us.

#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/core/DeviceGuard.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <array>
#include <initializer_list>
#include <string>

#include "dptq.h"

namespace {

// Set by init(): raises DptqError(status, what); returns the raw stream of a
// device index.
PyObject* g_raise = nullptr;
PyObject* g_stream = nullptr;

// A Python error is set.
struct Raised {};

const char* dtype_name(at::ScalarType t) {
  switch (t) {
    case at::kHalf: return "torch.float16";
    case at::kFloat: return "torch.float32";
    case at::kDouble: return "torch.float64";
    case at::kByte: return "torch.uint8";
    case at::kChar: return "torch.int8";
    case at::kInt: return "torch.int32";
    case at::kLong: return "torch.int64";
    case at::kFloat8_e4m3fn: return "torch.float8_e4m3fn";
    default: return "?";
  }
}

[[noreturn]] void fail(PyObject* type, const std::string& msg) {
  PyErr_SetString(type, msg.c_str());
  throw Raised{};
}

std::string shape_text(at::IntArrayRef s) {
  std::string r = "(";
  for (size_t i = 0; i < s.size(); ++i) r += (i ? ", " : "") + std::to_string(s[i]);
  return r + (s.size() == 1 ? ",)" : ")");
}

// The tensor o, of that dtype and on the GPU.
const at::Tensor& gpu_tensor(PyObject* o, const char* name, at::ScalarType dtype) {
  if (!THPVariable_Check(o)) fail(PyExc_TypeError, std::string(name) + " must be a torch.Tensor");
  const at::Tensor& t = THPVariable_Unpack(o);
  if (t.scalar_type() != dtype) {
    PyObject* d = PyObject_GetAttrString(o, "dtype");
    if (!d) throw Raised{};
    PyErr_Format(PyExc_TypeError, "%s must have dtype %s, got %S", name, dtype_name(dtype), d);
    Py_DECREF(d);
    throw Raised{};
  }
  if (!t.is_cuda()) fail(PyExc_ValueError, std::string(name) + " must be a GPU tensor");
  return t;
}

// The tensor o after its checks; shape only when `has_shape`.
const at::Tensor& tensor(PyObject* o, const char* name, at::ScalarType dtype, at::IntArrayRef shape = {},
                         bool has_shape = false) {
  const at::Tensor& t = gpu_tensor(o, name, dtype);
  if (!t.is_contiguous()) fail(PyExc_ValueError, std::string(name) + " must be contiguous");
  if (has_shape && t.sizes() != shape)
    fail(PyExc_ValueError, std::string(name) + " must have shape " + shape_text(shape) + ", got " +
                               shape_text(t.sizes()));
  return t;
}

const at::Tensor& tensor_of(PyObject* o, const char* name, at::ScalarType dtype,
                            std::initializer_list<int64_t> shape) {
  return tensor(o, name, dtype, at::IntArrayRef(shape.begin(), shape.size()), true);
}

void two_d(const at::Tensor& t, const char* what) {
  if (t.dim() != 2) fail(PyExc_ValueError, what);
}

int64_t dim(const at::Tensor& t, int i) {
  if (i >= t.dim()) fail(PyExc_IndexError, "tuple index out of range");
  return t.size(i);
}

// An integer argument; any_number: also another number of an integer's value.
int64_t integer(PyObject* o, const char* name, bool any_number = false) {
  PyObject* n = PyIndex_Check(o) ? PyNumber_Index(o) : any_number && PyNumber_Check(o) ? PyNumber_Long(o) : nullptr;
  if (!n) {
    if (!PyErr_Occurred()) PyErr_Format(PyExc_TypeError, "%s must be an integer, got %R", name, o);
    throw Raised{};
  }
  const int eq = PyIndex_Check(o) ? 1 : PyObject_RichCompareBool(o, n, Py_EQ);
  const int64_t v = PyLong_AsLongLong(n);
  Py_DECREF(n);
  if (PyErr_Occurred()) throw Raised{};
  if (eq != 1) {
    PyErr_Format(PyExc_ValueError, "%s must be an integer, got %R", name, o);
    throw Raised{};
  }
  return v;
}

// int(o) as a C int32 argument (taken modulo 2^32, as ctypes does).
int32_t integer32(PyObject* o) {
  if (PyLong_CheckExact(o)) return (int32_t)PyLong_AsUnsignedLongLongMask(o);
  PyObject* n = PyNumber_Long(o);
  if (!n) throw Raised{};
  const int32_t v = (int32_t)PyLong_AsUnsignedLongLongMask(n);
  Py_DECREF(n);
  return v;
}

// o == v, by value.
bool equals(PyObject* o, long v) {
  PyObject* n = PyLong_FromLong(v);
  const int eq = n ? PyObject_RichCompareBool(o, n, Py_EQ) : -1;
  Py_XDECREF(n);
  if (eq < 0) throw Raised{};
  return eq == 1;
}

int32_t bits_4_or_8(PyObject* o) {
  if (equals(o, 4)) return 4;
  if (equals(o, 8)) return 8;
  fail(PyExc_ValueError, "bits must be 4 or 8");
}

// Codes of the entry points that leave the check of bits to the library: packed
// where bits == 4, bytes for any other value.
at::ScalarType code_dtype(int32_t bits) { return bits == 4 ? at::kByte : at::kChar; }
int32_t code_bits(PyObject* bits) { return equals(bits, 4) ? 4 : 8; }

// The interpreter lock released for a scope, also when an exception leaves it.
class Unlocked {
 public:
  Unlocked() : state_(PyEval_SaveThread()) {}
  ~Unlocked() { PyEval_RestoreThread(state_); }
  Unlocked(const Unlocked&) = delete;

 private:
  PyThreadState* state_;
};

// An output: the caller's tensor after its checks, or a new one (allocate).
struct Out {
  PyObject* o = nullptr;   // a new reference
  at::Tensor t;
  std::array<int64_t, 3> shape{};
  int dims;
  at::TensorOptions options;
  Out(PyObject* given, const char* name, at::ScalarType dtype, std::initializer_list<int64_t> s,
      const at::Tensor& like)
      : dims((int)s.size()) {
    if (given != Py_None) {
      t = tensor_of(given, name, dtype, s);
      Py_INCREF(given);
      o = given;
    } else {
      std::copy(s.begin(), s.end(), shape.begin());
      options = at::TensorOptions().dtype(dtype).device(like.device());
    }
  }
  Out(const Out&) = delete;
  ~Out() { Py_XDECREF(o); }
  template <typename T = void>
  T* ptr() const { return static_cast<T*>(t.data_ptr()); }
  PyObject* release() {
    PyObject* r = o;
    o = nullptr;
    return r;
  }
};

// Allocates the outputs that the caller did not pass.  Without the interpreter
// lock: an allocation may wait for the device.
template <typename... O>
void allocate(O&... outs) {
  if ((outs.o && ...)) return;
  {
    Unlocked unlocked;
    const auto one = [](Out& out) {
      if (!out.o) out.t = at::empty(at::IntArrayRef(out.shape.data(), out.dims), out.options);
    };
    (one(outs), ...);
  }
  const auto wrap = [](Out& out) {
    if (!out.o) out.o = THPVariable_Wrap(out.t);
    if (!out.o) throw Raised{};
  };
  (wrap(outs), ...);
}

template <typename T = void>
T* ptr(const at::Tensor& t) { return static_cast<T*>(t.data_ptr()); }

void* stream_of(const at::Tensor& t) {
  PyObject* idx = PyLong_FromLong(t.device().index());
  if (!idx) throw Raised{};
  PyObject* s = PyObject_CallOneArg(g_stream, idx);
  Py_DECREF(idx);
  if (!s) throw Raised{};
  void* p = PyLong_AsVoidPtr(s);
  Py_DECREF(s);
  if (!p && PyErr_Occurred()) throw Raised{};
  return p;
}

// Calls the C entry f(args..., stream) on the current stream of t's device,
// without the interpreter lock, and raises on a nonzero status.  The arguments,
// data pointers among them, are values by then: what a tensor without storage
// throws leaves with the lock held.
template <typename F, typename... A>
void call(const char* what, const at::Tensor& t, F f, A... args) {
  void* stream = stream_of(t);
  int st;
  {
    Unlocked unlocked;
    st = f(args..., stream);
  }
  if (st == DPTQ_OK) return;
  PyObject* r = PyObject_CallFunction(g_raise, "is", st, what);
  Py_XDECREF(r);
  if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, what);
  throw Raised{};
}

template <typename... O>
PyObject* tuple(O&... outs) {
  PyObject* r = PyTuple_New(sizeof...(outs));
  if (!r) throw Raised{};
  Py_ssize_t i = 0;
  (PyTuple_SET_ITEM(r, i++, outs.release()), ...);
  return r;
}

void same_device(const at::Tensor& t, const char* name, const at::Tensor& x, const char* of) {
  if (t.device() != x.device())
    fail(PyExc_ValueError, std::string(name) + " must be on the same device as " + of);
}

const at::Tensor* signs_of(PyObject* o, int64_t K, const at::Tensor& x) {
  if (o == Py_None) return nullptr;
  const at::Tensor& s = tensor_of(o, "signs", at::kByte, {(K + 7) / 8});
  if (s.device() != x.device()) fail(PyExc_ValueError, "signs must be on the same device as x");
  return &s;
}

int64_t fp6_bytes(int64_t rows, int64_t K) {
  const int64_t n = dptq_fp6_bytes(rows, K);
  if (n < 0)
    fail(PyExc_ValueError, "no FP6 layout for rows=" + std::to_string(rows) + ", K=" + std::to_string(K) +
                               " (K must be a multiple of 128)");
  return n;
}

// rotate_quant(x, had_size, bits, codes, scales, signs)
PyObject* rotate_quant(PyObject* const* a) {
  const at::Tensor& x = tensor(a[0], "x", at::kHalf);
  two_d(x, "x must be 2-D [M, K]");
  const int64_t M = x.size(0), K = x.size(1);
  const int32_t bits = bits_4_or_8(a[2]);
  Out codes(a[3], "codes", code_dtype(bits), {M, bits == 4 ? K / 2 : K}, x);
  Out scales(a[4], "scales", at::kFloat, {M}, x);
  allocate(codes, scales);
  const at::Tensor* signs = signs_of(a[5], K, x);
  const int32_t h = integer32(a[1]);
  if (!signs)
    call("dptq_rotate_quant", x, dptq_rotate_quant, ptr(x), M, K, h, bits, codes.ptr(), scales.ptr<float>());
  else
    call("dptq_rotate_quant_ex", x, dptq_rotate_quant_ex, ptr(x), M, K, h, bits, ptr<uint8_t>(*signs),
         DPTQ_LAYOUT_PACKED, codes.ptr(), scales.ptr<float>());
  return tuple(codes, scales);
}

// rotate_quant_fp6(x, had_size, out, scales, signs)
PyObject* rotate_quant_fp6(PyObject* const* a) {
  const at::Tensor& x = tensor(a[0], "x", at::kHalf);
  two_d(x, "x must be 2-D [M, K]");
  const int64_t M = x.size(0), K = x.size(1);
  Out out(a[2], "out", at::kByte, {fp6_bytes(M, K)}, x);
  Out scales(a[3], "scales", at::kFloat, {M}, x);
  allocate(out, scales);
  const at::Tensor* signs = signs_of(a[4], K, x);
  const int32_t h = integer32(a[1]);
  if (!signs)
    call("dptq_rotate_quant_fp6", x, dptq_rotate_quant_fp6, ptr(x), M, K, h, out.ptr<uint8_t>(),
         scales.ptr<float>());
  else
    call("dptq_rotate_quant_ex", x, dptq_rotate_quant_ex, ptr(x), M, K, h, 4, ptr<uint8_t>(*signs),
         DPTQ_LAYOUT_FP6, out.ptr(), scales.ptr<float>());
  return tuple(out, scales);
}

// rotate_quant_range(x, had_size, bits, codes, scales, zeros)
PyObject* rotate_quant_range(PyObject* const* a) {
  const at::Tensor& x = tensor(a[0], "x", at::kHalf);
  if (x.dim() != 2) fail(PyExc_ValueError, "x must be 2-D [M, K]");
  const int64_t M = x.size(0), K = x.size(1);
  const int32_t cb = code_bits(a[2]);
  Out codes(a[3], "codes", code_dtype(cb), {M, cb == 4 ? K / 2 : K}, x);
  Out scales(a[4], "scales", at::kFloat, {M}, x);
  Out zeros(a[5], "zeros", at::kInt, {M}, x);
  allocate(codes, scales, zeros);
  const int32_t h = integer32(a[1]), bits = integer32(a[2]);
  call("dptq_rotate_quant_range", x, dptq_rotate_quant_range, ptr(x), M, K, h, bits, codes.ptr(),
       scales.ptr<float>(), zeros.ptr<int32_t>());
  return tuple(codes, scales, zeros);
}

struct Gemm {
  const at::Tensor &codes, &w;
  int64_t M, K, N;
};

Gemm gemm_args(PyObject* codes_o, int32_t bits, PyObject* w_o) {
  const at::Tensor& codes = tensor(codes_o, "codes", code_dtype(bits));
  const at::Tensor& w = tensor(w_o, "w_packed", at::kByte);
  const int64_t M = dim(codes, 0), K = dim(codes, 1) * (bits == 4 ? 2 : 1), N = dim(w, 0);
  if (dim(w, 1) * 2 != K)
    fail(PyExc_ValueError, "w_packed must be [N, K/2] with K = " + std::to_string(K));
  return Gemm{codes, w, M, K, N};
}

// qlinear(codes, a_scales, bits, w_packed, w_scales, y, kernel)
PyObject* qlinear(PyObject* const* a) {
  const int32_t bits = bits_4_or_8(a[2]);
  const Gemm g = gemm_args(a[0], bits, a[3]);
  const at::Tensor& as = tensor_of(a[1], "a_scales", at::kFloat, {g.M});
  const at::Tensor& ws = tensor_of(a[4], "w_scales", at::kFloat, {g.N});
  Out y(a[5], "y", at::kHalf, {g.M, g.N}, g.codes);
  allocate(y);
  const int32_t kernel = integer32(a[6]);
  if (kernel == DPTQ_GEMM_AUTO)
    call("dptq_qlinear", g.codes, dptq_qlinear, ptr(g.codes), ptr<float>(as), g.M, g.K, bits,
         ptr<uint8_t>(g.w), ptr<float>(ws), g.N, y.ptr());
  else
    call("dptq_qlinear_kernel", g.codes, dptq_qlinear_kernel, ptr(g.codes), ptr<float>(as), g.M, g.K, bits,
         ptr<uint8_t>(g.w), ptr<float>(ws), g.N, y.ptr(), nullptr, kernel);
  return y.release();
}

// qlinear_a8(codes, a_scales, w_a8, w_scales, y, kernel)
PyObject* qlinear_a8(PyObject* const* a) {
  const Gemm g = gemm_args(a[0], 8, a[2]);
  const at::Tensor& as = tensor_of(a[1], "a_scales", at::kFloat, {g.M});
  const at::Tensor& ws = tensor_of(a[3], "w_scales", at::kFloat, {g.N});
  Out y(a[4], "y", at::kHalf, {g.M, g.N}, g.codes);
  allocate(y);
  const int32_t kernel = integer32(a[5]);
  call("dptq_qlinear_a8", g.codes, dptq_qlinear_a8, ptr(g.codes), ptr<float>(as), g.M, g.K, ptr<uint8_t>(g.w),
       ptr<float>(ws), g.N, y.ptr(), kernel);
  return y.release();
}

// qlinear_decode_native(codes, a_scales, bits, w_dec, w_scales, y)
PyObject* qlinear_decode_native(PyObject* const* a) {
  if (!THPVariable_Check(a[4])) fail(PyExc_TypeError, "w_scales must be a torch.Tensor");
  const int64_t N = dim(THPVariable_Unpack(a[4]), 0);
  const int32_t bits = bits_4_or_8(a[2]);
  const at::Tensor& codes = tensor(a[0], "codes", code_dtype(bits));
  const int64_t M = dim(codes, 0), K = dim(codes, 1) * (bits == 4 ? 2 : 1);
  const int64_t n = dptq_prepacked_bytes(N, K, DPTQ_WEIGHTS_DECODE);
  if (n < 0)
    fail(PyExc_ValueError, "no layout 3 for N=" + std::to_string(N) + ", K=" + std::to_string(K) +
                               " (K must be a multiple of 128; the decode layout also needs N % 16 == 0)");
  const at::Tensor& w = tensor_of(a[3], "w_dec", at::kByte, {n});
  const at::Tensor& as = tensor_of(a[1], "a_scales", at::kFloat, {M});
  const at::Tensor& ws = tensor_of(a[4], "w_scales", at::kFloat, {N});
  Out y(a[5], "y", at::kHalf, {M, N}, codes);
  allocate(y);
  call("dptq_qlinear_decode_native", codes, dptq_qlinear_decode_native, ptr(codes), ptr<float>(as), M, K,
       bits, ptr<uint8_t>(w), ptr<float>(ws), N, y.ptr(), nullptr);
  return y.release();
}

// qlinear_fp6(a6, a_scales, w6, w_scales, M, K, N, y)
PyObject* qlinear_fp6(PyObject* const* a) {
  const int64_t M = integer(a[4], "M"), K = integer(a[5], "K"), N = integer(a[6], "N");
  const at::Tensor& a6 = tensor_of(a[0], "a_fp6", at::kByte, {fp6_bytes(M, K)});
  const at::Tensor& w6 = tensor_of(a[2], "w_fp6", at::kByte, {fp6_bytes(N, K)});
  const at::Tensor& as = tensor_of(a[1], "a_scales", at::kFloat, {M});
  const at::Tensor& ws = tensor_of(a[3], "w_scales", at::kFloat, {N});
  Out y(a[7], "y", at::kHalf, {M, N}, a6);
  allocate(y);
  call("dptq_qlinear_fp6", a6, dptq_qlinear_fp6, ptr<uint8_t>(a6), ptr<float>(as), M, K, ptr<uint8_t>(w6),
       ptr<float>(ws), N, y.ptr(), nullptr);
  return y.release();
}

// The activation of a gated block, by its name.
int32_t gate_activation(PyObject* o) {
  if (PyUnicode_Check(o)) {
    if (PyUnicode_CompareWithASCIIString(o, "silu") == 0) return DPTQ_GATE_SILU;
    if (PyUnicode_CompareWithASCIIString(o, "gelu_tanh") == 0) return DPTQ_GATE_GELU_TANH;
  }
  fail(PyExc_ValueError, "activation must be 'silu' or 'gelu_tanh'");
}

// The channels of a gated block with N rows of weights.
int64_t gated_channels(int64_t N) {
  if (N < 16 || N % 16) fail(PyExc_ValueError, "a gated block has 2 F rows of weights, F a multiple of 8");
  return N / 2;
}

// On weights in the layout `weights`, [N, K/2] or in the decode layout.
PyObject* gated(PyObject* o_codes, PyObject* o_as, int32_t bits, PyObject* o_w, int32_t weights, PyObject* o_ws,
                PyObject* o_y, PyObject* o_act) {
  const at::Tensor& codes = tensor(o_codes, "codes", code_dtype(bits));
  const int64_t M = dim(codes, 0), K = dim(codes, 1) * (bits == 4 ? 2 : 1);
  const at::Tensor& ws = tensor(o_ws, "w_scales", at::kFloat);
  if (ws.dim() != 1) fail(PyExc_ValueError, "w_scales must be 1-D [2 F]");
  const int64_t N = ws.size(0), F = gated_channels(N);
  const int64_t n = weights == DPTQ_WEIGHTS_DECODE ? dptq_prepacked_bytes(N, K, DPTQ_WEIGHTS_DECODE) : 0;
  if (n < 0) fail(PyExc_ValueError, "K must be a multiple of 128 in the decode layout");
  const at::Tensor& w = weights == DPTQ_WEIGHTS_DECODE ? tensor_of(o_w, "w_dec", at::kByte, {n})
                                                       : tensor_of(o_w, "w_packed", at::kByte, {N, K / 2});
  const at::Tensor& as = tensor_of(o_as, "a_scales", at::kFloat, {M});
  same_device(as, "a_scales", codes, "codes");
  same_device(w, "w", codes, "codes");
  same_device(ws, "w_scales", codes, "codes");
  const int32_t act = gate_activation(o_act);
  const c10::DeviceGuard on(codes.device());
  Out y(o_y, "y", at::kHalf, {M, F}, codes);
  allocate(y);
  same_device(y.t, "y", codes, "codes");
  call("dptq_qlinear_gated", codes, dptq_qlinear_gated, ptr(codes), ptr<float>(as), M, K, bits, ptr<uint8_t>(w),
       weights, ptr<float>(ws), F, act, y.ptr());
  return y.release();
}

// qlinear_gated(codes, a_scales, bits, w_packed, w_scales, y, activation)
PyObject* qlinear_gated(PyObject* const* a) {
  return gated(a[0], a[1], bits_4_or_8(a[2]), a[3], DPTQ_WEIGHTS_PACKED, a[4], a[5], a[6]);
}

// qlinear_gated_a8(codes, a_scales, w_a8, w_scales, y, activation)
PyObject* qlinear_gated_a8(PyObject* const* a) {
  return gated(a[0], a[1], 8, a[2], DPTQ_WEIGHTS_A8_ORDER, a[3], a[4], a[5]);
}

// qlinear_gated_decode_native(codes, a_scales, bits, w_dec, w_scales, y, activation)
PyObject* qlinear_gated_decode_native(PyObject* const* a) {
  return gated(a[0], a[1], bits_4_or_8(a[2]), a[3], DPTQ_WEIGHTS_DECODE, a[4], a[5], a[6]);
}

// qlinear_gated_fp6(a6, a_scales, w6, w_scales, M, K, F, y, activation)
PyObject* qlinear_gated_fp6(PyObject* const* a) {
  const int64_t M = integer(a[4], "M"), K = integer(a[5], "K"), F = integer(a[6], "F");
  if (F < 8 || F % 8 || F > 0x3FFFFFF8) fail(PyExc_ValueError, "F must be a positive multiple of 8");
  const at::Tensor& a6 = tensor_of(a[0], "a_fp6", at::kByte, {fp6_bytes(M, K)});
  const at::Tensor& w6 = tensor_of(a[2], "w_fp6", at::kByte, {fp6_bytes(2 * F, K)});
  const at::Tensor& as = tensor_of(a[1], "a_scales", at::kFloat, {M});
  const at::Tensor& ws = tensor_of(a[3], "w_scales", at::kFloat, {2 * F});
  same_device(as, "a_scales", a6, "a_fp6");
  same_device(w6, "w_fp6", a6, "a_fp6");
  same_device(ws, "w_scales", a6, "a_fp6");
  const int32_t act = gate_activation(a[8]);
  const c10::DeviceGuard on(a6.device());
  Out y(a[7], "y", at::kHalf, {M, F}, a6);
  allocate(y);
  same_device(y.t, "y", a6, "a_fp6");
  call("dptq_qlinear_gated_fp6", a6, dptq_qlinear_gated_fp6, ptr<uint8_t>(a6), ptr<float>(as), M, K,
       ptr<uint8_t>(w6), ptr<float>(ws), F, act, y.ptr());
  return y.release();
}

// qlinear_decode_fused(x, had_size, bits, w_packed, w_scales, y, codes, scales, mode)
PyObject* qlinear_decode_fused(PyObject* const* a) {
  const at::Tensor& x = tensor(a[0], "x", at::kHalf);
  two_d(x, "x must be 2-D [M, K]");
  const int64_t M = x.size(0), K = x.size(1);
  if (!THPVariable_Check(a[3])) fail(PyExc_TypeError, "w_packed must be a torch.Tensor");
  const int64_t N = dim(THPVariable_Unpack(a[3]), 0);
  const at::Tensor& w = tensor_of(a[3], "w_packed", at::kByte, {N, K / 2});
  const at::Tensor& ws = tensor_of(a[4], "w_scales", at::kFloat, {N});
  const int32_t cb = code_bits(a[2]);
  Out y(a[5], "y", at::kHalf, {M, N}, x);
  Out codes(a[6], "codes", code_dtype(cb), {M, cb == 4 ? K / 2 : K}, x);
  Out scales(a[7], "scales", at::kFloat, {M}, x);
  allocate(y, codes, scales);
  const int32_t h = integer32(a[1]), bits = integer32(a[2]), mode = integer32(a[8]);
  call("dptq_qlinear_decode_fused", x, dptq_qlinear_decode_fused, ptr(x), M, K, h, bits, ptr<uint8_t>(w),
       ptr<float>(ws), N, y.ptr(), codes.ptr(), scales.ptr<float>(), mode);
  return tuple(y, codes, scales);
}

// qlinear_range(codes, scales, zeros, bits, w_packed, w_scales, w_sums, y)
PyObject* qlinear_range(PyObject* const* a) {
  if (!THPVariable_Check(a[1])) fail(PyExc_TypeError, "scales must be a torch.Tensor");
  if (!THPVariable_Check(a[4])) fail(PyExc_TypeError, "w_packed must be a torch.Tensor");
  const int64_t M = dim(THPVariable_Unpack(a[1]), 0);
  const at::Tensor& wt = THPVariable_Unpack(a[4]);
  if (wt.dim() != 2) fail(PyExc_ValueError, "w_packed must be 2-D [N, K/2]");
  const int64_t N = wt.size(0), K = 2 * wt.size(1);
  const int32_t cb = code_bits(a[3]);
  const at::Tensor& codes = tensor_of(a[0], "codes", code_dtype(cb), {M, cb == 4 ? K / 2 : K});
  const at::Tensor& s = tensor_of(a[1], "scales", at::kFloat, {M});
  const at::Tensor& z = tensor_of(a[2], "zeros", at::kInt, {M});
  const at::Tensor& w = tensor_of(a[4], "w_packed", at::kByte, {N, K / 2});
  const at::Tensor& ws = tensor_of(a[5], "w_scales", at::kFloat, {N});
  const at::Tensor& sums = tensor_of(a[6], "w_sums", at::kInt, {N});
  Out y(a[7], "y", at::kHalf, {M, N}, codes);
  allocate(y);
  const int32_t bits = integer32(a[3]);
  call("dptq_qlinear_range", codes, dptq_qlinear_range, ptr(codes), ptr<float>(s), ptr<int32_t>(z), M, K,
       bits, ptr<uint8_t>(w), ptr<float>(ws), ptr<int32_t>(sums), N, y.ptr());
  return y.release();
}

// residual_dynamics(x, dx, had_size, bits, eps, jr, snr, means)
PyObject* residual_dynamics(PyObject* const* a) {
  const at::Tensor& x = tensor(a[0], "x", at::kHalf);
  two_d(x, "x must be 2-D [T, K]");
  const int64_t T = x.size(0), K = x.size(1);
  const at::Tensor& dx = tensor_of(a[1], "dx", at::kHalf, {T, K});
  const int32_t bits = bits_4_or_8(a[3]);
  Out jr(a[5], "jr", at::kFloat, {T}, x);
  Out snr(a[6], "snr", at::kFloat, {T}, x);
  Out means(a[7], "means", at::kDouble, {2}, x);
  allocate(jr, snr, means);
  const int32_t h = integer32(a[2]);
  PyObject* f = PyNumber_Float(a[4]);
  if (!f) throw Raised{};
  const double eps = PyFloat_AS_DOUBLE(f);
  Py_DECREF(f);
  call("dptq_residual_dynamics", x, dptq_residual_dynamics, ptr(x), ptr(dx), T, K, h, bits, (float)eps,
       jr.ptr<float>(), snr.ptr<float>(), means.ptr<double>());
  return tuple(jr, snr, means);
}

// kv_quant(kv, group, codes, scales, mins)
PyObject* kv_quant(PyObject* const* a) {
  const at::Tensor& kv = tensor(a[0], "kv", at::kHalf);
  two_d(kv, "kv must be 2-D [T, D]");
  const int64_t T = kv.size(0), D = kv.size(1), group = integer(a[1], "group", true);
  if (group <= 0 || D % group) fail(PyExc_ValueError, "D must be a multiple of group");
  if (a[3] == Py_None || a[4] == Py_None) integer(a[1], "group");   // sizes the new buffers
  Out codes(a[2], "codes", at::kByte, {T, D / 2}, kv);
  Out scales(a[3], "scales", at::kFloat, {T, D / group}, kv);
  Out mins(a[4], "mins", at::kFloat, {T, D / group}, kv);
  allocate(codes, scales, mins);
  const int32_t g = integer32(a[1]);
  call("dptq_kv_quant", kv, dptq_kv_quant, ptr(kv), T, D, g, codes.ptr<uint8_t>(), scales.ptr<float>(),
       mins.ptr<float>());
  return tuple(codes, scales, mins);
}

// kv_dequant(codes, scales, mins, group, out)
PyObject* kv_dequant(PyObject* const* a) {
  const at::Tensor& codes = tensor(a[0], "codes", at::kByte);
  two_d(codes, "codes must be 2-D [T, D/2]");
  const int64_t T = codes.size(0), D = 2 * codes.size(1), group = integer(a[3], "group", true);
  if (group <= 0 || D % group) fail(PyExc_ValueError, "D must be a multiple of group");
  const at::Tensor& scales = tensor_of(a[1], "scales", at::kFloat, {T, D / group});
  const at::Tensor& mins = tensor_of(a[2], "mins", at::kFloat, {T, D / group});
  Out out(a[4], "out", at::kHalf, {T, D}, codes);
  allocate(out);
  const int32_t g = integer32(a[3]);
  call("dptq_kv_dequant", codes, dptq_kv_dequant, ptr<uint8_t>(codes), ptr<float>(scales), ptr<float>(mins),
       T, D, g, out.ptr());
  return out.release();
}

// rms_norm_quant(x, weight, eps, residual, sum, codes, scales)
PyObject* rms_norm_quant(PyObject* const* a) {
  const at::Tensor& x = tensor(a[0], "x", at::kHalf);
  two_d(x, "x must be 2-D [M, K]");
  const int64_t M = x.size(0), K = x.size(1);
  const at::Tensor& weight = tensor_of(a[1], "weight", at::kHalf, {K});
  same_device(weight, "weight", x, "x");
  const bool add = a[3] != Py_None;
  const at::Tensor* residual = add ? &tensor_of(a[3], "residual", at::kHalf, {M, K}) : nullptr;
  if (add) same_device(*residual, "residual", x, "x");
  if (!add && a[4] != Py_None) fail(PyExc_ValueError, "sum is given without a residual");
  // Without a residual the sum is x itself.
  Out sum(add ? a[4] : a[0], "sum", at::kHalf, {M, K}, x);
  Out codes(a[5], "codes", at::kChar, {M, K}, x);
  Out scales(a[6], "scales", at::kFloat, {M}, x);
  allocate(sum, codes, scales);
  same_device(sum.t, "sum", x, "x");
  same_device(codes.t, "codes", x, "x");
  same_device(scales.t, "scales", x, "x");
  PyObject* f = PyNumber_Float(a[2]);
  if (!f) throw Raised{};
  const double eps = PyFloat_AS_DOUBLE(f);
  Py_DECREF(f);
  call("dptq_rms_norm_quant", x, dptq_rms_norm_quant, ptr(x), add ? ptr(*residual) : nullptr, ptr(weight), M, K,
       (float)eps, add ? sum.ptr() : nullptr, codes.ptr<int8_t>(), scales.ptr<float>());
  return tuple(codes, scales, sum);
}

// Token rows [T, heads, D] with dense heads; *ld: elements from a token to the next.
const at::Tensor& token_rows(PyObject* o, const char* name, int64_t T, int64_t heads, int64_t D, int64_t* ld) {
  const at::Tensor& t = gpu_tensor(o, name, at::kHalf);
  const std::array<int64_t, 3> shape{T < 0 && t.dim() == 3 ? t.size(0) : T,
                                     heads < 0 && t.dim() == 3 ? t.size(1) : heads, D};
  if (t.sizes() != at::IntArrayRef(shape))
    fail(PyExc_ValueError, std::string(name) + " must be 3-D [T, heads, head_dim] with " +
                               (T < 0 ? "" : "T = " + std::to_string(T) + ", ") +
                               (heads < 0 ? "" : "heads = " + std::to_string(heads) + ", ") +
                               "head_dim = " + std::to_string(D) + ", got " + shape_text(t.sizes()));
  const int64_t row = t.size(1) * D;
  *ld = t.size(0) > 1 ? t.stride(0) : (row + 7) / 8 * 8;
  if ((D > 1 && t.stride(2) != 1) || (t.size(1) > 1 && t.stride(1) != D) || *ld < row || *ld % 8)
    fail(PyExc_ValueError, std::string(name) + " must have dense heads and tokens a multiple of 8 elements apart");
  return t;
}

// The cache's four tensors and the sequences' three (from a[0]).
struct Cache {
  const at::Tensor &cu, &lengths, &table, &k, &v, &ks, &vs;
  int64_t B, max_pages, pages, heads, D;
};

Cache cache_args(PyObject* const* a) {
  const at::Tensor& k = tensor(a[3], "k_pages", at::kFloat8_e4m3fn);
  if (k.dim() != 4 || k.size(2) != DPTQ_KV8_PAGE)
    fail(PyExc_ValueError, "k_pages must be 4-D [pages, kv_heads, 64, head_dim]");
  const int64_t P = k.size(0), H = k.size(1), D = k.size(3);
  const at::Tensor& v = tensor_of(a[4], "v_pages", at::kFloat8_e4m3fn, {P, H, D, DPTQ_KV8_PAGE});
  const at::Tensor& ks = tensor_of(a[5], "k_scales", at::kFloat, {P, H});
  const at::Tensor& vs = tensor_of(a[6], "v_scales", at::kFloat, {P, H});
  const at::Tensor& lengths = tensor(a[1], "lengths", at::kInt);
  if (lengths.dim() != 1) fail(PyExc_ValueError, "lengths must be 1-D [B]");
  const int64_t B = lengths.size(0);
  const at::Tensor& cu = tensor_of(a[0], "cu_seqlens", at::kInt, {B + 1});
  const at::Tensor& table = tensor(a[2], "page_table", at::kInt);
  if (table.dim() != 2 || table.size(0) != B) fail(PyExc_ValueError, "page_table must be 2-D [B, max_pages]");
  same_device(v, "v_pages", k, "k_pages");
  same_device(ks, "k_scales", k, "k_pages");
  same_device(vs, "v_scales", k, "k_pages");
  same_device(cu, "cu_seqlens", k, "k_pages");
  same_device(lengths, "lengths", k, "k_pages");
  same_device(table, "page_table", k, "k_pages");
  return Cache{cu, lengths, table, k, v, ks, vs, B, table.size(1), P, H, D};
}

int64_t size_hint(PyObject* o, const char* name) {
  const int64_t n = o == Py_None ? 0 : integer(o, name);
  if (n < 0) fail(PyExc_ValueError, std::string(name) + " must not be negative");
  return n;
}

int32_t small_count(PyObject* o, const char* name) {
  const int64_t n = integer(o, name);
  if (n < 0 || n > 0x7FFFFFFF) fail(PyExc_ValueError, std::string(name) + " must be in [0, 2^31)");
  return (int32_t)n;
}

// kv8_append(k, v, cu_seqlens, lengths, page_table, k_pages, v_pages, k_scales, v_scales, max_new)
PyObject* kv8_append(PyObject* const* a) {
  const Cache c = cache_args(a + 2);
  int64_t ld_k, ld_v;
  const at::Tensor& k = token_rows(a[0], "k", -1, c.heads, c.D, &ld_k);
  const at::Tensor& v = token_rows(a[1], "v", k.size(0), c.heads, c.D, &ld_v);
  same_device(k, "k", c.k, "k_pages");
  same_device(v, "v", c.k, "k_pages");
  const int64_t max_new = size_hint(a[9], "max_new");
  call("dptq_kv8_append", k, dptq_kv8_append, ptr(k), ld_k, ptr(v), ld_v, k.size(0), ptr<int32_t>(c.cu),
       ptr<int32_t>(c.lengths), c.B, ptr<int32_t>(c.table), c.max_pages, c.pages, (int32_t)c.heads, (int32_t)c.D,
       ptr<uint8_t>(c.k), ptr<uint8_t>(c.v), ptr<float>(c.ks), ptr<float>(c.vs), max_new);
  Py_RETURN_NONE;
}

// An output of token rows [T, heads, D]: a new dense one, or the caller's, whose
// rows may be parts of wider ones.
struct RowsOut {
  Out out;
  int64_t ld;
  RowsOut(PyObject* given, const char* name, int64_t T, int64_t heads, int64_t D, const at::Tensor& x, const char* of)
      : out(Py_None, name, at::kHalf, {T, heads, D}, x), ld(heads * D) {
    if (given == Py_None) return;
    out.t = token_rows(given, name, T, heads, D, &ld);
    same_device(out.t, name, x, of);
    Py_INCREF(given);
    out.o = given;
  }
};

double real(PyObject* o) {
  PyObject* f = PyNumber_Float(o);
  if (!f) throw Raised{};
  const double v = PyFloat_AS_DOUBLE(f);
  Py_DECREF(f);
  return v;
}

bool truth(PyObject* o) {
  const int v = PyObject_IsTrue(o);
  if (v < 0) throw Raised{};
  return v == 1;
}

// The frequencies of rotary positions, at most head_dim / 2 of them.
const at::Tensor& frequencies(PyObject* o, int64_t D, const at::Tensor& x, const char* of) {
  const at::Tensor& f = tensor(o, "inv_freq", at::kDouble);
  if (f.dim() != 1 || f.size(0) < 1 || 2 * f.size(0) > D)
    fail(PyExc_ValueError, "inv_freq must be 1-D with 1 to head_dim / 2 frequencies");
  same_device(f, "inv_freq", x, of);
  return f;
}

int64_t head_dim_of(PyObject* o, const char* name) {
  const at::Tensor& t = gpu_tensor(o, name, at::kHalf);
  if (t.dim() != 3) fail(PyExc_ValueError, std::string(name) + " must be 3-D [T, heads, head_dim]");
  return t.size(2);
}

// rotary(q, k, positions, inv_freq, interleaved, scale, q_out, k_out)
PyObject* rotary(PyObject* const* a) {
  const int64_t D = head_dim_of(a[0], "q");
  int64_t ld_q, ld_k = 0;
  const at::Tensor& q = token_rows(a[0], "q", -1, -1, D, &ld_q);
  const int64_t T = q.size(0), H = q.size(1);
  const bool keys = a[1] != Py_None;
  if (!keys && a[7] != Py_None) fail(PyExc_ValueError, "k_out is given without k");
  const at::Tensor& k = keys ? token_rows(a[1], "k", T, -1, D, &ld_k) : q;
  const int64_t Hkv = keys ? k.size(1) : 0;
  if (keys) same_device(k, "k", q, "q");
  if (H < 1 || H > 8192 || Hkv > 8192 || D > 8192) fail(PyExc_ValueError, "q and k must have 1 to 8192 heads");
  const c10::DeviceGuard on(q.device());
  const at::Tensor& positions = tensor_of(a[2], "positions", at::kInt, {T});
  same_device(positions, "positions", q, "q");
  const at::Tensor& f = frequencies(a[3], D, q, "q");
  RowsOut q_out(a[6], "q_out", T, H, D, q, "q"), k_out(keys ? a[7] : a[0], "k_out", T, keys ? Hkv : H, D, q, "q");
  allocate(q_out.out, k_out.out);
  call("dptq_rotary", q, dptq_rotary, ptr(q), ld_q, (int32_t)H, keys ? ptr(k) : nullptr, ld_k, (int32_t)Hkv, T,
       (int32_t)D, ptr<int32_t>(positions), ptr<double>(f), (int32_t)(2 * f.size(0)), (int32_t)truth(a[4]),
       (float)real(a[5]), q_out.out.ptr(), q_out.ld, keys ? k_out.out.ptr() : nullptr, k_out.ld);
  if (keys) return tuple(q_out.out, k_out.out);
  PyObject* r = PyTuple_Pack(2, q_out.out.o, Py_None);
  if (!r) throw Raised{};
  return r;
}

// rotary_kv8_append(q, k, v, cu_seqlens, lengths, page_table, k_pages, v_pages, k_scales, v_scales, inv_freq,
//                   interleaved, scale, max_new, q_out)
PyObject* rotary_kv8_append(PyObject* const* a) {
  const Cache c = cache_args(a + 3);
  int64_t ld_q, ld_k, ld_v;
  const at::Tensor& q = token_rows(a[0], "q", -1, -1, c.D, &ld_q);
  const int64_t T = q.size(0), H = q.size(1);
  const at::Tensor& k = token_rows(a[1], "k", T, c.heads, c.D, &ld_k);
  const at::Tensor& v = token_rows(a[2], "v", T, c.heads, c.D, &ld_v);
  same_device(q, "q", c.k, "k_pages");
  same_device(k, "k", c.k, "k_pages");
  same_device(v, "v", c.k, "k_pages");
  if (H < 1 || H > 8192 || c.heads > 8192) fail(PyExc_ValueError, "q must have 1 to 8192 heads");
  const c10::DeviceGuard on(q.device());
  const at::Tensor& f = frequencies(a[10], c.D, q, "q");
  const int64_t max_new = size_hint(a[13], "max_new");
  RowsOut q_out(a[14], "q_out", T, H, c.D, q, "q");
  allocate(q_out.out);
  call("dptq_rotary_kv8_append", q, dptq_rotary_kv8_append, ptr(q), ld_q, (int32_t)H, ptr(k), ld_k, ptr(v), ld_v, T,
       ptr<int32_t>(c.cu), ptr<int32_t>(c.lengths), c.B, ptr<int32_t>(c.table), c.max_pages, c.pages,
       (int32_t)c.heads, (int32_t)c.D, ptr<uint8_t>(c.k), ptr<uint8_t>(c.v), ptr<float>(c.ks), ptr<float>(c.vs),
       ptr<double>(f), (int32_t)(2 * f.size(0)), (int32_t)truth(a[11]), (float)real(a[12]), q_out.out.ptr(), q_out.ld,
       max_new);
  return q_out.out.release();
}

// kv8_attention(q, cu_seqlens, lengths, page_table, k_pages, v_pages, k_scales, v_scales, max_q, max_len, scale,
//               window, sinks, out, lse)
PyObject* kv8_attention(PyObject* const* a) {
  const Cache c = cache_args(a + 1);
  int64_t ld;
  const at::Tensor& q = token_rows(a[0], "q", -1, -1, c.D, &ld);
  same_device(q, "q", c.k, "k_pages");
  const int64_t T = q.size(0), H = q.size(1);
  if (c.heads == 0 || H % c.heads != 0 || H == 0)
    fail(PyExc_ValueError, "the heads of q must be a multiple of the cache's kv_heads");
  const int64_t max_q = size_hint(a[8], "max_q"), max_len = size_hint(a[9], "max_len");
  PyObject* f = PyNumber_Float(a[10]);
  if (!f) throw Raised{};
  const double scale = PyFloat_AS_DOUBLE(f);
  Py_DECREF(f);
  const int32_t window = small_count(a[11], "window"), sinks = small_count(a[12], "sinks");
  Out out(a[13], "out", at::kHalf, {T, H, c.D}, q);
  Out lse(a[14], "lse", at::kFloat, {T, H}, q);
  const int64_t bytes = dptq_kv8_attention_workspace(T, c.B, c.max_pages, (int32_t)H, (int32_t)c.heads,
                                                     (int32_t)c.D, window, sinks, max_q, max_len);
  // The call's own scratch, in the order of the stream.  Sizes that the library
  // does not cover are its to refuse.
  Out work(Py_None, "workspace", at::kByte, {bytes > 0 ? bytes : 0}, q);
  if (bytes > 0) allocate(out, lse, work);
  else allocate(out, lse);
  same_device(out.t, "out", q, "q");
  same_device(lse.t, "lse", q, "q");
  call("dptq_kv8_attention", q, dptq_kv8_attention, ptr(q), ld, T, ptr<int32_t>(c.cu), ptr<int32_t>(c.lengths), c.B,
       ptr<int32_t>(c.table), c.max_pages, c.pages, (int32_t)H, (int32_t)c.heads, (int32_t)c.D, ptr<uint8_t>(c.k),
       ptr<uint8_t>(c.v), ptr<float>(c.ks), ptr<float>(c.vs), (float)scale, window, sinks, max_q, max_len, out.ptr(),
       lse.ptr<float>(), bytes > 0 ? work.ptr() : nullptr, bytes > 0 ? bytes : 0);
  return tuple(out, lse);
}

// Logits [M, V], fp16 or fp32, rows *ld apart.
const at::Tensor& logit_rows(PyObject* o, int32_t* dtype, int64_t* ld) {
  if (!THPVariable_Check(o)) fail(PyExc_TypeError, "logits must be a torch.Tensor");
  const at::ScalarType type = THPVariable_Unpack(o).scalar_type();
  const bool half = type == at::kHalf;
  if (!half && type != at::kFloat) fail(PyExc_TypeError, "logits must have dtype torch.float16 or torch.float32");
  const at::Tensor& x = gpu_tensor(o, "logits", type);
  two_d(x, "logits must be 2-D [M, V]");
  *ld = x.size(0) > 1 ? x.stride(0) : x.size(1);
  if ((x.size(1) > 1 && x.stride(1) != 1) || *ld < x.size(1)) fail(PyExc_ValueError, "logits must have dense rows");
  *dtype = half ? DPTQ_F16 : DPTQ_F32;
  return x;
}

// token_logprobs(logits, tokens, top, logprobs, entropy, top_logprobs, top_ids)
PyObject* token_logprobs(PyObject* const* a) {
  int32_t dtype;
  int64_t ld;
  const at::Tensor& x = logit_rows(a[0], &dtype, &ld);
  const int64_t M = x.size(0), V = x.size(1);
  const at::Tensor& tokens = tensor_of(a[1], "tokens", at::kLong, {M});
  same_device(tokens, "tokens", x, "logits");
  const int32_t top = small_count(a[2], "top");
  if (top > V || top > DPTQ_MAX_TOP)
    fail(PyExc_ValueError, "top must be at most min(V, " + std::to_string(DPTQ_MAX_TOP) + ")");
  Out lp(a[3], "logprobs", at::kFloat, {M}, x);
  Out entropy(a[4], "entropy", at::kFloat, {M}, x);
  Out top_lp(a[5], "top_logprobs", at::kFloat, {M, top}, x);
  Out ids(a[6], "top_ids", at::kLong, {M, top}, x);
  const int64_t bytes = dptq_token_logprobs_workspace(M, V, top, dtype);
  Out work(Py_None, "workspace", at::kByte, {bytes > 0 ? bytes : 0}, x);
  if (bytes > 0) allocate(lp, entropy, top_lp, ids, work);
  else allocate(lp, entropy, top_lp, ids);
  same_device(lp.t, "logprobs", x, "logits");
  same_device(entropy.t, "entropy", x, "logits");
  same_device(top_lp.t, "top_logprobs", x, "logits");
  same_device(ids.t, "top_ids", x, "logits");
  call("dptq_token_logprobs", x, dptq_token_logprobs, ptr(x), dtype, ld, M, V, ptr<int64_t>(tokens), top,
       lp.ptr<float>(), entropy.ptr<float>(), top_lp.ptr<float>(), ids.ptr<int64_t>(),
       bytes > 0 ? work.ptr() : nullptr, bytes > 0 ? bytes : 0);
  return tuple(lp, entropy, top_lp, ids);
}

// A parameter of each row, a tensor [M] (nullptr: a number for all).
const at::Tensor* of_rows(PyObject* o, const char* name, at::ScalarType type, int64_t M, const at::Tensor& x) {
  if (!THPVariable_Check(o)) return nullptr;
  const at::Tensor& t = tensor_of(o, name, type, {M});
  same_device(t, name, x, "logits");
  return &t;
}

// sample_tokens(logits, uniform, temperature, top_k, top_p, min_p, tokens, probs)
PyObject* sample_tokens(PyObject* const* a) {
  int32_t dtype;
  int64_t ld;
  const at::Tensor& x = logit_rows(a[0], &dtype, &ld);
  const int64_t M = x.size(0), V = x.size(1);
  const at::Tensor& u = tensor_of(a[1], "uniform", at::kFloat, {M});
  same_device(u, "uniform", x, "logits");
  const at::Tensor* t = of_rows(a[2], "temperature", at::kFloat, M, x);
  const at::Tensor* k = of_rows(a[3], "top_k", at::kInt, M, x);
  const at::Tensor* p = of_rows(a[4], "top_p", at::kFloat, M, x);
  const at::Tensor* m = of_rows(a[5], "min_p", at::kFloat, M, x);
  const double t_all = t ? 0 : real(a[2]), p_all = p ? 0 : real(a[4]), m_all = m ? 0 : real(a[5]);
  const int64_t k_all = k ? 0 : integer(a[3], "top_k");
  if (!t && !(t_all >= 0)) fail(PyExc_ValueError, "temperature must not be negative");
  if (k_all < 0 || k_all > 0x7FFFFFFF) fail(PyExc_ValueError, "top_k must be in [0, 2^31)");
  if (!p && !(p_all >= 0)) fail(PyExc_ValueError, "top_p must not be negative");
  if (!m && !(m_all >= 0)) fail(PyExc_ValueError, "min_p must not be negative");
  const c10::DeviceGuard on(x.device());   // of the workspace's size and the launch
  Out tokens(a[6], "tokens", at::kLong, {M}, x);
  Out probs(a[7], "probs", at::kFloat, {M}, x);
  const int64_t bytes = dptq_sample_tokens_workspace(M, V, dtype);
  Out work(Py_None, "workspace", at::kByte, {bytes > 0 ? bytes : 0}, x);
  if (bytes > 0) allocate(tokens, probs, work);
  else allocate(tokens, probs);
  same_device(tokens.t, "tokens", x, "logits");
  same_device(probs.t, "probs", x, "logits");
  call("dptq_sample_tokens", x, dptq_sample_tokens, ptr(x), dtype, ld, M, V, ptr<float>(u),
       t ? ptr<float>(*t) : nullptr, (float)t_all, k ? ptr<int32_t>(*k) : nullptr, (int32_t)k_all,
       p ? ptr<float>(*p) : nullptr, (float)p_all, m ? ptr<float>(*m) : nullptr, (float)m_all, tokens.ptr<int64_t>(),
       probs.ptr<float>(), bytes > 0 ? work.ptr() : nullptr, bytes > 0 ? bytes : 0);
  return tuple(tokens, probs);
}

// init(raise_error, raw_stream)
PyObject* init(PyObject* const* a) {
  Py_INCREF(a[0]);
  Py_INCREF(a[1]);
  Py_XSETREF(g_raise, a[0]);
  Py_XSETREF(g_stream, a[1]);
  Py_RETURN_NONE;
}

template <PyObject* (*F)(PyObject* const*), int NARGS>
PyObject* entry(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != NARGS) {
    PyErr_Format(PyExc_TypeError, "expected %d arguments, got %zd", NARGS, n);
    return nullptr;
  }
  try {
    return F(args);
  } catch (const Raised&) {
    return nullptr;
  }
  END_HANDLE_TH_ERRORS
}

#define DPTQ_ENTRY(f, n) \
  {#f, reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(&entry<f, n>)), METH_FASTCALL, nullptr}

PyMethodDef kMethods[] = {
    DPTQ_ENTRY(init, 2),
    DPTQ_ENTRY(rotate_quant, 6),
    DPTQ_ENTRY(rotate_quant_fp6, 5),
    DPTQ_ENTRY(rotate_quant_range, 6),
    DPTQ_ENTRY(qlinear, 7),
    DPTQ_ENTRY(qlinear_a8, 6),
    DPTQ_ENTRY(qlinear_decode_native, 6),
    DPTQ_ENTRY(qlinear_fp6, 8),
    DPTQ_ENTRY(qlinear_decode_fused, 9),
    DPTQ_ENTRY(qlinear_gated, 7),
    DPTQ_ENTRY(qlinear_gated_a8, 6),
    DPTQ_ENTRY(qlinear_gated_decode_native, 7),
    DPTQ_ENTRY(qlinear_gated_fp6, 9),
    DPTQ_ENTRY(qlinear_range, 8),
    DPTQ_ENTRY(residual_dynamics, 8),
    DPTQ_ENTRY(kv_quant, 5),
    DPTQ_ENTRY(kv_dequant, 5),
    DPTQ_ENTRY(rms_norm_quant, 7),
    DPTQ_ENTRY(kv8_append, 10),
    DPTQ_ENTRY(kv8_attention, 15),
    DPTQ_ENTRY(rotary, 8),
    DPTQ_ENTRY(rotary_kv8_append, 15),
    DPTQ_ENTRY(token_logprobs, 7),
    DPTQ_ENTRY(sample_tokens, 8),
    {nullptr, nullptr, 0, nullptr},
};

PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_dptq_torch", nullptr, -1, kMethods, nullptr, nullptr, nullptr,
                       nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__dptq_torch() { return PyModule_Create(&kModule); }
