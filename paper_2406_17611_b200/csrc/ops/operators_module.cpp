// Python's way into the operators of the residual block and the clipped step: checks of tensors, outputs, the call.
//
// A call on a few nodes keeps the GPU busy for 2 to 6 us; the same checks, allocations and argument marshalling in Python
// took 15 to 20 us around it (and 0.4 us for each tensor of a step).  Here a norm of one node takes 6.3 us of host time, of
// which the launch is 3, and a product 5.4.  The entry points' addresses come from the library that Python has loaded
// (bind), so there is one library and one place that picks it.
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <c10/util/SmallVector.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "varco.h"

namespace {

using at::ScalarType;
using at::Tensor;

constexpr int64_t kBlock = 128;

// what bind() was given
struct Bound {
  decltype(&varco_norm_fwd) norm_fwd = nullptr;
  decltype(&varco_norm_bwd) norm_bwd = nullptr;
  decltype(&varco_quantize_rows) quantize_rows = nullptr;
  decltype(&varco_quantize_weight) quantize_weight = nullptr;
  decltype(&varco_fp8_product) fp8_product = nullptr;
  decltype(&varco_weight_grad) weight_grad = nullptr;
  decltype(&varco_grad_norm) grad_norm = nullptr;
  decltype(&varco_grad_clip) grad_clip = nullptr;
  decltype(&varco_clip_step) clip_step = nullptr;
  PyTypeObject *Norm = nullptr, *NormGrad = nullptr, *Eight = nullptr, *EightWeight = nullptr, *Product = nullptr;   // subtypes of tuple
  PyObject *error = nullptr;
} bound;

// ------------------------------------------------------------------------------------------ arguments
struct Object {   // owns a reference
  PyObject *p;
  explicit Object(PyObject *o) : p(o) {
    if (!o) throw python_error();
  }
  Object(const Object &) = delete;
  Object &operator=(const Object &) = delete;
  ~Object() { Py_XDECREF(p); }
};

void count_args(Py_ssize_t n, Py_ssize_t want) { TORCH_CHECK_TYPE(n == want, "expected ", want, " arguments, got ", n); }
int64_t integer(PyObject *o) {
  const Py_ssize_t v = PyNumber_AsSsize_t(o, PyExc_OverflowError);
  if (v == -1 && PyErr_Occurred()) throw python_error();
  return v;
}
int32_t width(PyObject *o, const char *what) {
  const int64_t v = integer(o);
  TORCH_CHECK_VALUE(v > 0 && v <= INT32_MAX - 127, what, " must be positive and below 2^31, not ", v);
  return (int32_t)v;
}
float real(PyObject *o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw python_error();
  return (float)v;
}
bool truth(PyObject *o) {
  const int v = PyObject_IsTrue(o);
  if (v < 0) throw python_error();
  return v != 0;
}
const Tensor &tensor(PyObject *o, const char *what) {
  TORCH_CHECK_TYPE(THPVariable_Check(o), what, " must be a tensor");
  return THPVariable_Unpack(o);
}
// device of the call's first tensor
c10::Device device_of(const Tensor &t, const char *what) {
  TORCH_CHECK_VALUE(t.is_cuda(), what, " must lie on a CUDA device");
  return t.device();
}
varco_dtype_t dtype_of(const Tensor &t) {
  const ScalarType s = t.scalar_type();
  TORCH_CHECK_TYPE(s == at::kFloat || s == at::kBFloat16, "activations must be float32 or bfloat16");
  return s == at::kFloat ? VARCO_F32 : VARCO_BF16;
}
// Row stride of a [rows x ld] matrix with F columns in use (the library checks alignment and the stride itself).  rows < 0 and
// dtype Undefined: any.
int64_t matrix(const Tensor &t, const char *what, int64_t rows, int64_t F, ScalarType dtype, c10::Device dev) {
  TORCH_CHECK_VALUE(t.dim() == 2 && (t.size(1) <= 1 || t.stride(1) == 1), what, " must be a matrix with contiguous rows");
  TORCH_CHECK_VALUE(t.device() == dev, what, " must lie on the CUDA device of the call's first matrix");
  TORCH_CHECK_TYPE(dtype == ScalarType::Undefined || t.scalar_type() == dtype, what, " must be ", dtype, ", not ", t.scalar_type());
  TORCH_CHECK_VALUE((rows < 0 || t.size(0) == rows) && t.size(1) >= F, what, " is [", t.size(0), " x ", t.size(1), "]: ",
                    rows < 0 ? "any number of" : std::to_string(rows), " rows and at least ", F, " columns are wanted");
  if (t.size(0) > 1) return t.stride(0);
  // A single row has no stride of its own and torch reports any number.  Where it is one that rows could have (a row out of a
  // padded matrix), it tells that the padding is there; else the row ends with its columns.
  const int64_t ld = t.stride(0), vec = 16 / (int64_t)t.element_size();
  return ld >= t.size(1) && ld % vec == 0 ? ld : t.size(1);
}
const float *vector(const Tensor &t, const char *what, int64_t n, c10::Device dev) {
  TORCH_CHECK_TYPE(t.scalar_type() == at::kFloat, what, " must be float32");
  TORCH_CHECK_VALUE(t.dim() == 1 && t.size(0) == n && t.is_contiguous() && t.device() == dev, what, " must be a contiguous vector of ", n,
                    " values on the call's device");
  return t.const_data_ptr<float>();
}
// row stride of the [blocks x rows] scales of a [rows x F] matrix
int64_t row_scales(const Tensor &t, const char *what, int64_t rows, int64_t F, c10::Device dev) {
  const int64_t nb = (F + kBlock - 1) / kBlock;
  TORCH_CHECK_TYPE(t.scalar_type() == at::kFloat, what, " must be float32");
  TORCH_CHECK_VALUE(t.dim() == 2 && t.size(0) == nb && t.size(1) == rows && (rows <= 1 || t.stride(1) == 1) && t.device() == dev, what,
                    " must be [", nb, " x ", rows, "] with contiguous rows on the call's device");
  return nb > 1 ? t.stride(0) : rows;
}
struct Workspace {
  void *p = nullptr;
  size_t bytes = 0;
  Workspace() = default;
  Workspace(PyObject *o, c10::Device dev) {
    const Tensor *t = THPVariable_Check(o) ? &THPVariable_Unpack(o) : nullptr;
    TORCH_CHECK_VALUE(t && t->scalar_type() == at::kByte && t->device() == dev && t->is_contiguous(),
                      "workspace must be the uint8 tensor that varco_ops_workspace / varco_weight_grad_workspace returns, on the call's device");
    p = t->data_ptr();
    bytes = (size_t)t->numel();
  }
};

// ------------------------------------------------------------------------------------------ outputs and the call
// the calls write all of it
Tensor room(at::IntArrayRef size, ScalarType dtype, c10::Device dev) { return Tensor(at::detail::empty_cuda(size, dtype, dev, std::nullopt)); }
int64_t round_up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }

struct Eight {   // the 8-bit form of a [rows x F] matrix
  Tensor data, scales;
  int64_t ld = 0;
  Eight() = default;
  Eight(int64_t rows, int64_t F, c10::Device dev)
      : data(room({rows, round_up(F, 16)}, at::kFloat8_e4m3fn, dev)), scales(room({(F + kBlock - 1) / kBlock, rows}, at::kFloat, dev)), ld(round_up(F, 16)) {}
};
template <typename T = void> T *at_or_null(const Tensor &t) { return t.defined() ? (T *)t.data_ptr() : nullptr; }

struct NoGil {
  PyThreadState *s = PyEval_SaveThread();
  ~NoGil() { PyEval_RestoreThread(s); }
};
// `call` gets the current stream of the device, which is current meanwhile
template <typename F> void launch(const char *name, c10::Device dev, F call) {
  int status;
  {
    const c10::cuda::CUDAGuard guard(dev);
    void *stream = c10::cuda::getCurrentCUDAStream(dev.index()).stream();
    const NoGil no_gil;          // a full launch queue blocks
    status = call(stream);
  }
  if (status) {
    const Object e(PyObject_CallFunction(bound.error, "is", status, name));
    PyErr_SetObject((PyObject *)Py_TYPE(e.p), e.p);
    throw python_error();
  }
}
// a result tuple; an undefined tensor becomes None
PyObject *result(PyTypeObject *type, std::initializer_list<const Tensor *> of) {
  PyObject *r = type->tp_alloc(type, (Py_ssize_t)of.size());
  if (!r) throw python_error();
  Py_ssize_t i = 0;
  for (const Tensor *t : of) {
    PyObject *o = THPVariable_Wrap(*t);   // None for an undefined one
    if (!o) {
      Py_DECREF(r);
      throw python_error();
    }
    PyTuple_SET_ITEM(r, i++, o);
  }
  return r;
}

// ------------------------------------------------------------------------------------------ the operators
// X, F, gain, residual, eps, keep, quantize
PyObject *norm_fwd(PyObject *, PyObject *const *a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  count_args(n, 7);
  const Tensor &X = tensor(a[0], "X");
  const int32_t F = width(a[1], "F");
  const varco_dtype_t dt = dtype_of(X);
  const c10::Device dev = device_of(X, "X");
  const int64_t ldx = matrix(X, "X", -1, F, ScalarType::Undefined, dev), rows = X.size(0), ld = round_up(F, dt == VARCO_F32 ? 4 : 8);
  const void *R = nullptr;
  const float *gain = nullptr;
  int64_t ldr = 0;
  Tensor H, Y;
  Eight q;
  if (a[2] != Py_None) gain = vector(tensor(a[2], "gain"), "gain", F, dev);
  if (a[3] != Py_None) {
    const Tensor &r = tensor(a[3], "residual");
    ldr = matrix(r, "residual", rows, F, X.scalar_type(), dev);
    R = r.const_data_ptr();
    H = room({rows, ld}, X.scalar_type(), dev);
  }
  const float eps = real(a[4]);
  if (truth(a[5])) Y = room({rows, ld}, X.scalar_type(), dev);
  if (truth(a[6])) q = Eight(rows, F, dev);
  const Tensor rstd = room({rows}, at::kFloat, dev);
  const varco_norm_desc_t d = {rows, F, dt, eps, ldx, ldr, ld, ld, q.ld, rows};
  launch("varco_norm_fwd", dev, [&](void *stream) {
    return bound.norm_fwd(&d, X.const_data_ptr(), R, gain, at_or_null(H), at_or_null(Y), at_or_null(q.data), at_or_null<float>(q.scales),
                          at_or_null<float>(rstd), stream);
  });
  return result(bound.Norm, {&H, &Y, &q.data, &q.scales, &rstd});
  END_HANDLE_TH_ERRORS
}

// dY, H, rstd, F, gain, residual_grad, keep, quantize, workspace
PyObject *norm_bwd(PyObject *, PyObject *const *a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  count_args(n, 9);
  const Tensor &dY = tensor(a[0], "dY"), &H = tensor(a[1], "H");
  const int32_t F = width(a[3], "F");
  const varco_dtype_t dt = dtype_of(H);
  const c10::Device dev = device_of(H, "H");
  const int64_t ldh = matrix(H, "H", -1, F, ScalarType::Undefined, dev), rows = H.size(0), ld = round_up(F, dt == VARCO_F32 ? 4 : 8);
  const int64_t ldy = matrix(dY, "dY", rows, F, H.scalar_type(), dev);
  const float *rstd = vector(tensor(a[2], "rstd"), "rstd", rows, dev), *gain = nullptr;
  const void *R = nullptr;
  int64_t ldr = 0;
  Tensor dX, dgain;
  Eight q;
  Workspace ws;
  if (a[5] != Py_None) {
    const Tensor &r = tensor(a[5], "residual_grad");
    ldr = matrix(r, "residual_grad", rows, F, H.scalar_type(), dev);
    R = r.const_data_ptr();
  }
  if (a[4] != Py_None) {
    gain = vector(tensor(a[4], "gain"), "gain", F, dev);
    ws = Workspace(a[8], dev);
    dgain = room({F}, at::kFloat, dev);
  }
  if (truth(a[6])) dX = room({rows, ld}, H.scalar_type(), dev);
  if (truth(a[7])) q = Eight(rows, F, dev);
  const varco_norm_desc_t d = {rows, F, dt, 1.f, ld, ldr, ldh, ldy, q.ld, rows};
  launch("varco_norm_bwd", dev, [&](void *stream) {
    return bound.norm_bwd(&d, dY.const_data_ptr(), H.const_data_ptr(), rstd, gain, R, at_or_null(dX), at_or_null(q.data),
                          at_or_null<float>(q.scales), at_or_null<float>(dgain), ws.p, ws.bytes, stream);
  });
  return result(bound.NormGrad, {&dX, &q.data, &q.scales, &dgain});
  END_HANDLE_TH_ERRORS
}

// X, F
PyObject *quantize_rows(PyObject *, PyObject *const *a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  count_args(n, 2);
  const Tensor &X = tensor(a[0], "X");
  const int32_t F = width(a[1], "F");
  const varco_dtype_t dt = dtype_of(X);
  const c10::Device dev = device_of(X, "X");
  const int64_t ldx = matrix(X, "X", -1, F, ScalarType::Undefined, dev), rows = X.size(0);
  const Eight q(rows, F, dev);
  launch("varco_quantize_rows", dev, [&](void *stream) {
    return bound.quantize_rows(rows, F, dt, X.const_data_ptr(), ldx, q.data.data_ptr(), q.ld, at_or_null<float>(q.scales), rows, stream);
  });
  return result(bound.Eight, {&q.data, &q.scales});
  END_HANDLE_TH_ERRORS
}

// W, transposed
PyObject *quantize_weight(PyObject *, PyObject *const *a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  count_args(n, 2);
  const Tensor &W = tensor(a[0], "W");
  const varco_dtype_t dt = dtype_of(W);
  const c10::Device dev = device_of(W, "W");
  const int64_t ldw = matrix(W, "W", -1, 1, ScalarType::Undefined, dev), R = W.size(0), K = W.size(1);
  TORCH_CHECK_VALUE(R <= INT32_MAX - 127 && K <= INT32_MAX - 127, "W must have fewer than 2^31 rows and columns");
  const int64_t nk = (K + kBlock - 1) / kBlock, ld8 = round_up(K, 16), ldt = round_up(R, 16);
  const Tensor W8 = room({R, ld8}, at::kFloat8_e4m3fn, dev), scales = room({(R + kBlock - 1) / kBlock, nk}, at::kFloat, dev);
  Tensor T8;
  if (truth(a[1])) T8 = room({K, ldt}, at::kFloat8_e4m3fn, dev);
  launch("varco_quantize_weight", dev, [&](void *stream) {
    return bound.quantize_weight((int32_t)R, (int32_t)K, dt, W.const_data_ptr(), ldw, W8.data_ptr(), ld8, at_or_null(T8), ldt,
                                 at_or_null<float>(scales), nk, stream);
  });
  return result(bound.EightWeight, {&W8, &T8, &scales});
  END_HANDLE_TH_ERRORS
}

// A8, sA, B8, sB, K, bias, relu, mask, fp32 output, keep, quantize, workspace
PyObject *fp8_product(PyObject *, PyObject *const *a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  count_args(n, 12);
  const Tensor &A = tensor(a[0], "A8"), &sA = tensor(a[1], "sA"), &B = tensor(a[2], "B8"), &sB = tensor(a[3], "sB");
  const int32_t K = width(a[4], "K");
  const c10::Device dev = device_of(A, "A8");
  const int64_t lda = matrix(A, "A8", -1, K, at::kFloat8_e4m3fn, dev), M = A.size(0);
  const int64_t ldb = matrix(B, "B8", -1, K, at::kFloat8_e4m3fn, dev), N = B.size(0);
  TORCH_CHECK_VALUE(N <= INT32_MAX - 127, "B8 must have fewer than 2^31 rows");
  const int64_t ld_sa = row_scales(sA, "sA", M, K, dev);
  TORCH_CHECK_TYPE(sB.scalar_type() == at::kFloat, "sB must be float32");
  TORCH_CHECK_VALUE(sB.dim() == 2 && sB.size(0) == (N + kBlock - 1) / kBlock && sB.size(1) == (K + kBlock - 1) / kBlock && sB.device() == dev,
                    "sB must be [ceil(N/128) x ceil(K/128)] on the call's device");
  const bool f32 = truth(a[8]);
  const ScalarType dtype = f32 ? at::kFloat : at::kBFloat16;
  const float *bias = a[5] != Py_None ? vector(tensor(a[5], "bias"), "bias", N, dev) : nullptr;
  const int32_t relu = truth(a[6]);
  const void *mask = nullptr;
  int64_t ldm = 0;
  if (a[7] != Py_None) {
    const Tensor &m = tensor(a[7], "mask");
    ldm = matrix(m, "mask", M, N, dtype, dev);
    mask = m.const_data_ptr();
  }
  const Workspace ws(a[11], dev);
  const int64_t ld = round_up(N, f32 ? 4 : 8);
  Tensor Y;
  Eight q;
  if (truth(a[9])) Y = room({M, ld}, dtype, dev);
  if (truth(a[10])) q = Eight(M, N, dev);
  const varco_fp8_desc_t d = {M,   (int32_t)N,    K,             f32 ? VARCO_F32 : VARCO_BF16, relu, lda, ldb, ld_sa, sB.stride(0),
                              sB.stride(1), ldm, ld, q.ld, M};
  launch("varco_fp8_product", dev, [&](void *stream) {
    return bound.fp8_product(&d, A.const_data_ptr(), sA.const_data_ptr<float>(), B.const_data_ptr(), sB.const_data_ptr<float>(), bias, mask,
                             at_or_null(Y), at_or_null(q.data), at_or_null<float>(q.scales), ws.p, ws.bytes, stream);
  });
  return result(bound.Product, {&Y, &q.data, &q.scales});
  END_HANDLE_TH_ERRORS
}

// A, Fa, B, Fb, workspace, bias
PyObject *weight_grad(PyObject *, PyObject *const *a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  count_args(n, 6);
  const Tensor &A = tensor(a[0], "A"), &B = tensor(a[2], "B");
  const int32_t Fa = width(a[1], "Fa"), Fb = width(a[3], "Fb");
  const varco_dtype_t dt = dtype_of(A);
  const c10::Device dev = device_of(A, "A");
  const int64_t lda = matrix(A, "A", -1, Fa, ScalarType::Undefined, dev), rows = A.size(0);
  const int64_t ldb = matrix(B, "B", rows, Fb, A.scalar_type(), dev);
  const Workspace ws(a[4], dev);
  const Tensor dW = room({Fa, Fb}, at::kFloat, dev);
  Tensor db;
  if (truth(a[5])) db = room({Fa}, at::kFloat, dev);
  launch("varco_weight_grad", dev, [&](void *stream) {
    return bound.weight_grad(rows, Fa, Fb, dt, A.const_data_ptr(), lda, B.const_data_ptr(), ldb, at_or_null<float>(dW), at_or_null<float>(db),
                             ws.p, ws.bytes, stream);
  });
  return result(&PyTuple_Type, {&dW, &db});
  END_HANDLE_TH_ERRORS
}

// ------------------------------------------------------------------------------------------ lists of tensors
constexpr int kInline = 64;
struct Addresses {
  c10::SmallVector<void *, kInline> at;
  c10::SmallVector<int64_t, kInline> count;
  c10::SmallVector<int32_t, kInline> dtype;
};

bool any_twice(const Addresses &l) {
  size_t slots = 64;
  while (slots < l.at.size() * 2) slots *= 2;
  c10::SmallVector<void *, 4 * kInline> table(slots, nullptr);
  for (size_t i = 0; i < l.at.size(); ++i) {
    if (!l.count[i] || !l.at[i]) continue;
    size_t s = (size_t)(((uint64_t)(uintptr_t)l.at[i] >> 1) * 0x9E3779B97F4A7C15ull >> 32) & (slots - 1);
    for (; table[s]; s = (s + 1) & (slots - 1))
      if (table[s] == l.at[i]) return true;
    table[s] = l.at[i];
  }
  return false;
}

// contiguous tensors of `dev` and one of the types; None entries, where they are allowed, get address and size of `like`
// (NULL and the same size)
Addresses addresses(PyObject *list, const char *what, bool f32, bool bf16, c10::Device dev, const Addresses *like = nullptr) {
  const Object seq(PySequence_Fast(list, "a list of tensors is wanted"));
  const Py_ssize_t n = PySequence_Fast_GET_SIZE(seq.p);
  PyObject **o = PySequence_Fast_ITEMS(seq.p);
  TORCH_CHECK_VALUE(n <= INT32_MAX, "too many ", what);
  TORCH_CHECK_VALUE(!like || like->at.size() == (size_t)n, what, " and weights differ in number");
  Addresses l;
  l.at.reserve(n), l.count.reserve(n), l.dtype.reserve(n);
  for (Py_ssize_t i = 0; i < n; ++i) {
    if (like && o[i] == Py_None) {
      l.at.push_back(nullptr), l.count.push_back(like->count[i]), l.dtype.push_back(VARCO_BF16);
      continue;
    }
    const Tensor &t = tensor(o[i], what);
    TORCH_CHECK_VALUE(t.device() == dev, what, " must lie on one CUDA device");
    TORCH_CHECK_VALUE(t.is_contiguous(), what, " must be contiguous");
    const ScalarType s = t.scalar_type();
    TORCH_CHECK_TYPE((f32 && s == at::kFloat) || (bf16 && s == at::kBFloat16), what, " must be ",
                     f32 && bf16 ? "float32 or bfloat16" : f32 ? "float32" : "bfloat16", ", not ", s);
    l.at.push_back(t.data_ptr()), l.count.push_back(t.numel()), l.dtype.push_back(s == at::kFloat ? VARCO_F32 : VARCO_BF16);
  }
  TORCH_CHECK_VALUE(!any_twice(l), what, " holds a tensor twice");
  return l;
}
c10::Device gradients_device(PyObject *list) {
  const Object seq(PySequence_Fast(list, "a list of gradients is wanted"));
  TORCH_CHECK_VALUE(PySequence_Fast_GET_SIZE(seq.p) > 0, "no gradients");
  return device_of(tensor(PySequence_Fast_GET_ITEM(seq.p, 0), "grads"), "grads");
}

// grads, workspace
PyObject *grad_norm(PyObject *, PyObject *const *a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  count_args(n, 2);
  const c10::Device dev = gradients_device(a[0]);
  const Addresses g = addresses(a[0], "grads", true, true, dev);
  const Workspace ws(a[1], dev);
  const Tensor norm = room({1}, at::kFloat, dev);
  launch("varco_grad_norm", dev, [&](void *stream) {
    return bound.grad_norm(g.at.data(), g.count.data(), g.dtype.data(), (int32_t)g.at.size(), at_or_null<float>(norm), ws.p, ws.bytes, stream);
  });
  return THPVariable_Wrap(norm);
  END_HANDLE_TH_ERRORS
}

// grads, max_norm, workspace, eps
PyObject *grad_clip(PyObject *, PyObject *const *a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  count_args(n, 4);
  const c10::Device dev = gradients_device(a[0]);
  const Addresses g = addresses(a[0], "grads", true, true, dev);
  const float max_norm = real(a[1]), eps = real(a[3]);
  const Workspace ws(a[2], dev);
  const Tensor norm = room({1}, at::kFloat, dev);
  launch("varco_grad_clip", dev, [&](void *stream) {
    return bound.grad_clip(g.at.data(), g.count.data(), g.dtype.data(), (int32_t)g.at.size(), max_norm, eps, at_or_null<float>(norm), ws.p,
                           ws.bytes, stream);
  });
  return THPVariable_Wrap(norm);
  END_HANDLE_TH_ERRORS
}

// weights, grads, lr, max_norm, copies, eps, workspace
PyObject *clip_step(PyObject *, PyObject *const *a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  count_args(n, 7);
  const c10::Device dev = gradients_device(a[1]);
  const Addresses g = addresses(a[1], "grads", true, true, dev), w = addresses(a[0], "weights", true, false, dev);
  TORCH_CHECK_VALUE(w.count == g.count, "weights and gradients differ in number or size");
  Addresses c;
  if (a[4] != Py_None) {
    c = addresses(a[4], "copies", false, true, dev, &w);
    TORCH_CHECK_VALUE(c.count == w.count, "a copy and its weight differ in size");
  }
  const float lr = real(a[2]), max_norm = real(a[3]), eps = real(a[5]);
  const Workspace ws(a[6], dev);
  const Tensor norm = room({1}, at::kFloat, dev);
  launch("varco_clip_step", dev, [&](void *stream) {
    return bound.clip_step(g.at.data(), g.count.data(), g.dtype.data(), (float *const *)w.at.data(), a[4] != Py_None ? c.at.data() : nullptr,
                           (int32_t)g.at.size(), lr, max_norm, eps, at_or_null<float>(norm), ws.p, ws.bytes, stream);
  });
  return THPVariable_Wrap(norm);
  END_HANDLE_TH_ERRORS
}

// ------------------------------------------------------------------------------------------ the module
// addresses of the entry points by name, types of results by name, class of errors
PyObject *bind(PyObject *, PyObject *args) {
  HANDLE_TH_ERRORS
  PyObject *entries, *types, *error;
  if (!PyArg_ParseTuple(args, "O!O!O", &PyDict_Type, &entries, &PyDict_Type, &types, &error)) throw python_error();
  auto entry = [&](auto &to, const char *name) {
    PyObject *v = PyDict_GetItemString(entries, name);
    TORCH_CHECK_VALUE(v, "no address of ", name);
    void *p = PyLong_AsVoidPtr(v);
    if (!p && PyErr_Occurred()) throw python_error();
    to = reinterpret_cast<std::decay_t<decltype(to)>>(p);
  };
  auto type = [&](PyTypeObject *&to, const char *name) {
    PyObject *v = PyDict_GetItemString(types, name);
    TORCH_CHECK_TYPE(v && PyType_Check(v) && PyType_IsSubtype((PyTypeObject *)v, &PyTuple_Type), "no tuple type ", name);
    Py_INCREF(v);
    to = (PyTypeObject *)v;
  };
  entry(bound.norm_fwd, "varco_norm_fwd");
  entry(bound.norm_bwd, "varco_norm_bwd");
  entry(bound.quantize_rows, "varco_quantize_rows");
  entry(bound.quantize_weight, "varco_quantize_weight");
  entry(bound.fp8_product, "varco_fp8_product");
  entry(bound.weight_grad, "varco_weight_grad");
  entry(bound.grad_norm, "varco_grad_norm");
  entry(bound.grad_clip, "varco_grad_clip");
  entry(bound.clip_step, "varco_clip_step");
  type(bound.Norm, "Norm");
  type(bound.NormGrad, "NormGrad");
  type(bound.Eight, "Eight");
  type(bound.EightWeight, "EightWeight");
  type(bound.Product, "Product");
  Py_INCREF(error);
  bound.error = error;
  Py_RETURN_NONE;
  END_HANDLE_TH_ERRORS
}

#define ENTRY(f) {#f, (PyCFunction)(void (*)(void))f, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {{"bind", bind, METH_VARARGS, nullptr},
                         ENTRY(norm_fwd),
                         ENTRY(norm_bwd),
                         ENTRY(quantize_rows),
                         ENTRY(quantize_weight),
                         ENTRY(fp8_product),
                         ENTRY(weight_grad),
                         ENTRY(grad_norm),
                         ENTRY(grad_clip),
                         ENTRY(clip_step),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_operators", "Operators of the residual block: checks, outputs, calls.", -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__operators() { return PyModule_Create(&module); }
