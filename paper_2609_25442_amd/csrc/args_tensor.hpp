// What the binding's operators check of torch tensors, and how their results
// are made (args_ops.cpp, args_train.cpp).
#ifndef WB_ARGS_TENSOR_HPP
#define WB_ARGS_TENSOR_HPP

#include <ATen/ATen.h>
#include <c10/core/GradMode.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>
#include <initializer_list>
#include <stdexcept>
#include <string>
#include <utility>

#include "../../include/wb.h"

namespace wb_args {

using at::Tensor;

struct Refused : std::runtime_error {
  using std::runtime_error::runtime_error;
};

[[noreturn]] inline void refuse(const char* name, const char* what) { throw Refused(std::string(name) + " " + what); }

inline int32_t code_of(at::ScalarType t, const char* name) {
  switch (t) {
    case at::kFloat: return WB_F32;
    case at::kBFloat16: return WB_BF16;
    case at::kFloat8_e4m3fn: return WB_F8E4M3;
    default: refuse(name, "is neither float32 nor bfloat16 nor float8_e4m3fn");
  }
}

inline at::ScalarType type_of(int32_t code) {
  if (code != WB_F32 && code != WB_BF16 && code != WB_F8E4M3) throw Refused("unknown out_dtype");
  return code == WB_F32 ? at::kFloat : code == WB_BF16 ? at::kBFloat16 : at::kFloat8_e4m3fn;
}

// A tensor argument on the call's device; null for None. One with a tangent of
// forward-mode differentiation is refused: no result here would carry it on.
inline const Tensor* tensor(PyObject* o, const char* name, int64_t device) {
  if (o == Py_None) return nullptr;
  if (!THPVariable_Check(o)) refuse(name, "is no tensor");
  const Tensor& t = THPVariable_Unpack(o);
  if (!t.defined() || !t.is_cuda() || t.layout() != at::kStrided) refuse(name, "is not in device memory");
  if (t.get_device() != device) refuse(name, "is on another device than the current one");
  if (t._fw_grad(0).defined()) refuse(name, "has a forward-mode tangent, which the operators do not carry on");
  return &t;
}

inline const Tensor& needed(PyObject* o, const char* name, int64_t device) {
  const Tensor* t = tensor(o, name, device);
  if (!t) refuse(name, "is None");
  return *t;
}

// A result made here has no graph behind it: where one is being recorded, an
// argument that requires a gradient would lose it without a word.
inline void ungraded(std::initializer_list<std::pair<const Tensor*, const char*>> all) {
  if (!c10::GradMode::is_enabled()) return;
  for (const auto& [t, name] : all)
    if (t && t->requires_grad())
      refuse(name, "requires a gradient, which this operator does not have: detach it, or call under torch.no_grad()");
}

// [rows, cols], or [n, rows, cols] as its n * rows rows.
inline wb_matrix matrix(const Tensor& t, const char* name, bool stacked = false) {
  const int64_t d = t.dim();
  if (d != 2 && !(stacked && d == 3)) refuse(name, stacked ? "has neither two nor three dimensions" : "does not have two dimensions");
  wb_matrix m{};
  m.data = t.data_ptr();
  m.dtype = code_of(t.scalar_type(), name);
  m.rows = t.size(d - 2), m.cols = t.size(d - 1);
  if (m.cols > 1 && t.stride(d - 1) != 1) refuse(name, "has columns that are not neighbours");
  m.ld = m.rows > 1 ? t.stride(d - 2) : m.cols;
  if (d == 3) {
    const int64_t n = t.size(0);
    if (m.rows == 1 && n > 1) m.ld = t.stride(0);
    if (n > 1 && t.stride(0) != m.rows * m.ld) refuse(name, "has matrices that do not lie row after row");
    m.rows *= n;
  }
  if (m.ld < m.cols) refuse(name, "has rows that overlap");
  return m;
}

inline wb_matrix vector(const Tensor& t, const char* name) {
  if (t.dim() != 1 || (t.numel() > 1 && t.stride(0) != 1)) refuse(name, "is no contiguous vector");
  wb_matrix m{};
  m.data = t.data_ptr();
  m.dtype = code_of(t.scalar_type(), name);
  m.rows = 1, m.cols = m.ld = t.numel();
  return m;
}

inline const Tensor& plain(const Tensor& t, at::ScalarType type, int64_t count, const char* name) {
  if (t.scalar_type() != type) refuse(name, "has another dtype");
  if (!t.is_contiguous()) refuse(name, "is not contiguous");
  if (t.numel() != count) refuse(name, "has another number of elements");
  return t;
}

// One of the tensors that lie one after the other in `base`.
inline Tensor part(const Tensor& base, int64_t& at, at::IntArrayRef shape) {
  Tensor t = at::detail::make_tensor<c10::TensorImpl>(c10::Storage(base.storage()), base.key_set(), base.dtype());
  t.unsafeGetTensorImpl()->set_storage_offset(base.storage_offset() + at);
  t.unsafeGetTensorImpl()->set_sizes_contiguous(shape);
  at += t.numel();
  return t;
}

inline Tensor fresh(at::IntArrayRef shape, at::ScalarType type, const Tensor& like) {
  return at::empty(shape, like.options().dtype(type));
}

inline int64_t scale_cols(int64_t cols) { return (cols + 127) / 128; }

inline PyObject* wrap(const Tensor& t) {
  if (!t.defined()) Py_RETURN_NONE;
  return THPVariable_Wrap(t);
}

// A refusal becomes its text; what torch throws (no memory for a result) the
// Python exception that torch has for it.
template <class F>
PyObject* guarded(F&& f) {
  HANDLE_TH_ERRORS
  try {
    return f();
  } catch (const Refused& e) {
    return PyUnicode_FromString(e.what());
  }
  END_HANDLE_TH_ERRORS
}

inline bool counted(Py_ssize_t got, Py_ssize_t want, const char* call) {
  if (got == want) return true;
  PyErr_Format(PyExc_TypeError, "%s takes %zd arguments", call, want);
  return false;
}

template <class F>
F* function(PyObject* o) { return reinterpret_cast<F*>(PyLong_AsVoidPtr(o)); }

// What every call ends with: the device and the stream.
struct Where {
  int64_t device;
  void* stream;
  explicit Where(PyObject* const* args) : device(PyLong_AsLongLong(args[0])), stream(PyLong_AsVoidPtr(args[1])) {}
};

}  // namespace wb_args

#endif
