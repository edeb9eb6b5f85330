// The operators for tensors: what their translation units share.  Checks of shapes, types, places and history, outputs from PyTorch's
// allocator, the current stream.
#pragma once

#include <ATen/ATen.h>
#include <c10/core/AutogradState.h>
#include <c10/core/GradMode.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/utils/pybind.h>

#include <climits>
#include <optional>
#include <string>

#include "moe_cache.h"

namespace py = pybind11;
using at::Tensor;
using Maybe = std::optional<Tensor>;

void bind_attention(py::module &m);  // attend_torch.cpp

inline py::object *error_type;  // MoEError

[[noreturn]] inline void wrong(const std::string &what) { throw py::value_error(what); }

inline void check(int code, const char *where) {
  if (code == MOE_OK) return;
  const py::object e = (*error_type)(code, where);
  PyErr_SetObject(error_type->ptr(), e.ptr());
  throw py::error_already_set();
}

inline int format(const Tensor &t, const char *name, bool codes = false) {
  const at::ScalarType s = t.scalar_type();
  if (s == at::kFloat) return MOE_R_FP32;
  if (s == at::kBFloat16) return MOE_R_BF16;
  if (codes && s == at::kChar) return MOE_R_INT8;
  wrong(std::string(name) + ": " + c10::toString(s) + (codes ? " is none of float32, bfloat16 and int8" : " is neither float32 nor bfloat16"));
}

inline int32_t size32(int64_t v) {
  if (v > INT_MAX) wrong("a size of " + std::to_string(v) + " is too large");
  return (int32_t)v;
}

struct Rows {
  int32_t n, d;
  int64_t stride;
};
// a matrix whose rows are dense (they may lie apart)
inline Rows rows_of(const Tensor &t, const char *name) {
  if (t.dim() != 2 || (t.stride(1) != 1 && t.size(1) > 1)) wrong(std::string(name) + " has to be a matrix with dense rows");
  return {size32(t.size(0)), size32(t.size(1)), t.size(0) > 1 ? t.stride(0) : t.size(1)};
}

inline void dense(const Tensor &t, at::IntArrayRef shape, std::optional<at::ScalarType> type, const char *name) {
  if (t.sizes() == shape && t.is_contiguous() && (!type || t.scalar_type() == *type)) return;
  std::string s = std::string(name) + " has to be contiguous, (";
  for (size_t i = 0; i < shape.size(); ++i) s += (i ? ", " : "") + std::to_string(shape[i]);
  wrong(s + ")" + (type ? std::string(", ") + c10::toString(*type) : ""));
}
inline void dense(const Maybe &t, at::IntArrayRef shape, std::optional<at::ScalarType> type, const char *name) {
  if (t) dense(*t, shape, type, name);
}

inline const void *at_(const Maybe &t) { return t ? t->const_data_ptr() : nullptr; }
inline const float *floats(const Maybe &t) { return static_cast<const float *>(at_(t)); }
inline const int32_t *ints(const Tensor &t) { return static_cast<const int32_t *>(t.const_data_ptr()); }
inline void *to(const Maybe &t) { return t ? t->mutable_data_ptr() : nullptr; }
inline float *to_floats(const Maybe &t) { return static_cast<float *>(to(t)); }
inline int32_t *to_ints(const Tensor &t) { return static_cast<int32_t *>(t.mutable_data_ptr()); }
// within: what the library takes.  It refuses other sizes before it looks at a pointer, and nothing is allocated for them.
inline Tensor fresh(const Tensor &like, at::IntArrayRef shape, at::ScalarType type, bool within) {
  static constexpr int64_t nothing[] = {0};
  return at::empty(within ? shape : at::IntArrayRef(nothing), like.options().dtype(type));
}
inline bool within(int64_t rows, int64_t hidden) { return rows < MOE_ROWS_LIMIT && hidden <= MOE_ROWS_MAX_HIDDEN; }

inline bool differentiable(const Tensor &t) { return t.requires_grad(); }
inline bool differentiable(const Maybe &t) { return t && t->requires_grad(); }
inline bool has_tangent(const Tensor &t) { return t._fw_grad(0).defined(); }  // (there is one level)
inline bool has_tangent(const Maybe &t) { return t && has_tangent(*t); }
// The results have no history for automatic differentiation: a caller who would lose a gradient that way, or a tangent of the
// forward mode (which torch.no_grad() does not switch off), is told.
template <typename... T>
inline void no_history(const T &...t) {
  if (c10::GradMode::is_enabled() && (differentiable(t) || ...))
    wrong("an input requires a gradient, which this call does not record: call it under torch.no_grad(), or in a torch.autograd.Function with the backward calls");
  if (c10::AutogradState::get_tls_state().get_fw_grad_mode() && (has_tangent(t) || ...))
    wrong("an input has a tangent of forward-mode differentiation, which this call does not propagate: call it on the primal, or in a torch.autograd.Function with a jvp");
}

// The GPU that all tensors are on, current for the call, and its current stream
class Place {
 public:
  explicit Place(const Tensor &t) {
    if (!t.is_cuda()) wrong("the tensors have to be on a GPU");
    at_ = t.get_device();
    back_ = c10::hip::current_device();
    if (back_ != at_) c10::hip::set_device(at_);
  }
  Place(const Place &) = delete;
  ~Place() {
    if (back_ != at_) c10::hip::set_device(back_);
  }
  template <typename... T>
  void has(const T &...t) const {
    (one(t), ...);
  }
  void *stream() const { return c10::hip::getCurrentHIPStream(at_).stream(); }

 private:
  void one(const Tensor &t) const {
    if (!t.is_cuda() || t.get_device() != at_) wrong("all tensors have to be on one GPU");
  }
  void one(const Maybe &t) const {
    if (t) one(*t);
  }
  c10::DeviceIndex at_, back_;
};
