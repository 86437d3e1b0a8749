// What the calls that take PyTorch tensors share: checks of tensors, their layouts as the C ABI has them, allocation of outputs, errors.
#pragma once

#include <ATen/core/grad_mode.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/core/AutogradState.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <mutex>

#include "as_layer.h"

namespace as_calls {

inline PyObject *g_block_fp8 = nullptr, *g_as_error = nullptr;      // the classes BlockFp8 and AsError
inline std::mutex g_lock;
inline as_fp8_context_t g_contexts[64] = {};

// A refusal: the call, the argument's name and what is wrong with it.
inline bool refuse(const char* where, const char* name, const char* what) {
  PyErr_Format(PyExc_ValueError, "%s: %s %s", where, name, what);
  return false;
}
inline bool status(as_status_t s, const char* where) {
  if (s == AS_OK) return true;
  PyObject* e = PyObject_CallFunction(g_as_error, "is", (int)s, where);
  if (e != nullptr) {
    PyErr_SetObject(g_as_error, e);
    Py_DECREF(e);
  }
  return false;
}

// An object that is given back or let go.
struct Held {
  PyObject* o;
  explicit Held(PyObject* p = nullptr) : o(p) {}
  ~Held() { Py_XDECREF(o); }
  Held(const Held&) = delete;
  Held& operator=(const Held&) = delete;
  PyObject* give() { PyObject* p = o; o = nullptr; return p; }
  void take(PyObject* p) { Py_XDECREF(o); o = p; }
  void share(PyObject* p) { Py_INCREF(p); take(p); }
};

inline const at::Tensor* tensor_of(PyObject* o, int here, const char* where, const char* name) {
  if (!THPVariable_Check(o)) { refuse(where, name, "is no tensor"); return nullptr; }
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.is_cuda() || t.get_device() != here || t.layout() != at::kStrided) { refuse(where, name, "is not a strided tensor on the current CUDA device"); return nullptr; }
  if (t.requires_grad() && at::GradMode::is_enabled()) { refuse(where, name, "requires a gradient, which these calls have none of: detach it, or call under torch.no_grad()"); return nullptr; }
  if (t.is_neg()) { refuse(where, name, "is a view whose values count negated: resolve_neg() writes them out"); return nullptr; }
  if (t._fw_grad(0).defined() && c10::AutogradState::get_tls_state().get_fw_grad_mode()) { refuse(where, name, "carries a forward-mode tangent, which these calls would drop"); return nullptr; }
  return &t;
}
// A tensor of the caller's that the call has written: what autograd has saved of it is no longer there.  (Inference tensors keep no count.)
inline void written(PyObject* o) {
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}

// [rows, cols] or [B, H, N, d] as an as_rows_t.  A single row, column or head leaves its stride open.
inline const at::Tensor* rows_of(PyObject* o, int here, const char* where, const char* name, as_rows_t& r, int64_t& rows, int64_t& cols) {
  const at::Tensor* t = tensor_of(o, here, where, name);
  if (t == nullptr) return nullptr;
  const auto type = t->scalar_type();
  if (type != at::kBFloat16 && type != at::kFloat) { refuse(where, name, "is neither bf16 nor fp32"); return nullptr; }
  const auto size = t->sizes(), stride = t->strides();
  if (size.size() == 2) {
    rows = size[0]; cols = size[1];
    r = as_rows_t{t->data_ptr(), type == at::kFloat ? AS_DTYPE_F32 : AS_DTYPE_BF16, (int32_t)cols, rows, 0, 0, rows > 1 ? stride[0] : 0};
  } else if (size.size() == 4) {
    rows = size[0] * size[2]; cols = size[1] * size[3];
    r = as_rows_t{t->data_ptr(), type == at::kFloat ? AS_DTYPE_F32 : AS_DTYPE_BF16, (int32_t)size[3], size[2], size[0] > 1 ? stride[0] : 0, size[1] > 1 ? stride[1] : 0,
                  size[2] > 1 ? stride[2] : 0};
  } else {
    refuse(where, name, "is neither [rows, cols] nor [B, H, N, d]");
    return nullptr;
  }
  if (size.back() > INT32_MAX || cols > INT32_MAX) { refuse(where, name, "has too many columns"); return nullptr; }
  if (stride.back() != 1 && size.back() > 1) { refuse(where, name, "has columns that do not lie next to each other"); return nullptr; }
  return t;
}

// The tensors of a pair, held for as long as the call uses them: what hands them out need not keep them (an iterator does not).
struct Pair { Held data, scales; };
inline void written(const Pair& pair) { written(pair.data.o); written(pair.scales.o); }

// A pair (e4m3 values, scales) as an as_fp8_matrix_t.
inline bool matrix_of(PyObject* pair, int here, const char* where, const char* name, Pair& hold, as_fp8_matrix_t& m, int64_t& rows, int64_t& cols) {
  PyObject* fast = PySequence_Fast(pair, "a matrix in 8-bit form is a pair of tensors");
  if (fast == nullptr) return false;
  if (PySequence_Fast_GET_SIZE(fast) != 2) { Py_DECREF(fast); return refuse(where, name, "is no pair of tensors"); }
  hold.data.share(PySequence_Fast_GET_ITEM(fast, 0));
  hold.scales.share(PySequence_Fast_GET_ITEM(fast, 1));
  Py_DECREF(fast);
  const at::Tensor* data = tensor_of(hold.data.o, here, where, name);
  const at::Tensor* scales = data == nullptr ? nullptr : tensor_of(hold.scales.o, here, where, name);
  if (scales == nullptr) return false;
  if (data->scalar_type() != at::kFloat8_e4m3fn || scales->scalar_type() != at::kByte || data->dim() != 2 || scales->dim() != 3)
    return refuse(where, name, "is no pair of float8_e4m3fn [rows, cols] and uint8 [ceil(cols / 512), rows, 4]");
  rows = data->size(0); cols = data->size(1);
  const int64_t groups = (cols + 511) / 512;
  if (scales->size(0) != groups || scales->size(1) != rows || scales->size(2) != 4) return refuse(where, name, "has scales that are not [ceil(cols / 512), rows, 4]");
  const int64_t st = data->stride(0), sg = scales->stride(0);
  if ((data->stride(1) != 1 && cols > 1) || scales->stride(2) != 1 || (scales->stride(1) != 4 && rows > 1) || (groups > 1 && rows > 0 && (sg % 4 != 0 || sg < 4 * rows)))
    return refuse(where, name, "has values, or scales of a row or of one row and the next, that do not lie next to each other");
  m = as_fp8_matrix_t{data->data_ptr(), rows > 1 ? st : (cols + 15) / 16 * 16, scales->data_ptr(), groups > 1 ? sg / 4 : rows};
  return true;
}

inline bool vector_of(PyObject* o, int64_t n, bool f32, int here, const char* where, const char* name, const void*& data, int32_t& dtype) {
  const at::Tensor* t = tensor_of(o, here, where, name);
  if (t == nullptr) return false;
  const auto type = t->scalar_type();
  if (!(type == at::kBFloat16 || (f32 && type == at::kFloat)) || t->dim() != 1 || t->size(0) != n || (n > 1 && t->stride(0) != 1))
    return refuse(where, name, f32 ? "is not a value in bf16 or fp32 for each column, next to each other" : "is not a value in bf16 for each column, next to each other");
  data = t->data_ptr();
  dtype = type == at::kFloat ? AS_DTYPE_F32 : AS_DTYPE_BF16;
  return true;
}

inline PyObject* empty(at::IntArrayRef size, at::IntArrayRef stride, at::ScalarType type, int here) {
  return THPVariable_Wrap(at::Tensor(at::detail::empty_strided_cuda(size, stride, type, at::Device(at::kCUDA, (c10::DeviceIndex)here))));
}
inline PyObject* empty_contiguous(at::IntArrayRef size, at::ScalarType type, int here) {
  return THPVariable_Wrap(at::Tensor(at::detail::empty_cuda(size, type, at::Device(at::kCUDA, (c10::DeviceIndex)here), std::nullopt)));
}
// A BlockFp8 of new tensors, which share one allocation (two take 0.3 us more).
inline PyObject* empty_pair(int64_t rows, int64_t cols, int here) {
  const int64_t pitch = (cols + 15) / 16 * 16, groups = (cols + 511) / 512, values = (rows * pitch + 255) / 256 * 256;
  const at::Tensor whole(at::detail::empty_cuda({values + 4 * groups * rows}, at::kByte, at::Device(at::kCUDA, (c10::DeviceIndex)here), std::nullopt));
  auto part = [&](at::ScalarType type, at::IntArrayRef size, at::IntArrayRef stride, int64_t from) {
    at::Tensor t = at::detail::make_tensor<c10::TensorImpl>(c10::TensorImpl::VIEW, c10::Storage(whole.storage()), whole.key_set(), c10::scalarTypeToTypeMeta(type));
    t.unsafeGetTensorImpl()->set_sizes_and_strides(size, stride, from);
    return THPVariable_Wrap(std::move(t));
  };
  PyObject* two = PyTuple_New(2);
  if (two == nullptr) return nullptr;
  PyTuple_SET_ITEM(two, 0, part(at::kFloat8_e4m3fn, {rows, cols}, {pitch, 1}, 0));
  PyTuple_SET_ITEM(two, 1, part(at::kByte, {groups, rows, 4}, {4 * rows, 4, 1}, values));
  PyObject* args = PyTuple_Pack(1, two);
  Py_DECREF(two);
  if (args == nullptr) return nullptr;
  PyObject* made = PyTuple_Type.tp_new(reinterpret_cast<PyTypeObject*>(g_block_fp8), args, nullptr);
  Py_DECREF(args);
  return made;
}

inline bool context_of(int here, as_fp8_context_t& ctx) {
  if (here < 0 || here >= 64) return status(AS_ERR_UNSUPPORTED, "as_fp8_create");
  as_status_t s = AS_OK;
  {
    std::lock_guard<std::mutex> hold(g_lock);
    if (g_contexts[here] == nullptr) s = as_fp8_create(&g_contexts[here]);
    ctx = g_contexts[here];
  }
  return status(s, "as_fp8_create");        // behind the lock: making the exception runs Python code, which may let another thread in here
}

inline void* current_stream(int here) { return c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)here).stream(); }

#define ARGS(n)                                                               \
  if (nargs != n) {                                                           \
    PyErr_SetString(PyExc_TypeError, "wrong number of arguments");            \
    return nullptr;                                                           \
  }

// The calls of torch_layer_calls.cpp.
PyObject* rotary_table(PyObject*, PyObject* const* a, Py_ssize_t nargs);
PyObject* qk_norm_rotary(PyObject*, PyObject* const* a, Py_ssize_t nargs);
PyObject* qk_norm_rotary_backward(PyObject*, PyObject* const* a, Py_ssize_t nargs);
PyObject* linear(PyObject*, PyObject* const* a, Py_ssize_t nargs);
PyObject* linear_backward(PyObject*, PyObject* const* a, Py_ssize_t nargs);

}  // namespace as_calls
