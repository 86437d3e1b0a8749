// The calls of block_fp8.py: checks of the tensors, allocation of outputs, the argument structs of as_fp8.h, the call.  In C++ because these calls take 2 to 6 us on the GPU where
// there are few rows, and the same steps in Python took 9 to 11 us of the CPU's time (here 3 to 5).  A module of its own beside libas_hybrid_attn.so, which itself knows nothing of
// PyTorch.
#include "torch_args.h"

namespace {

using namespace as_calls;

// (x, weight, residual, eps, fp8, out, residual_out)
PyObject* rms_norm(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  ARGS(7)
  const char* where = "rms_norm";
  const int here = c10::cuda::current_device();
  as_rms_norm_t p{};
  int64_t rows, cols, r, c;
  const at::Tensor* x = rows_of(a[0], here, where, "x", p.x, rows, cols);
  if (x == nullptr) return nullptr;
  p.struct_size = sizeof p;
  p.rows = rows; p.cols = (int32_t)cols;
  p.eps = (float)PyFloat_AsDouble(a[3]);
  if (PyErr_Occurred()) return nullptr;
  if (a[1] != Py_None && !vector_of(a[1], cols, true, here, where, "weight", p.weight, p.weight_dtype)) return nullptr;
  Held out, total;
  Pair pair;
  if (a[2] != Py_None) {
    const at::Tensor* t = rows_of(a[2], here, where, "residual", p.residual, r, c);
    if (t == nullptr) return nullptr;
    if (r != rows || c != cols) { refuse(where, "residual", "has not x's rows and columns"); return nullptr; }
    if (a[6] != Py_None) total.share(a[6]);
    else total.take(empty_contiguous(t->sizes(), t->scalar_type(), here));
    const at::Tensor* u = rows_of(total.o, here, where, "residual_out", p.residual_out, r, c);
    if (u == nullptr) return nullptr;
    if (r != rows || c != cols || u->scalar_type() != t->scalar_type()) { refuse(where, "residual_out", "has not the residual's rows, columns and type"); return nullptr; }
  } else if (a[6] != Py_None) {
    refuse(where, "residual_out", "needs a residual");
    return nullptr;
  }
  const int fp8 = PyObject_IsTrue(a[4]);
  if (fp8 < 0) return nullptr;
  if (a[5] != Py_None) out.share(a[5]);
  else if (fp8) out.take(empty_pair(rows, cols, here));
  else out.take(empty_contiguous(x->sizes(), at::kBFloat16, here));
  if (out.o == nullptr) return nullptr;
  if (fp8 ? !matrix_of(out.o, here, where, "out", pair, p.out8, r, c) : rows_of(out.o, here, where, "out", p.out, r, c) == nullptr) return nullptr;
  if (r != rows || c != cols) { refuse(where, "out", "has not x's rows and columns"); return nullptr; }
  if (rows > 0 && cols > 0 && !status(as_rms_norm(&p, current_stream(here)), "as_rms_norm")) return nullptr;
  if (a[5] != Py_None) { if (fp8) written(pair); else written(out.o); }
  if (a[6] != Py_None) written(total.o);
  if (total.o == nullptr) return out.give();
  return PyTuple_Pack(2, out.o, total.o);
  END_HANDLE_TH_ERRORS
}

// (x, block_rows, out)
PyObject* quantize_fp8(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  ARGS(3)
  const char* where = "quantize_fp8";
  const int here = c10::cuda::current_device();
  as_quantize_fp8_t p{};
  int64_t rows, cols, r, c;
  if (rows_of(a[0], here, where, "x", p.x, rows, cols) == nullptr) return nullptr;
  p.struct_size = sizeof p;
  p.rows = rows; p.cols = (int32_t)cols;
  const long block = PyLong_AsLong(a[1]);
  if (PyErr_Occurred()) return nullptr;
  p.block_rows = block == 1 || block == 128 ? (int32_t)block : 0;
  Held out;
  Pair pair;
  if (a[2] != Py_None) out.share(a[2]);
  else out.take(empty_pair(rows, cols, here));
  if (out.o == nullptr || !matrix_of(out.o, here, where, "out", pair, p.out, r, c)) return nullptr;
  if (r != rows || c != cols) { refuse(where, "out", "has not x's rows and columns"); return nullptr; }
  if (rows > 0 && cols > 0 && !status(as_quantize_fp8(&p, current_stream(here)), "as_quantize_fp8")) return nullptr;
  if (a[2] != Py_None) written(pair);
  return out.give();
  END_HANDLE_TH_ERRORS
}

// (a, w, bias, out)
PyObject* matmul_fp8(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  ARGS(4)
  const char* where = "matmul_fp8";
  const int here = c10::cuda::current_device();
  as_matmul_fp8_t p{};
  int64_t m, k, n, wk, r, c;
  Pair of_a, of_w;
  if (!matrix_of(a[0], here, where, "a", of_a, p.a, m, k) || !matrix_of(a[1], here, where, "w", of_w, p.w, n, wk)) return nullptr;
  if (k != wk) { refuse(where, "w", "has not a's columns"); return nullptr; }
  if (k == 0 && m > 0 && n > 0) { refuse(where, "a", "has no columns to sum over"); return nullptr; }
  int32_t dtype;
  if (a[2] != Py_None && !vector_of(a[2], n, false, here, where, "bias", p.bias, dtype)) return nullptr;
  Held out;
  if (a[3] != Py_None) out.share(a[3]);
  else out.take(empty({m, n}, {n, 1}, at::kBFloat16, here));
  if (rows_of(out.o, here, where, "out", p.out, r, c) == nullptr) return nullptr;
  if (r != m || c != n || p.out.dtype != AS_DTYPE_BF16) { refuse(where, "out", "is not a's rows by w's rows in bf16"); return nullptr; }
  if (m > 0 && n > 0) {
    p.struct_size = sizeof p;
    p.rows = m; p.out_cols = n;
    p.cols = (int32_t)std::min<int64_t>(k, INT32_MAX);
    as_fp8_context_t ctx;
    if (!context_of(here, ctx) || !status(as_matmul_fp8(ctx, &p, current_stream(here)), "as_matmul_fp8")) return nullptr;
  }
  if (a[3] != Py_None) written(out.o);
  return out.give();
  END_HANDLE_TH_ERRORS
}

PyObject* last_status(PyObject*, PyObject*) {
  HANDLE_TH_ERRORS
  const int here = c10::cuda::current_device();
  as_fp8_context_t ctx;
  if (!context_of(here, ctx)) return nullptr;
  as_status_t s;
  Py_BEGIN_ALLOW_THREADS
  s = as_fp8_last_status(ctx, current_stream(here));
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(s);
  END_HANDLE_TH_ERRORS
}

// (BlockFp8, AsError)
PyObject* set_classes(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  ARGS(2)
  if (!PyType_Check(a[0]) || !PyType_IsSubtype(reinterpret_cast<PyTypeObject*>(a[0]), &PyTuple_Type)) {
    PyErr_SetString(PyExc_TypeError, "BlockFp8 is a tuple");
    return nullptr;
  }
  Py_INCREF(a[0]); Py_INCREF(a[1]);
  Py_XDECREF(g_block_fp8); Py_XDECREF(g_as_error);
  g_block_fp8 = a[0]; g_as_error = a[1];
  Py_RETURN_NONE;
}

template <typename F> PyCFunction fast(F f) { return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)); }
PyMethodDef methods[] = {{"rms_norm", fast(rms_norm), METH_FASTCALL, nullptr}, {"quantize_fp8", fast(quantize_fp8), METH_FASTCALL, nullptr},
                         {"matmul_fp8", fast(matmul_fp8), METH_FASTCALL, nullptr}, {"last_status", last_status, METH_NOARGS, nullptr},
                         {"set_classes", fast(set_classes), METH_FASTCALL, nullptr},
                         {"rotary_table", fast(rotary_table), METH_FASTCALL, nullptr}, {"qk_norm_rotary", fast(qk_norm_rotary), METH_FASTCALL, nullptr},
                         {"qk_norm_rotary_backward", fast(qk_norm_rotary_backward), METH_FASTCALL, nullptr}, {"linear", fast(linear), METH_FASTCALL, nullptr},
                         {"linear_backward", fast(linear_backward), METH_FASTCALL, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "as_torch_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit_as_torch_calls() { return PyModule_Create(&module); }
