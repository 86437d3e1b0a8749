// The calls of rotation.py and projection.py: checks of the tensors, allocation of outputs and workspaces, the argument structs of as_layer.h, the call.
#include "torch_args.h"

namespace as_calls {

namespace {

// Whole numbers of a tuple.
bool ints_of(PyObject* o, const char* where, const char* name, int most, int32_t* to, int& n) {
  if (!PyTuple_Check(o) || PyTuple_GET_SIZE(o) < 1 || PyTuple_GET_SIZE(o) > most) return refuse(where, name, "is not a tuple of one to four whole numbers");
  n = (int)PyTuple_GET_SIZE(o);
  for (int i = 0; i < n; ++i) {
    const long v = PyLong_AsLong(PyTuple_GET_ITEM(o, i));
    if (PyErr_Occurred()) return false;
    if (v < 1 || v > INT32_MAX) return refuse(where, name, "has numbers that are not positive");
    to[i] = (int32_t)v;
  }
  return true;
}

// [B, H, N, d] as an as_rows_t.
const at::Tensor* heads_of(PyObject* o, int here, const char* where, const char* name, as_rows_t& r, int64_t& rows, int32_t& heads) {
  int64_t cols;
  const at::Tensor* t = rows_of(o, here, where, name, r, rows, cols);
  if (t == nullptr) return nullptr;
  if (t->dim() != 4) { refuse(where, name, "is not [B, H, N, d]"); return nullptr; }
  heads = (int32_t)t->size(1);
  return t;
}
bool like(const at::Tensor* t, const at::Tensor* u, const char* where, const char* name) {
  if (t->sizes() != u->sizes() || t->scalar_type() != u->scalar_type()) return refuse(where, name, "has not the shape and type of what it belongs to");
  return true;
}

// A table (factors, sizes, pairs), and the tokens' positions.
bool rotation_of(PyObject* table, PyObject* positions, PyObject* first, bool half, bool inverse, int64_t B, int64_t N, int here, const char* where, as_rotation_t& r) {
  if (table == Py_None) {
    if (positions != Py_None) return refuse(where, "positions", "need a table");
    return true;
  }
  if (!PyTuple_Check(table) || PyTuple_GET_SIZE(table) != 3) return refuse(where, "table", "is no triple of factors, sizes and pairs");
  const at::Tensor* f = tensor_of(PyTuple_GET_ITEM(table, 0), here, where, "table");
  if (f == nullptr) return false;
  int n, m;
  if (!ints_of(PyTuple_GET_ITEM(table, 1), where, "table", AS_ROTARY_MAX_AXES, r.size, n) || !ints_of(PyTuple_GET_ITEM(table, 2), where, "table", AS_ROTARY_MAX_AXES, r.pairs, m)) return false;
  int64_t rows = 0, pairs = 0;
  for (int i = 0; i < n; ++i) rows += r.size[i];
  for (int i = 0; i < m; ++i) pairs += r.pairs[i];
  if (n != m || f->scalar_type() != at::kFloat || f->dim() != 3 || f->size(0) != rows || f->size(1) != pairs || f->size(2) != 2 || !f->is_contiguous())
    return refuse(where, "table", "has factors that are not contiguous fp32 [sum of sizes, sum of pairs, 2]");
  r.table = static_cast<const float*>(f->data_ptr());
  r.n_axes = n;
  r.layout = half ? AS_ROTARY_HALF : AS_ROTARY_INTERLEAVED;
  r.inverse = inverse;
  r.first = PyLong_AsLongLong(first);
  if (PyErr_Occurred()) return false;
  if (positions == Py_None) return true;
  if (r.first != 0) return refuse(where, "first", "does not go with positions");
  const at::Tensor* p = tensor_of(positions, here, where, "positions");
  if (p == nullptr) return false;
  const auto type = p->scalar_type();
  if (type != at::kInt && type != at::kLong) return refuse(where, "positions", "are neither int32 nor int64");
  // [N], [B, N] for one axis; [N, axes], [B, N, axes]
  const int inner = n > 1 || p->dim() == 3 ? 1 : 0;
  const int64_t dims = p->dim(), entries = dims == 2 + inner ? p->size(0) : 1, N_at = dims - 1 - inner;
  if ((dims != 1 + inner && dims != 2 + inner) || p->size(N_at) != N || (inner && p->size(dims - 1) != n) || (entries != B && entries != 1))
    return refuse(where, "positions", "are not [N] or [B, N] (with several axes: [N, axes] or [B, N, axes])");
  if ((inner && n > 1 && p->stride(dims - 1) != 1) || (N > 1 && p->stride(N_at) != n)) return refuse(where, "positions", "do not lie next to each other");
  r.positions = p->data_ptr();
  r.position_bytes = type == at::kLong ? 8 : 4;
  r.positions_stride = dims == 2 + inner && entries > 1 ? p->stride(0) : 0;
  return true;
}

bool flag_of(PyObject* o, bool& f) {
  const int v = PyObject_IsTrue(o);
  f = v > 0;
  return v >= 0;
}
bool int_of(PyObject* o, int32_t& v) {
  v = (int32_t)PyLong_AsLong(o);
  return !PyErr_Occurred();
}

// Room that a call needs while it runs: it belongs to the current stream, behind whose work it is used again.
bool workspace_of(uint64_t bytes, int here, Held& hold, void*& at, uint64_t& has) {
  at = nullptr;
  has = bytes;
  if (bytes == 0) return true;
  hold.take(empty_contiguous({(int64_t)bytes}, at::kByte, here));
  if (hold.o == nullptr) return false;
  at = THPVariable_Unpack(hold.o).data_ptr();
  return true;
}

}  // namespace

// (sizes, pairs, bases, scalings, factors, originals): tuples of one length
PyObject* rotary_table(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  ARGS(6)
  const char* where = "rotary_table";
  const int here = c10::cuda::current_device();
  int32_t sizes[AS_ROTARY_MAX_AXES], pairs[AS_ROTARY_MAX_AXES];
  int n, m;
  if (!ints_of(a[0], where, "sizes", AS_ROTARY_MAX_AXES, sizes, n) || !ints_of(a[1], where, "pairs", AS_ROTARY_MAX_AXES, pairs, m)) return nullptr;
  if (n != m) { refuse(where, "pairs", "are not one number for each size"); return nullptr; }
  as_rotary_axis_t axes[AS_ROTARY_MAX_AXES] = {};
  int64_t rows = 0, total = 0;
  for (int i = 0; i < n; ++i) {
    for (int j = 2; j < 6; ++j)
      if (!PyTuple_Check(a[j]) || PyTuple_GET_SIZE(a[j]) != n) { refuse(where, "base, scaling, factor or original", "is not one for each axis"); return nullptr; }
    axes[i].size = sizes[i];
    axes[i].pairs = pairs[i];
    axes[i].base = PyFloat_AsDouble(PyTuple_GET_ITEM(a[2], i));
    axes[i].scaling = (int32_t)PyLong_AsLong(PyTuple_GET_ITEM(a[3], i));
    axes[i].factor = PyFloat_AsDouble(PyTuple_GET_ITEM(a[4], i));
    axes[i].original = PyFloat_AsDouble(PyTuple_GET_ITEM(a[5], i));
    if (PyErr_Occurred()) return nullptr;
    rows += sizes[i];
    total += pairs[i];
  }
  if (total > 8192 || rows > INT32_MAX) { refuse(where, "sizes, pairs", "are too many"); return nullptr; }
  Held out(empty_contiguous({rows, total, 2}, at::kFloat, here));
  if (out.o == nullptr) return nullptr;
  if (!status(as_rotary_table(axes, n, static_cast<float*>(THPVariable_Unpack(out.o).data_ptr()), current_stream(here)), "as_rotary_table")) return nullptr;
  return out.give();
  END_HANDLE_TH_ERRORS
}

namespace {

struct TurnArgs { const at::Tensor *q, *k; as_qk_norm_rotary_t p; };
// (q, k, q_weight, k_weight, table, norm, eps, half, inverse, positions, first) from a[0] on
bool turn_args(PyObject* const* a, int here, const char* where, TurnArgs& t) {
  as_qk_norm_rotary_t& p = t.p;
  p.struct_size = sizeof p;
  int64_t rows;
  t.q = heads_of(a[0], here, where, "q", p.q, p.rows, p.q_heads);
  if (t.q == nullptr) return false;
  p.head_dim = (int32_t)t.q->size(3);
  if (a[1] != Py_None) {
    t.k = heads_of(a[1], here, where, "k", p.k, rows, p.k_heads);
    if (t.k == nullptr) return false;
    if (t.k->size(0) != t.q->size(0) || t.k->size(2) != t.q->size(2) || t.k->size(3) != t.q->size(3) || t.k->scalar_type() != t.q->scalar_type())
      return refuse(where, "k", "has not q's batch, tokens, head size and type");
  }
  if (!int_of(a[5], p.norm)) return false;
  p.eps = (float)PyFloat_AsDouble(a[6]);
  if (PyErr_Occurred()) return false;
  int32_t types[2] = {-1, -1};
  const char* names[2] = {"q_weight", "k_weight"};
  const void* data[2] = {nullptr, nullptr};
  for (int i = 0; i < 2; ++i)
    if (a[2 + i] != Py_None) {
      if (p.norm == AS_NORM_NONE) return refuse(where, names[i], "needs a norm");
      if (i == 1 && t.k == nullptr) return refuse(where, names[i], "needs a k");
      const int64_t n = p.norm == AS_NORM_ROW ? (int64_t)(i == 0 ? p.q_heads : p.k_heads) * p.head_dim : p.head_dim;
      if (!vector_of(a[2 + i], n, true, here, where, names[i], data[i], types[i])) return false;
    }
  if (types[0] >= 0 && types[1] >= 0 && types[0] != types[1]) return refuse(where, "k_weight", "has not q_weight's type");
  p.q_weight = data[0]; p.k_weight = data[1];
  p.weight_dtype = types[0] >= 0 ? types[0] : types[1] >= 0 ? types[1] : AS_DTYPE_BF16;
  bool half, inverse;
  if (!flag_of(a[7], half) || !flag_of(a[8], inverse)) return false;
  return rotation_of(a[4], a[9], a[10], half, inverse, t.q->size(0), t.q->size(2), here, where, p.rotation);
}
// An output: the one that is given, or a new one in [B, H, N, d] order.
bool out_of(PyObject* given, const at::Tensor* t, int here, const char* where, const char* name, Held& hold, as_rows_t& r) {
  if (given != Py_None) hold.share(given);
  else hold.take(empty_contiguous(t->sizes(), t->scalar_type(), here));
  int64_t rows;
  int32_t heads;
  if (hold.o == nullptr) return false;
  const at::Tensor* u = heads_of(hold.o, here, where, name, r, rows, heads);
  return u != nullptr && like(u, t, where, name);
}
bool anything(const at::Tensor* t) { return t->numel() > 0; }

}  // namespace

// (q, k, q_weight, k_weight, table, norm, eps, half, inverse, positions, first, q_out, k_out)
PyObject* qk_norm_rotary(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  ARGS(13)
  const int here = c10::cuda::current_device();
  TurnArgs t{};
  const char* where = a[1] == Py_None ? "rotary" : "qk_norm_rotary";
  if (!turn_args(a, here, where, t)) return nullptr;
  Held q, k;
  if (!out_of(a[11], t.q, here, where, "q_out", q, t.p.q_out)) return nullptr;
  if (t.k != nullptr) {
    if (!out_of(a[12], t.k, here, where, "k_out", k, t.p.k_out)) return nullptr;
  } else if (a[12] != Py_None) {
    refuse(where, "k_out", "needs a k");
    return nullptr;
  }
  const bool some = anything(t.q) && (t.k == nullptr || anything(t.k));
  if (!some && (anything(t.q) || (t.k != nullptr && anything(t.k)))) { refuse(where, "k", "or q has no heads"); return nullptr; }
  if (some && !status(as_qk_norm_rotary(&t.p, current_stream(here)), "as_qk_norm_rotary")) return nullptr;
  if (a[11] != Py_None) written(q.o);
  if (a[12] != Py_None) written(k.o);
  if (t.k == nullptr) return q.give();
  return PyTuple_Pack(2, q.o, k.o);
  END_HANDLE_TH_ERRORS
}

// (dq, dk, q, k, q_weight, k_weight, table, norm, eps, half, inverse, positions, first, dq_out, dk_out) -> (dq, dk, dq_weight, dk_weight)
PyObject* qk_norm_rotary_backward(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  ARGS(15)
  const char* where = "qk_norm_rotary_backward";
  const int here = c10::cuda::current_device();
  TurnArgs t{};
  if (!turn_args(a + 2, here, where, t)) return nullptr;
  as_qk_norm_rotary_backward_t b{};
  b.struct_size = sizeof b;
  b.fwd = &t.p;
  int64_t rows;
  int32_t heads;
  const at::Tensor* g = heads_of(a[0], here, where, "dq", b.dq, rows, heads);
  if (g == nullptr || !like(g, t.q, where, "dq")) return nullptr;
  if ((a[1] == Py_None) != (t.k == nullptr)) { refuse(where, "dk", "goes with k"); return nullptr; }
  if (t.k != nullptr) {
    g = heads_of(a[1], here, where, "dk", b.dk, rows, heads);
    if (g == nullptr || !like(g, t.k, where, "dk")) return nullptr;
  }
  Held q, k, w[2], room;
  if (!out_of(a[13], t.q, here, where, "dq_out", q, b.dq_out)) return nullptr;
  if (t.k != nullptr) {
    if (!out_of(a[14], t.k, here, where, "dk_out", k, b.dk_out)) return nullptr;
  } else if (a[14] != Py_None) {
    refuse(where, "dk_out", "needs a k");
    return nullptr;
  }
  void** to[2] = {&b.dq_weight, &b.dk_weight};
  for (int i = 0; i < 2; ++i)
    if (a[4 + i] != Py_None) {
      const at::Tensor& u = THPVariable_Unpack(a[4 + i]);
      w[i].take(empty_contiguous(u.sizes(), u.scalar_type(), here));
      if (w[i].o == nullptr) return nullptr;
      *to[i] = THPVariable_Unpack(w[i].o).data_ptr();
    }
  if (t.p.q_heads < 1 || t.p.head_dim < 1 || (t.k != nullptr && t.p.k_heads < 1)) { refuse(where, "q", "or k has no heads"); return nullptr; }
  if (t.p.rows == 0) {                       // (tensors of no elements have no address, which the C entry takes for no tensor)
    for (int i = 0; i < 2; ++i)
      if (w[i].o != nullptr) THPVariable_Unpack(w[i].o).zero_();
  } else {
    uint64_t bytes;
    if (!status(as_qk_norm_rotary_backward_workspace_bytes(&b, &bytes), "as_qk_norm_rotary_backward") || !workspace_of(bytes, here, room, b.workspace, b.workspace_bytes)) return nullptr;
    if (!status(as_qk_norm_rotary_backward(&b, current_stream(here)), "as_qk_norm_rotary_backward")) return nullptr;
  }
  if (a[13] != Py_None) written(q.o);
  if (a[14] != Py_None) written(k.o);
  auto or_none = [](Held& h) { return h.o != nullptr ? h.o : Py_None; };
  return PyTuple_Pack(4, q.o, or_none(k), or_none(w[0]), or_none(w[1]));
  END_HANDLE_TH_ERRORS
}

namespace {

// [N] or [gates, N].
bool gate_of(PyObject* o, int64_t rows, int64_t n, int here, const char* where, const void*& data, int32_t& dtype, int64_t& gates, int64_t& stride) {
  gates = 1;
  if (o == Py_None) return true;
  const at::Tensor* t = tensor_of(o, here, where, "gate");
  if (t == nullptr) return false;
  const auto type = t->scalar_type();
  const int64_t dims = t->dim();
  if ((type != at::kBFloat16 && type != at::kFloat) || (dims != 1 && dims != 2) || t->size(dims - 1) != n || (n > 1 && t->stride(dims - 1) != 1))
    return refuse(where, "gate", "is not [cols] or [entries, cols] in bf16 or fp32, columns next to each other");
  if (dims == 2) {
    gates = t->size(0);
    stride = t->stride(0);
    if (gates < 1 || rows % gates != 0) return refuse(where, "gate", "has entries that do not divide the rows");
  }
  data = t->data_ptr();
  dtype = type == at::kFloat ? AS_DTYPE_F32 : AS_DTYPE_BF16;
  return true;
}
bool bf16_of(PyObject* o, int here, const char* where, const char* name, as_rows_t& r, int64_t& rows, int64_t& cols, const at::Tensor** out = nullptr) {
  const at::Tensor* t = rows_of(o, here, where, name, r, rows, cols);
  if (t == nullptr) return false;
  if (r.dtype != AS_DTYPE_BF16) return refuse(where, name, "is not bf16");
  if (out != nullptr) *out = t;
  return true;
}
bool weight_of(PyObject* o, int64_t k, int here, const char* where, as_rows_t& r, int64_t& n) {
  int64_t cols;
  const at::Tensor* t;
  if (!bf16_of(o, here, where, "w", r, n, cols, &t)) return false;
  if (t->dim() != 2 || cols != k) return refuse(where, "w", "is not [out columns, x's columns]");
  return true;
}

}  // namespace

// (x, w, bias, activation, gate, residual, out, pre: None, True or a tensor)
PyObject* linear(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  ARGS(8)
  const char* where = "linear";
  const int here = c10::cuda::current_device();
  as_linear_t p{};
  p.struct_size = sizeof p;
  int64_t m, k, n, r, c;
  if (!bf16_of(a[0], here, where, "x", p.x, m, k) || !weight_of(a[1], k, here, where, p.w, n)) return nullptr;
  if (k == 0 && m > 0 && n > 0) { refuse(where, "x", "has no columns to sum over"); return nullptr; }
  if (a[2] != Py_None && !vector_of(a[2], n, true, here, where, "bias", p.bias, p.bias_dtype)) return nullptr;
  if (!int_of(a[3], p.activation) || !gate_of(a[4], m, n, here, where, p.gate, p.gate_dtype, p.gates, p.gate_stride)) return nullptr;
  Held out, pre, room;
  const at::Tensor* res = nullptr;
  if (a[5] != Py_None) {
    res = rows_of(a[5], here, where, "residual", p.residual, r, c);
    if (res == nullptr) return nullptr;
    if (r != m || c != n) { refuse(where, "residual", "has not x's rows and w's rows as columns"); return nullptr; }
  }
  if (a[6] != Py_None) out.share(a[6]);
  else if (res != nullptr) out.take(empty_contiguous(res->sizes(), res->scalar_type(), here));
  else out.take(empty_contiguous({m, n}, at::kBFloat16, here));
  if (out.o == nullptr || rows_of(out.o, here, where, "out", p.out, r, c) == nullptr) return nullptr;
  if (r != m || c != n) { refuse(where, "out", "is not x's rows by w's rows"); return nullptr; }
  const bool given = THPVariable_Check(a[7]);
  bool keep = given;
  if (!given && !flag_of(a[7], keep)) return nullptr;
  if (keep) {
    if (given) pre.share(a[7]);
    else pre.take(empty_contiguous({m, n}, at::kBFloat16, here));
    if (pre.o == nullptr || !bf16_of(pre.o, here, where, "pre", p.pre, r, c)) return nullptr;
    if (r != m || c != n) { refuse(where, "pre", "is not x's rows by w's rows"); return nullptr; }
  }
  if (m > 0 && n > 0) {
    p.rows = m; p.cols = k; p.out_cols = n;
    as_fp8_context_t ctx;
    uint64_t bytes;
    if (!context_of(here, ctx) || !status(as_linear_workspace_bytes(ctx, &p, &bytes), "as_linear") || !workspace_of(bytes, here, room, p.workspace, p.workspace_bytes)) return nullptr;
    if (!status(as_linear(ctx, &p, current_stream(here)), "as_linear")) return nullptr;
  }
  if (a[6] != Py_None) written(out.o);
  if (given) written(pre.o);
  if (!keep) return out.give();
  return PyTuple_Pack(2, out.o, pre.o);
  END_HANDLE_TH_ERRORS
}

// (dy, x, w, pre, activation, gate, bias, x_grad, w_grad, gate_grad) -> (dx, dw, dbias, dgate)
PyObject* linear_backward(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  ARGS(10)
  const char* where = "linear_backward";
  const int here = c10::cuda::current_device();
  as_linear_backward_t p{};
  p.struct_size = sizeof p;
  int64_t m, k, n, r, c;
  const at::Tensor* x;
  if (!bf16_of(a[1], here, where, "x", p.x, m, k, &x) || !weight_of(a[2], k, here, where, p.w, n)) return nullptr;
  if (rows_of(a[0], here, where, "dy", p.dy, r, c) == nullptr) return nullptr;
  if (r != m || c != n) { refuse(where, "dy", "is not x's rows by w's rows"); return nullptr; }
  if (a[3] != Py_None) {
    if (!bf16_of(a[3], here, where, "pre", p.pre, r, c)) return nullptr;
    if (r != m || c != n) { refuse(where, "pre", "is not x's rows by w's rows"); return nullptr; }
  }
  if (!int_of(a[4], p.activation) || !gate_of(a[5], m, n, here, where, p.gate, p.gate_dtype, p.gates, p.gate_stride)) return nullptr;
  const void* bias;
  bool x_grad, w_grad, gate_grad;
  if (a[6] != Py_None && !vector_of(a[6], n, true, here, where, "bias", bias, p.bias_dtype)) return nullptr;
  if (!flag_of(a[7], x_grad) || !flag_of(a[8], w_grad) || !flag_of(a[9], gate_grad)) return nullptr;
  gate_grad = gate_grad && p.gate != nullptr;
  if (a[3] == Py_None && p.activation != AS_ACT_NONE) { refuse(where, "pre", "is needed with an activation"); return nullptr; }
  if (a[3] == Py_None && gate_grad) { refuse(where, "pre", "is needed for the gate's gradient"); return nullptr; }
  Held dx, dw, db, dg, room;
  if (x_grad) {
    dx.take(empty_contiguous(x->sizes(), at::kBFloat16, here));
    if (dx.o == nullptr || !bf16_of(dx.o, here, where, "dx", p.dx, r, c)) return nullptr;
  }
  if (w_grad) {
    dw.take(empty_contiguous({n, k}, at::kBFloat16, here));
    if (dw.o == nullptr || !bf16_of(dw.o, here, where, "dw", p.dw, r, c)) return nullptr;
  }
  if (a[6] != Py_None) {
    db.take(empty_contiguous({n}, THPVariable_Unpack(a[6]).scalar_type(), here));
    if (db.o == nullptr) return nullptr;
    p.dbias = THPVariable_Unpack(db.o).data_ptr();
  }
  if (gate_grad) {
    const at::Tensor& g = THPVariable_Unpack(a[5]);
    dg.take(empty_contiguous(g.sizes(), g.scalar_type(), here));
    if (dg.o == nullptr) return nullptr;
    p.dgate = THPVariable_Unpack(dg.o).data_ptr();
  }
  if (m == 0 || n == 0 || k == 0) {          // sums over nothing
    if (k == 0 && m > 0 && n > 0) { refuse(where, "x", "has no columns"); return nullptr; }
    for (Held* h : {&dx, &dw, &db, &dg})
      if (h->o != nullptr) THPVariable_Unpack(h->o).zero_();
  } else {
    p.rows = m; p.cols = k; p.out_cols = n;
    as_fp8_context_t ctx;
    uint64_t bytes;
    if (!context_of(here, ctx) || !status(as_linear_backward_workspace_bytes(ctx, &p, &bytes), "as_linear_backward") || !workspace_of(bytes, here, room, p.workspace, p.workspace_bytes)) return nullptr;
    if (!status(as_linear_backward(ctx, &p, current_stream(here)), "as_linear_backward")) return nullptr;
  }
  auto or_none = [](Held& h) { return h.o != nullptr ? h.o : Py_None; };
  return PyTuple_Pack(4, or_none(dx), or_none(dw), or_none(db), or_none(dg));
  END_HANDLE_TH_ERRORS
}

}  // namespace as_calls
