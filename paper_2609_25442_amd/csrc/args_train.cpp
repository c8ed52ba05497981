// The trainer's operators' side of the binding's extension, as args_ops.cpp.
#include <c10/core/impl/VirtualGuardImpl.h>
#include <torch/csrc/autograd/function.h>
#include <torch/csrc/autograd/variable.h>

#include "args_ops.hpp"
#include "args_tensor.hpp"

using namespace wb_args;

namespace {

wb_tokens token_ids(const Tensor& t) {
  if (t.scalar_type() != at::kInt && t.scalar_type() != at::kLong) refuse("tokens", "is neither int32 nor int64");
  if (!t.is_contiguous()) refuse("tokens", "is not contiguous");
  wb_tokens k{};
  k.data = t.data_ptr(), k.bytes = t.scalar_type() == at::kInt ? 4 : 8, k.count = t.numel();
  return k;
}

// [..., cols] as rows: two dimensions with rows any distance apart, or others without gaps.
wb_matrix rows_of(const Tensor& t, const char* name) {
  if (t.dim() == 2) return matrix(t, name);
  if (t.dim() < 1 || !t.is_contiguous()) refuse(name, "is not contiguous");
  wb_matrix m{};
  m.data = t.data_ptr(), m.dtype = code_of(t.scalar_type(), name);
  m.cols = m.ld = t.size(t.dim() - 1);
  m.rows = 1;
  for (int64_t d = 0; d + 1 < t.dim(); ++d) m.rows *= t.size(d);
  return m;
}

struct Span {
  const int32_t *first = nullptr, *last = nullptr;
  explicit Span(const Tensor* span) {
    if (!span) return;
    if (span->scalar_type() != at::kInt || span->dim() != 1 || span->numel() < 1 || !span->is_contiguous())
      refuse("span", "is no contiguous int32 vector");
    first = span->data_ptr<int32_t>(), last = first + (span->numel() - 1);
  }
};

struct Places {
  const int32_t *positions, *tokens;
  int64_t rows, k, places;
  Places(const Tensor& p, const Tensor& t) {
    if (p.dim() != 2) refuse("positions", "does not have two dimensions");
    rows = p.size(0), k = p.size(1), places = t.numel();
    positions = plain(p, at::kInt, rows * k, "positions").data_ptr<int32_t>();
    tokens = plain(t, at::kInt, places, "tokens").data_ptr<int32_t>();
  }
};

Tensor workspace_of(size_t bytes, const Tensor& like) { return fresh({static_cast<int64_t>(bytes)}, at::kByte, like); }

void* data(const Tensor& t) { return t.defined() && t.numel() ? t.data_ptr() : nullptr; }

}  // namespace

// embedding(fn, tokens, weight, scale, first, out_dtype, device, stream) -> out
PyObject* wb_py_embedding(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (!counted(n, 8, "embedding")) return nullptr;
  return guarded([&]() -> PyObject* {
    const Where at(args + 6);
    const double scale = PyFloat_AsDouble(args[3]);
    const long long first = PyLong_AsLongLong(args[4]);
    const long type = PyLong_AsLong(args[5]);
    auto* fn = function<decltype(wb_embedding)>(args[0]);
    if (PyErr_Occurred()) return nullptr;
    const Tensor& tokens = needed(args[1], "tokens", at.device);
    const Tensor& weight = needed(args[2], "weight", at.device);
    ungraded({{&weight, "weight"}});
    const wb_tokens ids = token_ids(tokens);
    const wb_matrix mw = matrix(weight, "weight");
    at::DimVector shape(tokens.sizes());
    shape.push_back(mw.cols);
    Tensor out = fresh(shape, type_of(type < 0 ? mw.dtype : static_cast<int32_t>(type)), weight);
    const wb_matrix mo = rows_of(out, "out");
    const int rc = fn(&ids, &mw, static_cast<float>(scale), first, &mo, at.stream);
    return rc != WB_OK ? PyLong_FromLong(rc) : wrap(out);
  });
}

// embedding_backward(fn, workspace_fn, d_out, tokens, rows, scale, first, out_dtype, device, stream) -> d_weight
PyObject* wb_py_embedding_backward(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (!counted(n, 10, "embedding_backward")) return nullptr;
  return guarded([&]() -> PyObject* {
    const Where at(args + 8);
    const long long rows = PyLong_AsLongLong(args[4]), first = PyLong_AsLongLong(args[6]);
    const double scale = PyFloat_AsDouble(args[5]);
    const long type = PyLong_AsLong(args[7]);
    auto* fn = function<decltype(wb_embedding_backward)>(args[0]);
    auto* size = function<decltype(wb_embedding_backward_workspace)>(args[1]);
    if (PyErr_Occurred()) return nullptr;
    const Tensor& d_out = needed(args[2], "d_out", at.device);
    const Tensor& tokens = needed(args[3], "tokens", at.device);
    ungraded({{&d_out, "d_out"}});
    const wb_tokens ids = token_ids(tokens);
    const wb_matrix md = rows_of(d_out, "d_out");
    size_t bytes = 0;
    int rc = size(ids.count, rows, md.cols, &bytes);
    if (rc != WB_OK) return PyLong_FromLong(rc);
    Tensor d_weight = fresh({rows, md.cols}, type_of(type < 0 ? md.dtype : static_cast<int32_t>(type)), d_out);
    const Tensor workspace = workspace_of(bytes, d_out);
    const wb_matrix mw = matrix(d_weight, "d_weight");
    rc = fn(&ids, &md, static_cast<float>(scale), first, &mw, data(workspace), bytes, at.stream);
    return rc != WB_OK ? PyLong_FromLong(rc) : wrap(d_weight);
  });
}

// add_layer_norm(fn, x, weight, bias, residual, eps, center, out_dtype, device, stream) -> (out, total, mean, inv)
PyObject* wb_py_add_layer_norm(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (!counted(n, 10, "add_layer_norm")) return nullptr;
  return guarded([&]() -> PyObject* {
    const Where at(args + 8);
    const double eps = PyFloat_AsDouble(args[5]);
    const long center = PyLong_AsLong(args[6]), type = PyLong_AsLong(args[7]);
    auto* fn = function<decltype(wb_add_layer_norm)>(args[0]);
    if (PyErr_Occurred()) return nullptr;
    const Tensor& x = needed(args[1], "x", at.device);
    const Tensor& weight = needed(args[2], "weight", at.device);
    const Tensor* bias = tensor(args[3], "bias", at.device);
    const Tensor* residual = tensor(args[4], "residual", at.device);
    ungraded({{&x, "x"}, {&weight, "weight"}, {bias, "bias"}, {residual, "residual"}});
    const wb_matrix mx = matrix(x, "x"), mw = vector(weight, "weight");
    wb_matrix mb{}, mr{}, mt{};
    if (bias) mb = vector(*bias, "bias");
    Tensor out = fresh(x.sizes(), type_of(type < 0 ? mx.dtype : static_cast<int32_t>(type)), x), total, mean, inv;
    if (residual) {
      mr = matrix(*residual, "residual");
      total = fresh(x.sizes(), residual->scalar_type(), x), mt = matrix(total, "total");
    }
    const Tensor stats = fresh({center ? 2 * mx.rows : mx.rows}, at::kFloat, x);
    int64_t next = 0;
    inv = part(stats, next, {mx.rows});
    if (center) mean = part(stats, next, {mx.rows});
    const wb_matrix mo = matrix(out, "out");
    // rows of none have no addresses: the library asks for none, but mean's says that it is centred
    const int rc = fn(&mx, residual ? &mr : nullptr, &mw, bias ? &mb : nullptr, static_cast<float>(eps),
                      residual ? &mt : nullptr, &mo, center ? mean.data_ptr<float>() : nullptr, inv.data_ptr<float>(), at.stream);
    if (rc != WB_OK) return PyLong_FromLong(rc);
    return Py_BuildValue("(NNNN)", wrap(out), wrap(total), wrap(mean), wrap(inv));
  });
}

// add_layer_norm_backward(fn, workspace_fn, d_out, total, weight, d_total, mean, inv, x_type, residual_type, weight_type,
//                         bias_type, device, stream) -> (d_x, d_residual, d_weight, d_bias); types of -1: not computed
PyObject* wb_py_add_layer_norm_backward(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (!counted(n, 14, "add_layer_norm_backward")) return nullptr;
  return guarded([&]() -> PyObject* {
    const Where at(args + 12);
    const long x_type = PyLong_AsLong(args[8]), residual_type = PyLong_AsLong(args[9]);
    const long weight_type = PyLong_AsLong(args[10]), bias_type = PyLong_AsLong(args[11]);
    auto* fn = function<decltype(wb_add_layer_norm_backward)>(args[0]);
    auto* size = function<decltype(wb_add_layer_norm_backward_workspace)>(args[1]);
    if (PyErr_Occurred()) return nullptr;
    const Tensor& d_out = needed(args[2], "d_out", at.device);
    const Tensor& total = needed(args[3], "total", at.device);
    const Tensor& weight = needed(args[4], "weight", at.device);
    const Tensor* d_total = tensor(args[5], "d_total", at.device);
    const Tensor* mean = tensor(args[6], "mean", at.device);
    const Tensor& inv = needed(args[7], "inv", at.device);
    ungraded({{&d_out, "d_out"}, {&total, "total"}, {&weight, "weight"}, {d_total, "d_total"}});
    const wb_matrix md = matrix(d_out, "d_out"), mt = matrix(total, "total"), mw = vector(weight, "weight");
    wb_matrix mdt{}, mr{}, mdw{}, mdb{};
    if (d_total) mdt = matrix(*d_total, "d_total");
    if (mean) plain(*mean, at::kFloat, mt.rows, "mean");
    plain(inv, at::kFloat, mt.rows, "inv");
    size_t bytes = 0;
    int rc = size(mt.rows, mt.cols, &bytes);
    if (rc != WB_OK) return PyLong_FromLong(rc);
    Tensor d_x = fresh({mt.rows, mt.cols}, type_of(static_cast<int32_t>(x_type)), total), d_residual, d_weight, d_bias;
    const wb_matrix mx = matrix(d_x, "d_x");
    if (residual_type == x_type) {
      d_residual = d_x;
    } else if (residual_type >= 0) {
      d_residual = fresh({mt.rows, mt.cols}, type_of(static_cast<int32_t>(residual_type)), total);
      mr = matrix(d_residual, "d_residual");
    }
    if (weight_type >= 0) {
      d_weight = fresh({mt.cols}, type_of(static_cast<int32_t>(weight_type)), total), mdw = vector(d_weight, "d_weight");
      if (bias_type >= 0) d_bias = fresh({mt.cols}, type_of(static_cast<int32_t>(bias_type)), total), mdb = vector(d_bias, "d_bias");
    }
    const Tensor workspace = workspace_of(bytes, total);
    rc = fn(&md, &mt, &mw, d_total ? &mdt : nullptr, mean ? mean->data_ptr<float>() : nullptr, inv.data_ptr<float>(), &mx,
            mr.data ? &mr : nullptr, mdw.data ? &mdw : nullptr, mdb.data ? &mdb : nullptr, data(workspace), bytes, at.stream);
    if (rc != WB_OK) return PyLong_FromLong(rc);
    return Py_BuildValue("(NNNN)", wrap(d_x), wrap(d_residual), wrap(d_weight), wrap(d_bias));
  });
}

// dispatch(fn, x, positions, tokens, span, device, stream) -> rows
PyObject* wb_py_dispatch(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (!counted(n, 7, "dispatch")) return nullptr;
  return guarded([&]() -> PyObject* {
    const Where at(args + 5);
    auto* fn = function<decltype(wb_dispatch)>(args[0]);
    if (PyErr_Occurred()) return nullptr;
    const Tensor& x = needed(args[1], "x", at.device);
    ungraded({{&x, "x"}});
    const Places p(needed(args[2], "positions", at.device), needed(args[3], "tokens", at.device));
    const Span span(tensor(args[4], "span", at.device));
    const wb_matrix mx = matrix(x, "x");
    if (mx.rows != p.rows) refuse("x", "has another number of rows than the routing");
    Tensor out = fresh({p.places, mx.cols}, x.scalar_type(), x);
    const wb_matrix mo = matrix(out, "out");
    const int rc = fn(&mx, p.positions, p.tokens, static_cast<int32_t>(p.k), span.first, span.last, &mo, at.stream);
    return rc != WB_OK ? PyLong_FromLong(rc) : wrap(out);
  });
}

// dispatch_backward(fn, d_rows, positions, tokens, span, out_dtype, device, stream) -> d_x
PyObject* wb_py_dispatch_backward(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (!counted(n, 8, "dispatch_backward")) return nullptr;
  return guarded([&]() -> PyObject* {
    const Where at(args + 6);
    const long type = PyLong_AsLong(args[5]);
    auto* fn = function<decltype(wb_dispatch_backward)>(args[0]);
    if (PyErr_Occurred()) return nullptr;
    const Tensor& d_rows = needed(args[1], "d_rows", at.device);
    ungraded({{&d_rows, "d_rows"}});
    const Places p(needed(args[2], "positions", at.device), needed(args[3], "tokens", at.device));
    const Span span(tensor(args[4], "span", at.device));
    const wb_matrix md = matrix(d_rows, "d_rows");
    if (md.rows != p.places) refuse("d_rows", "has another number of rows than the routing has places");
    Tensor d_x = fresh({p.rows, md.cols}, type_of(type < 0 ? md.dtype : static_cast<int32_t>(type)), d_rows);
    const wb_matrix mx = matrix(d_x, "d_x");
    const int rc = fn(&md, p.positions, p.tokens, static_cast<int32_t>(p.k), span.first, span.last, &mx, at.stream);
    return rc != WB_OK ? PyLong_FromLong(rc) : wrap(d_x);
  });
}

// collect(fn, y, positions, tokens, gates, residual, span, out_dtype, device, stream) -> out
PyObject* wb_py_collect(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (!counted(n, 10, "collect")) return nullptr;
  return guarded([&]() -> PyObject* {
    const Where at(args + 8);
    const long type = PyLong_AsLong(args[7]);
    auto* fn = function<decltype(wb_collect)>(args[0]);
    if (PyErr_Occurred()) return nullptr;
    const Tensor& y = needed(args[1], "y", at.device);
    const Places p(needed(args[2], "positions", at.device), needed(args[3], "tokens", at.device));
    const Tensor& gates = needed(args[4], "gates", at.device);
    const Tensor* residual = tensor(args[5], "residual", at.device);
    const Span span(tensor(args[6], "span", at.device));
    ungraded({{&y, "y"}, {&gates, "gates"}, {residual, "residual"}});
    plain(gates, at::kFloat, p.rows * p.k, "gates");
    const wb_matrix my = matrix(y, "y");
    if (my.rows != p.places) refuse("y", "has another number of rows than the routing has places");
    wb_matrix mr{};
    if (residual) mr = matrix(*residual, "residual");
    Tensor out = fresh({p.rows, my.cols}, type_of(type < 0 ? my.dtype : static_cast<int32_t>(type)), y);
    const wb_matrix mo = matrix(out, "out");
    const int rc = fn(&my, p.positions, p.tokens, gates.data_ptr<float>(), static_cast<int32_t>(p.k), residual ? &mr : nullptr,
                      span.first, span.last, &mo, at.stream);
    return rc != WB_OK ? PyLong_FromLong(rc) : wrap(out);
  });
}

// collect_backward(fn, d_out, y, positions, tokens, gates, span, y_type, device, stream) -> (d_y, d_gates)
// y None: no d_gates; y_type -1: no d_y
PyObject* wb_py_collect_backward(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (!counted(n, 10, "collect_backward")) return nullptr;
  return guarded([&]() -> PyObject* {
    const Where at(args + 8);
    const long y_type = PyLong_AsLong(args[7]);
    auto* fn = function<decltype(wb_combine_backward)>(args[0]);
    if (PyErr_Occurred()) return nullptr;
    const Tensor& d_out = needed(args[1], "d_out", at.device);
    const Tensor* y = tensor(args[2], "y", at.device);
    const Places p(needed(args[3], "positions", at.device), needed(args[4], "tokens", at.device));
    const Tensor& gates = needed(args[5], "gates", at.device);
    const Span span(tensor(args[6], "span", at.device));
    ungraded({{&d_out, "d_out"}, {y, "y"}, {&gates, "gates"}});
    plain(gates, at::kFloat, p.rows * p.k, "gates");
    const wb_matrix md = matrix(d_out, "d_out");
    if (md.rows != p.rows) refuse("d_out", "has another number of rows than the routing");
    wb_matrix my{}, mdy{};
    Tensor d_y, d_gates;
    if (y) {
      my = matrix(*y, "y");
      if (my.rows != p.places) refuse("y", "has another number of rows than the routing has places");
      d_gates = fresh({p.rows, p.k}, at::kFloat, d_out);
    }
    if (y_type >= 0) d_y = fresh({p.places, md.cols}, type_of(static_cast<int32_t>(y_type)), d_out), mdy = matrix(d_y, "d_y");
    const int rc = fn(&md, y ? &my : nullptr, p.positions, p.tokens, gates.data_ptr<float>(), static_cast<int32_t>(p.k),
                      span.first, span.last, d_y.defined() ? &mdy : nullptr, y ? d_gates.data_ptr<float>() : nullptr, at.stream);
    if (rc != WB_OK) return PyLong_FromLong(rc);
    return Py_BuildValue("(NN)", wrap(d_y), wrap(d_gates));
  });
}

// activate(fn, x, activation, gated, keep, out_dtype, device, stream) -> (out, codes, scales)
PyObject* wb_py_activate(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (!counted(n, 8, "activate")) return nullptr;
  return guarded([&]() -> PyObject* {
    const Where at(args + 6);
    const long activation = PyLong_AsLong(args[2]), gated = PyLong_AsLong(args[3]), keep = PyLong_AsLong(args[4]);
    const long type = PyLong_AsLong(args[5]);
    auto* fn = function<decltype(wb_activate)>(args[0]);
    if (PyErr_Occurred()) return nullptr;
    const Tensor& x = needed(args[1], "x", at.device);
    ungraded({{&x, "x"}});
    const wb_matrix mx = matrix(x, "x");
    const int64_t cols = gated ? mx.cols / 2 : mx.cols;
    Tensor out = fresh({mx.rows, cols}, type_of(type < 0 ? mx.dtype : static_cast<int32_t>(type)), x), codes, scales;
    const wb_matrix mo = matrix(out, "out");
    wb_matrix mc{}, ms{};
    if (keep) {
      codes = fresh({mx.rows, mx.cols}, at::kFloat8_e4m3fn, x), mc = matrix(codes, "codes");
      scales = fresh({mx.rows, scale_cols(cols) * (gated ? 2 : 1)}, at::kFloat, x), ms = matrix(scales, "scales");
    }
    const int rc = fn(&mx, static_cast<int32_t>(activation), static_cast<int32_t>(gated), &mo, keep ? &mc : nullptr,
                      keep ? &ms : nullptr, at.stream);
    if (rc != WB_OK) return PyLong_FromLong(rc);
    return Py_BuildValue("(NNN)", wrap(out), wrap(codes), wrap(scales));
  });
}

// activate_backward(fn, d_out, x, scales, activation, gated, x_type, device, stream) -> d_x
PyObject* wb_py_activate_backward(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (!counted(n, 9, "activate_backward")) return nullptr;
  return guarded([&]() -> PyObject* {
    const Where at(args + 7);
    const long activation = PyLong_AsLong(args[4]), gated = PyLong_AsLong(args[5]), type = PyLong_AsLong(args[6]);
    auto* fn = function<decltype(wb_activate_backward)>(args[0]);
    if (PyErr_Occurred()) return nullptr;
    const Tensor& d_out = needed(args[1], "d_out", at.device);
    const Tensor& x = needed(args[2], "x", at.device);
    const Tensor* scales = tensor(args[3], "scales", at.device);
    ungraded({{&d_out, "d_out"}, {&x, "x"}});
    const wb_matrix md = matrix(d_out, "d_out"), mx = matrix(x, "x");
    wb_matrix ms{};
    if (scales) ms = matrix(*scales, "scales");
    Tensor d_x = fresh({mx.rows, mx.cols}, type_of(static_cast<int32_t>(type)), d_out);
    const wb_matrix mo = matrix(d_x, "d_x");
    const int rc = fn(&md, &mx, scales ? &ms : nullptr, static_cast<int32_t>(activation), static_cast<int32_t>(gated), &mo, at.stream);
    return rc != WB_OK ? PyLong_FromLong(rc) : wrap(d_x);
  });
}

// held_elsewhere(tensor): whether a graph that lives accumulates this leaf's
// gradient on another stream than the current one.
PyObject* wb_py_held_elsewhere(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (!counted(n, 1, "held_elsewhere")) return nullptr;
  return guarded([&]() -> PyObject* {
    if (!THPVariable_Check(args[0])) Py_RETURN_FALSE;
    const Tensor& t = THPVariable_Unpack(args[0]);
    if (!t.defined() || !t.is_cuda() || !t.requires_grad() || !t.is_leaf()) Py_RETURN_FALSE;
    const auto accumulator = torch::autograd::impl::try_get_grad_accumulator(t);
    if (!accumulator) Py_RETURN_FALSE;
    const auto on = accumulator->stream();
    const c10::impl::VirtualGuardImpl device(t.device().type());
    if (on && *on == device.getStream(t.device())) Py_RETURN_FALSE;
    Py_RETURN_TRUE;
  });
}
