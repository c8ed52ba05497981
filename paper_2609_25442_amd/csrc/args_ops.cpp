// The operators' side of the binding's extension: torch tensors in, the C
// call of include/wb.h, new torch tensors out. What the library cannot see is
// refused here (a tensor on the CPU or on another device, columns that are
// not neighbours); shapes, types and extents are the library's to refuse. In
// place of a result a call returns a text (what it refused) or the library's
// negative status.
#include "args_ops.hpp"

#include "args_tensor.hpp"

using namespace wb_args;

// add_rms_norm(fn, x, weight, residual, eps, out_dtype, device, stream) -> (out, scales, total)
PyObject* wb_py_add_rms_norm(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (!counted(n, 8, "add_rms_norm")) return nullptr;
  return guarded([&]() -> PyObject* {
    const Where at(args + 6);
    const double eps = PyFloat_AsDouble(args[4]);
    const long type = PyLong_AsLong(args[5]);
    auto* fn = function<decltype(wb_add_rms_norm)>(args[0]);
    if (PyErr_Occurred()) return nullptr;
    const Tensor& x = needed(args[1], "x", at.device);
    const Tensor& weight = needed(args[2], "weight", at.device);
    const Tensor* residual = tensor(args[3], "residual", at.device);
    ungraded({{&x, "x"}, {&weight, "weight"}, {residual, "residual"}});
    const wb_matrix mx = matrix(x, "x"), mw = vector(weight, "weight");
    const bool f8 = type == WB_F8E4M3;
    wb_matrix mr{}, mt{}, ms{};
    Tensor out = fresh(x.sizes(), type_of(type < 0 ? mx.dtype : static_cast<int32_t>(type)), x), scales, total;
    if (f8) scales = fresh({mx.rows, scale_cols(mx.cols)}, at::kFloat, x), ms = matrix(scales, "scales");
    if (residual) {
      mr = matrix(*residual, "residual");
      total = fresh(x.sizes(), residual->scalar_type(), x), mt = matrix(total, "total");
    }
    const wb_matrix mo = matrix(out, "out");
    const int rc = fn(&mx, residual ? &mr : nullptr, &mw, static_cast<float>(eps), residual ? &mt : nullptr, &mo,
                      f8 ? &ms : nullptr, at.stream);
    if (rc != WB_OK) return PyLong_FromLong(rc);
    return Py_BuildValue("(NNN)", wrap(out), wrap(scales), wrap(total));
  });
}

// route(fn, workspace_fn, logits, mask, k, renormalize, device, stream)
//   -> (experts, gates, positions, tokens, counts, offsets, loss, routed)
PyObject* wb_py_route(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (!counted(n, 8, "route")) return nullptr;
  return guarded([&]() -> PyObject* {
    const Where at(args + 6);
    const long k = PyLong_AsLong(args[4]), renormalize = PyLong_AsLong(args[5]);
    auto* fn = function<decltype(wb_route)>(args[0]);
    auto* size = function<decltype(wb_route_workspace)>(args[1]);
    if (PyErr_Occurred()) return nullptr;
    const Tensor& logits = needed(args[2], "logits", at.device);
    const Tensor* mask = tensor(args[3], "mask", at.device);
    const wb_matrix ml = matrix(logits, "logits");
    if (mask) plain(*mask, mask->scalar_type() == at::kBool ? at::kBool : at::kByte, ml.rows, "mask");
    if (k < 1 || k > ml.cols) throw Refused("k is outside 1..experts");
    size_t bytes = 0;
    int rc = size(ml.rows, static_cast<int32_t>(ml.cols), &bytes);
    if (rc != WB_OK) return PyLong_FromLong(rc);
    // the integers in one allocation (each costs about as much as the checks)
    const Tensor block = fresh({3 * ml.rows * k + 2 * ml.cols + 2}, at::kInt, logits);
    int64_t next = 0;
    Tensor experts = part(block, next, {ml.rows, k}), positions = part(block, next, {ml.rows, k});
    Tensor tokens = part(block, next, {ml.rows * k}), counts = part(block, next, {ml.cols});
    Tensor offsets = part(block, next, {ml.cols + 1}), routed = part(block, next, {1});
    Tensor gates = fresh({ml.rows, k}, at::kFloat, logits), loss = fresh({}, at::kFloat, logits);
    Tensor workspace = fresh({static_cast<int64_t>(bytes)}, at::kByte, logits);
    wb_routing r{};
    r.experts = experts.data_ptr<int32_t>(), r.gates = gates.data_ptr<float>();
    r.positions = positions.data_ptr<int32_t>(), r.tokens = tokens.data_ptr<int32_t>();
    r.counts = counts.data_ptr<int32_t>(), r.offsets = offsets.data_ptr<int32_t>(), r.loss = loss.data_ptr<float>();
    r.routed = routed.data_ptr<int32_t>();
    rc = fn(&ml, mask ? static_cast<const uint8_t*>(mask->data_ptr()) : nullptr, static_cast<int32_t>(k),
            static_cast<int32_t>(renormalize), &r, workspace.data_ptr(), bytes, at.stream);
    if (rc != WB_OK) return PyLong_FromLong(rc);
    return Py_BuildValue("(NNNNNNNN)", wrap(experts), wrap(gates), wrap(positions), wrap(tokens), wrap(counts),
                         wrap(offsets), wrap(loss), wrap(routed));
  });
}

// route_backward(fn, logits, mask, k, renormalize, experts, gates, counts, routed, d_gates, d_loss, device, stream)
//   -> d_logits
PyObject* wb_py_route_backward(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (!counted(n, 13, "route_backward")) return nullptr;
  return guarded([&]() -> PyObject* {
    const Where at(args + 11);
    const long k = PyLong_AsLong(args[3]), renormalize = PyLong_AsLong(args[4]);
    auto* fn = function<decltype(wb_route_backward)>(args[0]);
    if (PyErr_Occurred()) return nullptr;
    const Tensor& logits = needed(args[1], "logits", at.device);
    const Tensor* mask = tensor(args[2], "mask", at.device);
    const wb_matrix ml = matrix(logits, "logits");
    if (mask) plain(*mask, mask->scalar_type() == at::kBool ? at::kBool : at::kByte, ml.rows, "mask");
    if (k < 1 || k > ml.cols) throw Refused("k is outside 1..experts");
    const int64_t count = ml.rows * k;
    wb_routing r{};
    r.experts = plain(needed(args[5], "experts", at.device), at::kInt, count, "experts").data_ptr<int32_t>();
    r.gates = plain(needed(args[6], "gates", at.device), at::kFloat, count, "gates").data_ptr<float>();
    r.counts = plain(needed(args[7], "counts", at.device), at::kInt, ml.cols, "counts").data_ptr<int32_t>();
    r.routed = plain(needed(args[8], "routed", at.device), at::kInt, 1, "routed").data_ptr<int32_t>();
    const Tensor* d_gates = tensor(args[9], "d_gates", at.device);
    const Tensor* d_loss = tensor(args[10], "d_loss", at.device);
    ungraded({{d_gates, "d_gates"}, {d_loss, "d_loss"}});
    if (d_gates) plain(*d_gates, at::kFloat, count, "d_gates");
    if (d_loss) plain(*d_loss, at::kFloat, 1, "d_loss");
    Tensor d_logits = fresh(logits.sizes(), logits.scalar_type(), logits);
    const wb_matrix md = matrix(d_logits, "d_logits");
    const int rc = fn(&ml, mask ? static_cast<const uint8_t*>(mask->data_ptr()) : nullptr, static_cast<int32_t>(k),
                      static_cast<int32_t>(renormalize), &r, d_gates ? d_gates->data_ptr<float>() : nullptr,
                      d_loss ? d_loss->data_ptr<float>() : nullptr, &md, at.stream);
    if (rc != WB_OK) return PyLong_FromLong(rc);
    return wrap(d_logits);
  });
}

// linear(fn, workspace_fn, x, weight, offsets, tokens, x_scales, weight_scales, bias, residual, activation, gated, out_dtype, device,
//        stream) -> out or (out, scales)
PyObject* wb_py_linear(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (!counted(n, 15, "linear")) return nullptr;
  return guarded([&]() -> PyObject* {
    const Where at(args + 13);
    const long activation = PyLong_AsLong(args[10]), gated = PyLong_AsLong(args[11]), type = PyLong_AsLong(args[12]);
    auto* fn = function<decltype(wb_linear)>(args[0]);
    auto* size = function<decltype(wb_linear_workspace)>(args[1]);
    if (PyErr_Occurred()) return nullptr;
    const Tensor& x = needed(args[2], "x", at.device);
    const Tensor& weight = needed(args[3], "weight", at.device);
    const Tensor* offsets = tensor(args[4], "offsets", at.device);
    const Tensor* tokens = tensor(args[5], "tokens", at.device);
    const Tensor* x_scales = tensor(args[6], "x_scales", at.device);
    const Tensor* weight_scales = tensor(args[7], "weight_scales", at.device);
    const Tensor* bias = tensor(args[8], "bias", at.device);
    const Tensor* residual = tensor(args[9], "residual", at.device);
    ungraded({{&x, "x"}, {&weight, "weight"}, {x_scales, "x_scales"}, {weight_scales, "weight_scales"}, {bias, "bias"},
              {residual, "residual"}});
    wb_linear_args a{};
    a.x = matrix(x, "x"), a.weight = matrix(weight, "weight", offsets != nullptr);
    a.activation = static_cast<int32_t>(activation), a.gated = gated != 0;
    int64_t experts = 1, rows = a.x.rows;
    if (offsets) {
      if (offsets->scalar_type() != at::kInt || offsets->dim() != 1 || offsets->numel() < 2 || !offsets->is_contiguous())
        refuse("offsets", "is no contiguous int32 vector of one entry per expert and one more");
      experts = offsets->numel() - 1;
      if (experts != (weight.dim() == 3 ? weight.size(0) : 1)) refuse("offsets", "does not go with the weight's experts");
      a.offsets = offsets->data_ptr<int32_t>(), a.num_experts = static_cast<int32_t>(experts);
    }
    if (tokens) {
      if (!offsets) refuse("tokens", "is given without offsets");
      if (tokens->scalar_type() != at::kInt || tokens->dim() != 1 || !tokens->is_contiguous())
        refuse("tokens", "is no contiguous int32 vector");
      rows = tokens->numel(), a.tokens = tokens->data_ptr<int32_t>();
    }
    if (x_scales) a.x_scales = matrix(*x_scales, "x_scales");
    if (weight_scales) a.weight_scales = matrix(*weight_scales, "weight_scales", offsets != nullptr);
    if (bias) a.bias = bias->dim() == 1 && experts == 1 ? vector(*bias, "bias") : matrix(*bias, "bias");
    if (residual) a.residual = matrix(*residual, "residual");
    const int64_t cols = a.weight.rows / experts / (gated ? 2 : 1);
    const at::ScalarType t = type_of(static_cast<int32_t>(type));
    Tensor out = fresh({rows, cols}, t, x), scales;
    a.out = matrix(out, "out");
    Tensor workspace;
    size_t bytes = 0;
    int rc = WB_OK;
    const bool f8 = t == at::kFloat8_e4m3fn;
    if (f8) scales = fresh({rows, scale_cols(cols)}, at::kFloat, x), a.out_scales = matrix(scales, "scales");
    const int64_t es = x.element_size();
    const bool on_grid = ((reinterpret_cast<uintptr_t>(a.x.data) | reinterpret_cast<uintptr_t>(a.weight.data) |
                           static_cast<uintptr_t>((a.x.ld | a.weight.ld | a.x.cols) * es)) & 15) == 0;
    if (f8 || !on_grid) {  // else none is needed
      rc = size(&a, &bytes);
      if (rc == WB_OK && bytes) workspace = fresh({static_cast<int64_t>(bytes)}, at::kByte, x);
    }
    if (rc == WB_OK) rc = fn(&a, bytes ? workspace.data_ptr() : nullptr, bytes, at.stream);
    if (rc != WB_OK) return PyLong_FromLong(rc);
    if (!scales.defined()) return wrap(out);
    return Py_BuildValue("(NN)", wrap(out), wrap(scales));
  });
}

// combine(fn, y, positions, gates, residual, span, out_dtype, device, stream) -> out
PyObject* wb_py_combine(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (!counted(n, 9, "combine")) return nullptr;
  return guarded([&]() -> PyObject* {
    const Where at(args + 7);
    const long type = PyLong_AsLong(args[6]);
    auto* fn = function<decltype(wb_combine)>(args[0]);
    if (PyErr_Occurred()) return nullptr;
    const Tensor& y = needed(args[1], "y", at.device);
    const Tensor& positions = needed(args[2], "positions", at.device);
    const Tensor& gates = needed(args[3], "gates", at.device);
    const Tensor* residual = tensor(args[4], "residual", at.device);
    const Tensor* span = tensor(args[5], "span", at.device);
    ungraded({{&y, "y"}, {&gates, "gates"}, {residual, "residual"}});
    const wb_matrix my = matrix(y, "y");
    if (positions.dim() != 2) refuse("positions", "does not have two dimensions");
    const int64_t rows = positions.size(0), k = positions.size(1);
    plain(positions, at::kInt, rows * k, "positions");
    plain(gates, at::kFloat, rows * k, "gates");
    const int32_t *first = nullptr, *last = nullptr;
    if (span) {
      if (span->scalar_type() != at::kInt || span->dim() != 1 || span->numel() < 1 || !span->is_contiguous())
        refuse("span", "is no contiguous int32 vector");
      first = span->data_ptr<int32_t>(), last = first + (span->numel() - 1);
    }
    wb_matrix mr{};
    if (residual) mr = matrix(*residual, "residual");
    Tensor out = fresh({rows, my.cols}, type_of(type < 0 ? my.dtype : static_cast<int32_t>(type)), y);
    const wb_matrix mo = matrix(out, "out");
    const int rc = fn(&my, positions.data_ptr<int32_t>(), gates.data_ptr<float>(), static_cast<int32_t>(k),
                      residual ? &mr : nullptr, first, last, &mo, at.stream);
    if (rc != WB_OK) return PyLong_FromLong(rc);
    return wrap(out);
  });
}
