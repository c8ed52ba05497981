// C entries of the operators (declared in include/wb.h): what they refuse, and
// the launch arguments of norm.hip, route.hip and linear.hip.
#include <hip/hip_runtime_api.h>

#include <string>

#include "entry.hpp"
#include "ops.hpp"

namespace {

using wb::check_extent_as;
using wb::guarded;
using wb::hip_fail;
using wb::KnownRange;
using wb::set_error;

constexpr int64_t kMaxRows = 4194303;            // a row may take a workgroup of 1024 threads: 2^32 in a launch
constexpr int64_t kMaxCols = int64_t(1) << 26;  // 2048 to a workgroup in y of a launch
constexpr int64_t kMaxStride = int64_t(1) << 40;
constexpr int64_t kMaxExtent = int64_t(1) << 50;  // rows times row distance: bytes and offsets stay within 63 bits

bool is_float(int32_t t) { return t == WB_F32 || t == WB_BF16; }
int64_t type_bytes(int32_t t) { return t == WB_F32 ? 4 : t == WB_BF16 ? 2 : 1; }
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// One call's operands: each is refused for the first thing wrong with it, and
// `rc` keeps the first refusal.
struct Operands {
  KnownRange range;
  int rc = WB_OK;
  bool memory = true;  // look pointers up

  int refuse(const std::string& msg) {
    if (rc == WB_OK) rc = set_error(WB_EINVAL, msg);
    return rc;
  }

  void array(const void* p, int64_t count, int64_t bytes_each, const char* name) {
    if (rc != WB_OK || count == 0 || !memory) return;
    rc = check_extent_as(p, count * bytes_each, [&] { return std::string(name); }, static_cast<int>(bytes_each), &range);
  }

  void matrix(const wb_matrix& m, int64_t rows, int64_t cols, const char* name) {
    if (rc != WB_OK) return;
    if (m.rows != rows || m.cols != cols) {
      refuse(std::string(name) + " is " + std::to_string(m.rows) + " x " + std::to_string(m.cols) + ", not " +
             std::to_string(rows) + " x " + std::to_string(cols));
      return;
    }
    if (rows < 0 || cols < 1 || cols > kMaxCols || m.ld < cols || m.ld > kMaxStride || rows > kMaxExtent / m.ld) {
      refuse(std::string(name) + ": sizes or row distance out of range");
      return;
    }
    if (rows == 0 || !memory) return;
    const int64_t es = type_bytes(m.dtype);
    rc = check_extent_as(m.data, ((rows - 1) * m.ld + cols) * es, [&] { return std::string(name); }, static_cast<int>(es),
                         &range);
  }

  void floats(const wb_matrix& m, const char* name) {
    if (rc == WB_OK && !is_float(m.dtype)) refuse(std::string(name) + " is neither WB_F32 nor WB_BF16");
  }

  void scales(const wb_matrix& m, int64_t rows, int64_t cols, const char* name) {
    if (rc == WB_OK && m.data == nullptr && rows > 0) refuse(std::string(name) + " is null: fp8 values need scales");
    if (rc == WB_OK && m.dtype != WB_F32) refuse(std::string(name) + " is not WB_F32");
    matrix(m, rows, cols, name);
  }

  // a result of any of the three types
  void result(const wb_matrix& out, const wb_matrix* scales_of, int64_t rows, int64_t cols) {
    if (rc == WB_OK && !is_float(out.dtype) && out.dtype != WB_F8E4M3) refuse("out: unknown type");
    matrix(out, rows, cols, "out");
    const bool given = scales_of && scales_of->data;
    if (rc == WB_OK && out.dtype == WB_F8E4M3) {
      if (!scales_of) {
        refuse("fp8 out needs scales");
      } else {
        scales(*scales_of, rows, ceil_div(cols, wb::kScaleBlock), "scales of out");
      }
    } else if (rc == WB_OK && given) {
      refuse("scales are given for an out that is not fp8");
    }
  }
};

int too_many_rows(int64_t rows) {
  if (rows < 0) return set_error(WB_EINVAL, "negative number of rows");
  if (rows > kMaxRows) return set_error(WB_EUNSUPPORTED, "more than 4194303 rows");
  return WB_OK;
}

int launched(int e, const char* what) { return e == 0 ? WB_OK : hip_fail(static_cast<hipError_t>(e), what); }

int too_many_tiles() { return set_error(WB_EUNSUPPORTED, "more tiles than one launch takes"); }

int check_route(const wb_matrix* logits, const uint8_t* mask, int32_t k, Operands& ops) {
  if (!logits) return set_error(WB_EINVAL, "null argument");
  const int rc = too_many_rows(logits->rows);
  if (rc != WB_OK) return rc;
  if (logits->cols > wb::kMaxRouteExperts) return set_error(WB_EUNSUPPORTED, "more than 1024 experts");
  if (k < 1 || k > logits->cols) return set_error(WB_EINVAL, "k outside 1..experts");
  if (k > wb::kMaxRouteK) return set_error(WB_EUNSUPPORTED, "k past 64");
  if (logits->rows * k > INT32_MAX) return set_error(WB_EUNSUPPORTED, "rows * k past 2^31 - 1");
  ops.floats(*logits, "logits");
  ops.matrix(*logits, logits->rows, logits->cols, "logits");
  if (mask) ops.array(mask, logits->rows, 1, "mask");
  return ops.rc;
}

// The checks of wb_linear and, after them, its launch's arguments. Without
// `memory`, for the workspace's size, pointers are not looked up.
int check_linear(const wb_linear_args* p, Operands& ops, wb::LinearArgs& a, bool memory) {
  ops.memory = memory;
  if (!p) return set_error(WB_EINVAL, "null argument");
  const bool stacked = p->num_experts > 0;
  if (p->num_experts < 0 || p->num_experts > 65536) return set_error(WB_EINVAL, "num_experts outside 0..65536");
  int rc = too_many_rows(p->x.rows);
  if (rc == WB_OK) rc = too_many_rows(p->out.rows);
  if (rc != WB_OK) return rc;
  if (p->x.dtype != p->weight.dtype || (p->x.dtype != WB_BF16 && p->x.dtype != WB_F8E4M3))
    return set_error(WB_EUNSUPPORTED, "x and weight must both be bf16 or both fp8");
  if (p->activation < WB_ACT_NONE || p->activation > WB_ACT_GELU) return set_error(WB_EINVAL, "unknown activation");
  if (!stacked && (p->offsets || p->tokens)) return set_error(WB_EINVAL, "offsets and tokens need num_experts");
  if (stacked && !p->offsets) return set_error(WB_EINVAL, "stacked weights need offsets");
  const int64_t e = stacked ? p->num_experts : 1, k = p->x.cols;
  if (p->weight.rows < 1 || p->weight.rows % e != 0) return set_error(WB_EINVAL, "weight rows are no multiple of num_experts");
  const int64_t n = p->weight.rows / e;
  if (n > kMaxCols) return set_error(WB_EUNSUPPORTED, "weight of more than 2^26 rows");
  if (p->gated && n % 2 != 0) return set_error(WB_EINVAL, "gated weight with an odd number of rows");
  const int64_t n_out = p->gated ? n / 2 : n, rows = stacked ? p->out.rows : p->x.rows;
  if (stacked && !p->tokens && p->x.rows != rows)
    return set_error(WB_EINVAL, "without tokens, x has as many rows as out");
  if (stacked && p->tokens && p->x.rows == 0 && rows > 0) return set_error(WB_EINVAL, "tokens of an x without rows");
  const bool f8 = p->x.dtype == WB_F8E4M3;
  ops.matrix(p->x, p->x.rows, k, "x");
  ops.matrix(p->weight, p->weight.rows, k, "weight");
  if (f8) {
    ops.scales(p->x_scales, p->x.rows, ceil_div(k, wb::kScaleBlock), "x_scales");
    ops.scales(p->weight_scales, e * ceil_div(n, wb::kScaleBlock), ceil_div(k, wb::kScaleBlock), "weight_scales");
  } else if (p->x_scales.data || p->weight_scales.data) {
    return set_error(WB_EINVAL, "scales are given for operands that are not fp8");
  }
  if (p->bias.data) {
    ops.floats(p->bias, "bias");
    ops.matrix(p->bias, e, n, "bias");
  }
  if (p->residual.data) {
    ops.floats(p->residual, "residual");
    ops.matrix(p->residual, rows, n_out, "residual");
  }
  ops.result(p->out, &p->out_scales, rows, n_out);
  if (stacked) ops.array(p->offsets, e + 1, 4, "offsets");
  if (p->tokens) ops.array(p->tokens, rows, 4, "tokens");
  if (ops.rc != WB_OK) return ops.rc;

  const int64_t es = f8 ? 1 : 2;
  a.x = static_cast<const uint8_t*>(p->x.data), a.weight = static_cast<const uint8_t*>(p->weight.data);
  a.ld_x_bytes = p->x.ld * es, a.ld_w_bytes = p->weight.ld * es, a.stride_w_bytes = n * a.ld_w_bytes;
  a.rows = rows, a.x_rows = p->x.rows, a.n = static_cast<int32_t>(n), a.n_out = static_cast<int32_t>(n_out);
  a.k = static_cast<int32_t>(k), a.in_type = p->x.dtype, a.gated = p->gated != 0, a.activation = p->activation;
  a.num_experts = p->num_experts, a.offsets = p->offsets, a.tokens = p->tokens;
  if (f8) {
    a.x_scales = static_cast<const float*>(p->x_scales.data), a.ld_xs = p->x_scales.ld;
    a.weight_scales = static_cast<const float*>(p->weight_scales.data), a.ld_ws = p->weight_scales.ld;
    a.stride_ws = ceil_div(n, wb::kScaleBlock) * a.ld_ws;
  }
  if (p->bias.data) a.bias = p->bias.data, a.bias_type = p->bias.dtype, a.stride_bias = p->bias.ld;
  if (p->residual.data) a.residual = p->residual.data, a.residual_type = p->residual.dtype, a.ld_residual = p->residual.ld;
  a.out = p->out.data, a.out_type = p->out.dtype, a.ld_out = p->out.ld;
  if (p->out.dtype == WB_F8E4M3) a.out_scales = static_cast<float*>(p->out_scales.data), a.ld_os = p->out_scales.ld;
  const uintptr_t at = reinterpret_cast<uintptr_t>(a.x) | reinterpret_cast<uintptr_t>(a.weight) |
                       static_cast<uintptr_t>(a.ld_x_bytes) | static_cast<uintptr_t>(a.ld_w_bytes) |
                       static_cast<uintptr_t>(k * es);
  a.direct = at % 16 == 0 && wb::linear_near(a);
  return WB_OK;
}

}  // namespace

extern "C" {

int wb_add_rms_norm(const wb_matrix* x, const wb_matrix* residual, const wb_matrix* weight, float eps,
                    const wb_matrix* total, const wb_matrix* out, const wb_matrix* scales, void* stream) {
  return guarded([&]() -> int {
    if (!x || !weight || !out) return set_error(WB_EINVAL, "null argument");
    if (!(eps >= 0.0f)) return set_error(WB_EINVAL, "eps is negative or NaN");
    const int rc = too_many_rows(x->rows);
    if (rc != WB_OK) return rc;
    Operands ops;
    ops.floats(*x, "x");
    ops.matrix(*x, x->rows, x->cols, "x");
    ops.floats(*weight, "weight");
    ops.matrix(*weight, 1, x->cols, "weight");
    if (residual) {
      ops.floats(*residual, "residual");
      ops.matrix(*residual, x->rows, x->cols, "residual");
    }
    if (total) {
      ops.floats(*total, "total");
      ops.matrix(*total, x->rows, x->cols, "total");
    }
    ops.result(*out, scales, x->rows, x->cols);
    if (ops.rc != WB_OK) return ops.rc;
    wb::NormArgs a{};
    a.x = x->data, a.x_type = x->dtype, a.ld_x = x->ld, a.rows = x->rows, a.cols = x->cols;
    a.weight = weight->data, a.weight_type = weight->dtype, a.eps = eps;
    if (residual) a.residual = residual->data, a.residual_type = residual->dtype, a.ld_residual = residual->ld;
    if (total) a.total = total->data, a.total_type = total->dtype, a.ld_total = total->ld;
    a.out = out->data, a.out_type = out->dtype, a.ld_out = out->ld;
    if (out->dtype == WB_F8E4M3) a.scales = static_cast<float*>(scales->data), a.ld_scales = scales->ld;
    return launched(wb::launch_add_rms_norm(a, stream), "norm launch");
  });
}

int wb_route_workspace(int64_t rows, int32_t experts, size_t* bytes) {
  return guarded([&]() -> int {
    if (!bytes) return set_error(WB_EINVAL, "null argument");
    const int rc = too_many_rows(rows);
    if (rc != WB_OK) return rc;
    if (experts < 1) return set_error(WB_EINVAL, "no experts");
    if (experts > wb::kMaxRouteExperts) return set_error(WB_EUNSUPPORTED, "more than 1024 experts");
    *bytes = wb::route_workspace_bytes(rows, experts);
    return WB_OK;
  });
}

int wb_route(const wb_matrix* logits, const uint8_t* mask, int32_t k, int32_t renormalize, const wb_routing* out,
             void* workspace, size_t workspace_bytes, void* stream) {
  return guarded([&]() -> int {
    if (!out) return set_error(WB_EINVAL, "null argument");
    Operands ops;
    const int rc = check_route(logits, mask, k, ops);
    if (rc != WB_OK) return rc;
    const int64_t rows = logits->rows, n = rows * k;
    const int32_t experts = static_cast<int32_t>(logits->cols);
    const size_t need = wb::route_workspace_bytes(rows, experts);
    if (workspace_bytes < need) return set_error(WB_ESIZE, "workspace smaller than wb_route_workspace");
    ops.array(out->experts, n, 4, "experts");
    ops.array(out->gates, n, 4, "gates");
    ops.array(out->positions, n, 4, "positions");
    ops.array(out->tokens, n, 4, "tokens");
    ops.array(out->counts, experts, 4, "counts");
    ops.array(out->routed, 1, 4, "routed");
    ops.array(out->offsets, experts + 1, 4, "offsets");
    ops.array(out->loss, 1, 4, "loss");
    if (ops.rc == WB_OK)
      ops.rc = check_extent_as(workspace, static_cast<int64_t>(need), [] { return std::string("workspace"); }, 16, &ops.range);
    if (ops.rc != WB_OK) return ops.rc;
    wb::RouteArgs a{};
    a.logits = logits->data, a.logits_type = logits->dtype, a.ld_logits = logits->ld, a.rows = rows;
    a.mask = mask, a.num_experts = experts, a.k = k, a.renormalize = renormalize != 0;
    a.experts = out->experts, a.gates = out->gates, a.positions = out->positions, a.tokens = out->tokens;
    a.counts = out->counts, a.routed = out->routed, a.offsets = out->offsets, a.loss = out->loss, a.workspace = workspace;
    return launched(wb::launch_route(a, stream), "route launch");
  });
}

int wb_route_backward(const wb_matrix* logits, const uint8_t* mask, int32_t k, int32_t renormalize,
                      const wb_routing* routing, const float* d_gates, const float* d_loss,
                      const wb_matrix* d_logits, void* stream) {
  return guarded([&]() -> int {
    if (!routing || !d_logits) return set_error(WB_EINVAL, "null argument");
    Operands ops;
    const int rc = check_route(logits, mask, k, ops);
    if (rc != WB_OK) return rc;
    const int64_t rows = logits->rows, n = rows * k;
    ops.array(routing->experts, n, 4, "experts");
    ops.array(routing->gates, n, 4, "gates");
    ops.array(routing->counts, logits->cols, 4, "counts");
    ops.array(routing->routed, 1, 4, "routed");
    if (d_gates) ops.array(d_gates, n, 4, "d_gates");
    if (d_loss) ops.array(d_loss, 1, 4, "d_loss");
    if (ops.rc == WB_OK && d_logits->dtype != logits->dtype) return ops.refuse("d_logits has another type than the logits");
    ops.matrix(*d_logits, rows, logits->cols, "d_logits");
    if (ops.rc != WB_OK) return ops.rc;
    wb::RouteGradArgs a{};
    a.logits = logits->data, a.logits_type = logits->dtype, a.ld_logits = logits->ld, a.rows = rows;
    a.mask = mask, a.num_experts = static_cast<int32_t>(logits->cols), a.k = k, a.renormalize = renormalize != 0;
    a.experts = routing->experts, a.gates = routing->gates, a.counts = routing->counts, a.routed = routing->routed;
    a.d_gates = d_gates, a.d_loss = d_loss, a.d_logits = d_logits->data, a.ld_d_logits = d_logits->ld;
    return launched(wb::launch_route_grad(a, stream), "route gradient launch");
  });
}

int wb_linear_workspace(const wb_linear_args* p, size_t* bytes) {
  return guarded([&]() -> int {
    if (!bytes) return set_error(WB_EINVAL, "null argument");
    Operands ops;
    wb::LinearArgs a{};
    const int rc = check_linear(p, ops, a, false);
    if (rc != WB_OK) return rc;
    const int64_t need = wb::linear_workspace_bytes(a);
    if (need < 0) return too_many_tiles();
    *bytes = static_cast<size_t>(need);
    return WB_OK;
  });
}

int wb_linear(const wb_linear_args* p, void* workspace, size_t workspace_bytes, void* stream) {
  return guarded([&]() -> int {
    Operands ops;
    wb::LinearArgs a{};
    const int rc = check_linear(p, ops, a, true);
    if (rc != WB_OK) return rc;
    const int64_t need = wb::linear_workspace_bytes(a);
    if (need < 0) return too_many_tiles();
    if (workspace_bytes < static_cast<size_t>(need)) return set_error(WB_ESIZE, "workspace smaller than wb_linear_workspace");
    if (need) ops.rc = check_extent_as(workspace, need, [] { return std::string("workspace"); }, 16, &ops.range);
    if (ops.rc != WB_OK) return ops.rc;
    return launched(wb::launch_linear(a, workspace, stream), "product launch");
  });
}

int wb_combine(const wb_matrix* y, const int32_t* positions, const float* gates, int32_t k, const wb_matrix* residual,
               const int32_t* first, const int32_t* last, const wb_matrix* out, void* stream) {
  return guarded([&]() -> int {
    if (!y || !out) return set_error(WB_EINVAL, "null argument");
    if (k < 1) return set_error(WB_EINVAL, "k below 1");
    if (k > wb::kMaxRouteK) return set_error(WB_EUNSUPPORTED, "k past 64");
    if ((first == nullptr) != (last == nullptr)) return set_error(WB_EINVAL, "first and last go together");
    int rc = too_many_rows(out->rows);
    if (rc != WB_OK) return rc;
    Operands ops;
    ops.floats(*y, "y");
    if (y->rows > INT32_MAX) return set_error(WB_EUNSUPPORTED, "y of more than 2^31 - 1 rows");
    ops.matrix(*y, y->rows, out->cols, "y");
    ops.floats(*out, "out");
    ops.matrix(*out, out->rows, out->cols, "out");
    ops.array(positions, out->rows * k, 4, "positions");
    ops.array(gates, out->rows * k, 4, "gates");
    if (residual) {
      ops.floats(*residual, "residual");
      ops.matrix(*residual, out->rows, out->cols, "residual");
    }
    if (first) ops.array(first, 1, 4, "first");
    if (last) ops.array(last, 1, 4, "last");
    if (ops.rc != WB_OK) return ops.rc;
    wb::CombineArgs a{};
    a.y = y->data, a.y_type = y->dtype, a.ld_y = y->ld, a.y_rows = y->rows;
    a.positions = positions, a.gates = gates, a.k = k, a.first = first, a.last = last;
    if (residual) a.residual = residual->data, a.residual_type = residual->dtype, a.ld_residual = residual->ld;
    a.out = out->data, a.out_type = out->dtype, a.ld_out = out->ld, a.rows = out->rows, a.cols = out->cols;
    return launched(wb::launch_combine(a, stream), "combine launch");
  });
}

}  // extern "C"
