// C entries of the trainer's operators (declared in include/wb.h): what they
// refuse, and the launch arguments of embedding.hip, layer_norm.hip,
// expert_rows.hip and activate.hip.
#include <string>

#include "operands.hpp"
#include "train.hpp"

namespace {

using wb::ceil_div;
using wb::check_extent_as;
using wb::guarded;
using wb::kMaxCols;
using wb::kMaxRows;
using wb::launched;
using wb::Operands;
using wb::set_error;
using wb::too_many_rows;

constexpr int64_t kMaxFirst = int64_t(1) << 62;

int check_sizes(int64_t rows, int64_t cols) {
  const int rc = too_many_rows(rows);
  if (rc != WB_OK) return rc;
  if (cols < 1 || cols > kMaxCols) return set_error(WB_EINVAL, "columns outside 1..2^26");
  return WB_OK;
}

void floats(Operands& ops, const wb_matrix& m, int64_t rows, int64_t cols, const char* name) {
  ops.floats(m, name);
  ops.matrix(m, rows, cols, name);
}

int check_workspace(Operands& ops, const void* workspace, size_t bytes, size_t need, const char* of) {
  if (ops.rc != WB_OK) return ops.rc;
  if (bytes < need) return set_error(WB_ESIZE, std::string("workspace smaller than ") + of);
  if (need)
    ops.rc = check_extent_as(workspace, static_cast<int64_t>(need), [] { return std::string("workspace"); }, 16, &ops.range);
  return ops.rc;
}

// Token ids, and the table of `rows` that they name rows of.
int check_tokens(const wb_tokens* t, int64_t rows, int64_t first) {
  if (t->bytes != 4 && t->bytes != 8) return set_error(WB_EINVAL, "tokens are neither int32 nor int64");
  int rc = too_many_rows(t->count);
  if (rc == WB_OK) rc = too_many_rows(rows);
  if (rc != WB_OK) return rc;
  if (first < 0 || first > kMaxFirst) return set_error(WB_EINVAL, "first is outside 0..2^62");
  return WB_OK;
}

int check_places(const wb_matrix& by_row, const wb_matrix& by_place, const int32_t* positions, const int32_t* tokens, int32_t k,
                 const int32_t* first, const int32_t* last, Operands& ops, wb::PlacesArgs& a) {
  if (k < 1) return set_error(WB_EINVAL, "k below 1");
  if (k > wb::kMaxRouteK) return set_error(WB_EUNSUPPORTED, "k past 64");
  if ((first == nullptr) != (last == nullptr)) return set_error(WB_EINVAL, "first and last go together");
  const int rc = check_sizes(by_row.rows, by_row.cols);
  if (rc != WB_OK) return rc;
  if (by_place.rows < 0) return set_error(WB_EINVAL, "negative number of places");
  if (by_place.rows > INT32_MAX) return set_error(WB_EUNSUPPORTED, "more than 2^31 - 1 places");
  ops.array(positions, by_row.rows * k, 4, "positions");
  ops.array(tokens, by_place.rows, 4, "tokens");
  if (first) ops.array(first, 1, 4, "first");
  if (last) ops.array(last, 1, 4, "last");
  a.positions = positions, a.tokens = tokens, a.first = first, a.last = last;
  a.rows = by_row.rows, a.places = by_place.rows, a.cols = by_row.cols, a.k = k;
  return ops.rc;
}

int check_activation(int32_t activation, int32_t gated, int64_t rows, int64_t wide) {
  if (activation < WB_ACT_NONE || activation > WB_ACT_GELU) return set_error(WB_EINVAL, "unknown activation");
  const int rc = check_sizes(rows, wide);
  if (rc != WB_OK) return rc;
  if (gated && wide % 2 != 0) return set_error(WB_EINVAL, "gated x with an odd number of columns");
  return WB_OK;
}

// Scales of x in 8 bits: per 128 columns of each half.
int64_t kept_scales(int64_t cols, bool gated) { return ceil_div(cols, wb::kScaleBlock) * (gated ? 2 : 1); }

}  // namespace

extern "C" {

int wb_embedding(const wb_tokens* tokens, const wb_matrix* weight, float scale, int64_t first, const wb_matrix* out,
                 void* stream) {
  return guarded([&]() -> int {
    if (!tokens || !weight || !out) return set_error(WB_EINVAL, "null argument");
    Operands ops;
    int rc = check_tokens(tokens, weight->rows, first);
    if (rc == WB_OK) rc = check_sizes(weight->rows, weight->cols);
    if (rc != WB_OK) return rc;
    ops.array(tokens->data, tokens->count, tokens->bytes, "tokens");
    floats(ops, *weight, weight->rows, weight->cols, "weight");
    floats(ops, *out, tokens->count, weight->cols, "out");
    if (ops.rc != WB_OK) return ops.rc;
    wb::EmbedArgs a{};
    a.tokens = tokens->data, a.token_bytes = tokens->bytes, a.count = tokens->count, a.first = first, a.scale = scale;
    a.weight = weight->data, a.weight_type = weight->dtype, a.ld_weight = weight->ld, a.rows = weight->rows;
    a.cols = weight->cols, a.out = out->data, a.out_type = out->dtype, a.ld_out = out->ld;
    return launched(wb::launch_embed(a, stream), "embedding launch");
  });
}

int wb_embedding_backward_workspace(int64_t count, int64_t rows, int64_t cols, size_t* bytes) {
  return guarded([&]() -> int {
    if (!bytes) return set_error(WB_EINVAL, "null argument");
    int rc = too_many_rows(count);
    if (rc == WB_OK) rc = check_sizes(rows, cols);
    if (rc != WB_OK) return rc;
    *bytes = wb::embed_grad_workspace_bytes(count, rows, cols);
    return WB_OK;
  });
}

int wb_embedding_backward(const wb_tokens* tokens, const wb_matrix* d_out, float scale, int64_t first,
                          const wb_matrix* d_weight, void* workspace, size_t workspace_bytes, void* stream) {
  return guarded([&]() -> int {
    if (!tokens || !d_out || !d_weight) return set_error(WB_EINVAL, "null argument");
    Operands ops;
    int rc = check_tokens(tokens, d_weight->rows, first);
    if (rc == WB_OK) rc = check_sizes(d_weight->rows, d_weight->cols);
    if (rc != WB_OK) return rc;
    // ahead of its first launch: a refused call writes nothing
    if (!wb::embed_grad_fits(tokens->count, d_weight->rows, d_weight->cols))
      return launched(hipErrorInvalidConfiguration, "embedding gradient launch");
    ops.array(tokens->data, tokens->count, tokens->bytes, "tokens");
    floats(ops, *d_out, tokens->count, d_weight->cols, "d_out");
    floats(ops, *d_weight, d_weight->rows, d_weight->cols, "d_weight");
    rc = check_workspace(ops, workspace, workspace_bytes,
                         wb::embed_grad_workspace_bytes(tokens->count, d_weight->rows, d_weight->cols),
                         "wb_embedding_backward_workspace");
    if (rc != WB_OK) return rc;
    wb::EmbedGradArgs a{};
    a.tokens = tokens->data, a.token_bytes = tokens->bytes, a.count = tokens->count, a.first = first, a.scale = scale;
    a.d_out = d_out->data, a.d_out_type = d_out->dtype, a.ld_d_out = d_out->ld;
    a.d_weight = d_weight->data, a.d_weight_type = d_weight->dtype, a.ld_d_weight = d_weight->ld;
    a.rows = d_weight->rows, a.cols = d_weight->cols, a.workspace = workspace;
    return launched(wb::launch_embed_grad(a, stream), "embedding gradient launch");
  });
}

int wb_add_layer_norm(const wb_matrix* x, const wb_matrix* residual, const wb_matrix* weight, const wb_matrix* bias,
                      float eps, const wb_matrix* total, const wb_matrix* out, float* mean, float* inv, void* stream) {
  return guarded([&]() -> int {
    if (!x || !weight || !out) return set_error(WB_EINVAL, "null argument");
    if (!(eps >= 0.0f)) return set_error(WB_EINVAL, "eps is negative or NaN");
    if ((residual == nullptr) != (total == nullptr)) return set_error(WB_EINVAL, "residual and total go together");
    const int rc = check_sizes(x->rows, x->cols);
    if (rc != WB_OK) return rc;
    Operands ops;
    floats(ops, *x, x->rows, x->cols, "x");
    floats(ops, *weight, 1, x->cols, "weight");
    if (bias) floats(ops, *bias, 1, x->cols, "bias");
    if (residual) {
      floats(ops, *residual, x->rows, x->cols, "residual");
      floats(ops, *total, x->rows, x->cols, "total");
    }
    floats(ops, *out, x->rows, x->cols, "out");
    if (mean) ops.array(mean, x->rows, 4, "mean");
    ops.array(inv, x->rows, 4, "inv");
    if (ops.rc != WB_OK) return ops.rc;
    wb::LayerNormArgs a{};
    a.x = x->data, a.x_type = x->dtype, a.ld_x = x->ld, a.rows = x->rows, a.cols = x->cols, a.eps = eps;
    a.weight = weight->data, a.weight_type = weight->dtype;
    if (bias) a.bias = bias->data, a.bias_type = bias->dtype;
    if (residual) {
      a.residual = residual->data, a.residual_type = residual->dtype, a.ld_residual = residual->ld;
      a.total = total->data, a.total_type = total->dtype, a.ld_total = total->ld;
    }
    a.out = out->data, a.out_type = out->dtype, a.ld_out = out->ld, a.mean = mean, a.inv = inv;
    return launched(wb::launch_layer_norm(a, stream), "layer norm launch");
  });
}

int wb_add_layer_norm_backward_workspace(int64_t rows, int64_t cols, size_t* bytes) {
  return guarded([&]() -> int {
    if (!bytes) return set_error(WB_EINVAL, "null argument");
    const int rc = check_sizes(rows, cols);
    if (rc != WB_OK) return rc;
    *bytes = wb::layer_norm_grad_workspace_bytes(rows, cols);
    return WB_OK;
  });
}

int wb_add_layer_norm_backward(const wb_matrix* d_out, const wb_matrix* total, const wb_matrix* weight,
                               const wb_matrix* d_total, const float* mean, const float* inv, const wb_matrix* d_x,
                               const wb_matrix* d_residual, const wb_matrix* d_weight, const wb_matrix* d_bias,
                               void* workspace, size_t workspace_bytes, void* stream) {
  return guarded([&]() -> int {
    if (!d_out || !total || !weight || !d_x) return set_error(WB_EINVAL, "null argument");
    if (d_bias && !d_weight) return set_error(WB_EINVAL, "d_bias without d_weight");
    const int64_t rows = total->rows, cols = total->cols;
    int rc = check_sizes(rows, cols);
    if (rc != WB_OK) return rc;
    Operands ops;
    floats(ops, *total, rows, cols, "total");
    floats(ops, *d_out, rows, cols, "d_out");
    floats(ops, *weight, 1, cols, "weight");
    if (d_total) floats(ops, *d_total, rows, cols, "d_total");
    floats(ops, *d_x, rows, cols, "d_x");
    if (d_residual) floats(ops, *d_residual, rows, cols, "d_residual");
    if (d_weight) floats(ops, *d_weight, 1, cols, "d_weight");
    if (d_bias) floats(ops, *d_bias, 1, cols, "d_bias");
    if (mean) ops.array(mean, rows, 4, "mean");
    ops.array(inv, rows, 4, "inv");
    rc = check_workspace(ops, workspace, workspace_bytes, wb::layer_norm_grad_workspace_bytes(rows, cols),
                         "wb_add_layer_norm_backward_workspace");
    if (rc != WB_OK) return rc;
    wb::LayerNormGradArgs a{};
    a.d_out = d_out->data, a.d_out_type = d_out->dtype, a.ld_d_out = d_out->ld;
    a.total = total->data, a.total_type = total->dtype, a.ld_total = total->ld;
    a.weight = weight->data, a.weight_type = weight->dtype;
    if (d_total) a.d_total = d_total->data, a.d_total_type = d_total->dtype, a.ld_d_total = d_total->ld;
    a.mean = mean, a.inv = inv, a.rows = rows, a.cols = cols;
    a.d_x = d_x->data, a.d_x_type = d_x->dtype, a.ld_d_x = d_x->ld;
    if (d_residual) a.d_residual = d_residual->data, a.d_residual_type = d_residual->dtype, a.ld_d_residual = d_residual->ld;
    if (d_weight) a.d_weight = d_weight->data, a.d_weight_type = d_weight->dtype;
    if (d_bias) a.d_bias = d_bias->data, a.d_bias_type = d_bias->dtype;
    a.workspace = static_cast<float*>(workspace);
    return launched(wb::launch_layer_norm_grad(a, stream), "layer norm gradient launch");
  });
}

int wb_dispatch(const wb_matrix* x, const int32_t* positions, const int32_t* tokens, int32_t k, const int32_t* first,
                const int32_t* last, const wb_matrix* out, void* stream) {
  return guarded([&]() -> int {
    if (!x || !out) return set_error(WB_EINVAL, "null argument");
    Operands ops;
    wb::DispatchArgs a{};
    const int rc = check_places(*x, *out, positions, tokens, k, first, last, ops, a.at);
    if (rc != WB_OK) return rc;
    floats(ops, *x, x->rows, x->cols, "x");
    floats(ops, *out, out->rows, x->cols, "out");
    if (ops.rc != WB_OK) return ops.rc;
    a.x = x->data, a.x_type = x->dtype, a.ld_x = x->ld, a.out = out->data, a.out_type = out->dtype, a.ld_out = out->ld;
    return launched(wb::launch_dispatch(a, stream), "dispatch launch");
  });
}

int wb_dispatch_backward(const wb_matrix* d_out, const int32_t* positions, const int32_t* tokens, int32_t k,
                         const int32_t* first, const int32_t* last, const wb_matrix* d_x, void* stream) {
  return guarded([&]() -> int {
    if (!d_out || !d_x) return set_error(WB_EINVAL, "null argument");
    Operands ops;
    wb::DispatchGradArgs a{};
    const int rc = check_places(*d_x, *d_out, positions, tokens, k, first, last, ops, a.at);
    if (rc != WB_OK) return rc;
    floats(ops, *d_out, d_out->rows, d_x->cols, "d_out");
    floats(ops, *d_x, d_x->rows, d_x->cols, "d_x");
    if (ops.rc != WB_OK) return ops.rc;
    a.d_out = d_out->data, a.d_out_type = d_out->dtype, a.ld_d_out = d_out->ld;
    a.d_x = d_x->data, a.d_x_type = d_x->dtype, a.ld_d_x = d_x->ld;
    return launched(wb::launch_dispatch_grad(a, stream), "dispatch gradient launch");
  });
}

int wb_collect(const wb_matrix* y, const int32_t* positions, const int32_t* tokens, const float* gates, int32_t k,
               const wb_matrix* residual, const int32_t* first, const int32_t* last, const wb_matrix* out, void* stream) {
  return guarded([&]() -> int {
    if (!y || !out) return set_error(WB_EINVAL, "null argument");
    Operands ops;
    wb::CollectArgs a{};
    const int rc = check_places(*out, *y, positions, tokens, k, first, last, ops, a.at);
    if (rc != WB_OK) return rc;
    floats(ops, *y, y->rows, out->cols, "y");
    ops.array(gates, out->rows * k, 4, "gates");
    if (residual) {
      floats(ops, *residual, out->rows, out->cols, "residual");
      a.residual = residual->data, a.residual_type = residual->dtype, a.ld_residual = residual->ld;
    }
    floats(ops, *out, out->rows, out->cols, "out");
    if (ops.rc != WB_OK) return ops.rc;
    a.y = y->data, a.y_type = y->dtype, a.ld_y = y->ld, a.gates = gates;
    a.out = out->data, a.out_type = out->dtype, a.ld_out = out->ld;
    return launched(wb::launch_collect(a, stream), "collect launch");
  });
}

int wb_combine_backward(const wb_matrix* d_out, const wb_matrix* y, const int32_t* positions, const int32_t* tokens,
                        const float* gates, int32_t k, const int32_t* first, const int32_t* last, const wb_matrix* d_y,
                        float* d_gates, void* stream) {
  return guarded([&]() -> int {
    if (!d_out || (!y && !d_y)) return set_error(WB_EINVAL, "null argument");
    // gates of no rows have no address
    if ((y == nullptr) != (d_gates == nullptr) && !(y && d_out->rows == 0))
      return set_error(WB_EINVAL, "y and d_gates go together");
    Operands ops;
    wb::CombineGradArgs a{};
    const wb_matrix& by_place = y ? *y : *d_y;
    const int rc = check_places(*d_out, by_place, positions, tokens, k, first, last, ops, a.at);
    if (rc != WB_OK) return rc;
    floats(ops, *d_out, d_out->rows, d_out->cols, "d_out");
    ops.array(gates, d_out->rows * k, 4, "gates");
    if (y) {
      floats(ops, *y, y->rows, d_out->cols, "y");
      ops.array(d_gates, d_out->rows * k, 4, "d_gates");
      a.y = y->data, a.y_type = y->dtype, a.ld_y = y->ld, a.d_gates = d_gates;
    }
    if (d_y) {
      floats(ops, *d_y, by_place.rows, d_out->cols, "d_y");
      a.d_y = d_y->data, a.d_y_type = d_y->dtype, a.ld_d_y = d_y->ld;
    }
    if (ops.rc != WB_OK) return ops.rc;
    a.d_out = d_out->data, a.d_out_type = d_out->dtype, a.ld_d_out = d_out->ld, a.gates = gates;
    return launched(wb::launch_combine_grad(a, stream), "combine gradient launch");
  });
}

int wb_activate(const wb_matrix* x, int32_t activation, int32_t gated, const wb_matrix* out, const wb_matrix* codes,
                const wb_matrix* scales, void* stream) {
  return guarded([&]() -> int {
    if (!x || !out) return set_error(WB_EINVAL, "null argument");
    if ((codes == nullptr) != (scales == nullptr)) return set_error(WB_EINVAL, "codes and scales go together");
    const int rc = check_activation(activation, gated, x->rows, x->cols);
    if (rc != WB_OK) return rc;
    const int64_t cols = gated ? x->cols / 2 : x->cols;
    Operands ops;
    floats(ops, *x, x->rows, x->cols, "x");
    floats(ops, *out, x->rows, cols, "out");
    if (codes) {
      if (ops.rc == WB_OK && codes->dtype != WB_F8E4M3) return ops.refuse("codes are not WB_F8E4M3");
      ops.matrix(*codes, x->rows, x->cols, "codes");
      ops.scales(*scales, x->rows, kept_scales(cols, gated != 0), "scales");
    }
    if (ops.rc != WB_OK) return ops.rc;
    wb::ActivateArgs a{};
    a.x = x->data, a.x_type = x->dtype, a.ld_x = x->ld, a.out = out->data, a.out_type = out->dtype, a.ld_out = out->ld;
    a.rows = x->rows, a.cols = cols, a.activation = activation, a.gated = gated != 0;
    if (codes) {
      a.codes = static_cast<uint8_t*>(codes->data), a.ld_codes = codes->ld;
      a.scales = static_cast<float*>(scales->data), a.ld_scales = scales->ld;
    }
    return launched(wb::launch_activate(a, stream), "activation launch");
  });
}

int wb_activate_backward(const wb_matrix* d_out, const wb_matrix* x, const wb_matrix* scales, int32_t activation,
                         int32_t gated, const wb_matrix* d_x, void* stream) {
  return guarded([&]() -> int {
    if (!d_out || !x || !d_x) return set_error(WB_EINVAL, "null argument");
    const int rc = check_activation(activation, gated, x->rows, x->cols);
    if (rc != WB_OK) return rc;
    const int64_t cols = gated ? x->cols / 2 : x->cols;
    Operands ops;
    if (scales) {
      if (x->dtype != WB_F8E4M3) return ops.refuse("scales are given for an x that is not WB_F8E4M3");
      ops.matrix(*x, x->rows, x->cols, "x");
      ops.scales(*scales, x->rows, kept_scales(cols, gated != 0), "scales");
    } else {
      floats(ops, *x, x->rows, x->cols, "x");
    }
    floats(ops, *d_out, x->rows, cols, "d_out");
    floats(ops, *d_x, x->rows, x->cols, "d_x");
    if (ops.rc != WB_OK) return ops.rc;
    wb::ActivateGradArgs a{};
    a.d_out = d_out->data, a.d_out_type = d_out->dtype, a.ld_d_out = d_out->ld;
    a.x = x->data, a.x_type = x->dtype, a.ld_x = x->ld;
    if (scales) a.scales = static_cast<const float*>(scales->data), a.ld_scales = scales->ld;
    a.d_x = d_x->data, a.d_x_type = d_x->dtype, a.ld_d_x = d_x->ld;
    a.rows = x->rows, a.cols = cols, a.activation = activation, a.gated = gated != 0;
    return launched(wb::launch_activate_grad(a, stream), "activation gradient launch");
  });
}

}  // extern "C"
