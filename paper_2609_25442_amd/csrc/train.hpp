// Arguments of the trainer's operators' launches (embedding.hip, layer_norm.hip,
// expert_rows.hip, activate.hip), as train_api.cpp fills them in after its
// checks. Sizes and strides as in ops.hpp.
#ifndef WB_TRAIN_HPP
#define WB_TRAIN_HPP

#include <cstddef>
#include <cstdint>

#include "ops.hpp"

namespace wb {

struct EmbedArgs {
  const void* tokens;  // [count], of token_bytes
  const void* weight;
  void* out;
  int64_t count, rows, cols;  // rows: of the weight
  int64_t first, ld_weight, ld_out;
  int32_t token_bytes, weight_type, out_type;
  float scale;
};

struct EmbedGradArgs {
  const void* tokens;
  const void* d_out;
  void* d_weight;
  void* workspace;
  int64_t count, rows, cols;
  int64_t first, ld_d_out, ld_d_weight;
  int32_t token_bytes, d_out_type, d_weight_type;
  float scale;
};

struct LayerNormArgs {
  const void* x;
  const void* residual;  // null: none
  const void* weight;
  const void* bias;  // null: none
  void* total;       // with a residual
  void* out;
  float* mean;  // null: not centred
  float* inv;
  int64_t rows, cols;
  int64_t ld_x, ld_residual, ld_total, ld_out;
  int32_t x_type, residual_type, weight_type, bias_type, total_type, out_type;
  float eps;
};

struct LayerNormGradArgs {
  const void* d_out;
  const void* total;
  const void* weight;
  const void* d_total;  // null: zero
  const float* mean;    // null: not centred
  const float* inv;
  void* d_x;
  void* d_residual;  // null: not written
  void* d_weight;    // null: not computed
  void* d_bias;      // null: not written
  float* workspace;
  int64_t rows, cols;
  int64_t ld_d_out, ld_total, ld_d_total, ld_d_x, ld_d_residual;
  int32_t d_out_type, total_type, weight_type, d_total_type, d_x_type, d_residual_type, d_weight_type, d_bias_type;
};

// Rows that go to places, or come from them.
struct PlacesArgs {
  const int32_t* positions;  // [rows, k]
  const int32_t* tokens;     // [places]
  const int32_t* first;      // null: every place
  const int32_t* last;
  int64_t rows, places, cols;
  int32_t k;
};

struct DispatchArgs {
  PlacesArgs at;
  const void* x;
  void* out;
  int64_t ld_x, ld_out;
  int32_t x_type, out_type;
};

struct DispatchGradArgs {
  PlacesArgs at;
  const void* d_out;
  void* d_x;
  int64_t ld_d_out, ld_d_x;
  int32_t d_out_type, d_x_type;
};

struct CollectArgs {
  PlacesArgs at;
  const void* y;
  const float* gates;
  const void* residual;  // null: none
  void* out;
  int64_t ld_y, ld_residual, ld_out;
  int32_t y_type, residual_type, out_type;
};

struct CombineGradArgs {
  PlacesArgs at;
  const void* d_out;
  const void* y;  // null: no d_gates
  const float* gates;
  void* d_y;  // null: not written
  float* d_gates;
  int64_t ld_d_out, ld_y, ld_d_y;
  int32_t d_out_type, y_type, d_y_type;
};

struct ActivateArgs {
  const void* x;
  void* out;
  uint8_t* codes;  // null: none
  float* scales;
  int64_t rows, cols;  // of out
  int64_t ld_x, ld_out, ld_codes, ld_scales;
  int32_t x_type, out_type, activation;
  bool gated;
};

struct ActivateGradArgs {
  const void* d_out;
  const void* x;        // values, or codes where there are scales
  const float* scales;  // null: none
  void* d_x;
  int64_t rows, cols;  // of d_out
  int64_t ld_d_out, ld_x, ld_scales, ld_d_x;
  int32_t d_out_type, x_type, d_x_type, activation;
  bool gated;
};

bool embed_grad_fits(int64_t count, int64_t rows, int64_t cols);  // whether its launches take these sizes
size_t embed_grad_workspace_bytes(int64_t count, int64_t rows, int64_t cols);
size_t layer_norm_grad_workspace_bytes(int64_t rows, int64_t cols);

// Each enqueues its kernels on the stream and returns a hipError_t.
int launch_embed(const EmbedArgs& a, void* stream);
int launch_embed_grad(const EmbedGradArgs& a, void* stream);
int launch_layer_norm(const LayerNormArgs& a, void* stream);
int launch_layer_norm_grad(const LayerNormGradArgs& a, void* stream);
int launch_dispatch(const DispatchArgs& a, void* stream);
int launch_dispatch_grad(const DispatchGradArgs& a, void* stream);
int launch_collect(const CollectArgs& a, void* stream);
int launch_combine_grad(const CombineGradArgs& a, void* stream);
int launch_activate(const ActivateArgs& a, void* stream);
int launch_activate_grad(const ActivateGradArgs& a, void* stream);

}  // namespace wb

#endif
