// Arguments of the operators' launches (norm.hip, route.hip, linear.hip), as
// ops_api.cpp fills them in after its checks. Sizes and strides are in
// elements unless a name says bytes; rows may lie any distance apart, and a
// row starts at the alignment of its element type.
#ifndef WB_OPS_HPP
#define WB_OPS_HPP

#include <cstddef>
#include <cstdint>

namespace wb {

constexpr int kScaleBlock = 128;        // columns (and, for weights, rows) under one fp8 scale
constexpr int kMaxRouteExperts = 1024;  // columns of the router's rows
constexpr int kMaxRouteK = 64;          // experts a token is sent to

struct NormArgs {
  const void* x;
  const void* residual;  // null: none
  const void* weight;
  void* total;  // null: not written
  void* out;
  float* scales;  // fp8 output only
  int64_t rows, cols;
  int64_t ld_x, ld_residual, ld_total, ld_out, ld_scales;
  int32_t x_type, residual_type, weight_type, total_type, out_type;  // wb_dtype
  float eps;
};

struct RouteArgs {
  const void* logits;
  const uint8_t* mask;  // null: every row is routed
  int32_t* experts;     // [rows, k]
  float* gates;         // [rows, k]
  int32_t* positions;   // [rows, k]
  int32_t* tokens;      // [rows * k]
  int32_t* counts;      // [experts]
  int32_t* routed;      // [1]: rows sent anywhere
  int32_t* offsets;     // [experts + 1]
  float* loss;          // [1]
  void* workspace;
  int64_t rows, ld_logits;
  int32_t num_experts, k, logits_type;
  bool renormalize;
};

struct RouteGradArgs {
  const void* logits;
  const uint8_t* mask;
  const int32_t* experts;
  const float* gates;
  const int32_t* counts;
  const int32_t* routed;
  const float* d_gates;  // null: zero
  const float* d_loss;   // null: zero
  void* d_logits;
  int64_t rows, ld_logits, ld_d_logits;
  int32_t num_experts, k, logits_type;
  bool renormalize;
};

struct CombineArgs {
  const void* y;
  const int32_t* positions;
  const float* gates;
  const void* residual;  // null: none
  const int32_t* first;  // null: every row of y may be read
  const int32_t* last;
  void* out;
  int64_t rows, cols, y_rows, ld_y, ld_residual, ld_out;
  int32_t k, y_type, residual_type, out_type;
};

struct LinearArgs {
  const uint8_t* x;
  const float* x_scales;
  const uint8_t* weight;
  const float* weight_scales;
  const int32_t* offsets;  // null: one weight, every row
  const int32_t* tokens;   // null: row p of the output comes from row p of x
  const void* bias;        // null: none
  const void* residual;    // null: none
  void* out;
  float* out_scales;
  int64_t rows, x_rows;  // rows of the output and of x
  int64_t ld_x_bytes, ld_w_bytes, stride_w_bytes, ld_xs, ld_ws, stride_ws, stride_bias;
  int64_t ld_residual, ld_out, ld_os;
  int32_t num_experts;
  int32_t n, n_out;  // rows of the weight, columns of the output
  int32_t k;
  int32_t in_type, bias_type, residual_type, out_type, activation;
  bool gated;
  // rows of x and weight start at multiples of 16 bytes and hold a multiple of
  // 16, 32-bit offsets reach them, and sixteen rows of the weight share a scale
  bool direct;
};

size_t route_workspace_bytes(int64_t rows, int32_t experts);
int64_t linear_workspace_bytes(const LinearArgs& a);  // -1: more tiles than one launch takes, nothing to launch

// Whether 32-bit offsets reach the rows of x and weight, and sixteen rows of
// the weight share a scale.
bool linear_near(const LinearArgs& a);

// Each enqueues its kernels on the stream and returns a hipError_t.
int launch_add_rms_norm(const NormArgs& a, void* stream);
int launch_route(const RouteArgs& a, void* stream);
int launch_route_grad(const RouteGradArgs& a, void* stream);
int launch_combine(const CombineArgs& a, void* stream);
int launch_linear(const LinearArgs& a, void* workspace, void* stream);

}  // namespace wb

#endif
