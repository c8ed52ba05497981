// Layer norm of a residual sum, and its gradients:
//   t = x + residual, rounded to the type it is kept in;  h = (t - mean) inv,  out = h w + b
//   g = dout w;  dt = inv (g - mean(g) - h mean(g h)) + dtotal;  dw = sum_rows dout h,  db = sum_rows dout
// or without centring: mean 0, and the mean square in place of the variance.
//
// Forward, a row is held in registers between its two sums (mean, then squares
// of what is left) and its result, as in norm.hip.
#include <algorithm>

#include "ops_device.hpp"
#include "train.hpp"

namespace wb {
namespace {

constexpr int kMaxWaves = 16;
constexpr int64_t kManyRows = 2048;

__device__ __forceinline__ float rounded(float v, int type) {
  return type == WB_F32 ? v : __builtin_bit_cast(float, pack_bf16(v, v) << 16);
}

// The sum over a workgroup's wavefronts, in their order; `part` is free again after the next barrier.
__device__ __forceinline__ float sum_of_group(float v, float* part, int waves) {
  v = sum_of_wave(v);
  if (waves == 1) return v;
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
  __syncthreads();
  v = 0.0f;
  for (int w = 0; w < waves; ++w) v += part[w];
  return v;
}

// ---- forward -------------------------------------------------------------------
// A row takes `waves` wavefronts (ROWS > 1: one, and the workgroup holds ROWS
// rows), each lane V runs of eight columns. LOOP: rows wider than the registers
// are read again for each step.
template <int V, int ROWS, bool LOOP, bool NT>
__global__ __launch_bounds__(ROWS > 1 ? 64 * ROWS : 64 * kMaxWaves) void wb_layer_norm_kernel(LayerNormArgs a) {
  __shared__ float parts[2][kMaxWaves];
  const int wave = threadIdx.x >> 6;
  const int64_t row = ROWS > 1 ? int64_t(blockIdx.x) * ROWS + wave : int64_t(blockIdx.x);
  if (ROWS > 1 && row >= a.rows) return;
  const int lane = ROWS > 1 ? threadIdx.x & 63 : threadIdx.x;
  const int lanes = ROWS > 1 ? 64 : blockDim.x, waves = lanes / 64;
  const char* x = static_cast<const char*>(a.x) + row * a.ld_x * bytes_of(a.x_type);
  const char* res = static_cast<const char*>(a.residual) + row * a.ld_residual * bytes_of(a.residual_type);
  char* total = static_cast<char*>(a.total) + row * a.ld_total * bytes_of(a.total_type);
  char* out = static_cast<char*>(a.out) + row * a.ld_out * bytes_of(a.out_type);
  const int64_t step = int64_t(lanes) * 8, stride = LOOP ? step * V : a.cols;

  const auto load = [&](int64_t c, float(&t)[8]) {
    float r[8];
    if (c + 8 <= a.cols) {
      load_eight<NT>(x, c, a.x_type, t);
      if (!a.residual) return;
      load_eight<NT>(res, c, a.residual_type, r);
    } else {
      load_tail(x, c, a.cols, a.x_type, t);
      if (!a.residual) return;
      load_tail(res, c, a.cols, a.residual_type, r);
    }
    for (int i = 0; i < 8; ++i) t[i] = rounded(t[i] + r[i], a.total_type);
  };

  float t[V][8], sum = 0.0f;
  for (int64_t base = 0; base < a.cols; base += stride) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int64_t c = base + v * step + lane * 8;
      for (int i = 0; i < 8; ++i) t[v][i] = 0.0f;
      if (c < a.cols) load(c, t[v]);
    }
#pragma unroll
    for (int v = 0; v < V; ++v)
      for (int i = 0; i < 8; ++i) sum += t[v][i];
  }
  const float n = static_cast<float>(a.cols);
  const float mean = a.mean ? sum_of_group(sum, parts[0], waves) / n : 0.0f;
  float squares = 0.0f;
  for (int64_t base = 0; base < a.cols; base += stride) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int64_t c = base + v * step + lane * 8;
      if (c >= a.cols) continue;
      if (LOOP) load(c, t[v]);
      for (int i = 0; i < 8; ++i) {
        const float d = c + i < a.cols ? t[v][i] - mean : 0.0f;
        squares = __builtin_fmaf(d, d, squares);
      }
    }
  }
  const float inv = 1.0f / sqrtf(sum_of_group(squares, parts[1], waves) / n + a.eps);
  if (lane == 0) {
    a.inv[row] = inv;
    if (a.mean) a.mean[row] = mean;
  }
  for (int64_t base = 0; base < a.cols; base += stride) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int64_t c = base + v * step + lane * 8;
      if (c >= a.cols) continue;
      float w[8], b[8];
      if (LOOP) load(c, t[v]);
      load_run(static_cast<const char*>(a.weight), c, a.cols, a.weight_type, w);
      for (int i = 0; i < 8; ++i) b[i] = 0.0f;
      if (a.bias) load_run(static_cast<const char*>(a.bias), c, a.cols, a.bias_type, b);
      for (int i = 0; i < 8; ++i) w[i] = __builtin_fmaf((t[v][i] - mean) * inv, w[i], b[i]);
      if (c + 8 <= a.cols) {
        if (a.total) store_eight<NT>(total, c, a.total_type, t[v]);
        store_eight<NT>(out, c, a.out_type, w);
      } else {
        if (a.total) store_tail(total, c, a.cols, a.total_type, t[v]);
        store_tail(out, c, a.cols, a.out_type, w);
      }
    }
  }
}

template <int V, int ROWS, bool LOOP>
hipError_t launch(const LayerNormArgs& a, int waves, hipStream_t st) {
  const dim3 grid(static_cast<uint32_t>((a.rows + ROWS - 1) / ROWS)), block(64 * (ROWS > 1 ? ROWS : waves));
  const int64_t row_bytes = a.cols * (bytes_of(a.x_type) + (a.residual ? bytes_of(a.residual_type) + bytes_of(a.total_type) : 0) +
                                      bytes_of(a.out_type));
  if (a.rows * row_bytes > kStreamBytes)
    hipLaunchKernelGGL((wb_layer_norm_kernel<V, ROWS, LOOP, true>), grid, block, 0, st, a);
  else
    hipLaunchKernelGGL((wb_layer_norm_kernel<V, ROWS, LOOP, false>), grid, block, 0, st, a);
  return hipGetLastError();
}

// ---- gradients -------------------------------------------------------------------
// Rows wider than the registers hold: their two sums first, then slabs of
// columns over strips of rows, whose sums of dw and db meet in a third launch.

constexpr int kSlab = 2048, kSlabThreads = kSlab / 8;

// [rows][2]: mean of g, mean of g h
__global__ __launch_bounds__(64 * kMaxWaves) void wb_layer_norm_sums_kernel(LayerNormGradArgs a, float* sums) {
  __shared__ float parts[2][kMaxWaves];
  const int64_t row = blockIdx.x;
  const char* d_row = static_cast<const char*>(a.d_out) + row * a.ld_d_out * bytes_of(a.d_out_type);
  const char* t_row = static_cast<const char*>(a.total) + row * a.ld_total * bytes_of(a.total_type);
  const float mean = a.mean ? a.mean[row] : 0.0f, inv = a.inv[row];
  float s1 = 0.0f, s2 = 0.0f;
  for (int64_t c = threadIdx.x * 8; c < a.cols; c += blockDim.x * 8) {
    float d[8], t[8], w[8];
    load_run(d_row, c, a.cols, a.d_out_type, d);
    load_run(t_row, c, a.cols, a.total_type, t);
    load_run(static_cast<const char*>(a.weight), c, a.cols, a.weight_type, w);
    for (int i = 0; i < 8; ++i) {
      const float g = d[i] * w[i];
      if (c + i < a.cols) s1 += g, s2 = __builtin_fmaf(g, (t[i] - mean) * inv, s2);
    }
  }
  const int waves = blockDim.x / 64;
  s1 = sum_of_group(s1, parts[0], waves);
  s2 = sum_of_group(s2, parts[1], waves);
  if (threadIdx.x == 0) {
    const float n = static_cast<float>(a.cols);
    sums[row * 2] = a.mean ? s1 / n : 0.0f;
    sums[row * 2 + 1] = s2 / n;
  }
}

// parts: [2][strips][cols]
__global__ __launch_bounds__(kSlabThreads) void wb_layer_norm_slab_kernel(LayerNormGradArgs a, const float* sums, float* parts) {
  const int64_t c = (int64_t(blockIdx.y) * kSlabThreads + threadIdx.x) * 8;
  if (c >= a.cols) return;
  float w[8], dw[8], db[8];
  for (int i = 0; i < 8; ++i) dw[i] = db[i] = 0.0f;
  load_run(static_cast<const char*>(a.weight), c, a.cols, a.weight_type, w);
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const float mean = a.mean ? a.mean[row] : 0.0f, inv = a.inv[row], m1 = sums[row * 2], m2 = sums[row * 2 + 1];
    float d[8], t[8], more[8];
    load_run(static_cast<const char*>(a.d_out) + row * a.ld_d_out * bytes_of(a.d_out_type), c, a.cols, a.d_out_type, d);
    load_run(static_cast<const char*>(a.total) + row * a.ld_total * bytes_of(a.total_type), c, a.cols, a.total_type, t);
    for (int i = 0; i < 8; ++i) more[i] = 0.0f;
    if (a.d_total)
      load_run(static_cast<const char*>(a.d_total) + row * a.ld_d_total * bytes_of(a.d_total_type), c, a.cols, a.d_total_type,
               more);
    for (int i = 0; i < 8; ++i) {
      const float h = (t[i] - mean) * inv;
      dw[i] = __builtin_fmaf(d[i], h, dw[i]);
      db[i] += d[i];
      t[i] = __builtin_fmaf(inv, __builtin_fmaf(-h, m2, d[i] * w[i] - m1), more[i]);
    }
    store_run(static_cast<char*>(a.d_x) + row * a.ld_d_x * bytes_of(a.d_x_type), c, a.cols, a.d_x_type, t);
    if (a.d_residual)
      store_run(static_cast<char*>(a.d_residual) + row * a.ld_d_residual * bytes_of(a.d_residual_type), c, a.cols,
                a.d_residual_type, t);
  }
  if (!a.d_weight) return;
  char* to = reinterpret_cast<char*>(parts + int64_t(blockIdx.x) * a.cols);
  store_run(to, c, a.cols, WB_F32, dw);
  store_run(to + int64_t(gridDim.x) * a.cols * 4, c, a.cols, WB_F32, db);
}

// dw and db of the strips' sums: 16 lanes of four columns, 16 groups of strips.
constexpr int kColumns = 64;

__global__ __launch_bounds__(256) void wb_layer_norm_columns_kernel(LayerNormGradArgs a, const float* parts, int strips) {
  __shared__ float sums[16][kColumns];
  void* to = blockIdx.y ? a.d_bias : a.d_weight;
  if (!to) return;
  const int type = blockIdx.y ? a.d_bias_type : a.d_weight_type;
  parts += int64_t(blockIdx.y) * strips * a.cols;
  const int col = (threadIdx.x & 15) * 4, group = threadIdx.x >> 4;
  const int64_t c = int64_t(blockIdx.x) * kColumns + col;
  float sum[4] = {0, 0, 0, 0};
  for (int s = group; s < strips; s += 16) {
    const float* from = parts + int64_t(s) * a.cols + c;
    if (c + 4 <= a.cols) {
      const f32x4 v = *reinterpret_cast<const f32x4_a4*>(from);
      for (int i = 0; i < 4; ++i) sum[i] += v[i];
    } else {
      for (int i = 0; i < 4; ++i)
        if (c + i < a.cols) sum[i] += from[i];
    }
  }
  for (int i = 0; i < 4; ++i) sums[group][col + i] = sum[i];
  __syncthreads();
  const int64_t out = int64_t(blockIdx.x) * kColumns + threadIdx.x;
  if (threadIdx.x >= kColumns || out >= a.cols) return;
  float all = 0.0f;
  for (int g = 0; g < 16; ++g) all += sums[g][threadIdx.x];
  store_one(to, out, type, all);
}

int64_t strips_of(int64_t rows, int64_t cols) {
  const int64_t slabs = (cols + kSlab - 1) / kSlab;
  return std::max<int64_t>(1, std::min(rows, (2048 + slabs - 1) / slabs));
}

}  // namespace

size_t layer_norm_grad_workspace_bytes(int64_t rows, int64_t cols) {
  return static_cast<size_t>((rows * 2 + 2 * strips_of(rows, cols) * cols) * 4);
}

int launch_layer_norm(const LayerNormArgs& a, void* stream) {
  const auto st = static_cast<hipStream_t>(stream);
  if (a.rows == 0) return hipSuccess;
  const int64_t runs = (a.cols + 7) / 8;
  const auto waves = [&](int v) { return static_cast<int>((runs + 64 * v - 1) / (64 * v)); };
  if (runs <= 64) return launch<1, 4, false>(a, 1, st);
  if (runs <= 128) return launch<2, 4, false>(a, 1, st);
  if (a.rows >= kManyRows && runs <= 512) return launch<1, 1, false>(a, waves(1), st);
  if (a.rows < kManyRows && waves(2) <= kMaxWaves) return launch<2, 1, false>(a, waves(2), st);
  if (waves(4) <= kMaxWaves) return launch<4, 1, false>(a, waves(4), st);
  return launch<4, 1, true>(a, kMaxWaves, st);
}

int launch_layer_norm_grad(const LayerNormGradArgs& a, void* stream) {
  const auto st = static_cast<hipStream_t>(stream);
  float *sums = a.workspace, *parts = a.workspace + a.rows * 2;
  const int64_t strips = strips_of(a.rows, a.cols);
  if (a.rows > 0) {
    const int64_t runs = (a.cols + 7) / 8;
    const int waves = static_cast<int>(std::min<int64_t>(kMaxWaves, (runs + 63) / 64));
    hipLaunchKernelGGL(wb_layer_norm_sums_kernel, dim3(static_cast<uint32_t>(a.rows)), dim3(64 * waves), 0, st, a, sums);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(wb_layer_norm_slab_kernel,
                     dim3(static_cast<uint32_t>(strips), static_cast<uint32_t>((a.cols + kSlab - 1) / kSlab)),
                     dim3(kSlabThreads), 0, st, a, sums, parts);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !a.d_weight) return e;
  hipLaunchKernelGGL(wb_layer_norm_columns_kernel,
                     dim3(static_cast<uint32_t>((a.cols + kColumns - 1) / kColumns), a.d_bias ? 2 : 1), dim3(256), 0, st, a,
                     parts, static_cast<int>(strips));
  return hipGetLastError();
}

}  // namespace wb
