// Layer norm of a residual sum, and its gradients:
//   t = x + residual, rounded to the type it is kept in;  h = (t - mean) inv,  out = h w + b
//   g = dout w;  dt = inv (g - mean(g) - h mean(g h)) + dtotal;  dw = sum_rows dout h,  db = sum_rows dout
// or without centring: mean 0, and the mean square in place of the variance.
//
// Bandwidth bound. Forward, a row is held in registers between its two sums
// (mean, then squares of what is left) and its result, as in norm.hip: 16384 x
// 4096 bf16 with a residual in 99 us, 5.4 TB/s. Back, each operand is read once
// too: rows pass through a workgroup that keeps the sums of dw and db of its
// columns in registers, the next rows' loads ahead of the work on the present
// ones, and a second launch adds the workgroups' sums: the same rows in 96 us,
// 5.6 TB/s, and 5 for the sums.
#include <algorithm>

#include "ops_device.hpp"
#include "train.hpp"

namespace wb {
namespace {

constexpr int kMaxWaves = 16;

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

// Rows that registers hold: a row lies over W wavefronts, V runs of eight columns
// to a lane, and a workgroup has G of them at a time, whose raw values come while
// the rows before are worked on. dw and db of a lane's columns stay in registers
// over the workgroup's rows.
constexpr int kGradWaves = 8;  // of a workgroup

template <int TYPE>
struct Raw;
template <>
struct Raw<WB_BF16> {
  u32x4 v;
};
template <>
struct Raw<WB_F32> {
  f32x4 v[2];
};

template <int TYPE, bool NT>
__device__ __forceinline__ void raw_load(Raw<TYPE>& to, const char* row, uint32_t c) {
  if constexpr (TYPE == WB_BF16) {
    to.v = get_u4<NT>(reinterpret_cast<const u32x4_a2*>(row + c * 2u));
  } else {
    const auto* p = reinterpret_cast<const f32x4_a4*>(row + c * 4u);
    to.v[0] = get_f4<NT>(p), to.v[1] = get_f4<NT>(p + 1);
  }
}

template <int TYPE>
__device__ __forceinline__ float raw_get(const Raw<TYPE>& r, int i) {
  if constexpr (TYPE == WB_BF16)
    return __builtin_bit_cast(float, (i & 1) ? r.v[i >> 1] & 0xffff0000u : r.v[i >> 1] << 16);
  else
    return r.v[i >> 2][i & 3];
}

// Zeros in place of the first `n` values.
template <int TYPE>
__device__ __forceinline__ void raw_clear(Raw<TYPE>& r, int n) {
  if constexpr (TYPE == WB_BF16) {
    for (int j = 0; j < 4; ++j) r.v[j] &= n > 2 * j + 1 ? 0u : n > 2 * j ? 0xffff0000u : ~0u;
  } else {
    for (int i = 0; i < 8; ++i)
      if (i < n) r.v[i >> 2][i & 3] = 0.0f;
  }
}

template <int TT, int DT, int W, int V, bool NT>
__global__ __launch_bounds__(64 * kGradWaves) void wb_layer_norm_grad_kernel(LayerNormGradArgs a, float* parts) {
  constexpr int G = kGradWaves / W;
  __shared__ float sums[2][kGradWaves][2];
  extern __shared__ float meet[];  // [2][cols], where G > 1
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), group = wave / W;
  const int lane = threadIdx.x - group * (W * 64);
  const int tb = TT == WB_F32 ? 4 : 2, db = DT == WB_F32 ? 4 : 2;
  const uint32_t cols = static_cast<uint32_t>(a.cols);
  // A lane past the row's last whole run has the row's last eight columns: those before its own, `skip` of them, are
  // another lane's. Their gradient and their weight are zero here, so that they count once, infinite or not.
  uint32_t at_col[V];
  int skip[V];
  bool partial = false;  // of the wavefront: whether a lane skips any
  float w[V][8], dw[V][8], sb[V][8];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const uint32_t c = (v * (W * 64) + lane) * 8;
    at_col[v] = min(c, cols - 8);
    skip[v] = static_cast<int>(min(c - at_col[v], 8u));
    partial = partial || __any(skip[v] > 0);
    load_eight(a.weight, at_col[v], a.weight_type, w[v]);
    for (int i = 0; i < 8; ++i) {
      if (i < skip[v]) w[v][i] = 0.0f;
      dw[v][i] = sb[v][i] = 0.0f;
    }
  }
  Raw<TT> t[V], more[V];
  Raw<DT> d[V];
#pragma unroll
  for (int v = 0; v < V; ++v) more[v] = Raw<TT>{};
  const int64_t step = int64_t(gridDim.x) * G, last = a.rows - 1;
  float mean = 0.0f, inv = 0.0f;
  const auto fetch = [&](int64_t row) {  // rows past the end read the last one again
    row = min(row, last);
    mean = a.mean ? a.mean[row] : 0.0f, inv = a.inv[row];
    const char *tr = static_cast<const char*>(a.total) + row * a.ld_total * tb, *dr = static_cast<const char*>(a.d_out) + row * a.ld_d_out * db;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      raw_load<TT, NT>(t[v], tr, at_col[v]);
      raw_load<DT, NT>(d[v], dr, at_col[v]);
    }
    if (a.d_total) {
      const char* mr = static_cast<const char*>(a.d_total) + row * a.ld_d_total * tb;
#pragma unroll
      for (int v = 0; v < V; ++v) raw_load<TT, NT>(more[v], mr, at_col[v]);
    }
  };
  const int64_t first = int64_t(blockIdx.x) * G;  // of the workgroup: every group takes as many turns
  fetch(first + group);
  const float n = static_cast<float>(a.cols);
  int turn = 0;
  for (int64_t at = first; at < a.rows; at += step, turn ^= 1) {
    const int64_t row = at + group;
    Raw<TT> tc[V], mc[V];
    Raw<DT> dc[V];
    const float mean_now = mean, inv_now = inv;
#pragma unroll
    for (int v = 0; v < V; ++v) tc[v] = t[v], mc[v] = more[v], dc[v] = d[v];
    fetch(row + step);
    if (partial) {
#pragma unroll
      for (int v = 0; v < V; ++v) raw_clear(dc[v], skip[v]);
    }
    float s1 = 0.0f, s2 = 0.0f;
    if (row < a.rows) {
#pragma unroll
      for (int v = 0; v < V; ++v) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float dv = raw_get(dc[v], i), h = (raw_get(tc[v], i) - mean_now) * inv_now, g = dv * w[v][i];
          s1 += g;
          s2 = __builtin_fmaf(g, h, s2);
          dw[v][i] = __builtin_fmaf(dv, h, dw[v][i]);
          sb[v][i] += dv;
        }
      }
    }
    s1 = sum_of_wave(s1), s2 = sum_of_wave(s2);
    if (W > 1) {
      if ((threadIdx.x & 63) == 0) sums[turn][wave][0] = s1, sums[turn][wave][1] = s2;
      __syncthreads();
      s1 = s2 = 0.0f;
#pragma unroll
      for (int i = 0; i < W; ++i) s1 += sums[turn][group * W + i][0], s2 += sums[turn][group * W + i][1];
    }
    if (row >= a.rows) continue;
    const float m1 = a.mean ? s1 / n : 0.0f, m2 = s2 / n;
    char* x_row = static_cast<char*>(a.d_x) + row * a.ld_d_x * bytes_of(a.d_x_type);
    char* r_row = static_cast<char*>(a.d_residual) + row * a.ld_d_residual * bytes_of(a.d_residual_type);
#pragma unroll
    for (int v = 0; v < V; ++v) {
      if (skip[v] == 8) continue;
      float x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float h = (raw_get(tc[v], i) - mean_now) * inv_now;
        x[i] = __builtin_fmaf(inv_now, __builtin_fmaf(-h, m2, raw_get(dc[v], i) * w[v][i] - m1), raw_get(mc[v], i));
      }
      if (skip[v] == 0) {
        store_eight<NT>(x_row, at_col[v], a.d_x_type, x);
        if (a.d_residual) store_eight<NT>(r_row, at_col[v], a.d_residual_type, x);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          if (i < skip[v]) continue;
          store_one(x_row, at_col[v] + i, a.d_x_type, x[i]);
          if (a.d_residual) store_one(r_row, at_col[v] + i, a.d_residual_type, x[i]);
        }
      }
    }
  }
  if (!a.d_weight) return;
  for (int g = 0; g < G; ++g) {
    if (g > 0) __syncthreads();
    if (group != g) continue;
#pragma unroll
    for (int v = 0; v < V; ++v) {
#pragma unroll
      for (int which = 0; which < 2; ++which) {
        float* mine = meet + which * cols + at_col[v];
        float* out = parts + (int64_t(which) * gridDim.x + blockIdx.x) * cols + at_col[v];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          if (i < skip[v]) continue;
          float sum = which ? sb[v][i] : dw[v][i];
          if (g > 0) sum += mine[i];
          if (g + 1 < G)
            mine[i] = sum;
          else
            out[i] = sum;
        }
      }
    }
  }
}

// dw and db of the strips' sums: 16 lanes of four columns, 64 groups of strips.
constexpr int kColumns = 64, kGroups = 64;

__global__ __launch_bounds__(16 * kGroups) void wb_layer_norm_columns_kernel(LayerNormGradArgs a, const float* parts, int strips) {
  __shared__ float sums[kGroups][kColumns + 4];
  void* to = blockIdx.y ? a.d_bias : a.d_weight;
  const int type = blockIdx.y ? a.d_bias_type : a.d_weight_type;
  parts += int64_t(blockIdx.y) * strips * a.cols;
  const int col = (threadIdx.x & 15) * 4, group = threadIdx.x >> 4;
  const int64_t c = int64_t(blockIdx.x) * kColumns + col;
  float sum[4] = {0, 0, 0, 0};
  if (c + 4 <= a.cols) {
#pragma unroll 4
    for (int s = group; s < strips; s += kGroups) {
      const f32x4 v = *reinterpret_cast<const f32x4_a4*>(parts + int64_t(s) * a.cols + c);
      for (int i = 0; i < 4; ++i) sum[i] += v[i];
    }
  } else {
    for (int s = group; s < strips; s += kGroups)
      for (int i = 0; i < 4; ++i)
        if (c + i < a.cols) sum[i] += parts[int64_t(s) * a.cols + c + i];
  }
  for (int i = 0; i < 4; ++i) sums[group][col + i] = sum[i];
  __syncthreads();
  if (threadIdx.x >= kColumns * 4) return;
  // four lanes a column, sixteen groups each
  const int mine = threadIdx.x >> 2, part = threadIdx.x & 3;
  float all = 0.0f;
  for (int g = 0; g < kGroups / 4; ++g) all += sums[part * (kGroups / 4) + g][mine];
  all += __shfl_xor(all, 1);
  all += __shfl_xor(all, 2);
  const int64_t out = int64_t(blockIdx.x) * kColumns + mine;
  if (part == 0 && out < a.cols) store_one(to, out, type, all);
}

// How the gradient's launch goes: strips of rows, each with its sums of dw and
// db, and wavefronts and runs a row; no wavefronts for rows that registers do
// not hold, for rows of fewer than eight columns, and for no rows at all, where the
// kernel above would have none to load.
struct GradPlan {
  int64_t strips;
  int waves, runs;
};

// One run a lane up to 2048 columns, two above (16384 x 4096 bf16, there and
// back: 191 us against 215; 1777 x 1501 on an fp32 residual: 31 against 28). A
// strip per CU: more of them have fewer rows to fetch ahead, and more sums to
// add (16384 x 4096: 219 us with 512), except narrow rows, of which two
// workgroups fit a CU (16384 x 2048: 106 us with 512, 114 with 256).
GradPlan grad_plan(int64_t rows, int64_t cols) {
  GradPlan p{};
  p.runs = cols <= 2048 ? 1 : 2;
  p.waves = 1;
  while (p.waves * 64 * 8 * p.runs < cols) p.waves *= 2;
  if (p.waves > kGradWaves || cols < 8 || rows == 0) {
    const int64_t slabs = (cols + kSlab - 1) / kSlab;
    p.waves = 0;
    p.strips = std::max<int64_t>(1, std::min(rows, (2048 + slabs - 1) / slabs));
    return p;
  }
  const int64_t groups = kGradWaves / p.waves;
  p.strips = std::min<int64_t>((rows + groups - 1) / groups, p.runs == 1 && rows >= 8192 ? 512 : 256);
  p.strips = std::max<int64_t>(1, p.strips);
  return p;
}

template <int TT, int DT, int W, int V>
hipError_t launch_grad(const LayerNormGradArgs& a, const GradPlan& p, float* parts, hipStream_t st) {
  const int64_t row_bytes = a.cols * (bytes_of(TT) * (a.d_total ? 2 : 1) + bytes_of(DT) + bytes_of(a.d_x_type) +
                                      (a.d_residual ? bytes_of(a.d_residual_type) : 0));
  const size_t lds = kGradWaves > W && a.d_weight ? a.cols * 8 : 0;
  const auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3(static_cast<uint32_t>(p.strips)), dim3(64 * kGradWaves), lds, st, a, parts);
    return hipGetLastError();
  };
  return a.rows * row_bytes > kStreamBytes ? go(wb_layer_norm_grad_kernel<TT, DT, W, V, true>)
                                           : go(wb_layer_norm_grad_kernel<TT, DT, W, V, false>);
}

template <int TT, int DT, int V>
hipError_t by_waves(const LayerNormGradArgs& a, const GradPlan& p, float* parts, hipStream_t st) {
  switch (p.waves) {
    case 1: return launch_grad<TT, DT, 1, V>(a, p, parts, st);
    case 2: return launch_grad<TT, DT, 2, V>(a, p, parts, st);
    case 4: return launch_grad<TT, DT, 4, V>(a, p, parts, st);
    default: return launch_grad<TT, DT, 8, V>(a, p, parts, st);
  }
}

template <int TT, int DT>
hipError_t by_runs(const LayerNormGradArgs& a, const GradPlan& p, float* parts, hipStream_t st) {
  return p.runs == 1 ? by_waves<TT, DT, 1>(a, p, parts, st) : by_waves<TT, DT, 2>(a, p, parts, st);
}

}  // namespace

size_t layer_norm_grad_workspace_bytes(int64_t rows, int64_t cols) {
  return static_cast<size_t>((rows * 2 + 2 * grad_plan(rows, cols).strips * cols) * 4);
}

int launch_layer_norm(const LayerNormArgs& a, void* stream) {
  const auto st = static_cast<hipStream_t>(stream);
  if (a.rows == 0) return hipSuccess;
  const int64_t runs = (a.cols + 7) / 8;
  const auto waves = [&](int v) { return static_cast<int>((runs + 64 * v - 1) / (64 * v)); };
  // Narrow rows: one wavefront each, four to a workgroup. Wider ones: two runs
  // a lane (16384 x 4096 bf16 with a residual, at least: 96 us against 115 of one, 105 of
  // four and 123 of a wavefront a row; 512 x 7168: 9.0 us against 11.0 and 10.7),
  // past sixteen wavefronts four, past those several steps.
  if (runs <= 64) return launch<1, 4, false>(a, 1, st);
  if (runs <= 128) return launch<2, 4, false>(a, 1, st);
  if (waves(2) <= kMaxWaves) return launch<2, 1, false>(a, waves(2), st);
  if (waves(4) <= kMaxWaves) return launch<4, 1, false>(a, waves(4), st);
  return launch<4, 1, true>(a, kMaxWaves, st);
}

int launch_layer_norm_grad(const LayerNormGradArgs& a, void* stream) {
  const auto st = static_cast<hipStream_t>(stream);
  float *sums = a.workspace, *parts = a.workspace + a.rows * 2;
  const GradPlan p = grad_plan(a.rows, a.cols);
  if (p.waves == 0 || (a.d_total && a.d_total_type != a.total_type)) {
    if (a.rows > 0) {
      const int64_t runs = (a.cols + 7) / 8;
      const int waves = static_cast<int>(std::min<int64_t>(kMaxWaves, (runs + 63) / 64));
      hipLaunchKernelGGL(wb_layer_norm_sums_kernel, dim3(static_cast<uint32_t>(a.rows)), dim3(64 * waves), 0, st, a, sums);
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL(wb_layer_norm_slab_kernel,
                       dim3(static_cast<uint32_t>(p.strips), static_cast<uint32_t>((a.cols + kSlab - 1) / kSlab)),
                       dim3(kSlabThreads), 0, st, a, sums, parts);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  } else {
    const bool t32 = a.total_type == WB_F32, d32 = a.d_out_type == WB_F32;
    const hipError_t e = t32 ? (d32 ? by_runs<WB_F32, WB_F32>(a, p, parts, st) : by_runs<WB_F32, WB_BF16>(a, p, parts, st))
                             : (d32 ? by_runs<WB_BF16, WB_F32>(a, p, parts, st) : by_runs<WB_BF16, WB_BF16>(a, p, parts, st));
    if (e != hipSuccess) return e;
  }
  if (!a.d_weight) return hipSuccess;
  hipLaunchKernelGGL(wb_layer_norm_columns_kernel,
                     dim3(static_cast<uint32_t>((a.cols + kColumns - 1) / kColumns), a.d_bias ? 2 : 1), dim3(16 * kGroups), 0, st,
                     a, parts, static_cast<int>(p.strips));
  return hipGetLastError();
}

}  // namespace wb
