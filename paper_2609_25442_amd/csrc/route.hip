// Routing of tokens to experts, its balance loss and the gradient of both, and
// the weighted sum that brings a token's expert rows together again.
//
//   p_t   = softmax(z_t);  the k largest z of a row are chosen, ties to the
//           lower expert; -inf is never chosen, a masked row chooses nothing
//   gates = p at the chosen, or those divided by their sum
//   loss  = E / (k n^2) * sum_e counts_e * sum_t p_te   over the n routed rows
//   dz    = p (dp - sum_e p_e dp_e),  dp_e = dloss E counts_e / (k n^2) + the
//           gates' own; normalised gates: g_i (dg_i - sum_j g_j dg_j) at the
//           chosen instead
//   out_t = residual_t + sum_i gates_ti y[positions_ti]
//
// Bandwidth bound on paper, by latency in fact: a row's logits are a few
// hundred bytes. Sixteen lanes hold a row (four rows to a wavefront), so every
// reduction is four steps inside a row of lanes, and choosing an expert costs
// two passes over E / 16 registers.
//
// Places in expert order need every row's choice first: two launches, the
// first over blocks of rows (choices, gates, and per block the counts and the
// sums of p), the second over the same blocks (places) and one more (totals
// and loss). Sums run over the blocks in their order and counts are integers,
// so results do not depend on which workgroup ran first. Few rows take one
// workgroup and one launch.
#include <algorithm>
#include <type_traits>

#include "ops_device.hpp"

namespace wb {
namespace {

constexpr int kRouteThreads = 256, kGroups = kRouteThreads / 16;
constexpr int kOneBlockRows = 64;  // up to here one launch
constexpr int kMaxBlocks = 256;    // blocks of rows: one per CU

int64_t rows_per_block(int64_t rows) {
  if (rows <= kOneBlockRows) return kOneBlockRows;
  const int64_t per = (rows + kMaxBlocks - 1) / kMaxBlocks;
  return (per + kGroups - 1) / kGroups * kGroups;
}

// Per block: its sum of p and its count of every expert, and the rows it routed.
struct Partials {
  float* sums;      // [blocks][experts]
  int32_t* counts;  // [blocks][experts]
  int32_t* routed;  // [blocks]
};

__host__ __device__ Partials partials(void* workspace, int64_t blocks, int32_t experts) {
  Partials p;
  p.sums = static_cast<float*>(workspace);
  p.counts = reinterpret_cast<int32_t*>(p.sums + blocks * experts);
  p.routed = p.counts + blocks * experts;
  return p;
}

__device__ __forceinline__ int min16(int v) {
  for (int off = 8; off > 0; off >>= 1) v = min(v, __shfl_xor(v, off, 16));
  return v;
}

__device__ __forceinline__ float sum16(float v) {
  for (int off = 8; off > 0; off >>= 1) v += __shfl_xor(v, off, 16);
  return v;
}

// The logits of a row: lane l of the sixteen holds experts l, l + 16, ...
template <int R>
__device__ __forceinline__ void load_logits(const void* base, int64_t row, int64_t ld, int type, int experts, int l,
                                            float (&z)[R]) {
  const char* at = static_cast<const char*>(base) + row * ld * (type == WB_F32 ? 4 : 2);
#pragma unroll
  for (int j = 0; j < R; ++j) z[j] = l + 16 * j < experts ? load_one(at, l + 16 * j, type) : -__builtin_inff();
}

// p of a row, its largest logit and whether it has one above -inf. A NaN or
// +inf logit makes every p of the row NaN.
template <int R>
__device__ __forceinline__ bool softmax_row(const float (&z)[R], float (&p)[R], float& top) {
  top = -__builtin_inff();
#pragma unroll
  for (int j = 0; j < R; ++j) top = fmaxf(top, z[j]);
  top = reduce16(top, FMax());
  float sum = 0.0f;
#pragma unroll
  for (int j = 0; j < R; ++j) {
    p[j] = expf(z[j] - top);
    sum += z[j] == -__builtin_inff() ? 0.0f : p[j];
  }
  sum = sum16(sum);
  const float r = 1.0f / sum;
#pragma unroll
  for (int j = 0; j < R; ++j) p[j] = z[j] == -__builtin_inff() ? (r == r ? 0.0f : r) : p[j] * r;
  return sum != 0.0f;
}

// Choices, gates and partial sums of one block of rows.
template <int R>
__device__ void route_block(const RouteArgs& a, const Partials& part, int64_t block, int64_t per) {
  __shared__ float s_sum[kRouteThreads / 64][16 * R];
  __shared__ int32_t s_count[16 * R];
  __shared__ int32_t s_routed;
  const int l = threadIdx.x & 15, group = threadIdx.x >> 4;
  for (int e = threadIdx.x; e < 16 * R; e += kRouteThreads) s_count[e] = 0;
  if (threadIdx.x == 0) s_routed = 0;
  __syncthreads();
  float acc[R];
#pragma unroll
  for (int j = 0; j < R; ++j) acc[j] = 0.0f;
  const int64_t end = min(a.rows, (block + 1) * per);
  for (int64_t row = block * per + group; row < end; row += kGroups) {
    float z[R], p[R], top;
    load_logits<R>(a.logits, row, a.ld_logits, a.logits_type, a.num_experts, l, z);
    bool routed = softmax_row<R>(z, p, top);
    if (a.mask && !a.mask[row]) routed = false;
    if (routed) {
#pragma unroll
      for (int j = 0; j < R; ++j) acc[j] += p[j];
      if (l == 0) atomicAdd(&s_routed, 1);
    }
    float chosen_sum = 0.0f, gate = 0.0f;
    int expert = -1;
    // lane i % 16 keeps choice i and writes it with its fifteen neighbours'
    for (int i = 0; i < a.k; ++i) {
      float best = -__builtin_inff();
#pragma unroll
      for (int j = 0; j < R; ++j) best = fmaxf(best, z[j]);
      best = reduce16(best, FMax());
      int at = 16 * R;
#pragma unroll
      for (int j = R - 1; j >= 0; --j) at = z[j] == best ? l + 16 * j : at;
      at = min16(at);
      float g = -1.0f;
#pragma unroll
      for (int j = 0; j < R; ++j)
        if (at == l + 16 * j) g = p[j], z[j] = -__builtin_inff();
      const bool none = !routed || best == -__builtin_inff();
      // p of the chosen, from the lane that holds it
      g = __shfl(g, at & 15, 16);
      if (none) at = -1, g = 0.0f;
      if (!none && l == 0) atomicAdd(&s_count[at], 1);
      chosen_sum += a.renormalize && !none ? expf(best - top) : 0.0f;
      if (l == (i & 15)) expert = at, gate = a.renormalize && !none ? (g == g ? expf(best - top) : g) : g;
      if ((i & 15) == 15 || i == a.k - 1) {
        const int first = i & ~15;
        if (l <= i - first) {
          a.experts[row * a.k + first + l] = expert;
          a.gates[row * a.k + first + l] = gate;
        }
      }
    }
    if (a.renormalize && routed) {
      const float r = 1.0f / chosen_sum;
      for (int i = l; i < a.k; i += 16) a.gates[row * a.k + i] *= r;
    }
  }
  // four rows of a wavefront, then the wavefronts in order
  const int wave = threadIdx.x >> 6;
#pragma unroll
  for (int j = 0; j < R; ++j) {
    acc[j] += __shfl_xor(acc[j], 16);
    acc[j] += __shfl_xor(acc[j], 32);
    if ((threadIdx.x & 63) < 16) s_sum[wave][l + 16 * j] = acc[j];
  }
  __syncthreads();
  for (int e = threadIdx.x; e < a.num_experts; e += kRouteThreads) {
    float s = 0.0f;
    for (int w = 0; w < kRouteThreads / 64; ++w) s += s_sum[w][e];
    part.sums[block * a.num_experts + e] = s;
    part.counts[block * a.num_experts + e] = s_count[e];
  }
  if (threadIdx.x == 0) part.routed[block] = s_routed;
}

// Places of one block of rows; block == blocks: totals and loss.
template <int R>
__device__ void place_block(const RouteArgs& a, const Partials& part, int64_t block, int64_t blocks, int64_t per) {
  constexpr int E = 16 * R, kRows = 64, kWords = kRows / 32;
  __shared__ int32_t s_total[E], s_base[E], s_scan[kRouteThreads];
  __shared__ uint32_t s_bits[E][kWords];
  __shared__ float s_loss[kRouteThreads / 64];
  const int t = threadIdx.x;
  // counts over all blocks, and over those before this one
  for (int e = t; e < E; e += kRouteThreads) {
    int32_t total = 0, before = 0;
    if (e < a.num_experts) {
#pragma unroll 8
      for (int64_t b = 0; b < blocks; ++b) {
        const int32_t c = part.counts[b * a.num_experts + e];
        total += c;
        before += b < block ? c : 0;
      }
    }
    s_total[e] = total;
    s_base[e] = before;
  }
  __syncthreads();
  // exclusive prefix of the totals: each thread sums a run, then a scan of the threads
  constexpr int kRun = (E + kRouteThreads - 1) / kRouteThreads;
  int32_t run = 0;
  for (int i = 0; i < kRun; ++i) run += t * kRun + i < E ? s_total[t * kRun + i] : 0;
  s_scan[t] = run;
  __syncthreads();
  for (int off = 1; off < kRouteThreads; off <<= 1) {
    const int32_t add = t >= off ? s_scan[t - off] : 0;
    __syncthreads();
    s_scan[t] += add;
    __syncthreads();
  }
  const int32_t all = s_scan[kRouteThreads - 1];
  int32_t at = s_scan[t] - run;
  for (int i = 0; i < kRun && t * kRun + i < E; ++i) {
    const int e = t * kRun + i;
    s_base[e] += at;
    if (block == blocks && e < a.num_experts) a.offsets[e] = at;
    at += s_total[e];
  }
  if (block == blocks) {
    int32_t n = 0;
    for (int64_t b = 0; b < blocks; ++b) n += part.routed[b];
    float loss = 0.0f;
    for (int e = t; e < a.num_experts; e += kRouteThreads) {
      float s = 0.0f;
#pragma unroll 8
      for (int64_t b = 0; b < blocks; ++b) s += part.sums[b * a.num_experts + e];
      loss += s * static_cast<float>(s_total[e]);
      a.counts[e] = s_total[e];
    }
    loss = sum_of_wave(loss);
    if ((t & 63) == 0) s_loss[t >> 6] = loss;
    __syncthreads();
    if (t == 0) {
      loss = 0.0f;
      for (int w = 0; w < kRouteThreads / 64; ++w) loss += s_loss[w];
      const float rows = static_cast<float>(n);
      *a.loss = n ? loss / rows / rows * (static_cast<float>(a.num_experts) / static_cast<float>(a.k)) : 0.0f;
      *a.routed = n;
      a.offsets[a.num_experts] = all;
    }
    return;
  }
  // rows by sixty-four: a bit per row and expert, a place is the bits before it
  const int64_t end = min(a.rows, (block + 1) * per);
  for (int64_t first = block * per; first < end; first += kRows) {
    __syncthreads();
    for (int i = t; i < E * kWords; i += kRouteThreads) s_bits[i / kWords][i % kWords] = 0;
    __syncthreads();
    const int rows = static_cast<int>(min(int64_t(kRows), end - first)), n = rows * a.k;
    for (int i = t; i < n; i += kRouteThreads) {
      const int32_t e = a.experts[first * a.k + i];
      const int r = i / a.k;
      if (e >= 0) atomicOr(&s_bits[e][r >> 5], 1u << (r & 31));
    }
    __syncthreads();
    for (int i = t; i < n; i += kRouteThreads) {
      const int32_t e = a.experts[first * a.k + i];
      const int r = i / a.k;
      int32_t place = -1;
      if (e >= 0) {
        place = s_base[e];
        for (int w = 0; w < kWords; ++w) {
          const uint32_t before = w < (r >> 5) ? ~0u : w == (r >> 5) ? (1u << (r & 31)) - 1u : 0u;
          place += __builtin_popcount(s_bits[e][w] & before);
        }
        a.tokens[place] = static_cast<int32_t>(first + r);
      }
      a.positions[first * a.k + i] = place;
      if (first * a.k + i >= all) a.tokens[first * a.k + i] = -1;
    }
    __syncthreads();
    for (int e = t; e < E; e += kRouteThreads)
      for (int w = 0; w < kWords; ++w) s_base[e] += __builtin_popcount(s_bits[e][w]);
  }
}

template <int R>
__global__ __launch_bounds__(kRouteThreads) void wb_route_kernel(RouteArgs a, int64_t blocks, int64_t per) {
  route_block<R>(a, partials(a.workspace, blocks, a.num_experts), blockIdx.x, per);
}

template <int R>
__global__ __launch_bounds__(kRouteThreads) void wb_route_place_kernel(RouteArgs a, int64_t blocks, int64_t per) {
  place_block<R>(a, partials(a.workspace, blocks, a.num_experts), blockIdx.x, blocks, per);
}

// All of it for the rows of one block.
template <int R>
__global__ __launch_bounds__(kRouteThreads) void wb_route_few_kernel(RouteArgs a, int64_t per) {
  const Partials part = partials(a.workspace, 1, a.num_experts);
  if (a.rows) {
    route_block<R>(a, part, 0, per);
  } else {
    for (int e = threadIdx.x; e < a.num_experts; e += kRouteThreads) part.sums[e] = 0.0f, part.counts[e] = 0;
    if (threadIdx.x == 0) part.routed[0] = 0;
  }
  __threadfence_block();
  __syncthreads();
  place_block<R>(a, part, 0, 1, per);
  __syncthreads();
  place_block<R>(a, part, 1, 1, per);
}

template <int R>
__global__ __launch_bounds__(kRouteThreads) void wb_route_grad_kernel(RouteGradArgs a) {
  const int l = threadIdx.x & 15;
  const float n = static_cast<float>(*a.routed);
  const float scale = a.d_loss && n > 0.0f
                          ? *a.d_loss / n / n * (static_cast<float>(a.num_experts) / static_cast<float>(a.k))
                          : 0.0f;
  float of_loss[R];
#pragma unroll
  for (int j = 0; j < R; ++j)
    of_loss[j] = l + 16 * j < a.num_experts ? scale * static_cast<float>(a.counts[l + 16 * j]) : 0.0f;
  const int64_t stride = int64_t(gridDim.x) * kGroups;
  for (int64_t row = int64_t(blockIdx.x) * kGroups + (threadIdx.x >> 4); row < a.rows; row += stride) {
    float z[R], p[R], d[R], top;
    load_logits<R>(a.logits, row, a.ld_logits, a.logits_type, a.num_experts, l, z);
    const bool routed = softmax_row<R>(z, p, top) && (!a.mask || a.mask[row]);
    const int32_t* experts = a.experts + row * a.k;
    const float* gates = a.gates + row * a.k;
    const float* d_gates = a.d_gates ? a.d_gates + row * a.k : nullptr;
    float mean = 0.0f;
#pragma unroll
    for (int j = 0; j < R; ++j) d[j] = of_loss[j];
    if (d_gates && !a.renormalize)
      for (int i = 0; i < a.k; ++i) {
        const int e = experts[i];
        const float g = d_gates[i];
#pragma unroll
        for (int j = 0; j < R; ++j) d[j] += e == l + 16 * j ? g : 0.0f;
      }
#pragma unroll
    for (int j = 0; j < R; ++j) mean += p[j] * d[j];
    mean = sum16(mean);
#pragma unroll
    for (int j = 0; j < R; ++j) d[j] = p[j] * (d[j] - mean);
    if (d_gates && a.renormalize) {
      float dot = 0.0f;
      for (int i = 0; i < a.k; ++i) dot += experts[i] >= 0 ? gates[i] * d_gates[i] : 0.0f;
      for (int i = 0; i < a.k; ++i) {
        const int e = experts[i];
        const float g = gates[i] * (d_gates[i] - dot);
#pragma unroll
        for (int j = 0; j < R; ++j) d[j] += e == l + 16 * j ? g : 0.0f;
      }
    }
    char* to = static_cast<char*>(a.d_logits) + row * a.ld_d_logits * (a.logits_type == WB_F32 ? 4 : 2);
#pragma unroll
    for (int j = 0; j < R; ++j)
      if (l + 16 * j < a.num_experts) store_one(to, l + 16 * j, a.logits_type, routed ? d[j] : 0.0f);
  }
}

// One row per workgroup in x, runs of eight columns per thread; y of the
// row's places is read once, summed in fp32 in the order of the choices.
constexpr int kCombineThreads = 256;

__global__ __launch_bounds__(kCombineThreads) void wb_combine_kernel(CombineArgs a) {
  const int64_t row = blockIdx.x;
  const int64_t c = (int64_t(blockIdx.y) * kCombineThreads + threadIdx.x) * 8;
  if (c >= a.cols) return;
  const bool whole = c + 8 <= a.cols;
  const int32_t first = a.first ? max(0, *a.first) : 0;
  const int64_t last = a.last ? min(a.y_rows, int64_t(*a.last)) : a.y_rows;
  const int yb = a.y_type == WB_F32 ? 4 : 2, rb = a.residual_type == WB_F32 ? 4 : 2, ob = a.out_type == WB_F32 ? 4 : 2;
  float sum[8], v[8];
  for (int i = 0; i < 8; ++i) sum[i] = 0.0f;
  for (int i = 0; i < a.k; ++i) {
    const int32_t at = a.positions[row * a.k + i];
    if (at < first || at >= last) continue;
    const float g = a.gates[row * a.k + i];
    const char* y = static_cast<const char*>(a.y) + at * a.ld_y * yb;
    if (whole)
      load_eight(y, c, a.y_type, v);
    else
      load_tail(y, c, a.cols, a.y_type, v);
    for (int m = 0; m < 8; ++m) sum[m] = __builtin_fmaf(g, v[m], sum[m]);
  }
  if (a.residual) {
    const char* r = static_cast<const char*>(a.residual) + row * a.ld_residual * rb;
    if (whole)
      load_eight(r, c, a.residual_type, v);
    else
      load_tail(r, c, a.cols, a.residual_type, v);
    for (int m = 0; m < 8; ++m) sum[m] += v[m];
  }
  char* out = static_cast<char*>(a.out) + row * a.ld_out * ob;
  if (whole)
    store_eight(out, c, a.out_type, sum);
  else
    store_tail(out, c, a.cols, a.out_type, sum);
}

// Registers per lane for a row of E experts.
template <class F>
hipError_t by_width(int experts, F&& f) {
  const int r = (experts + 15) / 16;
  if (r <= 1) return f(std::integral_constant<int, 1>());
  if (r <= 4) return f(std::integral_constant<int, 4>());
  if (r <= 8) return f(std::integral_constant<int, 8>());
  if (r <= 16) return f(std::integral_constant<int, 16>());
  if (r <= 32) return f(std::integral_constant<int, 32>());
  return f(std::integral_constant<int, 64>());
}

}  // namespace

size_t route_workspace_bytes(int64_t rows, int32_t experts) {
  const int64_t per = rows_per_block(rows), blocks = rows <= per ? 1 : (rows + per - 1) / per;
  return static_cast<size_t>(blocks) * (8 * size_t(experts) + 4);
}

int launch_route(const RouteArgs& a, void* stream) {
  const auto st = static_cast<hipStream_t>(stream);
  const int64_t per = rows_per_block(a.rows), blocks = (a.rows + per - 1) / per;
  return by_width(a.num_experts, [&](auto width) {
    constexpr int R = decltype(width)::value;
    if (blocks <= 1) {
      hipLaunchKernelGGL((wb_route_few_kernel<R>), dim3(1), dim3(kRouteThreads), 0, st, a, per);
      return hipGetLastError();
    }
    const uint32_t n = static_cast<uint32_t>(blocks);
    hipLaunchKernelGGL((wb_route_kernel<R>), dim3(n), dim3(kRouteThreads), 0, st, a, blocks, per);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((wb_route_place_kernel<R>), dim3(n + 1), dim3(kRouteThreads), 0, st, a, blocks, per);
    return hipGetLastError();
  });
}

int launch_route_grad(const RouteGradArgs& a, void* stream) {
  if (a.rows == 0) return hipSuccess;
  const auto st = static_cast<hipStream_t>(stream);
  const int64_t blocks = std::min<int64_t>((a.rows + kGroups - 1) / kGroups, 2048);
  return by_width(a.num_experts, [&](auto width) {
    hipLaunchKernelGGL((wb_route_grad_kernel<decltype(width)::value>), dim3(static_cast<uint32_t>(blocks)),
                       dim3(kRouteThreads), 0, st, a);
    return hipGetLastError();
  });
}

int launch_combine(const CombineArgs& a, void* stream) {
  if (a.rows == 0) return hipSuccess;
  const int64_t per = 8 * kCombineThreads;
  hipLaunchKernelGGL(wb_combine_kernel, dim3(static_cast<uint32_t>(a.rows), static_cast<uint32_t>((a.cols + per - 1) / per)),
                     dim3(kCombineThreads), 0, static_cast<hipStream_t>(stream), a);
  return hipGetLastError();
}

}  // namespace wb
