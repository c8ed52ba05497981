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

constexpr int kOneBlockRows = 64;  // up to here one launch
constexpr int kMaxBlocks = 256;    // blocks of rows: one per CU
constexpr int kGradThreads = 256, kGradBlocks = 1024;

// Threads of a workgroup whose lanes hold R logits: as many as the registers allow.
constexpr int route_threads(int r) { return r <= 16 ? 1024 : r <= 32 ? 512 : 256; }

int64_t rows_per_block(int64_t rows) {
  if (rows <= kOneBlockRows) return kOneBlockRows;
  const int64_t per = (rows + kMaxBlocks - 1) / kMaxBlocks;
  return (per + 63) / 64 * 64;
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

// The logits of a row: lane l of the sixteen holds experts l, l + 16, ...
template <int R>
__device__ __forceinline__ void load_logits(const void* base, int64_t row, int64_t ld, int type, int experts, int l,
                                            float (&z)[R]) {
  const char* at = static_cast<const char*>(base) + row * ld * (type == WB_F32 ? 4 : 2);
#pragma unroll
  for (int j = 0; j < R; ++j) z[j] = l + 16 * j < experts ? load_one(at, l + 16 * j, type) : -__builtin_inff();
}

// exp(z - top) of a row, its largest logit and one over the sum, and whether
// the row has a logit above -inf. A NaN or +inf logit makes the sum NaN.
template <int R>
__device__ __forceinline__ bool softmax_row(const float (&z)[R], float (&e)[R], float& r) {
  float top = -__builtin_inff();
#pragma unroll
  for (int j = 0; j < R; ++j) top = fmaxf(top, z[j]);
  top = reduce16(top, FMax());
  float sum = 0.0f;
#pragma unroll
  for (int j = 0; j < R; ++j) {
    e[j] = z[j] == -__builtin_inff() ? 0.0f : expf(z[j] - top);
    sum += e[j];
  }
  sum = reduce16(sum, Sum());
  r = 1.0f / sum;
  return sum != 0.0f;
}

// Choices, gates and partial sums of one block of rows.
template <int R>
__device__ void route_block(const RouteArgs& a, const Partials& part, int64_t block, int64_t per) {
  constexpr int T = route_threads(R);
  __shared__ float s_sum[T / 64][16 * R];
  __shared__ int32_t s_count[16 * R];
  __shared__ int32_t s_routed;
  const int l = threadIdx.x & 15, group = threadIdx.x >> 4;
  for (int e = threadIdx.x; e < 16 * R; e += T) s_count[e] = 0;
  if (threadIdx.x == 0) s_routed = 0;
  __syncthreads();
  float acc[R];
#pragma unroll
  for (int j = 0; j < R; ++j) acc[j] = 0.0f;
  const int64_t end = min(a.rows, (block + 1) * per);
  for (int64_t row = block * per + group; row < end; row += T / 16) {
    float z[R], e[R], r;
    load_logits<R>(a.logits, row, a.ld_logits, a.logits_type, a.num_experts, l, z);
    bool routed = softmax_row<R>(z, e, r);
    if (a.mask && !a.mask[row]) routed = false;
    if (routed) {
#pragma unroll
      for (int j = 0; j < R; ++j) acc[j] = __builtin_fmaf(e[j], r, acc[j]);
      if (l == 0) atomicAdd(&s_routed, 1);
    }
    // lane i % 16 keeps choice i and writes it with its fifteen neighbours'
    float chosen = 0.0f, gate = 0.0f;
    int expert = -1;
    for (int i = 0; i < a.k; ++i) {
      float best = -__builtin_inff();
#pragma unroll
      for (int j = 0; j < R; ++j) best = fmaxf(best, z[j]);
      best = reduce16(best, FMax());
      int at = 16 * R;
#pragma unroll
      for (int j = R - 1; j >= 0; --j) at = z[j] == best ? l + 16 * j : at;
      at = reduce16(at, IMin());
      float g = 0.0f;
#pragma unroll
      for (int j = 0; j < R; ++j)
        if (at == l + 16 * j) g = e[j], z[j] = -__builtin_inff();
      g = __shfl(g, at & 15, 16);  // from the lane that holds it
      const bool none = !routed || best == -__builtin_inff();
      if (none) at = -1, g = 0.0f;
      if (!none && l == 0) atomicAdd(&s_count[at], 1);
      chosen += g;
      if (l == (i & 15)) expert = at, gate = g * r;
      if ((i & 15) == 15 || i == a.k - 1) {
        const int first = i & ~15;
        if (l <= i - first) {
          a.experts[row * a.k + first + l] = expert;
          a.gates[row * a.k + first + l] = expert < 0 ? 0.0f : gate;
        }
      }
    }
    if (a.renormalize && routed) {
      // over the sum of the chosen instead: r is 1 / the sum of all, so the
      // quotient of both is what the gates are still to be multiplied by
      const float more = 1.0f / (chosen * r);
      for (int i = l; i < a.k; i += 16)
        if (a.experts[row * a.k + i] >= 0) a.gates[row * a.k + i] *= more;
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
  for (int e = threadIdx.x; e < a.num_experts; e += T) {
    float s = 0.0f;
    for (int w = 0; w < T / 64; ++w) s += s_sum[w][e];
    part.sums[block * a.num_experts + e] = s;
    part.counts[block * a.num_experts + e] = s_count[e];
  }
  if (threadIdx.x == 0) part.routed[block] = s_routed;
}

// Places of one block of rows; block == blocks: totals and loss.
template <int R>
__device__ void place_block(const RouteArgs& a, const Partials& part, int64_t block, int64_t blocks, int64_t per) {
  constexpr int E = 16 * R, T = route_threads(R), G = T / E > 0 ? T / E : 1, kRows = 64, kWords = kRows / 32;
  __shared__ int32_t s_part[G][E], s_before[G][E], s_total[E], s_base[E], s_wave[T / 64];
  __shared__ uint32_t s_bits[E][kWords];
  __shared__ float s_loss[T / 64];
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  // counts over all blocks, and over those before this one: G sets of threads
  // take every G-th block
  for (int e = t % E; e < E; e += T) {
    int32_t total = 0, before = 0;
    if (e < a.num_experts) {
#pragma unroll 16
      for (int64_t b = t / E; b < blocks; b += G) {
        const int32_t c = part.counts[b * a.num_experts + e];
        total += c;
        before += b < block ? c : 0;
      }
    }
    s_part[t / E % G][e] = total;
    s_before[t / E % G][e] = before;
  }
  __syncthreads();
  // exclusive prefix of the totals, T experts at a time
  int32_t all = 0;
  for (int first = 0; first < E; first += T) {
    const int e = first + t;
    int32_t total = 0, before = 0;
    if (e < E)
      for (int g = 0; g < G; ++g) total += s_part[g][e], before += s_before[g][e];
    int32_t upto = total;
    for (int off = 1; off < 64; off <<= 1) {
      const int32_t add = __shfl_up(upto, off);
      upto += lane >= off ? add : 0;
    }
    if (lane == 63) s_wave[wave] = upto;
    __syncthreads();
    int32_t at = all + upto - total;
    for (int w = 0; w < T / 64; ++w) {
      at += w < wave ? s_wave[w] : 0;
      all += s_wave[w];
    }
    if (e < E) {
      s_total[e] = total;
      s_base[e] = at + before;
      if (block == blocks && e < a.num_experts) a.offsets[e] = at, a.counts[e] = total;
    }
    __syncthreads();
  }
  if (block == blocks) {
    float loss = 0.0f;
    for (int e = t % E; e < a.num_experts; e += T) {
      float s = 0.0f;
#pragma unroll 16
      for (int64_t b = t / E; b < blocks; b += G) s += part.sums[b * a.num_experts + e];
      loss = __builtin_fmaf(s, static_cast<float>(s_total[e]), loss);
    }
    int32_t n = 0;
    for (int64_t b = t; b < blocks; b += T) n += part.routed[b];
    for (int off = 32; off > 0; off >>= 1) n += __shfl_xor(n, off);
    loss = sum_of_wave(loss);
    if (lane == 0) s_loss[wave] = loss, s_wave[wave] = n;
    __syncthreads();
    if (t == 0) {
      loss = 0.0f, n = 0;
      for (int w = 0; w < T / 64; ++w) loss += s_loss[w], n += s_wave[w];
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
    for (int i = t; i < E * kWords; i += T) s_bits[i / kWords][i % kWords] = 0;
    __syncthreads();
    const int rows = static_cast<int>(min(int64_t(kRows), end - first)), n = rows * a.k;
    for (int i = t; i < n; i += T) {
      const int32_t e = a.experts[first * a.k + i];
      const int r = i / a.k;
      if (e >= 0) atomicOr(&s_bits[e][r >> 5], 1u << (r & 31));
    }
    __syncthreads();
    for (int i = t; i < n; i += T) {
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
    for (int e = t; e < E; e += T)
      for (int w = 0; w < kWords; ++w) s_base[e] += __builtin_popcount(s_bits[e][w]);
  }
}

template <int R>
__global__ __launch_bounds__(route_threads(R)) void wb_route_kernel(RouteArgs a, int64_t blocks, int64_t per) {
  route_block<R>(a, partials(a.workspace, blocks, a.num_experts), blockIdx.x, per);
}

template <int R>
__global__ __launch_bounds__(route_threads(R)) void wb_route_place_kernel(RouteArgs a, int64_t blocks, int64_t per) {
  place_block<R>(a, partials(a.workspace, blocks, a.num_experts), blockIdx.x, blocks, per);
}

// All of it for the rows of one block.
template <int R>
__global__ __launch_bounds__(route_threads(R)) void wb_route_few_kernel(RouteArgs a, int64_t per) {
  const Partials part = partials(a.workspace, 1, a.num_experts);
  if (a.rows) {
    route_block<R>(a, part, 0, per);
  } else {
    for (int e = threadIdx.x; e < a.num_experts; e += route_threads(R)) part.sums[e] = 0.0f, part.counts[e] = 0;
    if (threadIdx.x == 0) part.routed[0] = 0;
  }
  __threadfence_block();
  __syncthreads();
  place_block<R>(a, part, 0, 1, per);
  __syncthreads();
  place_block<R>(a, part, 1, 1, per);
}

// Sixteen lanes a row. What the gates add at a row's choices goes through the
// row's copy in LDS, lane i adding choice i's (the choices are different
// experts): k times E / 16 selections between registers take longer.
template <int R>
__global__ __launch_bounds__(kGradThreads) void wb_route_grad_kernel(RouteGradArgs a) {
  constexpr int E = 16 * R, kGroups = kGradThreads / 16, kPitch = E + 1;
  __shared__ float s_row[kGroups * kPitch];
  const int l = threadIdx.x & 15, group = threadIdx.x >> 4;
  float* const mine = s_row + group * kPitch;
  const float n = static_cast<float>(*a.routed);
  const float scale = a.d_loss && n > 0.0f
                          ? *a.d_loss / n / n * (static_cast<float>(a.num_experts) / static_cast<float>(a.k))
                          : 0.0f;
  float of_loss[R];
#pragma unroll
  for (int j = 0; j < R; ++j)
    of_loss[j] = l + 16 * j < a.num_experts ? scale * static_cast<float>(a.counts[l + 16 * j]) : 0.0f;
  const int64_t stride = int64_t(gridDim.x) * kGroups;
  for (int64_t row = int64_t(blockIdx.x) * kGroups + group; row < a.rows; row += stride) {
    float z[R], p[R], d[R], r;
    load_logits<R>(a.logits, row, a.ld_logits, a.logits_type, a.num_experts, l, z);
    const bool routed = softmax_row<R>(z, p, r) && (!a.mask || a.mask[row]);
    const int32_t* experts = a.experts + row * a.k;
    const float* gates = a.gates + row * a.k;
    const float* d_gates = a.d_gates ? a.d_gates + row * a.k : nullptr;
#pragma unroll
    for (int j = 0; j < R; ++j) p[j] *= r, d[j] = of_loss[j];
    if (d_gates && !a.renormalize) {
#pragma unroll
      for (int j = 0; j < R; ++j) mine[l + 16 * j] = d[j];
      order_lanes();
      for (int i = l; i < a.k; i += 16) {
        const int e = experts[i];
        if (e >= 0) mine[e] += d_gates[i];
      }
      order_lanes();
#pragma unroll
      for (int j = 0; j < R; ++j) d[j] = mine[l + 16 * j];
    }
    float mean = 0.0f;
#pragma unroll
    for (int j = 0; j < R; ++j) mean = __builtin_fmaf(p[j], d[j], mean);
    mean = reduce16(mean, Sum());
#pragma unroll
    for (int j = 0; j < R; ++j) d[j] = p[j] * (d[j] - mean);
    if (d_gates && a.renormalize) {
#pragma unroll
      for (int j = 0; j < R; ++j) mine[l + 16 * j] = d[j];
      float dot = 0.0f;
      for (int i = l; i < a.k; i += 16) dot += experts[i] >= 0 ? gates[i] * d_gates[i] : 0.0f;
      dot = reduce16(dot, Sum());
      order_lanes();
      for (int i = l; i < a.k; i += 16) {
        const int e = experts[i];
        if (e >= 0) mine[e] += gates[i] * (d_gates[i] - dot);
      }
      order_lanes();
#pragma unroll
      for (int j = 0; j < R; ++j) d[j] = mine[l + 16 * j];
    }
    char* to = static_cast<char*>(a.d_logits) + row * a.ld_d_logits * (a.logits_type == WB_F32 ? 4 : 2);
#pragma unroll
    for (int j = 0; j < R; ++j)
      if (l + 16 * j < a.num_experts) store_one(to, l + 16 * j, a.logits_type, routed ? d[j] : 0.0f);
  }
}

// One row per workgroup in x, runs of eight columns per thread; y of the
// row's places is read once, summed in fp32 in the order of the choices. NT:
// streamed past the caches (4096 rows of 8 x 7168 bf16: 106 us against 122; at
// 256 rows 9.5 us against 7.8).
constexpr int kCombineThreads = 256;

template <bool NT>
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
      load_eight<NT>(y, c, a.y_type, v);
    else
      load_tail(y, c, a.cols, a.y_type, v);
    for (int m = 0; m < 8; ++m) sum[m] = __builtin_fmaf(g, v[m], sum[m]);
  }
  if (a.residual) {
    const char* r = static_cast<const char*>(a.residual) + row * a.ld_residual * rb;
    if (whole)
      load_eight<NT>(r, c, a.residual_type, v);
    else
      load_tail(r, c, a.cols, a.residual_type, v);
    for (int m = 0; m < 8; ++m) sum[m] += v[m];
  }
  char* out = static_cast<char*>(a.out) + row * a.ld_out * ob;
  if (whole)
    store_eight<NT>(out, c, a.out_type, sum);
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
      hipLaunchKernelGGL((wb_route_few_kernel<R>), dim3(1), dim3(route_threads(R)), 0, st, a, per);
      return hipGetLastError();
    }
    const uint32_t n = static_cast<uint32_t>(blocks);
    hipLaunchKernelGGL((wb_route_kernel<R>), dim3(n), dim3(route_threads(R)), 0, st, a, blocks, per);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((wb_route_place_kernel<R>), dim3(n + 1), dim3(route_threads(R)), 0, st, a, blocks, per);
    return hipGetLastError();
  });
}

int launch_route_grad(const RouteGradArgs& a, void* stream) {
  if (a.rows == 0) return hipSuccess;
  const auto st = static_cast<hipStream_t>(stream);
  const int64_t blocks = std::min<int64_t>((a.rows + kGradThreads / 16 - 1) / (kGradThreads / 16), kGradBlocks);
  return by_width(a.num_experts, [&](auto width) {
    hipLaunchKernelGGL((wb_route_grad_kernel<decltype(width)::value>), dim3(static_cast<uint32_t>(blocks)),
                       dim3(kGradThreads), 0, st, a);
    return hipGetLastError();
  });
}

int launch_combine(const CombineArgs& a, void* stream) {
  if (a.rows == 0) return hipSuccess;
  const int64_t per = 8 * kCombineThreads;
  const int64_t row_bytes = a.cols * (a.k * bytes_of(a.y_type) + (a.residual ? bytes_of(a.residual_type) : 0) + bytes_of(a.out_type));
  const auto kernel = a.rows * row_bytes > kStreamBytes ? wb_combine_kernel<true> : wb_combine_kernel<false>;
  hipLaunchKernelGGL(kernel, dim3(static_cast<uint32_t>(a.rows), static_cast<uint32_t>((a.cols + per - 1) / per)),
                     dim3(kCombineThreads), 0, static_cast<hipStream_t>(stream), a);
  return hipGetLastError();
}

}  // namespace wb
