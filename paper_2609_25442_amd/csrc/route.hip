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
// The bytes are few; choosing is what takes time, k times a row's largest and
// its place. Eight lanes hold a row (sixteen past 256 experts), so that the
// steps of a reduction serve eight rows at once. Measured with 32768 x 256
// fp32 logits, k = 8: choices 23 us (27 with a pass over every lane's registers
// for each choice, 29 with sixteen lanes a row), places 14 (every block sums the
// counts of all), gradient 19 (the 67 MB that it moves take 10; a group of lanes
// loads its row and then works on it); 35 us the forward calls, 54 with the
// gradient. Gates and p are quotients with the exponential's remainder kept, as
// exact as elementary operations in fp32; reciprocals made it 52 us and the
// gates' error 1.1 to 1.3 times theirs.
//
// Places in expert order need every row's choice first: two launches, the
// first over blocks of rows (choices, gates, and per block the counts and the
// sums of p), the second over the same blocks (places) and one more (totals
// and loss). Sums are taken in a fixed order and counts are integers,
// so results do not depend on which workgroup ran first. Few rows take one
// workgroup and one launch.
#include <algorithm>
#include <type_traits>

#include "ops_device.hpp"

namespace wb {
namespace {

// A lane's neighbour within eight.
template <int CTRL, class V>
__device__ __forceinline__ V lanes8(V v) {
  const int i = __builtin_bit_cast(int, v);
  return __builtin_bit_cast(V, __builtin_amdgcn_update_dpp(i, i, CTRL, 0xf, 0xf, false));
}

constexpr int kOneBlockRows = 64;  // up to here one launch
constexpr int kMaxBlocks = 256;    // blocks of rows: one per CU
constexpr int kGradThreads = 256, kGradBlocks = 1024, kPlaceThreads = 1024;

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
typedef i32x4 i32x4_a4 __attribute__((aligned(4)));

// Rows lie over L lanes with R registers each: lane l holds experts 4 l, ...,
// 4 l + 3 of every 4 L, or l of every L where R is 1. T: threads of a
// workgroup, as many as the registers allow.
template <int L_, int R_>
struct Row {
  static constexpr int L = L_, R = R_, E = L * R, T = R <= 8 ? 1024 : R <= 32 ? 512 : 256;
  __device__ static int expert(int l, int j) { return R == 1 ? l : (j >> 2) * (4 * L) + 4 * l + (j & 3); }
  // and back
  __device__ static int lane(int e) { return R == 1 ? e % L : e / 4 % L; }
  __device__ static int place(int e) { return R == 1 ? 0 : e / (4 * L) % (R / 4 > 0 ? R / 4 : 1) * 4 + e % 4; }
  template <class V, class Op>
  __device__ __forceinline__ static V reduce(V v, Op op) {
    if constexpr (L == 16) {
      return reduce16(v, op);
    } else {
      v = op(v, lanes8<0xB1>(v));    // pairs
      v = op(v, lanes8<0x4E>(v));    // fours
      return op(v, lanes8<0x141>(v));  // eights, mirrored
    }
  }
};

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

template <class W>
__device__ __forceinline__ void load_logits(const void* base, int64_t row, int64_t ld, int type, int experts, int l,
                                            float (&z)[W::R]) {
  const char* at = static_cast<const char*>(base) + row * ld * (type == WB_F32 ? 4 : 2);
  if constexpr (W::R == 1) {
    z[0] = l < experts ? load_one(at, l, type) : -__builtin_inff();
  } else {
#pragma unroll
    for (int j = 0; j < W::R; j += 4) {
      const int e = W::expert(l, j);
      float v[4];
      if (e + 4 <= experts) {
        load_four(at, e, type, v);
      } else {
        for (int i = 0; i < 4; ++i) v[i] = e + i < experts ? load_one(at, e + i, type) : -__builtin_inff();
      }
      for (int i = 0; i < 4; ++i) z[j + i] = v[i];
    }
  }
}

// The sum of a lane's registers, by halves: as many roundings on the way of
// each as there are halvings.
template <int N>
__device__ __forceinline__ float sum_of(const float* v) {
  if constexpr (N == 1)
    return v[0];
  else
    return sum_of<N / 2>(v) + sum_of<N / 2>(v + N / 2);
}

// exp(z - top) of a row, their sum, one over it, and whether the row has a
// logit above -inf. A NaN or +inf logit makes the sum NaN.
template <class W>
__device__ __forceinline__ bool softmax_row(const float (&z)[W::R], float (&e)[W::R], float& sum, float& r, float& top) {
  top = -__builtin_inff();
#pragma unroll
  for (int j = 0; j < W::R; ++j) top = fmaxf(top, z[j]);
  top = W::reduce(top, FMax());
  if (top == -__builtin_inff()) top = 0.0f;
#pragma unroll
  for (int j = 0; j < W::R; ++j) e[j] = exp_below(z[j] - top);
  sum = W::reduce(sum_of<W::R>(e), Sum());
  r = 1.0f / sum;
  return sum != 0.0f;
}

// Choices, gates and partial sums of one block of rows.
template <class W>
__device__ void route_block(const RouteArgs& a, const Partials& part, int64_t block, int64_t per) {
  constexpr int T = W::T, R = W::R, L = W::L;
  __shared__ float s_sum[T / 64][W::E];
  __shared__ int32_t s_count[W::E];
  __shared__ int32_t s_routed;
  constexpr bool kShared = R >= 2 * L;
  constexpr int kPitch = R + 1;  // of a lane's logits
  __shared__ float s_row[kShared ? T / L * L * kPitch : 1];
  __shared__ float s_gate[T / L][kMaxRouteK + 1];  // a row's, until their sum is known
  __shared__ int32_t s_expert[T / L][kMaxRouteK + 1];
  const int l = threadIdx.x % L, group = threadIdx.x / L;
  for (int e = threadIdx.x; e < W::E; e += T) s_count[e] = 0;
  if (threadIdx.x == 0) s_routed = 0;
  __syncthreads();
  float acc[R];
#pragma unroll
  for (int j = 0; j < R; ++j) acc[j] = 0.0f;
  const int64_t end = min(a.rows, (block + 1) * per);
  for (int64_t row = block * per + group; row < end; row += T / L) {
    float z[R], e[R], sum, r, top;
    const bool masked = a.mask && !a.mask[row];
    load_logits<W>(a.logits, row, a.ld_logits, a.logits_type, a.num_experts, l, z);
    const bool routed = softmax_row<W>(z, e, sum, r, top) && !masked;
    if (routed) {
#pragma unroll
      for (int j = 0; j < R; ++j) acc[j] = __builtin_fmaf(e[j], r, acc[j]);
      if (l == 0) atomicAdd(&s_routed, 1);
    }
    // Every lane knows its largest; a choice asks for the row's, and only the
    // lane that had it needs its next, which all the lanes of the row look for
    // in the row's copy in LDS: a third of the instructions of a pass over
    // every lane's registers, where those are many.
    float lane_best = -__builtin_inff();
    int lane_at = W::E;
    float* const mine = s_row + group * (L * kPitch);
    if constexpr (kShared) {
      order_lanes();
#pragma unroll
      for (int j = 0; j < R; ++j) lane_best = fmaxf(lane_best, z[j]), mine[l * kPitch + j] = z[j];
#pragma unroll
      for (int j = R - 1; j >= 0; --j) lane_at = z[j] == lane_best ? W::expert(l, j) : lane_at;
    }
    for (int i = 0; i < a.k; ++i) {
      float best;
      int at;
      if constexpr (kShared) {
        best = W::reduce(lane_best, FMax());
        at = W::reduce(lane_best == best ? lane_at : W::E, IMin());
        // its lane's next, looked for by all the lanes of the row
        const int from = W::lane(at), here = l * (R / L);
        order_lanes();
        if (l == 0) mine[from * kPitch + W::place(at)] = -__builtin_inff();
        order_lanes();
        float v[R / L], most = -__builtin_inff();
#pragma unroll
        for (int j = 0; j < R / L; ++j) v[j] = mine[from * kPitch + here + j], most = fmaxf(most, v[j]);
        most = W::reduce(most, FMax());
        int next = R;
#pragma unroll
        for (int j = R / L - 1; j >= 0; --j) next = v[j] == most ? here + j : next;
        next = W::reduce(next, IMin());
        if (l == from) lane_best = most, lane_at = W::expert(l, next < R ? next : 0);
      } else {
        best = -__builtin_inff();
#pragma unroll
        for (int j = 0; j < R; ++j) best = fmaxf(best, z[j]);
        best = W::reduce(best, FMax());
        at = W::E;
#pragma unroll
        for (int j = R - 1; j >= 0; --j) at = z[j] == best ? W::expert(l, j) : at;
        at = W::reduce(at, IMin());
#pragma unroll
        for (int j = 0; j < R; ++j) z[j] = at == W::expert(l, j) ? -__builtin_inff() : z[j];
      }
      float g = exp_below(best - top) + (r - r);  // NaN where the row's sum is
      const bool none = !routed || best == -__builtin_inff();
      if (none) at = -1, g = 0.0f;
      if (l == 0) {
        s_gate[group][i] = g;
        s_expert[group][i] = at;
        if (!none) atomicAdd(&s_count[at], 1);
      }
    }
    order_lanes();
    // over the sum of the chosen, or of all
    float over = 0.0f;
    for (int i = l; i < a.k; i += L) over += s_gate[group][i];
    over = W::reduce(over, Sum());
    if (!a.renormalize) over = sum;
    for (int i = l; i < a.k; i += L) {
      const int at = s_expert[group][i];
      a.experts[row * a.k + i] = at;
      a.gates[row * a.k + i] = at < 0 ? 0.0f : s_gate[group][i] / over;
    }
    order_lanes();
  }
  // the rows of a wavefront, then the wavefronts in order
  const int wave = threadIdx.x >> 6;
#pragma unroll
  for (int j = 0; j < R; ++j) {
#pragma unroll
    for (int off = L; off < 64; off <<= 1) acc[j] += __shfl_xor(acc[j], off);
    if ((threadIdx.x & 63) < L) s_sum[wave][W::expert(l, j)] = acc[j];
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
template <class W, int T>
__device__ void place_block(const RouteArgs& a, const Partials& part, int64_t block, int64_t blocks, int64_t per) {
  constexpr int E = W::E, Q = E / 4, G = T / Q < 16 ? T / Q : 16, kRows = 64, kWords = kRows / 32;
  static_assert(G >= 1, "a thread for every four experts");
  __shared__ int32_t s_part[G][E], s_before[G][E], s_total[E], s_base[E], s_wave[T / 64];
  __shared__ uint32_t s_bits[E][kWords];
  __shared__ float s_loss[T / 64];
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  // counts over all blocks, and over those before this one: G sets of threads
  // take every G-th block, a thread four experts
  if (t < Q * G) {
    const int e = t % Q * 4, in = a.num_experts - e;
    i32x4 total = {0, 0, 0, 0}, before = {0, 0, 0, 0};
    if (in >= 4) {
#pragma unroll 8
      for (int64_t b = t / Q; b < blocks; b += G) {
        const i32x4 c = *reinterpret_cast<const i32x4_a4*>(part.counts + b * a.num_experts + e);
        total += c;
        before += b < block ? c : i32x4{0, 0, 0, 0};
      }
    } else {
      for (int64_t b = t / Q; b < blocks; b += G)
        for (int i = 0; i < 4; ++i) {
          const int32_t c = i < in ? part.counts[b * a.num_experts + e + i] : 0;
          total[i] += c;
          before[i] += b < block ? c : 0;
        }
    }
    for (int i = 0; i < 4; ++i) s_part[t / Q][e + i] = total[i], s_before[t / Q][e + i] = before[i];
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
    if (t < Q * G) {
      const int e = t % Q * 4, in = min(4, a.num_experts - e);
      float sum[4] = {0, 0, 0, 0};
      if (in == 4) {
#pragma unroll 8
        for (int64_t b = t / Q; b < blocks; b += G) {
          const f32x4 p = *reinterpret_cast<const f32x4_a4*>(part.sums + b * a.num_experts + e);
          for (int i = 0; i < 4; ++i) sum[i] += p[i];
        }
      } else {
        for (int64_t b = t / Q; b < blocks; b += G)
          for (int i = 0; i < in; ++i) sum[i] += part.sums[b * a.num_experts + e + i];
      }
      for (int i = 0; i < in; ++i) loss = __builtin_fmaf(sum[i], static_cast<float>(s_total[e + i]), loss);
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

template <class W>
__global__ __launch_bounds__(W::T) void wb_route_kernel(RouteArgs a, int64_t blocks, int64_t per) {
  route_block<W>(a, partials(a.workspace, blocks, a.num_experts), blockIdx.x, per);
}

template <class W>
__global__ __launch_bounds__(kPlaceThreads) void wb_route_place_kernel(RouteArgs a, int64_t blocks, int64_t per) {
  place_block<W, kPlaceThreads>(a, partials(a.workspace, blocks, a.num_experts), blockIdx.x, blocks, per);
}

// All of it for the rows of one block.
template <class W>
__global__ __launch_bounds__(W::T) void wb_route_few_kernel(RouteArgs a, int64_t per) {
  const Partials part = partials(a.workspace, 1, a.num_experts);
  if (a.rows) {
    route_block<W>(a, part, 0, per);
  } else {
    for (int e = threadIdx.x; e < a.num_experts; e += W::T) part.sums[e] = 0.0f, part.counts[e] = 0;
    if (threadIdx.x == 0) part.routed[0] = 0;
  }
  __threadfence_block();
  __syncthreads();
  place_block<W, W::T>(a, part, 0, 1, per);
  __syncthreads();
  place_block<W, W::T>(a, part, 1, 1, per);
}

// What the gates add at a row's choices goes through the
// row's copy in LDS, lane i adding choice i's (the choices are different
// experts): k times R selections between registers take longer. A choice that
// is no expert's number is none, as -1 is: it has no place in the copy.
template <class W>
__global__ __launch_bounds__(kGradThreads) void wb_route_grad_kernel(RouteGradArgs a) {
  constexpr int R = W::R, L = W::L, kGroups = kGradThreads / L, kPitch = W::E + 1;
  __shared__ float s_row[kGroups * kPitch];
  const int l = threadIdx.x % L, group = threadIdx.x / L;
  float* const mine = s_row + group * kPitch;
  const float n = static_cast<float>(*a.routed);
  const float scale = a.d_loss && n > 0.0f
                          ? *a.d_loss / n / n * (static_cast<float>(a.num_experts) / static_cast<float>(a.k))
                          : 0.0f;
  float of_loss[R];
#pragma unroll
  for (int j = 0; j < R; ++j)
    of_loss[j] = W::expert(l, j) < a.num_experts ? scale * static_cast<float>(a.counts[W::expert(l, j)]) : 0.0f;
  const int64_t stride = int64_t(gridDim.x) * kGroups;
  for (int64_t row = int64_t(blockIdx.x) * kGroups + group; row < a.rows; row += stride) {
    float z[R], p[R], d[R], sum, r, top;
    // the lane's first choice, on its way with the logits
    struct {
      int32_t expert;
      float gate, d;
    } first = {-1, 0.0f, 0.0f};
    auto there = [&](int32_t e) { return static_cast<uint32_t>(e) < static_cast<uint32_t>(a.num_experts); };
    if (a.d_gates && l < a.k) first = {a.experts[row * a.k + l], a.gates[row * a.k + l], a.d_gates[row * a.k + l]};
    const bool masked = a.mask && !a.mask[row];
    load_logits<W>(a.logits, row, a.ld_logits, a.logits_type, a.num_experts, l, z);
    const bool routed = softmax_row<W>(z, p, sum, r, top) && !masked;
    const int32_t* experts = a.experts + row * a.k;
    const float* gates = a.gates + row * a.k;
    const float* d_gates = a.d_gates ? a.d_gates + row * a.k : nullptr;
#pragma unroll
    for (int j = 0; j < R; ++j) {
      const float q = p[j] * r;  // p / sum: the product, its remainder, one correction
      p[j] = __builtin_fmaf(__builtin_fmaf(-q, sum, p[j]), r, q);
      d[j] = of_loss[j];
    }
    if (d_gates && !a.renormalize) {
#pragma unroll
      for (int j = 0; j < R; ++j) mine[W::expert(l, j)] = d[j];
      order_lanes();
      if (there(first.expert)) mine[first.expert] += first.d;
      for (int i = l + L; i < a.k; i += L)
        if (there(experts[i])) mine[experts[i]] += d_gates[i];
      order_lanes();
#pragma unroll
      for (int j = 0; j < R; ++j) d[j] = mine[W::expert(l, j)];
    }
    float mean[4] = {0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < R; ++j) mean[j & 3] = __builtin_fmaf(p[j], d[j], mean[j & 3]);
    const float of_all = W::reduce(sum_of<4>(mean), Sum());
#pragma unroll
    for (int j = 0; j < R; ++j) d[j] = p[j] * (d[j] - of_all);
    if (d_gates && a.renormalize) {
#pragma unroll
      for (int j = 0; j < R; ++j) mine[W::expert(l, j)] = d[j];
      float dot = there(first.expert) ? first.gate * first.d : 0.0f;
      for (int i = l + L; i < a.k; i += L) dot += there(experts[i]) ? gates[i] * d_gates[i] : 0.0f;
      dot = W::reduce(dot, Sum());
      order_lanes();
      if (there(first.expert)) mine[first.expert] += first.gate * (first.d - dot);
      for (int i = l + L; i < a.k; i += L)
        if (there(experts[i])) mine[experts[i]] += gates[i] * (d_gates[i] - dot);
      order_lanes();
#pragma unroll
      for (int j = 0; j < R; ++j) d[j] = mine[W::expert(l, j)];
    }
    char* to = static_cast<char*>(a.d_logits) + row * a.ld_d_logits * (a.logits_type == WB_F32 ? 4 : 2);
    if constexpr (R == 1) {
      if (l < a.num_experts) store_one(to, l, a.logits_type, routed ? d[0] : 0.0f);
    } else {
#pragma unroll
      for (int j = 0; j < R; j += 4) {
        const int e = W::expert(l, j);
        float v[4];
        for (int i = 0; i < 4; ++i) v[i] = routed ? d[j + i] : 0.0f;
        if (e + 4 <= a.num_experts) {
          store_four(to, e, a.logits_type, v);
        } else {
          for (int i = 0; i < 4; ++i)
            if (e + i < a.num_experts) store_one(to, e + i, a.logits_type, v[i]);
        }
      }
    }
  }
}

// One row per workgroup in x, runs of eight columns per thread; y of the
// row's places is read once, summed in fp32 in the order of the choices. NT:
// streamed past the caches (4096 rows of 8 x 7168 bf16 and a residual: 106 us
// against 122, 5.5 TB/s of bytes that cannot be saved, which is what bounds it;
// at 256 rows 9.5 us against 7.8).
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

// How a row of E experts lies over lanes and registers.
template <class F>
hipError_t by_width(int experts, F&& f) {
  if (experts <= 8) return f(Row<8, 1>());
  if (experts <= 32) return f(Row<8, 4>());
  if (experts <= 64) return f(Row<8, 8>());
  if (experts <= 128) return f(Row<8, 16>());
  if (experts <= 256) return f(Row<8, 32>());
  if (experts <= 512) return f(Row<16, 32>());
  return f(Row<16, 64>());
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
    using W = decltype(width);
    if (blocks <= 1) {
      hipLaunchKernelGGL((wb_route_few_kernel<W>), dim3(1), dim3(W::T), 0, st, a, per);
      return hipGetLastError();
    }
    const uint32_t n = static_cast<uint32_t>(blocks);
    hipLaunchKernelGGL((wb_route_kernel<W>), dim3(n), dim3(W::T), 0, st, a, blocks, per);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((wb_route_place_kernel<W>), dim3(n + 1), dim3(kPlaceThreads), 0, st, a, blocks, per);
    return hipGetLastError();
  });
}

int launch_route_grad(const RouteGradArgs& a, void* stream) {
  if (a.rows == 0) return hipSuccess;
  const auto st = static_cast<hipStream_t>(stream);
  return by_width(a.num_experts, [&](auto width) {
    using W = decltype(width);
    const int64_t per = kGradThreads / W::L, blocks = std::min<int64_t>((a.rows + per - 1) / per, kGradBlocks);
    hipLaunchKernelGGL((wb_route_grad_kernel<W>), dim3(static_cast<uint32_t>(blocks)),
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
