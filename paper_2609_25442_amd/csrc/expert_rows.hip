// Rows sorted by expert and back, and their gradients.
//   dispatch: out_p = x_t for p = positions_ti, zeros elsewhere;  dx_t = sum_i dout_p
//   collect: out_t = r_t + sum_i g_ti y_p;  dy_p = g_ti dout_t, zeros elsewhere;  dg_ti = <dout_t, y_p>
// Work goes by tokens: a token's row is read
// once and its k places are written, or read, from there. A place is a token's
// own if tokens says so, so no two rows write one place, and counts once in a
// row; the places that are nobody's are filled with zeros by workgroups of their own.
//
// Bandwidth bound: eight columns a thread, one run of them. bf16 rows are waited
// for one by one (load_eight widens them inside its branch on the type), so that
// only the number of wavefronts hides a row's way to memory (the gradient of collect of
// 8192 x 7168, k = 8: 420 us, and 560 with four runs a lane). Past the caches' size
// places' rows are stored, and read, with the non-temporal hint, a token's own row without:
// dispatch of the same in 182 us, 5.8 TB/s (213 with none, 220 with its row hinted too),
// back in 179, 5.9 TB/s (198 without); the gradient of collect at 4.8 TB/s: a lane has one
// place under way, and stores its row of d_y and fetches its gate before the next.
#include <algorithm>

#include "ops_device.hpp"
#include "train.hpp"

namespace wb {
namespace {

constexpr int kThreads = 256;
constexpr int kFillPlaces = 16;  // to a workgroup

__device__ __forceinline__ int64_t first_place(const PlacesArgs& a) { return a.first ? max(0, *a.first) : 0; }
__device__ __forceinline__ int64_t last_place(const PlacesArgs& a) {
  return a.last ? min(a.places, int64_t(*a.last)) : a.places;
}

// A row's own places into LDS, -1 for what is left out: a place outside the
// call's, one that tokens gives to another row, and, with ONCE, one that an earlier
// choice of the row has. A row's choices are those of one wavefront's lanes.
template <bool ONCE>
__device__ __forceinline__ void own_places(const PlacesArgs& a, int64_t row, int lane, int lanes, int32_t* to) {
  const int64_t first = first_place(a), last = last_place(a);
  for (int i = lane; i < a.k; i += lanes) {
    const int32_t p = row < a.rows ? a.positions[row * a.k + i] : -1;
    const int32_t of = p >= first && p < last ? a.tokens[p] : -1;
    bool again = false;
    if (ONCE) {
      to[i] = p;
      order_lanes();
      // what is -1 here already was left out itself, and so is the same place after it
      for (int j = 0; j < i; j += 8) {
        int32_t before[8];
#pragma unroll
        for (int m = 0; m < 8; ++m) before[m] = to[min(j + m, i - 1)];
#pragma unroll
        for (int m = 0; m < 8; ++m) again = again || before[m] == p;
      }
      order_lanes();
    }
    to[i] = of == row && !again ? p : -1;
  }
}

// Zeros in those of a workgroup's places that are no row's own.
template <bool NT>
__device__ __forceinline__ void fill_places(const PlacesArgs& a, int64_t block, char* out, int64_t ld_bytes, int type) {
  __shared__ int left_out[kFillPlaces];
  const int64_t p = block * kFillPlaces + threadIdx.x;
  if (threadIdx.x < kFillPlaces) {
    bool none = p < a.places;
    if (none && p >= first_place(a) && p < last_place(a)) {
      const int32_t t = a.tokens[p];
      if (t >= 0 && t < a.rows)
        for (int i = 0; i < a.k; ++i) none = none && a.positions[int64_t(t) * a.k + i] != p;
    }
    left_out[threadIdx.x] = none;
  }
  __syncthreads();
  const float zero[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  for (int i = 0; i < kFillPlaces; ++i) {
    if (!left_out[i]) continue;
    char* row = out + (block * kFillPlaces + i) * ld_bytes;
    for (int64_t c = (int64_t(blockIdx.y) * kThreads + threadIdx.x) * 8; c < a.cols; c += int64_t(gridDim.y) * kThreads * 8)
      store_run<NT>(row, c, a.cols, type, zero);
  }
}

template <bool NT>
__global__ __launch_bounds__(kThreads) void wb_dispatch_kernel(DispatchArgs a, int shift, int64_t fills) {
  __shared__ int32_t places[32 * kMaxRouteK];
  const int ob = a.out_type == WB_F32 ? 4 : 2, xb = a.x_type == WB_F32 ? 4 : 2;
  if (int64_t(blockIdx.x) < fills) {
    fill_places<NT>(a.at, blockIdx.x, static_cast<char*>(a.out), a.ld_out * ob, a.out_type);
    return;
  }
  const int lanes = 1 << shift, lane = threadIdx.x & (lanes - 1), sub = threadIdx.x >> shift;
  const int64_t row = (int64_t(blockIdx.x) - fills) * (kThreads >> shift) + sub;
  const int64_t c = (int64_t(blockIdx.y) * lanes + lane) * 8;
  int32_t* mine = places + sub * a.at.k;
  float v[8];
  if (row < a.at.rows && c < a.at.cols)
    load_run(static_cast<const char*>(a.x) + row * a.ld_x * xb, c, a.at.cols, a.x_type, v);
  own_places<false>(a.at, row, lane, lanes, mine);  // written twice, a place holds the same
  __syncthreads();
  if (row >= a.at.rows || c >= a.at.cols) return;
  for (int i = 0; i < a.at.k; ++i)
    if (mine[i] >= 0) store_run<NT>(static_cast<char*>(a.out) + mine[i] * a.ld_out * ob, c, a.at.cols, a.out_type, v);
}

constexpr int kBatch = 4;  // rows of a token; whole fp32 ones are under way together

template <bool NT>
__global__ __launch_bounds__(kThreads) void wb_dispatch_grad_kernel(DispatchGradArgs a, int shift) {
  __shared__ int32_t places[32 * kMaxRouteK];
  const int lanes = 1 << shift, lane = threadIdx.x & (lanes - 1), sub = threadIdx.x >> shift;
  const int64_t row = int64_t(blockIdx.x) * (kThreads >> shift) + sub;
  int32_t* mine = places + sub * a.at.k;
  own_places<true>(a.at, row, lane, lanes, mine);
  __syncthreads();
  const int64_t c = (int64_t(blockIdx.y) * lanes + lane) * 8;
  if (row >= a.at.rows || c >= a.at.cols) return;
  const int db = a.d_out_type == WB_F32 ? 4 : 2, ob = a.d_x_type == WB_F32 ? 4 : 2;
  float sum[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  for (int i = 0; i < a.at.k; i += kBatch) {
    float v[kBatch][8];
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
      for (int m = 0; m < 8; ++m) v[j][m] = 0.0f;
      if (i + j < a.at.k && mine[i + j] >= 0)
        load_run<NT>(static_cast<const char*>(a.d_out) + mine[i + j] * a.ld_d_out * db, c, a.at.cols, a.d_out_type, v[j]);
    }
#pragma unroll
    for (int j = 0; j < kBatch; ++j)
      for (int m = 0; m < 8; ++m) sum[m] += v[j][m];
  }
  store_run<NT>(static_cast<char*>(a.d_x) + row * a.ld_d_x * ob, c, a.at.cols, a.d_x_type, sum);
}

// The sum of combine in route.hip, over the choices that the gradients know of:
// the same terms in the same order, so the same bits over a router's places. A row
// has one wavefront or more. Whose a place is, and whether an earlier choice has it,
// is known while y's row is on its way (a row of y that does not count is read for
// nothing): 8192 x 7168 of 8, bf16, in 201 us, combine 203; 333 x 1111 of 3, fp32, 4.8
// and 4.6 (5.6 with the places in LDS first).
template <bool NT>
__global__ __launch_bounds__(kThreads) void wb_collect_kernel(CollectArgs a, int shift) {
  static_assert(kMaxRouteK <= 64, "a lane of each wavefront has a choice");
  const int yb = a.y_type == WB_F32 ? 4 : 2, rb = a.residual_type == WB_F32 ? 4 : 2, ob = a.out_type == WB_F32 ? 4 : 2;
  const int lanes = 1 << shift, lane = threadIdx.x & 63;
  const int64_t row = int64_t(blockIdx.x) * (kThreads >> shift) + (__builtin_amdgcn_readfirstlane(threadIdx.x) >> shift);
  if (row >= a.at.rows) return;
  const int64_t c = (int64_t(blockIdx.y) * lanes + (threadIdx.x & (lanes - 1))) * 8;
  const bool on = c < a.at.cols;  // the other lanes stay for their choice
  const int32_t* places = a.at.positions + row * a.at.k;
  const int32_t mine = lane < a.at.k ? places[lane] : -1;
  const int64_t first = first_place(a.at), last = last_place(a.at);
  float sum[8] = {0, 0, 0, 0, 0, 0, 0, 0}, v[8];
  for (int i = 0; i < a.at.k; ++i) {
    const int32_t at = places[i];
    if (at < first || at >= last) continue;
    const float g = a.gates[row * a.at.k + i];
    const int32_t of = a.at.tokens[at];
    if (on) load_run<NT>(static_cast<const char*>(a.y) + at * a.ld_y * yb, c, a.at.cols, a.y_type, v);
    const uint64_t before = __ballot(mine == at) & ((uint64_t(1) << i) - 1);
    if (of != row || before != 0) continue;
    for (int m = 0; m < 8; ++m) sum[m] = __builtin_fmaf(g, v[m], sum[m]);
  }
  if (!on) return;
  if (a.residual) {
    load_run<NT>(static_cast<const char*>(a.residual) + row * a.ld_residual * rb, c, a.at.cols, a.residual_type, v);
    for (int m = 0; m < 8; ++m) sum[m] += v[m];
  }
  store_run<NT>(static_cast<char*>(a.out) + row * a.ld_out * ob, c, a.at.cols, a.out_type, sum);
}

// The sum over 8, 16, 32 or at least 64 neighbouring lanes.
__device__ __forceinline__ float sum_of_lanes(float v, int lanes) {
  if (lanes >= 16) {
    v = reduce16(v, Sum());
    if (lanes >= 32) v += __shfl_xor(v, 16);
    if (lanes >= 64) v += __shfl_xor(v, 32);
    return v;
  }
  for (int off = 4; off > 0; off >>= 1) v += __shfl_xor(v, off);
  return v;
}

// A row lies over 1 << shift lanes, wider ones over all of a workgroup's in
// steps; the sums of d_gates over lanes, then steps, then wavefronts.
template <bool NT>
__global__ __launch_bounds__(kThreads) void wb_combine_grad_kernel(CombineGradArgs a, int shift, int64_t fills) {
  __shared__ int32_t places[32 * kMaxRouteK];
  __shared__ float dots[32 * kMaxRouteK];  // of each wavefront, or of each row
  const int db = a.d_out_type == WB_F32 ? 4 : 2, yb = a.y_type == WB_F32 ? 4 : 2, ob = a.d_y_type == WB_F32 ? 4 : 2;
  if (int64_t(blockIdx.x) < fills) {
    fill_places<NT>(a.at, blockIdx.x, static_cast<char*>(a.d_y), a.ld_d_y * ob, a.d_y_type);
    return;
  }
  const int k = a.at.k;
  const int lanes = 1 << shift, lane = threadIdx.x & (lanes - 1), sub = threadIdx.x >> shift;
  const int64_t row = (int64_t(blockIdx.x) - fills) * (kThreads >> shift) + sub;
  const int group = lanes < 64 ? sub : int(threadIdx.x >> 6), groups = lanes < 64 ? 1 : lanes >> 6;
  int32_t* mine = places + sub * k;
  own_places<true>(a.at, row, lane, lanes, mine);
  for (int i = threadIdx.x; i < (kThreads / min(lanes, 64)) * k; i += kThreads) dots[i] = 0.0f;
  __syncthreads();
  if (row < a.at.rows) {
    const char* d_row = static_cast<const char*>(a.d_out) + row * a.ld_d_out * db;
    for (int64_t base = 0; base < a.at.cols; base += lanes * 8) {
      const int64_t c = base + lane * 8;
      const bool on = c < a.at.cols;  // lanes past the row add zeros
      float d[8], y[8], v[8];
      for (int m = 0; m < 8; ++m) d[m] = y[m] = 0.0f;
      if (on) load_run(d_row, c, a.at.cols, a.d_out_type, d);
      for (int i = 0; i < k; ++i) {
        const int32_t p = mine[i];
        if (p < 0) continue;
        float dot = 0.0f;
        if (a.y && on) load_run<NT>(static_cast<const char*>(a.y) + p * a.ld_y * yb, c, a.at.cols, a.y_type, y);
        if (a.d_y && on) {
          const float g = a.gates[row * k + i];
          for (int m = 0; m < 8; ++m) v[m] = g * d[m];
          store_run<NT>(static_cast<char*>(a.d_y) + p * a.ld_d_y * ob, c, a.at.cols, a.d_y_type, v);
        }
        if (a.y) {
          for (int m = 0; m < 8; ++m) dot = __builtin_fmaf(d[m], y[m], dot);
          dot = sum_of_lanes(dot, lanes);
          if ((threadIdx.x & (min(lanes, 64) - 1)) == 0) dots[group * k + i] += dot;
        }
      }
    }
  }
  if (!a.d_gates) return;
  __syncthreads();
  if (row < a.at.rows)
    for (int i = lane; i < k; i += lanes) {
      float sum = 0.0f;
      for (int g = 0; g < groups; ++g) sum += dots[(lanes < 64 ? sub : sub * groups + g) * k + i];
      a.d_gates[row * k + i] = mine[i] < 0 ? 0.0f : sum;
    }
}

struct Grid {
  int shift;
  int64_t rows;
  uint32_t y;
};

Grid grid_of(const PlacesArgs& a, int least = 0) {
  Grid g;
  g.shift = std::max(row_shift(a.cols), least);
  const int64_t per = kThreads >> g.shift, slab = int64_t(8) << g.shift;
  g.rows = (a.rows + per - 1) / per;
  g.y = static_cast<uint32_t>((a.cols + slab - 1) / slab);
  return g;
}

}  // namespace

int launch_dispatch(const DispatchArgs& a, void* stream) {
  const Grid g = grid_of(a.at);
  const int64_t fills = (a.at.places + kFillPlaces - 1) / kFillPlaces;
  if (g.rows + fills == 0) return hipSuccess;
  if (!one_launch((g.rows + fills) * g.y)) return hipErrorInvalidConfiguration;
  const bool nt = a.at.places * a.at.cols * bytes_of(a.out_type) > kStreamBytes;
  hipLaunchKernelGGL(nt ? wb_dispatch_kernel<true> : wb_dispatch_kernel<false>, dim3(static_cast<uint32_t>(g.rows + fills), g.y),
                     dim3(kThreads), 0, static_cast<hipStream_t>(stream), a, g.shift, fills);
  return hipGetLastError();
}

int launch_dispatch_grad(const DispatchGradArgs& a, void* stream) {
  const Grid g = grid_of(a.at);
  if (g.rows == 0) return hipSuccess;
  if (!one_launch(g.rows * g.y)) return hipErrorInvalidConfiguration;
  const bool nt = a.at.places * a.at.cols * bytes_of(a.d_out_type) > kStreamBytes;
  hipLaunchKernelGGL(nt ? wb_dispatch_grad_kernel<true> : wb_dispatch_grad_kernel<false>, dim3(static_cast<uint32_t>(g.rows), g.y),
                     dim3(kThreads), 0, static_cast<hipStream_t>(stream), a, g.shift);
  return hipGetLastError();
}

int launch_collect(const CollectArgs& a, void* stream) {
  const Grid g = grid_of(a.at, 6);  // a wavefront or more a row
  if (g.rows == 0) return hipSuccess;
  if (!one_launch(g.rows * g.y)) return hipErrorInvalidConfiguration;
  const int64_t row_bytes = a.at.cols * (a.at.k * bytes_of(a.y_type) + (a.residual ? bytes_of(a.residual_type) : 0) + bytes_of(a.out_type));
  const auto kernel = a.at.rows * row_bytes > kStreamBytes ? wb_collect_kernel<true> : wb_collect_kernel<false>;
  hipLaunchKernelGGL(kernel, dim3(static_cast<uint32_t>(g.rows), g.y), dim3(kThreads), 0, static_cast<hipStream_t>(stream), a, g.shift);
  return hipGetLastError();
}

int launch_combine_grad(const CombineGradArgs& a, void* stream) {
  const Grid g = grid_of(a.at);
  const int64_t fills = a.d_y ? (a.at.places + kFillPlaces - 1) / kFillPlaces : 0;
  if (g.rows + fills == 0) return hipSuccess;
  if (!one_launch(g.rows + fills)) return hipErrorInvalidConfiguration;
  const bool nt = a.at.places * a.at.cols * (bytes_of(a.y_type) + bytes_of(a.d_y_type)) > kStreamBytes;
  hipLaunchKernelGGL(nt ? wb_combine_grad_kernel<true> : wb_combine_grad_kernel<false>, dim3(static_cast<uint32_t>(g.rows + fills)),
                     dim3(kThreads), 0, static_cast<hipStream_t>(stream), a, g.shift, fills);
  return hipGetLastError();
}

}  // namespace wb
