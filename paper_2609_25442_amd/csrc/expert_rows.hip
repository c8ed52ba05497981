// Rows sorted by expert and back, and their gradients.
//   dispatch: out_p = x_t for p = positions_ti, zeros elsewhere;  dx_t = sum_i dout_p
//   combine's gradient: dy_p = g_ti dout_t, zeros elsewhere;  dg_ti = <dout_t, y_p>
// (the sum itself is in route.hip). Work goes by tokens: a token's row is read
// once and its k places are written, or read, from there. A place is a token's
// own if tokens says so, so no two rows write one place; the places that are
// nobody's are filled with zeros by workgroups of their own.
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

// A row's own places into LDS, -1 for what is left out.
__device__ __forceinline__ void own_places(const PlacesArgs& a, int64_t row, int lane, int lanes, int32_t* to) {
  const int64_t first = first_place(a), last = last_place(a);
  for (int i = lane; i < a.k; i += lanes) {
    int32_t p = -1;
    if (row < a.rows) {
      p = a.positions[row * a.k + i];
      if (p < first || p >= last || a.tokens[p] != row) p = -1;
    }
    to[i] = p;
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

template <int V, bool NT>
__global__ __launch_bounds__(kThreads) void wb_dispatch_kernel(DispatchArgs a, int shift, int64_t fills) {
  __shared__ int32_t places[32 * kMaxRouteK];
  const int ob = a.out_type == WB_F32 ? 4 : 2, xb = a.x_type == WB_F32 ? 4 : 2;
  if (int64_t(blockIdx.x) < fills) {
    fill_places<NT>(a.at, blockIdx.x, static_cast<char*>(a.out), a.ld_out * ob, a.out_type);
    return;
  }
  const int lanes = 1 << shift, lane = threadIdx.x & (lanes - 1), sub = threadIdx.x >> shift;
  const int64_t row = (int64_t(blockIdx.x) - fills) * (kThreads >> shift) + sub;
  int32_t* mine = places + sub * a.at.k;
  float v[V][8];
  const char* x = static_cast<const char*>(a.x) + row * a.ld_x * xb;
  const auto col = [&](int i) { return ((int64_t(blockIdx.y) * V + i) * lanes + lane) * 8; };
#pragma unroll
  for (int i = 0; i < V; ++i)
    if (row < a.at.rows && col(i) < a.at.cols) load_run(x, col(i), a.at.cols, a.x_type, v[i]);
  own_places(a.at, row, lane, lanes, mine);
  __syncthreads();
  if (row >= a.at.rows) return;
  for (int i = 0; i < a.at.k; ++i) {
    if (mine[i] < 0) continue;
    char* to = static_cast<char*>(a.out) + mine[i] * a.ld_out * ob;
#pragma unroll
    for (int j = 0; j < V; ++j)
      if (col(j) < a.at.cols) store_run<NT>(to, col(j), a.at.cols, a.out_type, v[j]);
  }
}

template <bool NT>
__global__ __launch_bounds__(kThreads) void wb_dispatch_grad_kernel(DispatchGradArgs a, int shift) {
  __shared__ int32_t places[32 * kMaxRouteK];
  const int lanes = 1 << shift, lane = threadIdx.x & (lanes - 1), sub = threadIdx.x >> shift;
  const int64_t row = int64_t(blockIdx.x) * (kThreads >> shift) + sub;
  int32_t* mine = places + sub * a.at.k;
  own_places(a.at, row, lane, lanes, mine);
  __syncthreads();
  const int64_t c = (int64_t(blockIdx.y) * lanes + lane) * 8;
  if (row >= a.at.rows || c >= a.at.cols) return;
  const int db = a.d_out_type == WB_F32 ? 4 : 2, ob = a.d_x_type == WB_F32 ? 4 : 2;
  float sum[8] = {0, 0, 0, 0, 0, 0, 0, 0}, v[8];
  for (int i = 0; i < a.at.k; ++i) {
    if (mine[i] < 0) continue;
    load_run(static_cast<const char*>(a.d_out) + mine[i] * a.ld_d_out * db, c, a.at.cols, a.d_out_type, v);
    for (int j = 0; j < 8; ++j) sum[j] += v[j];
  }
  store_run<NT>(static_cast<char*>(a.d_x) + row * a.ld_d_x * ob, c, a.at.cols, a.d_x_type, sum);
}

// A row lies over 1 << shift lanes, wider ones over all of a workgroup's in
// steps; the sums of d_gates over lanes, then wavefronts, then steps.
template <int V, bool NT>
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
  own_places(a.at, row, lane, lanes, mine);
  for (int i = threadIdx.x; i < (kThreads / min(lanes, 64)) * k; i += kThreads) dots[i] = 0.0f;
  __syncthreads();
  if (row < a.at.rows) {
    const char* d_row = static_cast<const char*>(a.d_out) + row * a.ld_d_out * db;
    for (int64_t base = 0; base < a.at.cols; base += int64_t(lanes) * V * 8) {
      float d[V][8];
      const auto col = [&](int j) { return base + (int64_t(j) * lanes + lane) * 8; };
#pragma unroll
      for (int j = 0; j < V; ++j) {
        for (int m = 0; m < 8; ++m) d[j][m] = 0.0f;
        if (col(j) < a.at.cols) load_run(d_row, col(j), a.at.cols, a.d_out_type, d[j]);
      }
      for (int i = 0; i < k; ++i) {
        const int32_t p = mine[i];
        if (p < 0) continue;
        if (a.y) {
          const char* y = static_cast<const char*>(a.y) + p * a.ld_y * yb;
          float dot = 0.0f, v[8];
#pragma unroll
          for (int j = 0; j < V; ++j)
            if (col(j) < a.at.cols) {
              load_run(y, col(j), a.at.cols, a.y_type, v);
              for (int m = 0; m < 8; ++m) dot = __builtin_fmaf(d[j][m], v[m], dot);
            }
          for (int off = min(lanes, 64) / 2; off > 0; off >>= 1) dot += __shfl_xor(dot, off);
          if ((threadIdx.x & (min(lanes, 64) - 1)) == 0) dots[group * k + i] += dot;
        }
        if (a.d_y) {
          const float g = a.gates[row * k + i];
          char* to = static_cast<char*>(a.d_y) + p * a.ld_d_y * ob;
#pragma unroll
          for (int j = 0; j < V; ++j)
            if (col(j) < a.at.cols) {
              float v[8];
              for (int m = 0; m < 8; ++m) v[m] = g * d[j][m];
              store_run<NT>(to, col(j), a.at.cols, a.d_y_type, v);
            }
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
  int64_t rows, per, lanes;
  uint32_t y;
};

Grid grid_of(const PlacesArgs& a, int v) {
  Grid g;
  g.shift = row_shift(a.cols), g.lanes = int64_t(1) << g.shift, g.per = kThreads >> g.shift;
  g.rows = (a.rows + g.per - 1) / g.per;
  g.y = static_cast<uint32_t>((a.cols + g.lanes * v * 8 - 1) / (g.lanes * v * 8));
  return g;
}

}  // namespace

int launch_dispatch(const DispatchArgs& a, void* stream) {
  const Grid g = grid_of(a.at, a.at.cols <= 2048 ? 1 : 2);
  const int64_t fills = (a.at.places + kFillPlaces - 1) / kFillPlaces;
  if (g.rows + fills == 0) return hipSuccess;
  const bool nt = a.at.places * a.at.cols * bytes_of(a.out_type) > kStreamBytes;
  const auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3(static_cast<uint32_t>(g.rows + fills), g.y), dim3(kThreads), 0,
                       static_cast<hipStream_t>(stream), a, g.shift, fills);
    return hipGetLastError();
  };
  if (a.at.cols <= 2048) return nt ? go(wb_dispatch_kernel<1, true>) : go(wb_dispatch_kernel<1, false>);
  return nt ? go(wb_dispatch_kernel<2, true>) : go(wb_dispatch_kernel<2, false>);
}

int launch_dispatch_grad(const DispatchGradArgs& a, void* stream) {
  const Grid g = grid_of(a.at, 1);
  if (g.rows == 0) return hipSuccess;
  hipLaunchKernelGGL(wb_dispatch_grad_kernel<false>, dim3(static_cast<uint32_t>(g.rows), g.y), dim3(kThreads), 0,
                     static_cast<hipStream_t>(stream), a, g.shift);
  return hipGetLastError();
}

int launch_combine_grad(const CombineGradArgs& a, void* stream) {
  const Grid g = grid_of(a.at, 1);
  const int64_t fills = a.d_y ? (a.at.places + kFillPlaces - 1) / kFillPlaces : 0;
  if (g.rows + fills == 0) return hipSuccess;
  const bool nt = a.at.places * a.at.cols * (bytes_of(a.y_type) + bytes_of(a.d_y_type)) > kStreamBytes;
  const auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3(static_cast<uint32_t>(g.rows + fills)), dim3(kThreads), 0,
                       static_cast<hipStream_t>(stream), a, g.shift, fills);
    return hipGetLastError();
  };
  if (a.at.cols <= 2048) return nt ? go(wb_combine_grad_kernel<1, true>) : go(wb_combine_grad_kernel<1, false>);
  if (a.at.cols <= 4096) return nt ? go(wb_combine_grad_kernel<2, true>) : go(wb_combine_grad_kernel<2, false>);
  return nt ? go(wb_combine_grad_kernel<4, true>) : go(wb_combine_grad_kernel<4, false>);
}

}  // namespace wb
