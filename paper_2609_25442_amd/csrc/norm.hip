// Residual addition and root-mean-square norm of rows, with the normed row in
// bf16, fp32, or fp8 E4M3 with one fp32 scale per 128 columns:
//   t = x + residual,  y_j = t_j w_j / sqrt(mean_j t_j^2 + eps),
//   s = max |y| / 448 over 128 columns,  q = E4M3(y / s).
// Bandwidth bound: each operand is read once and each result written once. A
// row is held in registers between the sum of squares and the output; its sum
// is taken in fp32, eight columns per lane, then over the wavefronts. Both
// outputs are rounded once, from the fp32 values (the norm sees t before it is
// rounded to the residual's type). Sixteen neighbouring lanes hold the 128
// columns of a scale, so its maximum needs no shared memory. Measured with
// bf16 rows and a residual, fp8 out: 16384 x 7168 in 141 us, 5.85 TB/s (88 % of
// a large copy); 4 rows in 5 us, 7 with the call.
#include "ops_device.hpp"

namespace wb {
namespace {

constexpr int kMaxWaves = 16;
constexpr int64_t kManyRows = 2048;

// A row takes `waves` wavefronts (ROWS > 1: one, and the workgroup holds ROWS
// rows), each lane V runs of eight columns. LOOP: rows wider than the registers; the
// second pass reads its operands again. NT: more bytes than the caches keep
// for the next reader, streamed past them (16384 x 7168 to fp8: 141 us against
// 158; at 2048 rows 23 us against 21).
template <int V, int ROWS, bool LOOP, bool NT>
__global__ __launch_bounds__(ROWS > 1 ? 64 * ROWS : 64 * kMaxWaves) void wb_add_rms_norm_kernel(NormArgs a) {
  __shared__ float part[kMaxWaves];
  const int wave = threadIdx.x >> 6;
  const int64_t row = ROWS > 1 ? int64_t(blockIdx.x) * ROWS + wave : int64_t(blockIdx.x);
  if (ROWS > 1 && row >= a.rows) return;
  const int lane = ROWS > 1 ? threadIdx.x & 63 : threadIdx.x;
  const int lanes = ROWS > 1 ? 64 : blockDim.x;
  const int xb = a.x_type == WB_F32 ? 4 : 2, rb = a.residual_type == WB_F32 ? 4 : 2, tb = a.total_type == WB_F32 ? 4 : 2;
  const int ob = a.out_type == WB_F32 ? 4 : a.out_type == WB_BF16 ? 2 : 1;
  const char* x = static_cast<const char*>(a.x) + row * a.ld_x * xb;
  const char* res = static_cast<const char*>(a.residual) + row * a.ld_residual * rb;
  char* total = static_cast<char*>(a.total) + row * a.ld_total * tb;
  char* out = static_cast<char*>(a.out) + row * a.ld_out * ob;

  auto load = [&](int64_t c, float(&t)[8]) {
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
    for (int i = 0; i < 8; ++i) t[i] += r[i];
  };

  float t[V][8], sum = 0.0f;
  const int64_t step = int64_t(lanes) * 8;
  for (int64_t base = 0; base < a.cols; base += LOOP ? step * V : a.cols) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int64_t c = base + v * step + lane * 8;
      if (c < a.cols) {
        load(c, t[v]);
      } else {
        for (int i = 0; i < 8; ++i) t[v][i] = 0.0f;
      }
    }
#pragma unroll
    for (int v = 0; v < V; ++v)
      for (int i = 0; i < 8; ++i) sum = __builtin_fmaf(t[v][i], t[v][i], sum);
  }
  sum = sum_of_wave(sum);
  if (ROWS == 1 && lanes > 64) {
    if ((lane & 63) == 0) part[wave] = sum;
    __syncthreads();
    sum = 0.0f;
    for (int w = 0; w < lanes / 64; ++w) sum += part[w];
  }
  const float inv = 1.0f / sqrtf(sum / static_cast<float>(a.cols) + a.eps);

  for (int64_t base = 0; base < a.cols; base += LOOP ? step * V : a.cols) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int64_t c = base + v * step + lane * 8;
      // the 16 lanes of a scale stay together: lanes past the row add zeros
      if (c - (lane & 15) * 8 >= a.cols) continue;
      const bool whole = c + 8 <= a.cols;
      float y[8];
      if (LOOP) {
        for (int i = 0; i < 8; ++i) t[v][i] = 0.0f;
        if (c < a.cols) load(c, t[v]);
      }
      if (whole) {
        if (a.total) store_eight<NT>(total, c, a.total_type, t[v]);
        load_eight(a.weight, c, a.weight_type, y);
      } else {
        if (a.total) store_tail(total, c, a.cols, a.total_type, t[v]);
        load_tail(a.weight, c, a.cols, a.weight_type, y);
      }
      for (int i = 0; i < 8; ++i) y[i] *= t[v][i] * inv;
      if (a.out_type == WB_F8E4M3) {
        float amax = 0.0f;
        for (int i = 0; i < 8; ++i) amax = fmaxf(amax, fabsf(y[i]));
        const RowScale q = row_scale(reduce16(amax, FMax()));
        if ((lane & 15) == 0) a.scales[row * a.ld_scales + c / kScaleBlock] = q.s;
        quotients(y, q);
        const u32x2 p = {pack_fp8(y[0], y[1], y[2], y[3]), pack_fp8(y[4], y[5], y[6], y[7])};
        if (whole) {
          put_u2<NT>(reinterpret_cast<u32x2_a1*>(out + c), p);
        } else {
          for (int i = 0; i < 8; ++i)
            if (c + i < a.cols) out[c + i] = static_cast<char>(p[i >> 2] >> (8 * (i & 3)));
        }
      } else if (whole) {
        store_eight<NT>(out, c, a.out_type, y);
      } else {
        store_tail(out, c, a.cols, a.out_type, y);
      }
    }
  }
}

template <int V, int ROWS, bool LOOP>
hipError_t launch(const NormArgs& a, int waves, hipStream_t st) {
  const dim3 grid(static_cast<uint32_t>((a.rows + ROWS - 1) / ROWS)), block(64 * (ROWS > 1 ? ROWS : waves));
  const int64_t row_bytes = a.cols * (bytes_of(a.x_type) + (a.residual ? bytes_of(a.residual_type) : 0) +
                                      (a.total ? bytes_of(a.total_type) : 0) + bytes_of(a.out_type));
  if (a.rows * row_bytes > kStreamBytes)
    hipLaunchKernelGGL((wb_add_rms_norm_kernel<V, ROWS, LOOP, true>), grid, block, 0, st, a);
  else
    hipLaunchKernelGGL((wb_add_rms_norm_kernel<V, ROWS, LOOP, false>), grid, block, 0, st, a);
  return hipGetLastError();
}

}  // namespace

int launch_add_rms_norm(const NormArgs& a, void* stream) {
  const auto st = static_cast<hipStream_t>(stream);
  if (a.rows == 0) return hipSuccess;
  // Narrow rows: one wavefront each, four to a workgroup. Wider ones: with
  // many rows four runs a lane (16384 x 7168 to fp8: 141 us against 148 of two
  // and 189 of one), one up to eight wavefronts (16384 x 4096 to bf16: 87 us
  // against 90 of two and 97 of four); with few rows two, which gives a row
  // more wavefronts (512 x 7168: 8.2 us against 10.2 of four). Past sixteen
  // wavefronts of four, two passes.
  const int64_t runs = (a.cols + 7) / 8;
  const auto waves = [&](int v) { return static_cast<int>((runs + 64 * v - 1) / (64 * v)); };
  if (runs <= 64) return launch<1, 4, false>(a, 1, st);
  if (runs <= 128) return launch<2, 4, false>(a, 1, st);
  if (a.rows >= kManyRows && runs <= 512) return launch<1, 1, false>(a, waves(1), st);
  if (a.rows < kManyRows && waves(2) <= kMaxWaves) return launch<2, 1, false>(a, waves(2), st);
  if (waves(4) <= kMaxWaves) return launch<4, 1, false>(a, waves(4), st);
  return launch<4, 1, true>(a, kMaxWaves, st);
}

}  // namespace wb
