// Activation of rows, or of their gate halves times their up halves, with a
// checkpoint of the input in 8 bits, and the gradient from either.
//   out = act(x), or act(g) u;   codes = E4M3(x / s), s = max |x| / 448 over 128 columns of a half
//   dx = dout act'(x), or dg = dout u act'(g), du = dout act(g)   at x, or at codes s
//   silu: z p, slope p (1 + z (1 - p)), p = 1 / (1 + e^-z);   gelu: z P, slope P + z e^(-z^2/2) / sqrt(2 pi), P = erfc(-z / sqrt 2) / 2
// Sixteen lanes hold the 128 columns of a scale, eight each, of both halves.
//
// Bandwidth bound once the instructions are few: 8192 x 28672 bf16, gated silu, in 8
// bits: there 170 us, 5.6 TB/s, back 156, 6.1 TB/s (least 156 and 150). With a 64-bit division for a unit's row, a divided sigmoid and a divided
// scale a pass of both took 362 us, now 315.
#include <type_traits>

#include "ops_device.hpp"
#include "train.hpp"

namespace wb {
namespace {

constexpr int kThreads = 256, kUnits = kThreads / 16;  // units of 128 columns to a workgroup
constexpr uint64_t kMaxBlocks = (uint64_t(1) << 24) - 1;  // a launch has fewer than 2^32 threads

// Units over rows: 128 columns of a row each, in.a_row of them, fewer than 2^32
// in all. A unit's row by multiplication (Granlund and Montgomery).
struct Units {
  uint32_t a_row, magic, shift;
  uint64_t all;
  __device__ __forceinline__ uint32_t row(uint32_t unit) const {
    const uint32_t t = __umulhi(unit, magic);
    return a_row == 1 ? unit : (t + ((unit - t) >> 1)) >> shift;
  }
};

Units units_of(int64_t rows, int64_t cols) {
  Units u{};
  u.a_row = static_cast<uint32_t>((cols + 127) / 128);
  u.all = static_cast<uint64_t>(rows) * u.a_row;
  uint32_t bits = 0;  // the smallest power of two not below a_row
  while ((uint64_t(1) << bits) < u.a_row) ++bits;
  u.magic = static_cast<uint32_t>(((uint64_t(1) << 32) * ((uint64_t(1) << bits) - u.a_row)) / u.a_row + 1);
  u.shift = bits ? bits - 1 : 0;
  return u;
}

uint32_t blocks_of(const Units& u) {
  const uint64_t blocks = (u.all + kUnits - 1) / kUnits;
  return static_cast<uint32_t>(blocks < kMaxBlocks ? blocks : kMaxBlocks);
}

// The activation of z and its slope.
struct Curve {
  float value, slope;
};

template <int ACT>
__device__ __forceinline__ Curve curve(float z) {
  if (ACT == WB_ACT_SILU) {
    // p by way of t = e^-|z|: 1 / (1 + t), or t / (1 + t) below zero, the reciprocal with one correction
    const float t = exp_below(-fabsf(z)), s = 1.0f + t;
    float r = __builtin_amdgcn_rcpf(s);
    r = __builtin_fmaf(__builtin_fmaf(-s, r, 1.0f), r, r);
    const float p = z < 0.0f ? t * r : r, q = z < 0.0f ? r : t * r;  // q = 1 - p
    const float v = z * p;
    return {v, __builtin_fmaf(v, q, p)};
  }
  if (ACT == WB_ACT_GELU) {
    const float below = 0.5f * erfcf(z * -0.70710678118654752f);
    const float v = z * below;
    return {v, __builtin_fmaf(z * 0.39894228040143268f, exp_below(-0.5f * z * z), below)};
  }
  return {z, 1.0f};
}

// row_scale of ops_device.hpp with fewer instructions: where the product with
// 1 / 448, itself rounded, and its remainder stay normal, one correction gives the
// quotient rounded once.
__device__ __forceinline__ RowScale scale_of(float amax) {
  if (!(amax > 0x1p-90f && amax < 0x1p90f)) return row_scale(amax);
  constexpr float inv = 1.0f / 448.0f;
  RowScale q;
  q.s = amax * inv;
  q.s = __builtin_fmaf(__builtin_fmaf(-q.s, 448.0f, amax), inv, q.s);
  q.r = 1.0f / q.s;
  q.near = q.s > 0x1p-90f;
  return q;
}

// x in 8 bits: sixteen lanes have the columns of a scale.
template <bool NT>
__device__ __forceinline__ void keep(const float (&x)[8], uint8_t* codes, float* scale, int64_t c, int64_t cols, int lane) {
  float amax = 0.0f, v[8];
  for (int i = 0; i < 8; ++i) amax = fmaxf(amax, fabsf(x[i])), v[i] = x[i];
  const RowScale q = scale_of(reduce16(amax, FMax()));
  if (lane == 0) *scale = q.s;
  quotients(v, q);
  const u32x2 p = {pack_fp8(v[0], v[1], v[2], v[3]), pack_fp8(v[4], v[5], v[6], v[7])};
  if (c + 8 <= cols) {
    put_u2<NT>(reinterpret_cast<u32x2_a1*>(codes + c), p);
  } else {
    for (int i = 0; i < 8; ++i)
      if (c + i < cols) codes[c + i] = static_cast<uint8_t>(p[i >> 2] >> (8 * (i & 3)));
  }
}

// Eight codes' values.
__device__ __forceinline__ void load_kept(const uint8_t* codes, float s, int64_t c, int64_t cols, float (&v)[8]) {
  u32x2 p = {0, 0};
  if (c + 8 <= cols) {
    p = *reinterpret_cast<const u32x2_a1*>(codes + c);
  } else {
    for (int i = 0; i < 8; ++i)
      if (c + i < cols) p[i >> 2] |= uint32_t(codes[c + i]) << (8 * (i & 3));
  }
  for (int i = 0; i < 2; ++i) {
    const int w = static_cast<int>(p[i]);
    const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
    v[4 * i] = lo[0] * s, v[4 * i + 1] = lo[1] * s, v[4 * i + 2] = hi[0] * s, v[4 * i + 3] = hi[1] * s;
  }
}

template <int ACT, bool GATED, bool NT>
__global__ __launch_bounds__(kThreads) void wb_activate_kernel(ActivateArgs a, Units in) {
  const int lane = threadIdx.x & 15;
  const int xb = a.x_type == WB_F32 ? 4 : 2, ob = a.out_type == WB_F32 ? 4 : 2;
  for (uint64_t unit = blockIdx.x * uint64_t(kUnits) + (threadIdx.x >> 4); unit < in.all; unit += gridDim.x * uint64_t(kUnits)) {
    const uint32_t r = in.row(static_cast<uint32_t>(unit)), block = static_cast<uint32_t>(unit) - r * in.a_row;
    const int64_t row = r, c = int64_t(block) * 128 + lane * 8;
    const char* x = static_cast<const char*>(a.x) + row * a.ld_x * xb;
    float g[8], u[8];
    for (int i = 0; i < 8; ++i) g[i] = u[i] = 0.0f;
    if (c < a.cols) {
      load_run(x, c, a.cols, a.x_type, g);
      if (GATED) load_run(x + a.cols * xb, c, a.cols, a.x_type, u);
    }
    if (a.codes) {  // all sixteen lanes, those past the row with zeros
      uint8_t* codes = a.codes + row * a.ld_codes;
      float* s = a.scales + row * a.ld_scales + block;
      keep<NT>(g, codes, s, c, a.cols, lane);
      if (GATED) keep<NT>(u, codes + a.cols, s + in.a_row, c, a.cols, lane);
    }
    if (c >= a.cols) continue;
    for (int i = 0; i < 8; ++i) {
      g[i] = curve<ACT>(g[i]).value;
      if (GATED) g[i] *= u[i];
    }
    store_run<NT>(static_cast<char*>(a.out) + row * a.ld_out * ob, c, a.cols, a.out_type, g);
  }
}

template <int ACT, bool GATED, bool NT>
__global__ __launch_bounds__(kThreads) void wb_activate_grad_kernel(ActivateGradArgs a, Units in) {
  const int lane = threadIdx.x & 15;
  const int xb = a.scales ? 1 : a.x_type == WB_F32 ? 4 : 2, db = a.d_out_type == WB_F32 ? 4 : 2;
  const int ob = a.d_x_type == WB_F32 ? 4 : 2;
  for (uint64_t unit = blockIdx.x * uint64_t(kUnits) + (threadIdx.x >> 4); unit < in.all; unit += gridDim.x * uint64_t(kUnits)) {
    const uint32_t r = in.row(static_cast<uint32_t>(unit)), block = static_cast<uint32_t>(unit) - r * in.a_row;
    const int64_t row = r, c = int64_t(block) * 128 + lane * 8;
    if (c >= a.cols) continue;
    const char* x = static_cast<const char*>(a.x) + row * a.ld_x * xb;
    float d[8], g[8], u[8];
    load_run(static_cast<const char*>(a.d_out) + row * a.ld_d_out * db, c, a.cols, a.d_out_type, d);
    if (a.scales) {
      const float* s = a.scales + row * a.ld_scales + block;
      load_kept(reinterpret_cast<const uint8_t*>(x), s[0], c, a.cols, g);
      if (GATED) load_kept(reinterpret_cast<const uint8_t*>(x) + a.cols, s[in.a_row], c, a.cols, u);
    } else {
      load_run(x, c, a.cols, a.x_type, g);
      if (GATED) load_run(x + a.cols * xb, c, a.cols, a.x_type, u);
    }
    for (int i = 0; i < 8; ++i) {
      const Curve f = curve<ACT>(g[i]);
      g[i] = d[i] * f.slope;
      if (GATED) g[i] *= u[i], u[i] = d[i] * f.value;
    }
    char* to = static_cast<char*>(a.d_x) + row * a.ld_d_x * ob;
    store_run<NT>(to, c, a.cols, a.d_x_type, g);
    if (GATED) store_run<NT>(to + a.cols * ob, c, a.cols, a.d_x_type, u);
  }
}

template <class F>
hipError_t by_act(int act, bool gated, F&& f) {
  const auto by_gate = [&](auto kind) {
    return gated ? f(kind, std::integral_constant<bool, true>()) : f(kind, std::integral_constant<bool, false>());
  };
  if (act == WB_ACT_SILU) return by_gate(std::integral_constant<int, WB_ACT_SILU>());
  if (act == WB_ACT_GELU) return by_gate(std::integral_constant<int, WB_ACT_GELU>());
  return by_gate(std::integral_constant<int, WB_ACT_NONE>());
}

}  // namespace

int launch_activate(const ActivateArgs& a, void* stream) {
  if (a.rows == 0) return hipSuccess;
  const Units in = units_of(a.rows, a.cols);
  if (in.all >> 32) return hipErrorInvalidValue;
  return by_act(a.activation, a.gated, [&](auto act, auto gated) {
    const int64_t bytes = a.rows * a.cols * ((bytes_of(a.x_type) + (a.codes ? 1 : 0)) * (a.gated ? 2 : 1) + bytes_of(a.out_type));
    const auto kernel = bytes > kStreamBytes ? wb_activate_kernel<act(), gated(), true> : wb_activate_kernel<act(), gated(), false>;
    hipLaunchKernelGGL(kernel, dim3(blocks_of(in)), dim3(kThreads), 0, static_cast<hipStream_t>(stream), a, in);
    return hipGetLastError();
  });
}

int launch_activate_grad(const ActivateGradArgs& a, void* stream) {
  if (a.rows == 0) return hipSuccess;
  const Units in = units_of(a.rows, a.cols);
  if (in.all >> 32) return hipErrorInvalidValue;
  return by_act(a.activation, a.gated, [&](auto act, auto gated) {
    const int64_t bytes = a.rows * a.cols * ((bytes_of(a.x_type) + bytes_of(a.d_x_type)) * (a.gated ? 2 : 1) + bytes_of(a.d_out_type));
    const auto kernel =
        bytes > kStreamBytes ? wb_activate_grad_kernel<act(), gated(), true> : wb_activate_grad_kernel<act(), gated(), false>;
    hipLaunchKernelGGL(kernel, dim3(blocks_of(in)), dim3(kThreads), 0, static_cast<hipStream_t>(stream), a, in);
    return hipGetLastError();
  });
}

}  // namespace wb
