// Device helpers the operators' kernels share: rows of bf16 or fp32 read and
// written eight columns at a time, reductions over 16 lanes and over a
// wavefront, and the quotient of the fp8 quantiser.
#ifndef WB_OPS_DEVICE_HPP
#define WB_OPS_DEVICE_HPP

#include <hip/hip_runtime.h>

#include "../../include/wb.h"
#include "ops.hpp"

namespace wb {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ float bf16_to_f32(uint16_t v) { return __builtin_bit_cast(float, uint32_t(v) << 16); }

// Round to nearest even (v_cvt_pk_bf16_f32), NaN stays NaN.
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const f32x2 v = {lo, hi};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
}

// Four E4M3FN codes of |v| <= 448.00003 or NaN (v_cvt_pk_fp8_f32).
__device__ __forceinline__ uint32_t pack_fp8(float a, float b, float c, float d) {
  int p = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(c, d, p, true));
}

constexpr int64_t kStreamBytes = int64_t(128) << 20;  // from here on a launch's data goes past the caches

__host__ __device__ __forceinline__ int64_t bytes_of(int type) { return type == WB_F32 ? 4 : type == WB_BF16 ? 2 : 1; }

// One element of a row.
__device__ __forceinline__ float load_one(const void* row, int64_t col, int type) {
  return type == WB_F32 ? static_cast<const float*>(row)[col] : bf16_to_f32(static_cast<const uint16_t*>(row)[col]);
}

__device__ __forceinline__ void store_one(void* row, int64_t col, int type, float v) {
  if (type == WB_F32)
    static_cast<float*>(row)[col] = v;
  else
    static_cast<uint16_t*>(row)[col] = static_cast<uint16_t>(pack_bf16(v, 0.0f));
}

// Eight columns of a row, 16 bytes at a time. A row starts at any element
// address: the hardware takes vector accesses there, and the types below say
// so to the compiler.
typedef u32x4 u32x4_a2 __attribute__((aligned(2)));
typedef f32x4 f32x4_a4 __attribute__((aligned(4)));
typedef u32x2 u32x2_a1 __attribute__((aligned(1)));

// NT: with the non-temporal hint, for data that is touched once. (One function
// a type: a template parameter would lose the type's alignment.)
template <bool NT>
__device__ __forceinline__ f32x4 get_f4(const f32x4_a4* p) { return NT ? __builtin_nontemporal_load(p) : *p; }
template <bool NT>
__device__ __forceinline__ u32x4 get_u4(const u32x4_a2* p) { return NT ? __builtin_nontemporal_load(p) : *p; }
template <bool NT>
__device__ __forceinline__ void put_f4(f32x4_a4* p, f32x4 v) {
  if (NT)
    __builtin_nontemporal_store(v, p);
  else
    *p = v;
}
template <bool NT>
__device__ __forceinline__ void put_u4(u32x4_a2* p, u32x4 v) {
  if (NT)
    __builtin_nontemporal_store(v, p);
  else
    *p = v;
}
template <bool NT>
__device__ __forceinline__ void put_u2(u32x2_a1* p, u32x2 v) {
  if (NT)
    __builtin_nontemporal_store(v, p);
  else
    *p = v;
}

template <bool NT = false>
__device__ __forceinline__ void load_eight(const void* row, int64_t col, int type, float (&v)[8]) {
  if (type == WB_F32) {
    const auto* p = reinterpret_cast<const f32x4_a4*>(static_cast<const float*>(row) + col);
    const f32x4 a = get_f4<NT>(p), b = get_f4<NT>(p + 1);
    for (int i = 0; i < 4; ++i) v[i] = a[i], v[4 + i] = b[i];
  } else {
    const u32x4 a = get_u4<NT>(reinterpret_cast<const u32x4_a2*>(static_cast<const uint16_t*>(row) + col));
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __builtin_bit_cast(float, a[i] << 16);
      v[2 * i + 1] = __builtin_bit_cast(float, a[i] & 0xffff0000u);
    }
  }
}

// The columns from col on of a row that ends before col + 8, zeros past its
// end. A row of eight or more gives them as its last eight, moved down.
__device__ __forceinline__ void load_tail(const void* row, int64_t col, int64_t cols, int type, float (&v)[8]) {
  if (cols < 8) {
    for (int i = 0; i < 8; ++i) v[i] = col + i < cols ? load_one(row, col + i, type) : 0.0f;
    return;
  }
  load_eight(row, cols - 8, type, v);
  const int by = col >= cols ? 8 : static_cast<int>(col - (cols - 8));
#pragma unroll
  for (int bit = 4; bit > 0; bit >>= 1)
    for (int i = 0; i < 8; ++i) v[i] = (by & bit) ? (i + bit < 8 ? v[i + bit] : 0.0f) : v[i];
  for (int i = 0; i < 8; ++i) v[i] = by >= 8 ? 0.0f : v[i];
}

template <bool NT = false>
__device__ __forceinline__ void store_eight(void* row, int64_t col, int type, const float (&v)[8]) {
  if (type == WB_F32) {
    auto* p = reinterpret_cast<f32x4_a4*>(static_cast<float*>(row) + col);
    put_f4<NT>(p, f32x4{v[0], v[1], v[2], v[3]});
    put_f4<NT>(p + 1, f32x4{v[4], v[5], v[6], v[7]});
  } else {
    put_u4<NT>(reinterpret_cast<u32x4_a2*>(static_cast<uint16_t*>(row) + col),
               u32x4{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])});
  }
}

__device__ __forceinline__ void store_tail(void* row, int64_t col, int64_t cols, int type, const float (&v)[8]) {
  for (int i = 0; i < 8; ++i)
    if (col + i < cols) store_one(row, col + i, type, v[i]);
}

// Eight columns of a row that may end before the eighth.
template <bool NT = false>
__device__ __forceinline__ void load_run(const char* row, int64_t c, int64_t cols, int type, float (&v)[8]) {
  if (c + 8 <= cols)
    load_eight<NT>(row, c, type, v);
  else
    load_tail(row, c, cols, type, v);
}

template <bool NT = false>
__device__ __forceinline__ void store_run(char* row, int64_t c, int64_t cols, int type, const float (&v)[8]) {
  if (c + 8 <= cols)
    store_eight<NT>(row, c, type, v);
  else
    store_tail(row, c, cols, type, v);
}

// Lanes of a workgroup of 256 over rows: 1 << row_shift lanes hold a row's runs
// of eight columns, wider rows all of them.
inline int row_shift(int64_t cols) {
  int shift = 3;
  while (shift < 8 && (int64_t(8) << shift) < cols) ++shift;
  return shift;
}

// Whether a launch takes as many workgroups of 256: it has fewer than 2^32 threads.
inline bool one_launch(int64_t blocks) { return blocks < (int64_t(1) << 24); }

// Four neighbouring columns.
typedef u32x2 u32x2_a2 __attribute__((aligned(2)));

__device__ __forceinline__ void load_four(const void* row, int64_t col, int type, float (&v)[4]) {
  if (type == WB_F32) {
    const f32x4 f = *reinterpret_cast<const f32x4_a4*>(static_cast<const float*>(row) + col);
    for (int r = 0; r < 4; ++r) v[r] = f[r];
  } else {
    const u32x2 u = *reinterpret_cast<const u32x2_a2*>(static_cast<const uint16_t*>(row) + col);
    for (int r = 0; r < 4; ++r) v[r] = __builtin_bit_cast(float, (r & 1) ? u[r >> 1] & 0xffff0000u : u[r >> 1] << 16);
  }
}

__device__ __forceinline__ void store_four(void* row, int64_t col, int type, const float (&v)[4]) {
  if (type == WB_F32)
    *reinterpret_cast<f32x4_a4*>(static_cast<float*>(row) + col) = f32x4{v[0], v[1], v[2], v[3]};
  else
    *reinterpret_cast<u32x2_a2*>(static_cast<uint16_t*>(row) + col) = u32x2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
}

// The sixteen lanes of a row, turned by N: every lane gets the result of a
// reduction after N = 8, 4, 2, 1, in vector instructions alone.
template <int N, class T>
__device__ __forceinline__ T turned16(T v) {
  const int i = __builtin_bit_cast(int, v);
  return __builtin_bit_cast(T, __builtin_amdgcn_update_dpp(i, i, 0x120 + N, 0xf, 0xf, false));
}

template <class T, class Op>
__device__ __forceinline__ T reduce16(T v, Op op) {
  v = op(v, turned16<8>(v));
  v = op(v, turned16<4>(v));
  v = op(v, turned16<2>(v));
  return op(v, turned16<1>(v));
}

// Between writes to LDS and reads of them by other lanes of the wavefront:
// the hardware keeps their order, this keeps the compiler to it.
__device__ __forceinline__ void order_lanes() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); }

__device__ __forceinline__ float sum_of_wave(float v) {
  for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off);
  return v;
}

// exp(x) of x <= 0 as 2^n 2^f, x log2 e = n + f with the constant in two parts:
// f is off by a rounding of a number of at most a half, so that the
// instruction's unit is nearly all that the result is off by.
__device__ __forceinline__ float exp_below(float x) {
  x = x < -150.0f ? -150.0f : x;  // 0; NaN stays
  const float n = __builtin_rintf(x * 1.44269502f);
  const float f = __builtin_fmaf(x, 1.92596299e-8f, __builtin_fmaf(x, 1.44269502f, -n));
  return __builtin_ldexpf(__builtin_amdgcn_exp2f(f), static_cast<int>(n));
}

struct Sum {
  __device__ __forceinline__ float operator()(float a, float b) const { return a + b; }
};

struct IMin {
  __device__ __forceinline__ int operator()(int a, int b) const { return min(a, b); }
};

struct FMax {
  __device__ __forceinline__ float operator()(float a, float b) const { return fmaxf(a, b); }
};

// The scale of values whose largest magnitude is amax, as the weight
// quantiser's: amax / 448 in IEEE fp32, and 1 where that is zero. NaN values
// are left out of amax (fmaxf) and become NaN codes.
struct RowScale {
  float s, r;
  bool near;  // 1 / s and the remainders below stay inside the normal range
};

__device__ __forceinline__ RowScale row_scale(float amax) {
  RowScale q;
  q.s = amax / 448.0f;
  if (!(q.s > 0.0f)) q.s = 1.0f;
  q.r = 1.0f / q.s;
  q.near = q.s > 0x1p-90f && q.s < 0x1p90f;
  return q;
}

// v / s rounded to fp32: one product, its remainder, one correction. A scale
// among the smallest numbers can be rounded down by a third, so quotients of
// such a one are held to what E4M3 has (a NaN stays one).
template <int N>
__device__ __forceinline__ void quotients(float (&v)[N], const RowScale& q) {
  if (q.near) {
    for (int i = 0; i < N; ++i) {
      const float a = v[i] * q.r;
      v[i] = __builtin_fmaf(__builtin_fmaf(-a, q.s, v[i]), q.r, a);
    }
  } else {
    for (int i = 0; i < N; ++i) {
      v[i] /= q.s;
      if (fabsf(v[i]) > 448.0f) v[i] = __builtin_copysignf(448.0f, v[i]);
    }
  }
}

}  // namespace wb

#endif
