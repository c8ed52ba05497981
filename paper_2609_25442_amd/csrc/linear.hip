// Products of activations with a rollout rank's weights, as they lie after
// unpacking: plain [n, k] or stacked [experts, n, k], bf16, or fp8 E4M3 with
// an fp32 scale per 128x128 block (activations: one per row and 128 columns).
//
//   z = x W^T + bias     fp8: z = sum over blocks b of k of
//                             (sum_{i in b} qx_i qw_i) sx_b sw_b
//   gated (W = [gate; up]): a = act(z_gate) z_up, else a = act(z)
//   out = a + residual   in bf16, fp32, or fp8 with a scale per 128 columns
//
// fp8 codes are widened to bf16 (exactly) on their way to the matrix cores;
// the sums of a block are scaled and added in fp32.
#include <algorithm>
#include <atomic>
#include <cmath>
#include <type_traits>

#include "ops_device.hpp"

namespace wb {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef u32x4 u32x4_a1 __attribute__((aligned(1)));
typedef uint32_t u32_a1 __attribute__((aligned(1)));

constexpr int kStageBytes = 128;  // of a row, per step over k: a scale block of fp8, half as many bf16

// Sixteen zero bytes: what a tile's 16-byte pieces and scales past the end of k are read from.
__device__ const u32x4 zero_piece = {0, 0, 0, 0};

// z / (1 + e^-z) by way of t = e^-|z|, which neither overflows nor takes its
// relative precision from a large sum: 1 / (1 + t) for z >= 0, t / (1 + t) below,
// the reciprocal with one correction. Within nine half units of fp32.
__device__ __forceinline__ float silu(float z) {
  const float t = exp_below(-fabsf(z)), d = 1.0f + t;
  float r = __builtin_amdgcn_rcpf(d);
  r = __builtin_fmaf(__builtin_fmaf(-d, r, 1.0f), r, r);
  return (z < 0.0f ? z * t : z) * r;
}
// The same for a bf16 result, whose half unit is 2^-9: the argument of e^ is
// rounded once (2^-24 of itself, so 2^-17.5 of the result at most where that is
// not below 2^-120), a third of the instructions (8192 rows, 28672 x 4096 bf16, gated:
// 20 us of 1480).
__device__ __forceinline__ float silu_to_bf16(float z) { return z * __builtin_amdgcn_rcpf(1.0f + __expf(-z)); }
// 1 + erf loses relative precision far below zero, where the result is small:
// it is off by roundings of z, as the same formula in elementary operations is.
__device__ __forceinline__ float gelu(float z) { return 0.5f * z * (1.0f + erff(z * 0.70710678118654752f)); }

__device__ __forceinline__ void activate(float (&v)[4], int kind, int out_type) {
  if (kind == WB_ACT_GELU) {
    for (int e = 0; e < 4; ++e) v[e] = gelu(v[e]);
  } else if (kind == WB_ACT_SILU) {
    if (out_type == WB_BF16) {
      for (int e = 0; e < 4; ++e) v[e] = silu_to_bf16(v[e]);
    } else {
      for (int e = 0; e < 4; ++e) v[e] = silu(v[e]);
    }
  }
}

// The rows of the output that tile `mt` of `per` rows covers, and their expert.
struct RowTile {
  int64_t first, end;  // end: of the expert's rows
  int expert;
};

// Tiles are counted over the experts in order, each starting anew; every
// wavefront scans the offsets, sixty-four experts at a time. False where the
// launch has more tiles than the rows fill.
__device__ __forceinline__ bool find_rows(const LinearArgs& a, int64_t mt, int per, RowTile& t) {
  if (!a.offsets) {
    t = RowTile{mt * per, a.rows, 0};
    return t.first < t.end;
  }
  const int lane = threadIdx.x & 63, rows = static_cast<int>(a.rows);
  int before = 0;
  for (int base = 0; base < a.num_experts; base += 64) {
    const int e = base + lane;
    int lo = 0, hi = 0;
    if (e < a.num_experts) {
      lo = min(max(a.offsets[e], 0), rows);
      hi = min(max(a.offsets[e + 1], lo), rows);
    }
    const int tiles = (hi - lo + per - 1) / per;
    int upto = tiles;
    for (int off = 1; off < 64; off <<= 1) {
      const int add = __shfl_up(upto, off);
      upto += lane >= off ? add : 0;
    }
    const int all = __builtin_amdgcn_readlane(upto, 63);
    if (mt < before + all) {
      const int src = __builtin_ctzll(__ballot(mt < before + upto));
      const int in = static_cast<int>(mt) - before - (__builtin_amdgcn_readlane(upto, src) - __builtin_amdgcn_readlane(tiles, src));
      t.expert = base + src;
      t.first = int64_t(__builtin_amdgcn_readlane(lo, src)) + int64_t(in) * per;
      t.end = __builtin_amdgcn_readlane(hi, src);
      return true;
    }
    before += all;
  }
  return false;
}

// The row of x behind row m of the output.
__device__ __forceinline__ int64_t x_row(const LinearArgs& a, int64_t m) {
  if (!a.tokens) return m;
  return min(max(int64_t(a.tokens[m]), int64_t(0)), a.x_rows - 1);
}

// The weight's row r of a tile that starts at output column `col`: plain
// tiles are rows in order, gated ones sixteen gate rows, then the sixteen up
// rows of the same columns. Rows past the end repeat the last one.
__device__ __forceinline__ int w_row(const LinearArgs& a, int col, int r) {
  if (!a.gated) return min(col + r, a.n - 1);
  const int o = min(col + ((r >> 5) << 4) + (r & 15), a.n_out - 1);
  return o + ((r >> 4) & 1) * a.n_out;
}

__device__ __forceinline__ float load_bias(const LinearArgs& a, int expert, int row) {
  return load_one(a.bias, expert * a.stride_bias + row, a.bias_type);
}

// 16 bytes of a row of `bytes` bytes at `at`; zeros past its end. Rows start
// anywhere. A row's last piece is its last 16 bytes moved down.
__device__ __forceinline__ u32x4 load_piece(const uint8_t* row, int64_t at, int64_t bytes) {
  if (at + 16 <= bytes) return *reinterpret_cast<const u32x4_a1*>(row + at);
  u32x4 v = {0, 0, 0, 0};
  if (at >= bytes) return v;
  if (bytes >= 16) {
    v = *reinterpret_cast<const u32x4_a1*>(row + bytes - 16);
    const int by = static_cast<int>(at + 16 - bytes) * 8;  // bits to drop, 8..120
    uint64_t lo = uint64_t(v[1]) << 32 | v[0], hi = uint64_t(v[3]) << 32 | v[2];
    if (by >= 64) {
      lo = hi >> (by - 64);
      hi = 0;
    } else {
      lo = lo >> by | hi << (64 - by);
      hi >>= by;
    }
    return u32x4{uint32_t(lo), uint32_t(lo >> 32), uint32_t(hi), uint32_t(hi >> 32)};
  }
  for (int i = 0; i < 16; ++i)
    if (at + i < bytes) v[i >> 2] |= uint32_t(row[at + i]) << (8 * (i & 3));
  return v;
}

// Four neighbouring columns of a row as they lie in memory, and as numbers; in:
// how many of them exist.
__device__ __forceinline__ u32x4 fetch_four(const void* base, int64_t at, int type, int in) {
  u32x4 v = {0, 0, 0, 0};
  const auto* wide = static_cast<const float*>(base) + at;
  const auto* half = static_cast<const uint16_t*>(base) + at;
  if (in >= 4) {
    if (type == WB_F32) return __builtin_bit_cast(u32x4, *reinterpret_cast<const f32x4_a4*>(wide));
    const u32x2 u = *reinterpret_cast<const u32x2_a2*>(half);
    return u32x4{u[0], u[1], 0, 0};
  }
  for (int r = 0; r < 4; ++r) {
    if (r >= in) continue;
    if (type == WB_F32)
      v[r] = __builtin_bit_cast(uint32_t, wide[r]);
    else
      v[r >> 1] |= uint32_t(half[r]) << (16 * (r & 1));
  }
  return v;
}

__device__ __forceinline__ float of_four(const u32x4& u, int type, int r) {
  return __builtin_bit_cast(float, type == WB_F32 ? u[r] : r & 1 ? u[r >> 1] & 0xffff0000u : u[r >> 1] << 16);
}

__device__ __forceinline__ void store_four(void* base, int64_t at, int type, int in, const float (&v)[4]) {
  if (type == WB_F8E4M3) {
    const uint32_t p = pack_fp8(v[0], v[1], v[2], v[3]);
    auto* to = static_cast<uint8_t*>(base) + at;
    if (in >= 4)
      *reinterpret_cast<u32_a1*>(to) = p;
    else
      for (int r = 0; r < in; ++r) to[r] = static_cast<uint8_t>(p >> (8 * r));
  } else if (in >= 4) {
    wb::store_four(base, at, type, v);
  } else {
    for (int r = 0; r < in; ++r) store_one(base, at + r, type, v[r]);
  }
}

__device__ __forceinline__ float largest(const float (&v)[4], int in_row, float top) {
  for (int r = 0; r < 4; ++r)
    if (r < in_row) top = fmaxf(top, fabsf(v[r]));
  return top;
}

// One 16x16 block of sums: the weight's rows down, tokens across (lane l
// holds token l % 16 and rows 4 (l / 16) ..+3).
__device__ __forceinline__ f32x4 mfma(bf16x8 w, bf16x8 x, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, x, c, 0, 0, 0);
}

// A lane's 32 bytes of a row and stage as operands: two of bf16, or four of
// fp8 codes as the same numbers in bf16. The fp8 instructions are not used:
// they drop what lies 14 bits below the largest of each eight products
// (measured: 2e-6 of the sum of magnitudes on average, 2e-5 at worst, of 128
// normal values), while products of bf16 are summed like fp32.
template <bool F8>
struct Operand {
  bf16x8 v[F8 ? 4 : 2];
  Operand() = default;
  __device__ __forceinline__ Operand(i32x4 a, i32x4 b) {
    if constexpr (F8) {
      v[0] = widen(a[0], a[1]), v[1] = widen(a[2], a[3]), v[2] = widen(b[0], b[1]), v[3] = widen(b[2], b[3]);
    } else {
      v[0] = __builtin_bit_cast(bf16x8, a), v[1] = __builtin_bit_cast(bf16x8, b);
    }
  }
  __device__ __forceinline__ static bf16x8 widen(int a, int b) {
    const bf16x2 p = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.0f, false), q = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.0f, true);
    const bf16x2 r = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, false), s = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, true);
    return bf16x8{p[0], p[1], q[0], q[1], r[0], r[1], s[0], s[1]};
  }
};

// The same rows of the weight against M blocks of tokens: the sums of one
// block depend on each other, those of different blocks do not.
template <bool F8, int M>
__device__ __forceinline__ void block_sums(const Operand<F8>& w, const Operand<F8>* x, f32x4* c) {
#pragma unroll
  for (int h = 0; h < (F8 ? 4 : 2); ++h)
#pragma unroll
    for (int j = 0; j < M; ++j) c[j] = mfma(w.v[h], x[j].v[h], c[j]);
}

// A workgroup's tile: BM rows of the output by BN rows of the weight, WM x WN
// wavefronts. LDS holds a ring of RING slots of STEP stages of every row of
// both; a barrier stands between slots, so small tiles take more stages at
// once, and KG such sets of wavefronts share them out (their sums meet in LDS
// at the end, in order). The pieces of a row are permuted by its number so
// that sixteen rows' pieces at one place of k fall into different banks.
template <int BM_, int BN_, int WM_, int WN_, int KG_, int STEP_, int RING_>
struct Shape {
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, KG = KG_, STEP = STEP_, RING = RING_;
  static constexpr int kThreads = 64 * WM * WN * KG, TM = BM / WM, TN = BN / WN, FM = TM / 16, FN = TN / 16;
  static constexpr int kRows = BM + BN, kStage = kRows * kStageBytes;
  // behind the slots: for each, the scales of its stages' rows, of x and then
  // of the weight; the epilogue's maxima lie over them
  static constexpr int kSlot = STEP * kStage, kRounds = (STEP * kRows + kThreads - 1) / kThreads;
  static constexpr int kScales = kRounds * kThreads * 4, kLds = RING * (kSlot + kScales);
  static_assert(kLds <= 160 * 1024, "");
  static_assert(WN * BM * 4 <= RING * kScales, "maxima fit");
  static_assert((KG - 1) * BM * BN * 4 <= RING * kSlot, "the ring holds the groups' sums");
  static_assert(kRows * STEP * 8 % kThreads == 0 && kRows % 16 == 0 && STEP % KG == 0, "the pieces share out evenly");
};

__device__ __forceinline__ int swizzle(int row) { return (row >> 1) & 7; }

// F8: fp8 operands, else bf16. DIRECT: rows start at multiples of 16 bytes and
// hold a multiple of 16, and the sixteen rows of a block share a weight
// scale: tiles go from memory to LDS without registers between. Otherwise
// through registers, piece by piece, and scales by row.
//
// What bounds it, as measured (rates of a large copy and of a large bf16
// product on this card: 6.7 TB/s, 1.54 PFLOP/s):
//   8192 rows, 28672 x 4096 bf16, gated    1.50 ms, 1.28 PFLOP/s: the matrix
//     cores, 62 % of the cycles (the rest: barriers, operands from LDS)
//   4096 rows, 7168 x 2048 fp8, and 8192 of 32 experts' 4096 x 7168, gated:
//     0.135 and 0.67 ms, 0.89 and 0.72 PFLOP/s: widening (in every wavefront that
//     reads a code, so two or three times) and scaling in the vector units,
//     beside matrix cores busy 38 to 40 %
//   128 rows of the same 32 experts: 0.18 ms, the weight's bytes at 5.3 TB/s
//   1 row, 6144 x 4096 bf16: 10 us, 5.0 TB/s with the launch and the call
//   333 rows, 3442 x 1500 bf16, by way of registers: 18 us; 14 were the rows
//     1504 long and on the 16-byte grid
template <class S, bool F8, bool DIRECT>
__global__ __launch_bounds__(S::kThreads, 2) void wb_linear_tile_kernel(LinearArgs a, uint32_t tiles_n, uint32_t group) {
  extern __shared__ __align__(128) uint8_t lds[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int kg = wave / (S::WM * S::WN), wm = wave / S::WN % S::WM, wn = wave % S::WN;
  const int l15 = lane & 15, quad = lane >> 4;

  // tiles of `group` neighbouring row tiles side by side, so that the rows of
  // the weight they share are read while they are in cache; neighbouring
  // tiles on one XCD
  const uint32_t xcd = blockIdx.x % 8, each = gridDim.x / 8, more = gridDim.x % 8;
  const uint32_t id = xcd * each + min(xcd, more) + blockIdx.x / 8;
  const uint32_t tiles_m = gridDim.x / tiles_n;
  const uint32_t g0 = id / (group * tiles_n) * group, gm = min(group, tiles_m - g0);
  const uint32_t in = id - g0 * tiles_n;
  RowTile rows;
  if (!find_rows(a, g0 + in % gm, S::BM, rows)) return;
  const int step_out = a.gated ? S::BN / 2 : S::BN;
  const int col0 = static_cast<int>(in / gm) * step_out;
  const int64_t k_bytes = F8 ? int64_t(a.k) : 2 * int64_t(a.k);
  const int stages = static_cast<int>((k_bytes + kStageBytes - 1) / kStageBytes);
  const uint8_t* weight = a.weight + rows.expert * a.stride_w_bytes;

  // sources of the tile's pieces: a row of the weight or of x
  auto row_of = [&](int r) {
    return r < S::BN ? weight + int64_t(w_row(a, col0, r)) * a.ld_w_bytes
                     : a.x + x_row(a, min(rows.first + (r - S::BN), rows.end - 1)) * a.ld_x_bytes;
  };
  constexpr int kWaves = S::kThreads / 64, kPieces = S::kRows * S::STEP * 8 / S::kThreads;  // per lane and step
  static_assert(kWaves % 2 == 0, "the pieces of a lane are permuted alike");
  const int piece = ((lane & 7) ^ swizzle(wave * 8 + (lane >> 3))) * 16;
  // DIRECT keeps a piece as its 32-bit offset from the weight or from x (the
  // tile's first row, where rows are not gathered), which the loads add to an
  // address that is the same for the wavefront; the launch sees to its range
  const uint8_t* const x_base = a.tokens ? a.x : a.x + rows.first * a.ld_x_bytes;
  const uint8_t* src[DIRECT ? 1 : kPieces];
  uint32_t off[DIRECT ? kPieces : 1];
  constexpr bool kApart = S::STEP == 1 && S::BN % (kWaves * 8) == 0;  // the weight's pieces come first, in every wavefront
  auto of_weight = [&](int i) { return kApart ? i * kWaves * 8 < S::BN : (wave + i * kWaves) * 8 % S::kRows < S::BN; };
#pragma unroll
  for (int i = 0; i < kPieces; ++i) {
    const int r = (wave + i * kWaves) * 8;  // of the step's rows; its stage is the same for the wavefront
    const uint8_t* from = row_of(r % S::kRows + (lane >> 3)) + r / S::kRows * kStageBytes;
    if constexpr (DIRECT)
      off[i] = static_cast<uint32_t>(from - (of_weight(i) ? weight : x_base)) + piece;
    else
      src[i] = from;
  }
  // scales: a row of x, then of the weight, per thread and round
  const float* scale_src[S::kRounds];
  // otherwise two steps' pieces and scales are in registers on their way
  struct Held {
    u32x4 piece[DIRECT ? 1 : kPieces];
    float scale[S::kRounds];
  };
  uint8_t* const scales = lds + S::RING * S::kSlot;
  if constexpr (F8) {
#pragma unroll
    for (int i = 0; i < S::kRounds; ++i) {
      const int g = min(tid + i * S::kThreads, S::STEP * S::kRows - 1), r = g % S::kRows;
      scale_src[i] = r < S::BM ? a.x_scales + x_row(a, min(rows.first + r, rows.end - 1)) * a.ld_xs
                               : a.weight_scales + rows.expert * a.stride_ws +
                                     int64_t(w_row(a, col0, r - S::BM) / kScaleBlock) * a.ld_ws;
    }
  }

  // the scale of a step that thread and round have to bring; zero of a stage past
  // the end, whose sums are zeros (an infinite scale would make them NaN)
  auto scale_at = [&](int t, int i) -> const float* {
    if constexpr (S::STEP == 1) return scale_src[i] + t;
    const int stage = t * S::STEP + min(tid + i * S::kThreads, S::STEP * S::kRows - 1) / S::kRows;
    return stage < stages ? scale_src[i] + stage : reinterpret_cast<const float*>(&zero_piece);
  };
  auto send_scales = [&](int t, int slot) {
    if constexpr (F8) {
#pragma unroll
      for (int i = 0; i < S::kRounds; ++i)
        __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)scale_at(t, i),
                                         (__attribute__((address_space(3))) void*)(scales + slot * S::kScales + (wave * 64 + i * S::kThreads) * 4),
                                         4, 0, 0);
    }
  };
  auto send = [&](const uint8_t* p, int slot, int i) {
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)p,
                                     (__attribute__((address_space(3))) void*)(lds + slot * S::kSlot + (wave + i * kWaves) * 1024), 16, 0, 0);
  };
  struct At {  // where a step lies in every row
    const uint8_t *weight, *x;
  };
  auto step_at = [&](int t) {
    return At{weight + int64_t(t) * (S::STEP * kStageBytes), x_base + int64_t(t) * (S::STEP * kStageBytes)};
  };
  // piece i of a step that lies within k
  auto send_whole = [&](const At& at, int slot, int i) {
    if constexpr (DIRECT) send((of_weight(i) ? at.weight : at.x) + off[i], slot, i);
  };
  // start step t's stages on their way into a slot of the ring; stages past
  // the end are zeros
  auto fetch = [&](int t, int slot) {
    if constexpr (DIRECT) {
      send_scales(t, slot);
      const At from = step_at(t);
      if ((t + 1) * int64_t(S::STEP * kStageBytes) <= k_bytes) {
#pragma unroll
        for (int i = 0; i < kPieces; ++i) send_whole(from, slot, i);
      } else {
        const int64_t at = int64_t(t) * (S::STEP * kStageBytes) + piece;
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
          const int64_t in_row = at + (wave + i * kWaves) * 8 / S::kRows * kStageBytes;
          const uint8_t* p = (of_weight(i) ? from.weight : from.x) + off[i];
          send(in_row < k_bytes ? p : reinterpret_cast<const uint8_t*>(&zero_piece), slot, i);
        }
      }
    }
  };
  // the same by way of registers
  auto take = [&](int t, Held& held) {
    if constexpr (!DIRECT) {
      const int64_t at = int64_t(t) * (S::STEP * kStageBytes) + piece;
      if ((t + 1) * int64_t(S::STEP * kStageBytes) <= k_bytes) {
#pragma unroll
        for (int i = 0; i < kPieces; ++i) held.piece[i] = *reinterpret_cast<const u32x4_a1*>(src[i] + at);
      } else {
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
          const int stage = (wave + i * kWaves) * 8 / S::kRows * kStageBytes;
          held.piece[i] = load_piece(src[i] - stage, at + stage, k_bytes);
        }
      }
      if constexpr (F8) {
#pragma unroll
        for (int i = 0; i < S::kRounds; ++i) held.scale[i] = *scale_at(t, i);
      }
    }
  };
  auto put = [&](const Held& held, int slot) {
    if constexpr (!DIRECT) {
      uint8_t* to = lds + slot * S::kSlot + wave * 1024 + lane * 16;
#pragma unroll
      for (int i = 0; i < kPieces; ++i) *reinterpret_cast<u32x4*>(to + i * kWaves * 1024) = held.piece[i];
      if constexpr (F8) {
#pragma unroll
        for (int i = 0; i < S::kRounds; ++i)
          *reinterpret_cast<float*>(scales + slot * S::kScales + (tid + i * S::kThreads) * 4) = held.scale[i];
      }
    }
  };

  f32x4 acc[S::FN][S::FM];
#pragma unroll
  for (int i = 0; i < S::FN; ++i)
#pragma unroll
    for (int j = 0; j < S::FM; ++j) acc[i][j] = f32x4{0, 0, 0, 0};

  const int frag = l15 * kStageBytes + ((quad ^ swizzle(l15)) << 4);
  const int w_frag = wn * S::TN * kStageBytes + frag, x_frag = (S::BN + wm * S::TM) * kStageBytes + frag;

  const int steps = (stages + S::STEP - 1) / S::STEP;

  // the products of the stages in a slot, `between` in front of each block of
  // sixteen rows of the weight
  auto compute = [&](int slot, auto&& between) {
#pragma unroll
    for (int h = 0; h < S::STEP / S::KG; ++h) {
    const int stage = h * S::KG + kg;
    const uint8_t* buf = lds + slot * S::kSlot + stage * S::kStage;
    const float* sc = reinterpret_cast<const float*>(scales + slot * S::kScales) + stage * S::kRows;
    auto operand = [&](int at) {
      return Operand<F8>(*reinterpret_cast<const i32x4*>(buf + at), *reinterpret_cast<const i32x4*>(buf + (at ^ 64)));
    };
    constexpr int kTogether = S::FM < 2 ? 1 : 2;  // chains of products that do not wait for each other
    Operand<F8> x[S::FM];
    float sx[S::FM];
#pragma unroll
    for (int j = 0; j < S::FM; ++j) {
      x[j] = operand(x_frag + j * 16 * kStageBytes);
      if constexpr (F8) sx[j] = sc[wm * S::TM + j * 16 + l15];
    }
#pragma unroll
    for (int i = 0; i < S::FN; ++i) {
      between(h * S::FN + i);
      const Operand<F8> w = operand(w_frag + i * 16 * kStageBytes);
      if constexpr (F8) {
        const float* sw = sc + S::BM + wn * S::TN + i * 16;
        const f32x4 sr = DIRECT ? f32x4{sw[0], sw[0], sw[0], sw[0]} : *reinterpret_cast<const f32x4*>(sw + quad * 4);
#pragma unroll
        for (int j0 = 0; j0 < S::FM; j0 += kTogether) {
          f32x4 part[kTogether];
#pragma unroll
          for (int j = 0; j < kTogether; ++j) part[j] = f32x4{0, 0, 0, 0};
          block_sums<F8, kTogether>(w, x + j0, part);
#pragma unroll
          for (int j = 0; j < kTogether; ++j) {
            f32x4& to = acc[i][j0 + j];
            if constexpr (DIRECT) {
              const float both = sx[j0 + j] * sr[0];
              for (int r = 0; r < 4; ++r) to[r] = __builtin_fmaf(part[j][r], both, to[r]);
            } else {
              for (int r = 0; r < 4; ++r) to[r] = __builtin_fmaf(part[j][r], sx[j0 + j] * sr[r], to[r]);
            }
          }
        }
      } else {
        block_sums<F8, S::FM>(w, x, acc[i]);
      }
    }
    }
  };
  if constexpr (DIRECT) {
    constexpr int kBlocks = S::STEP / S::KG * S::FN;                    // calls of `between`
    constexpr int kAhead = S::RING - 1;                                 // steps in flight
    constexpr int kLoads = kPieces + (F8 ? S::kRounds : 0);             // of a wavefront and step
    static_assert((kAhead - 1) * kLoads < 64, "the counter of loads in flight");
    auto next = [](int slot, int by) { return slot + by >= S::RING ? slot + by - S::RING : slot + by; };
    int slot = 0, t = 0;
    for (int i = 0; i < min(kAhead, steps); ++i) fetch(i, i);
    // As long as the step to fetch lies within k, its loads go out one by one
    // between the products: issued together, they hold up the matrix cores
    // (8192 x 8192 x 8192 bf16: 10 % of the time).
    const int whole_steps = static_cast<int>(k_bytes / (S::STEP * kStageBytes));
    for (; t + kAhead < whole_steps; ++t) {
      // after this, step t is in LDS for every wavefront, and the step before
      // it has been read by all: its slot can be filled
      asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((kAhead - 1) * kLoads) : "memory");
      const int to = next(slot, kAhead);
      const At from = step_at(t + kAhead);
      send_scales(t + kAhead, to);
      compute(slot, [&](int block) {
#pragma unroll
        for (int i = 0; i < kPieces; ++i)
          if (i * kBlocks / kPieces == block) send_whole(from, to, i);
      });
      slot = next(slot, 1);
    }
    for (; t < steps; ++t) {
      if (t + kAhead <= steps)
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((kAhead - 1) * kLoads) : "memory");
      else
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
      if (t + kAhead < steps) fetch(t + kAhead, next(slot, kAhead));
      compute(slot, [](int) {});
      slot = next(slot, 1);
    }
  } else {
    // step t is in slot t % 2, step t + 1 in registers when the barrier in
    // front of step t is passed, and step t + 2 then sets out
    Held even, odd;
    auto one = [&](int t, const Held& ready, Held& free) {
      asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
      if (t + 2 < steps) take(t + 2, free);
      compute(t & 1, [](int) {});
      if (t + 1 < steps) put(ready, (t + 1) & 1);
    };
    take(0, even);
    if (steps > 1) take(1, odd);
    put(even, 0);
    for (int t = 0; t < steps; t += 2) {
      one(t, odd, even);
      if (t + 1 < steps) one(t + 1, even, odd);
    }
  }

  // epilogue, sixteen rows at a time through LDS: a wavefront puts its sums
  // down by row and takes them up again four neighbouring columns per lane, a
  // row by neighbouring lanes, which is also how they are stored
  constexpr int kPitch = S::TN + 4;  // floats
  static_assert(S::WM * S::WN * 16 * kPitch * 4 <= S::RING * S::kSlot, "the ring holds the sums");
  float* const mine = reinterpret_cast<float*>(lds) + wave % (S::WM * S::WN) * 16 * kPitch;
  float* const tops = reinterpret_cast<float*>(scales);
  const int cols = a.gated ? S::TN / 2 : S::TN, lanes = cols / 4, span = kScaleBlock / cols;
  const int wave_col = col0 + wn * cols, c = lane % lanes * 4, per = 64 / lanes, col = wave_col + c;
  const int at = a.gated ? (c >> 4) * 32 + (c & 15) : c;
  const int in_row = a.n_out - col, first_r = kg == 0 ? lane / lanes : 16;
  const bool f8_out = a.out_type == WB_F8E4M3;
  const int64_t m0 = rows.first + wm * S::TM;
  const int there = static_cast<int>(min(rows.end - m0, int64_t(S::TM)));  // rows of the wavefront that exist
  float bias[4] = {0, 0, 0, 0}, bias_up[4] = {0, 0, 0, 0};
  if (a.bias && in_row > 0) {
    for (int e = 0; e < 4; ++e) {
      const int b = min(col + e, a.n_out - 1);
      bias[e] = load_bias(a, rows.expert, b);
      if (a.gated) bias_up[e] = load_bias(a, rows.expert, a.n_out + b);
    }
  }
  // The residual's loads are some of the lane's rows ahead, and in front
  // of the stores: a wait for loads is one for the stores before them as well
  // (4096 rows by 7168 x 2048 fp8: 133 us, 142 with the loads in between).
  auto residual_of = [&](int j, int r) {
    return fetch_four(a.residual, (m0 + min(j * 16 + r, there - 1)) * a.ld_residual + col, a.residual_type, in_row);
  };
  constexpr int kAhead = S::FN > 4 ? 2 : S::FN;  // more spill, of the largest tile
  u32x4 add[kAhead];
  if (a.residual && there > 0) {
#pragma unroll
    for (int h = 0; h < kAhead; ++h)
      if (first_r + h * per < 16) add[h] = residual_of(0, first_r + h * per);
  }

  if constexpr (S::KG > 1) {
    float* const sums = reinterpret_cast<float*>(lds);
    const int own = (wave % (S::WM * S::WN) * S::FN * S::FM) * 256 + lane * 4;
    __syncthreads();
    if (kg > 0) {
#pragma unroll
      for (int i = 0; i < S::FN; ++i)
#pragma unroll
        for (int j = 0; j < S::FM; ++j)
          *reinterpret_cast<f32x4*>(sums + (kg - 1) * S::BM * S::BN + own + (i * S::FM + j) * 256) = acc[i][j];
    }
    __syncthreads();
    if (kg == 0) {
#pragma unroll
      for (int i = 0; i < S::FN; ++i)
#pragma unroll
        for (int j = 0; j < S::FM; ++j)
          for (int g = 0; g < S::KG - 1; ++g) {
            const f32x4 more = *reinterpret_cast<const f32x4*>(sums + g * S::BM * S::BN + own + (i * S::FM + j) * 256);
            for (int r = 0; r < 4; ++r) acc[i][j][r] += more[r];
          }
    }
  }

  auto finish_rows = [&](int j, auto with_residual) {
#pragma unroll
    for (int h = 0; h < S::FN; ++h) {
      const int r = first_r + h * per;
      if (r >= 16) break;
      const int in = j * 16 + r < there ? in_row : 0;
      float* p = mine + r * kPitch + at;
      const f32x4 g = *reinterpret_cast<const f32x4*>(p);
      float v[4];
      for (int e = 0; e < 4; ++e) v[e] = g[e] + bias[e];
      activate(v, a.activation, a.out_type);
      if (a.gated) {
        const f32x4 u = *reinterpret_cast<const f32x4*>(p + 16);
        for (int e = 0; e < 4; ++e) v[e] *= u[e] + bias_up[e];
      }
      if constexpr (with_residual) {
        u32x4& of_row = add[h % kAhead];
        for (int e = 0; e < 4; ++e) v[e] += of_four(of_row, a.residual_type, e);
        if (r + kAhead * per < 16)
          of_row = residual_of(j, r + kAhead * per);
        else if (j + 1 < S::FM)
          of_row = residual_of(j + 1, first_r + h % kAhead * per);
      }
      if (f8_out) {
        *reinterpret_cast<f32x4*>(p) = f32x4{v[0], v[1], v[2], v[3]};
        float top = largest(v, in, 0.0f);
        for (int off = lanes / 2; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor(top, off));
        if (c == 0) tops[wn * S::BM + wm * S::TM + j * 16 + r] = top;
      } else if (in > 0) {
        store_four(a.out, (m0 + j * 16 + r) * a.ld_out + col, a.out_type, in, v);
      }
    }
  };
  __syncthreads();
#pragma unroll 1
  for (int j = 0; j < S::FM; ++j) {
    if (kg == 0) {
#pragma unroll
      for (int k = 0; k < S::FM; ++k)
        if (k == j) {  // a register has no index
#pragma unroll
          for (int i = 0; i < S::FN; ++i) *reinterpret_cast<f32x4*>(mine + l15 * kPitch + i * 16 + quad * 4) = acc[i][k];
        }
    }
    order_lanes();
    if (a.residual && there > 0)  // the same for the wavefront: lanes exchange maxima within
      finish_rows(j, std::true_type());
    else if (!a.residual || f8_out)
      finish_rows(j, std::false_type());
    order_lanes();
    if (f8_out) {
      // the largest magnitude of 128 columns, over the wavefronts that hold them
      __syncthreads();
#pragma unroll 1
      for (int r = first_r; r < 16; r += per) {
        if (j * 16 + r >= there || in_row <= 0) continue;
        float most = 0.0f;
        for (int w = wn / span * span; w < wn / span * span + span; ++w)
          most = fmaxf(most, tops[w * S::BM + wm * S::TM + j * 16 + r]);
        const RowScale q = row_scale(most);
        const int64_t m = m0 + j * 16 + r;
        if (c == 0 && wn % span == 0) a.out_scales[m * a.ld_os + wave_col / kScaleBlock] = q.s;
        const f32x4 g = *reinterpret_cast<const f32x4*>(mine + r * kPitch + at);
        float v[4] = {g[0], g[1], g[2], g[3]};
        quotients(v, q);
        store_four(a.out, m * a.ld_out + col, WB_F8E4M3, in_row, v);
      }
    }
  }
}

// fp8 codes and scales of fp32 rows, for tiles too narrow to hold the 128
// columns of a scale: sixteen lanes a scale, eight columns each. Rows that
// belong to no expert are left alone. Bound by the launch for few rows (128 rows
// of 2048: 5 us), by its bytes for many (8192 rows: 15 us).
__global__ __launch_bounds__(256) void wb_linear_codes_kernel(const float* sums, LinearArgs a) {
  const int64_t row = blockIdx.x, c = (int64_t(blockIdx.y) * 256 + threadIdx.x) * 8;
  if (a.offsets && (row < a.offsets[0] || row >= a.offsets[a.num_experts])) return;
  if (c - (threadIdx.x & 15) * 8 >= a.n_out) return;
  const float* from = sums + row * a.n_out;
  float v[8];
  if (c + 8 <= a.n_out)
    load_eight(from, c, WB_F32, v);
  else
    load_tail(from, c, a.n_out, WB_F32, v);
  float top = 0.0f;
  for (int i = 0; i < 8; ++i) top = fmaxf(top, fabsf(v[i]));
  const RowScale q = row_scale(reduce16(top, FMax()));
  if ((threadIdx.x & 15) == 0) a.out_scales[row * a.ld_os + c / kScaleBlock] = q.s;
  quotients(v, q);
  uint8_t* to = static_cast<uint8_t*>(a.out) + row * a.ld_out + c;
  const u32x2 p = {pack_fp8(v[0], v[1], v[2], v[3]), pack_fp8(v[4], v[5], v[6], v[7])};
  if (c + 8 <= a.n_out) {
    *reinterpret_cast<u32x2_a1*>(to) = p;
  } else {
    for (int i = 0; i < 8; ++i)
      if (c + i < a.n_out) to[i] = static_cast<uint8_t>(p[i >> 2] >> (8 * (i & 3)));
  }
}

// Rows of x and of the weight that start off the 16-byte grid, onto it: 16-byte
// pieces in order, zeros past a row's end (in both operands, so that sums stay
// as they are), four pieces a thread. Bound by its bytes.
struct Realign {
  const uint8_t* from;
  u32x4* to;
  int64_t ld, bytes;       // a row's distance and length
  uint32_t pieces, count;  // of a row, of all rows
};

__global__ __launch_bounds__(256) void wb_linear_realign_kernel(Realign x, Realign weight, uint32_t x_blocks) {
  const bool second = blockIdx.x >= x_blocks;
  const Realign a = second ? weight : x;
  const uint32_t base = (blockIdx.x - (second ? x_blocks : 0)) * 1024 + threadIdx.x;
  u32x4 v[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t at = base + i * 256;
    if (at >= a.count) continue;
    const uint32_t row = at / a.pieces;
    v[i] = load_piece(a.from + row * a.ld, int64_t(at - row * a.pieces) * 16, a.bytes);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (base + i * 256 < a.count) a.to[base + i * 256] = v[i];
}

// Row tiles of `per` rows: each expert's last may be part of one, so there is
// at most one more per expert with rows.
int64_t row_tiles(const LinearArgs& a, int per) {
  if (!a.offsets) return (a.rows + per - 1) / per;
  return std::min<int64_t>(a.rows, a.rows / per + std::min<int64_t>(a.num_experts, a.rows));
}

int64_t col_tiles(const LinearArgs& a, int bn) {
  const int step = a.gated ? bn / 2 : bn;
  return (a.n_out + step - 1) / step;
}

constexpr int64_t kMaxTiles = 0x3fffff;  // of a launch, whose threads (up to 512 a tile) stay below 2^32

template <class S, bool F8, bool DIRECT>
hipError_t launch_tile(const LinearArgs& a, hipStream_t st) {
  const auto kernel = wb_linear_tile_kernel<S, F8, DIRECT>;
  // the kernel's LDS is past the default limit; once for each GPU of a process
  static std::atomic<uint64_t> raised{0};
  int device = 0;
  hipError_t e = hipGetDevice(&device);
  if (e != hipSuccess) return e;
  const uint64_t bit = device < 64 ? uint64_t(1) << device : 0;
  if (!(raised.load(std::memory_order_acquire) & bit) || !bit) {
    e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, S::kLds);
    if (e != hipSuccess) return e;
    raised.fetch_or(bit, std::memory_order_release);
  }
  const int64_t tiles_n = col_tiles(a, S::BN), all = row_tiles(a, S::BM) * tiles_n;
  hipLaunchKernelGGL(kernel, dim3(static_cast<uint32_t>(all)), dim3(S::kThreads), S::kLds, st, a,
                     static_cast<uint32_t>(tiles_n), 8u);
  return hipGetLastError();
}

// The tiles in use. A launch takes the one whose rounds over the 256 CUs are
// expected to be done first; memory's rate has no part in that (128 rows of 32
// experts' 4096 x 7168 fp8: 75 us expected, 178 taken), nor do offsets, which
// are on the device: every row of the result counts as some expert's. A round
// takes us per stage of k (128 bytes of a row) and `fixed` for its start and
// its results; `resident` workgroups share a CU. Measured with 1024 tiles, and
// with 256 (`few`: up to there every tile has a CU to itself), for bf16 and
// fp8; the last two are us, with 512 and with 256 tiles, of rows that come by
// way of registers (0: not in use). Large tiles read less per product; small
// ones give every CU work, and keep more of the weight on its way when few rows
// meet it. 8192 x 8192 x 8192 bf16: 0.85 ms with 256 x 256, 0.99 with 128 x
// 128; 1024 x 7168 x 2048 fp8: 67 us and 37; one row by 6144 x 4096 bf16: 12 us
// with 16 x 32, 31 with 64 x 64.
struct Choice {
  int bm, bn, resident;
  float us[2], fixed, few_us[2], few_fixed;
  float by_registers[2], few_by_registers[2];
};
constexpr Choice kChoices[] = {
    {16, 32, 2, {0.105f, 0.137f}, 3.9f, {0.057f, 0.085f}, 4.8f, {}, {}},
    {32, 32, 1, {0.075f, 0.129f}, 3.2f, {0.075f, 0.128f}, 4.4f, {0.264f, 0.358f}, {0.264f, 0.358f}},
    {32, 64, 2, {0.28f, 0.437f}, 3.0f, {0.129f, 0.251f}, 4.3f, {}, {}},
    {64, 64, 2, {0.43f, 0.645f}, 2.0f, {0.25f, 0.333f}, 6.0f, {0.78f, 1.82f}, {0.54f, 0.77f}},
    {64, 64, 1, {0.22f, 0.345f}, 2.0f, {0.162f, 0.334f}, 6.0f, {}, {}},
    {128, 64, 1, {0.355f, 0.632f}, 2.5f, {0.396f, 0.635f}, 3.0f, {1.0f, 1.5f}, {1.0f, 1.5f}},
    {128, 128, 2, {0.95f, 1.8f}, 6.5f, {0.87f, 1.0f}, 5.0f, {1.72f, 0.0f}, {1.71f, 0.0f}},
    {128, 128, 1, {0.655f, 0.90f}, 5.0f, {0.74f, 0.914f}, 6.0f, {}, {}},
    {256, 256, 1, {1.5f, 3.24f}, 14.5f, {1.65f, 3.31f}, 11.5f, {}, {}},
};
constexpr double kCodesUs = 6.0;  // the second launch, of few rows (8192 rows of 2048: 16 us, which is not priced)
constexpr int kNumChoices = sizeof(kChoices) / sizeof(kChoices[0]);

// Whether a tile holds whole scales of an fp8 output.
bool holds_scales(const LinearArgs& a, int choice) {
  return (a.gated ? kChoices[choice].bn / 2 : kChoices[choice].bn) % kScaleBlock == 0;
}

// The tile, and the us that it is expected to take; -1 where one launch takes
// the tiles of no shape.
int choose(const LinearArgs& a, double* expected) {
  const int f8 = a.in_type == WB_F8E4M3;
  const double stages = std::ceil(double(a.k) * (f8 ? 1 : 2) / kStageBytes);
  int best = -1;
  double least = 0.0;
  for (int i = 0; i < kNumChoices; ++i) {
    const Choice& c = kChoices[i];
    if (!a.direct && c.by_registers[f8] == 0.0f) continue;
    const int64_t tiles_n = col_tiles(a, c.bn);
    if (row_tiles(a, c.bm) * tiles_n > kMaxTiles) continue;
    // of the experts' last tiles about half are empty
    double tiles_m = double(row_tiles(a, c.bm));
    if (a.offsets) tiles_m = std::min(double(a.rows), double(a.rows) / c.bm + 0.5 * std::min<int64_t>(a.num_experts, a.rows));
    const double tiles = tiles_m * double(tiles_n);
    // a residual is read between the products and the stores, at about the
    // stores' cost; what is left of 256 tiles or fewer has the CUs to itself
    const int more = a.residual ? 2 : 1;
    const double full = (a.direct ? c.us : c.by_registers)[f8] * stages + c.fixed * more;
    const double few = (a.direct ? c.few_us : c.few_by_registers)[f8] * stages + c.few_fixed * more;
    const double rounds = std::floor(tiles / (256 * c.resident)), left = tiles - rounds * 256 * c.resident;
    const double us = rounds * full + (left <= 0 ? 0.0 : left <= 256 ? few : full) +
                      (a.out_type == WB_F8E4M3 && !holds_scales(a, i) ? kCodesUs : 0.0);
    if (best < 0 || us < least) best = i, least = us;
  }
  *expected = least;
  return best;
}

// How a launch goes: its tile, and for rows off the 16-byte grid whether
// copies of them, in the workspace, are expected to be done first.
struct Form {
  LinearArgs a;  // the product; x and weight are set where they are copied
  int choice;
  bool copy_x = false, copy_weight = false;
  size_t x_bytes = 0, weight_bytes = 0, sums_bytes = 0;
};
// Measured: 4 to 6 us for the launch, and 3.2 TB/s (what comes back from the caches
// included). 4000 rows, 4096 x 1001: bf16 69 us by way of registers and 51 by
// way of copies, fp8 116 and 54; 2 rows, 1337 x 7543 bf16 39 and 22; 333 rows,
// 3442 x 1500 bf16 18 and 24; 40 rows, 300 x 700 6.5 and 10.6.
constexpr double kCopyUs = 6.0, kCopyBytesPerUs = 3.2e6;

Form form_of(const LinearArgs& a) {
  Form f;
  double us = 0.0, copied_us = 0.0;
  f.a = a, f.choice = choose(a, &us);
  const int64_t es = a.in_type == WB_F8E4M3 ? 1 : 2, pitch = (a.k * es + 15) / 16 * 16;
  auto off_grid = [&](const uint8_t* p, int64_t ld) {
    return ((reinterpret_cast<uintptr_t>(p) | static_cast<uintptr_t>(ld) | static_cast<uintptr_t>(a.k * es)) & 15) != 0;
  };
  const bool x = off_grid(a.x, a.ld_x_bytes), weight = off_grid(a.weight, a.ld_w_bytes);
  if (!a.direct && (x || weight)) {
    LinearArgs b = a;
    b.k = static_cast<int32_t>(pitch / es);
    if (x) b.ld_x_bytes = pitch;
    if (weight) b.ld_w_bytes = pitch, b.stride_w_bytes = b.n * pitch;
    b.direct = linear_near(b);
    const int64_t x_rows = x ? a.x_rows : 0, w_rows = weight ? int64_t(a.n) * std::max(1, a.num_experts) : 0;
    const int64_t most = (int64_t(1) << 32) - 4096;  // pieces are counted in 32 bits
    if (b.direct && x_rows <= most / (pitch / 16) && w_rows <= most / (pitch / 16)) {
      const int choice = choose(b, &copied_us);
      copied_us += kCopyUs + double(x_rows + w_rows) * pitch / kCopyBytesPerUs;
      if (choice >= 0 && (f.choice < 0 || copied_us < us))
        f.a = b, f.choice = choice, f.copy_x = x, f.copy_weight = weight, f.x_bytes = x_rows * pitch, f.weight_bytes = w_rows * pitch;
    }
  }
  if (a.out_type == WB_F8E4M3 && f.choice >= 0 && !holds_scales(a, f.choice)) f.sums_bytes = static_cast<size_t>(a.rows) * a.n_out * sizeof(float);
  return f;
}

template <class S, int CHOICE>
hipError_t launch_shape(const LinearArgs& a, hipStream_t st) {
  constexpr Choice c = kChoices[CHOICE];
  static_assert(c.bm == S::BM && c.bn == S::BN, "the tile of the table");
  const bool f8 = a.in_type == WB_F8E4M3;
  if (a.direct) return f8 ? launch_tile<S, true, true>(a, st) : launch_tile<S, false, true>(a, st);
  if constexpr (c.by_registers[1] > 0.0f) {
    if (f8) return launch_tile<S, true, false>(a, st);
  }
  if constexpr (c.by_registers[0] > 0.0f) {
    if (!f8) return launch_tile<S, false, false>(a, st);
  }
  return hipErrorInvalidConfiguration;  // not chosen
}

hipError_t launch_choice(const LinearArgs& a, int choice, hipStream_t st) {
  switch (choice) {
    case 0: return launch_shape<Shape<16, 32, 1, 1, 4, 4, 3>, 0>(a, st);
    case 1: return launch_shape<Shape<32, 32, 2, 1, 4, 4, 4>, 1>(a, st);
    case 2: return launch_shape<Shape<32, 64, 2, 2, 2, 2, 3>, 2>(a, st);
    case 3: return launch_shape<Shape<64, 64, 2, 2, 2, 2, 2>, 3>(a, st);
    case 4: return launch_shape<Shape<64, 64, 2, 2, 2, 2, 4>, 4>(a, st);
    case 5: return launch_shape<Shape<128, 64, 4, 2, 1, 2, 3>, 5>(a, st);
    case 6: return launch_shape<Shape<128, 128, 2, 2, 1, 1, 2>, 6>(a, st);
    case 7: return launch_shape<Shape<128, 128, 2, 2, 2, 2, 2>, 7>(a, st);
    default: return launch_shape<Shape<256, 256, 4, 2, 1, 1, 2>, 8>(a, st);
  }
}

}  // namespace

bool linear_near(const LinearArgs& a) {
  const int64_t reach = (int64_t(1) << 32) - 4096;
  return a.n * a.ld_w_bytes < reach && (a.tokens ? a.x_rows : 256) * a.ld_x_bytes < reach &&
         !(a.in_type == WB_F8E4M3 && a.gated && a.n_out % 16 != 0);
}

int64_t linear_workspace_bytes(const LinearArgs& a) {
  if (a.rows == 0) return 0;
  const Form f = form_of(a);
  if (f.choice < 0) return -1;
  return f.x_bytes + f.weight_bytes + f.sums_bytes;
}

int launch_linear(const LinearArgs& a, void* workspace, void* stream) {
  if (a.rows == 0) return hipSuccess;
  const auto st = static_cast<hipStream_t>(stream);
  Form f = form_of(a);
  auto* at = static_cast<uint8_t*>(workspace);
  if (f.copy_x || f.copy_weight) {
    const int64_t bytes = a.k * (a.in_type == WB_F8E4M3 ? 1 : 2);
    auto realign = [&](const uint8_t*& p, int64_t ld, size_t size) {
      const Realign r{p, reinterpret_cast<u32x4*>(at), ld, bytes, static_cast<uint32_t>((bytes + 15) / 16), static_cast<uint32_t>(size / 16)};
      if (size) p = at;
      at += size;
      return r;
    };
    const Realign x = realign(f.a.x, a.ld_x_bytes, f.x_bytes), weight = realign(f.a.weight, a.ld_w_bytes, f.weight_bytes);
    auto blocks = [](const Realign& r) { return (r.count + 1023) / 1024; };
    hipLaunchKernelGGL(wb_linear_realign_kernel, dim3(blocks(x) + blocks(weight)), dim3(256), 0, st, x, weight, blocks(x));
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (!f.sums_bytes) return launch_choice(f.a, f.choice, st);
  LinearArgs sums = f.a;
  sums.out = at, sums.out_type = WB_F32, sums.ld_out = a.n_out;
  const hipError_t e = launch_choice(sums, f.choice, st);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(wb_linear_codes_kernel, dim3(static_cast<uint32_t>(a.rows), static_cast<uint32_t>((a.n_out + 2047) / 2048)),
                     dim3(256), 0, st, reinterpret_cast<const float*>(at), a);
  return hipGetLastError();
}

}  // namespace wb
