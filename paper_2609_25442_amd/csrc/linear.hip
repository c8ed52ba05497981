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

#include "ops_device.hpp"

namespace wb {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef u32x4 u32x4_a1 __attribute__((aligned(1)));
typedef u32x2 u32x2_a2 __attribute__((aligned(2)));
typedef uint32_t u32_a1 __attribute__((aligned(1)));

// Read through the scalar cache: the same for the whole wavefront.
typedef __attribute__((address_space(4))) float ConstFloat;

constexpr int kStageBytes = 128;  // of a row, per step over k: a scale block of fp8, half as many bf16

// Sixteen zero bytes: what a tile's 16-byte pieces past the end of k are read from.
__device__ const u32x4 zero_piece = {0, 0, 0, 0};

__device__ __forceinline__ float silu(float z) { return z * __builtin_amdgcn_rcpf(1.0f + __expf(-z)); }
__device__ __forceinline__ float gelu(float z) { return 0.5f * z * (1.0f + erff(z * 0.70710678118654752f)); }
__device__ __forceinline__ float activate(float z, int kind) {
  return kind == WB_ACT_SILU ? silu(z) : kind == WB_ACT_GELU ? gelu(z) : z;
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

// Four neighbouring columns of a row; in: how many of them exist.
__device__ __forceinline__ void load_four(const void* base, int64_t at, int type, int in, float (&v)[4]) {
  if (in >= 4) {
    if (type == WB_F32) {
      const f32x4 f = *reinterpret_cast<const f32x4_a4*>(static_cast<const float*>(base) + at);
      for (int r = 0; r < 4; ++r) v[r] = f[r];
    } else {
      const u32x2 u = *reinterpret_cast<const u32x2_a2*>(static_cast<const uint16_t*>(base) + at);
      for (int r = 0; r < 4; ++r)
        v[r] = __builtin_bit_cast(float, (r & 1) ? u[r >> 1] & 0xffff0000u : u[r >> 1] << 16);
    }
  } else {
    for (int r = 0; r < 4; ++r) v[r] = r < in ? load_one(base, at + r, type) : 0.0f;
  }
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
    if (type == WB_F32)
      *reinterpret_cast<f32x4_a4*>(static_cast<float*>(base) + at) = f32x4{v[0], v[1], v[2], v[3]};
    else
      *reinterpret_cast<u32x2_a2*>(static_cast<uint16_t*>(base) + at) = u32x2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
  } else {
    for (int r = 0; r < in; ++r) store_one(base, at + r, type, v[r]);
  }
}

// What follows the sums of a row m and four columns from col on; u are the
// sums of the up rows where the weight is gated. in_row: columns that exist
// (none for a row past the end).
__device__ __forceinline__ void finish(const LinearArgs& a, int expert, int64_t m, int col, int in_row, float (&v)[4],
                                       float (&u)[4]) {
  if (a.bias && in_row > 0) {
    for (int r = 0; r < 4; ++r) {
      const int c = min(col + r, a.n_out - 1);
      v[r] += load_bias(a, expert, c);
      if (a.gated) u[r] += load_bias(a, expert, a.n_out + c);
    }
  }
  for (int r = 0; r < 4; ++r) v[r] = a.gated ? activate(v[r], a.activation) * u[r] : activate(v[r], a.activation);
  if (a.residual && in_row > 0) {
    float add[4];
    load_four(a.residual, m * a.ld_residual + col, a.residual_type, in_row, add);
    for (int r = 0; r < 4; ++r) v[r] += add[r];
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

template <bool F8>
__device__ __forceinline__ f32x4 block_sum(const Operand<F8>& w, const Operand<F8>& x, f32x4 c) {
#pragma unroll
  for (int h = 0; h < (F8 ? 4 : 2); ++h) c = mfma(w.v[h], x.v[h], c);
  return c;
}

// A workgroup's tile: BM rows of the output by BN rows of the weight, WM x WN
// wavefronts. LDS holds two stages of 128 bytes of every row of both; the
// pieces of a row are permuted by its number so that sixteen rows' pieces at
// one place of k fall into different banks.
template <int BM_, int BN_, int WM_, int WN_>
struct Shape {
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_;
  static constexpr int kThreads = 64 * WM * WN, TM = BM / WM, TN = BN / WN, FM = TM / 16, FN = TN / 16;
  static constexpr int kRows = BM + BN, kStage = kRows * kStageBytes;
  // behind the stages: scales of x by row and of the weight by row, for each
  // of the two; the epilogue's maxima lie over them
  static constexpr int kScales = (BM + BN) * 4, kLds = 2 * kStage + 2 * kScales;
  static_assert(WN * BM * 4 <= 2 * kScales, "maxima fit");
};

__device__ __forceinline__ int swizzle(int row) { return (row >> 1) & 7; }

// F8: fp8 operands, else bf16. DIRECT: rows start at multiples of 16 bytes and
// hold a multiple of 16, and the sixteen rows of a block share a weight
// scale: tiles go from memory to LDS without registers between. Otherwise
// through registers, piece by piece, and scales by row.
template <class S, bool F8, bool DIRECT>
__global__ __launch_bounds__(S::kThreads) void wb_linear_tile_kernel(LinearArgs a, uint32_t tiles_n, uint32_t group) {
  extern __shared__ __align__(128) uint8_t lds[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / S::WN, wn = wave % S::WN, l15 = lane & 15, quad = lane >> 4;

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
  constexpr int kPieces = S::kRows * 8 / S::kThreads;  // per lane and stage
  const uint8_t* src[kPieces];
  u32x4 held[DIRECT ? 1 : kPieces];
#pragma unroll
  for (int i = 0; i < kPieces; ++i) {
    const int r = (wave + i * (S::kThreads / 64)) * 8 + (lane >> 3);
    src[i] = row_of(r);
  }
  const int r0 = wave * 8 + (lane >> 3);
  static_assert((S::kThreads / 64 * 8) % 16 == 0, "the pieces of a lane are permuted alike");
  const int piece = ((lane & 7) ^ swizzle(r0)) * 16;

  auto fetch = [&](int s) {
    const int64_t at = int64_t(s) * kStageBytes + piece;
    if constexpr (DIRECT) {
      uint8_t* to = lds + (s & 1) * S::kStage;
      const bool past = at >= k_bytes;
#pragma unroll
      for (int i = 0; i < kPieces; ++i) {
        const uint8_t* p = past ? reinterpret_cast<const uint8_t*>(&zero_piece) : src[i] + at;
        __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)p,
                                         (__attribute__((address_space(3))) void*)(to + (wave + i * (S::kThreads / 64)) * 1024),
                                         16, 0, 0);
      }
    } else {
#pragma unroll
      for (int i = 0; i < kPieces; ++i) held[i] = load_piece(src[i], at, k_bytes);
    }
  };
  auto put = [&](int s) {
    if constexpr (!DIRECT) {
      uint8_t* to = lds + (s & 1) * S::kStage;
#pragma unroll
      for (int i = 0; i < kPieces; ++i)
        *reinterpret_cast<u32x4*>(to + (wave + i * (S::kThreads / 64)) * 1024 + lane * 16) = held[i];
    }
  };

  // scales of a stage, one row (of x, then of the weight) per thread and round
  constexpr int kScaleRows = F8 ? S::BM + S::BN : 0, kScaleRounds = (kScaleRows + S::kThreads - 1) / S::kThreads;
  const float* scale_src[kScaleRounds > 0 ? kScaleRounds : 1];
  float scale_held[kScaleRounds > 0 ? kScaleRounds : 1];
  float* const scales = reinterpret_cast<float*>(lds + 2 * S::kStage);
  if constexpr (F8) {
#pragma unroll
    for (int i = 0; i < kScaleRounds; ++i) {
      const int r = tid + i * S::kThreads;
      scale_src[i] = r < S::BM ? a.x_scales + x_row(a, min(rows.first + r, rows.end - 1)) * a.ld_xs
                               : a.weight_scales + rows.expert * a.stride_ws +
                                     int64_t(w_row(a, col0, min(r, kScaleRows - 1) - S::BM) / kScaleBlock) * a.ld_ws;
    }
  }
  auto fetch_scales = [&](int s) {
    if constexpr (F8) {
#pragma unroll
      for (int i = 0; i < kScaleRounds; ++i) scale_held[i] = scale_src[i][s];
    }
  };
  auto put_scales = [&](int s) {
    if constexpr (F8) {
#pragma unroll
      for (int i = 0; i < kScaleRounds; ++i)
        if (tid + i * S::kThreads < kScaleRows) scales[(s & 1) * kScaleRows + tid + i * S::kThreads] = scale_held[i];
    }
  };

  f32x4 acc[S::FN][S::FM];
#pragma unroll
  for (int i = 0; i < S::FN; ++i)
#pragma unroll
    for (int j = 0; j < S::FM; ++j) acc[i][j] = f32x4{0, 0, 0, 0};

  const int frag = l15 * kStageBytes + ((quad ^ swizzle(l15)) << 4);
  const int w_frag = wn * S::TN * kStageBytes + frag, x_frag = (S::BN + wm * S::TM) * kStageBytes + frag;

  fetch_scales(0);
  fetch(0);
  put(0);
  put_scales(0);
  for (int s = 0; s < stages; ++s) {
    // this stage is in LDS, and the one before it has been read
    __syncthreads();
    if (s + 1 < stages) {
      fetch_scales(s + 1);
      fetch(s + 1);
    }
    const uint8_t* buf = lds + (s & 1) * S::kStage;
    const float* sc = scales + (s & 1) * kScaleRows;
    auto operand = [&](int at) {
      return Operand<F8>(*reinterpret_cast<const i32x4*>(buf + at), *reinterpret_cast<const i32x4*>(buf + (at ^ 64)));
    };
    Operand<F8> x[S::FM];
    float sx[S::FM];
#pragma unroll
    for (int j = 0; j < S::FM; ++j) {
      x[j] = operand(x_frag + j * 16 * kStageBytes);
      if constexpr (F8) sx[j] = sc[wm * S::TM + j * 16 + l15];
    }
#pragma unroll
    for (int i = 0; i < S::FN; ++i) {
      const Operand<F8> w = operand(w_frag + i * 16 * kStageBytes);
      if constexpr (F8) {
        const float* sw = sc + S::BM + wn * S::TN + i * 16;
        const f32x4 sr = DIRECT ? f32x4{sw[0], sw[0], sw[0], sw[0]} : *reinterpret_cast<const f32x4*>(sw + quad * 4);
#pragma unroll
        for (int j = 0; j < S::FM; ++j) {
          const f32x4 part = block_sum<F8>(w, x[j], f32x4{0, 0, 0, 0});
          if constexpr (DIRECT) {
            const float both = sx[j] * sr[0];
            for (int r = 0; r < 4; ++r) acc[i][j][r] = __builtin_fmaf(part[r], both, acc[i][j][r]);
          } else {
            for (int r = 0; r < 4; ++r) acc[i][j][r] = __builtin_fmaf(part[r], sx[j] * sr[r], acc[i][j][r]);
          }
        }
      } else {
#pragma unroll
        for (int j = 0; j < S::FM; ++j) acc[i][j] = block_sum<F8>(w, x[j], acc[i][j]);
      }
    }
    if (s + 1 < stages) {
      put(s + 1);
      put_scales(s + 1);
    }
  }

  // epilogue: lane l holds token l % 16 of each j, four columns of each block.
  // A gated tile's blocks come in pairs, gate and up of the same columns.
  const int blocks = a.gated ? S::FN / 2 : S::FN;
  const int wave_col = col0 + wn * (a.gated ? S::TN / 2 : S::TN) + quad * 4;
  float top[S::FM];
#pragma unroll
  for (int j = 0; j < S::FM; ++j) {
    const int64_t m = rows.first + wm * S::TM + j * 16 + l15;
    const bool there = m < rows.end;
    top[j] = 0.0f;
#pragma unroll
    for (int b = 0; b < S::FN; ++b) {
      if (b >= blocks) break;
      const int col = wave_col + b * 16, in_row = there ? a.n_out - col : 0;
      float v[4], u[4];
      if (a.gated) {
        for (int r = 0; r < 4; ++r) v[r] = acc[2 * b < S::FN ? 2 * b : 0][j][r], u[r] = acc[2 * b + 1 < S::FN ? 2 * b + 1 : 0][j][r];
      } else {
        for (int r = 0; r < 4; ++r) v[r] = acc[b][j][r], u[r] = 1.0f;
      }
      finish(a, rows.expert, m, col, in_row, v, u);
      if (a.out_type == WB_F8E4M3) {
        for (int r = 0; r < 4; ++r) acc[b][j][r] = v[r];
        top[j] = largest(v, in_row, top[j]);
      } else if (in_row > 0) {
        store_four(a.out, m * a.ld_out + col, a.out_type, in_row, v);
      }
    }
  }
  if (a.out_type != WB_F8E4M3) return;

  // fp8: the largest magnitude of 128 columns, over the wavefronts that hold them
  float* tops = reinterpret_cast<float*>(lds + 2 * S::kStage);
  const int span = kScaleBlock / (a.gated ? S::TN / 2 : S::TN);  // wavefronts
  __syncthreads();
#pragma unroll
  for (int j = 0; j < S::FM; ++j) {
    top[j] = fmaxf(top[j], __shfl_xor(top[j], 16));
    top[j] = fmaxf(top[j], __shfl_xor(top[j], 32));
    if (quad == 0) tops[wn * S::BM + wm * S::TM + j * 16 + l15] = top[j];
  }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < S::FM; ++j) {
    const int64_t m = rows.first + wm * S::TM + j * 16 + l15;
    if (m >= rows.end) continue;
    float most = 0.0f;
    for (int w = wn / span * span; w < wn / span * span + span; ++w)
      most = fmaxf(most, tops[w * S::BM + wm * S::TM + j * 16 + l15]);
    const RowScale q = row_scale(most);
    if (quad == 0 && wn % span == 0 && wave_col < a.n_out) a.out_scales[m * a.ld_os + wave_col / kScaleBlock] = q.s;
#pragma unroll
    for (int b = 0; b < S::FN; ++b) {
      if (b >= blocks) break;
      const int col = wave_col + b * 16, in_row = a.n_out - col;
      if (in_row <= 0) continue;
      float v[4];
      for (int r = 0; r < 4; ++r) v[r] = quotient(acc[b][j][r], q);
      store_four(a.out, m * a.ld_out + col, WB_F8E4M3, in_row, v);
    }
  }
}

// Few rows: the weight is read once, so its bytes are the floor. A wavefront
// takes CB blocks of sixteen rows of the weight (gated: gate and up of the
// same columns) against NT * 16 tokens and every KS-th stage of k, straight
// from memory into operands; the KS partial sums meet in LDS and are added in
// order. FB such groups make a workgroup: eight where the output is fp8, so
// that it holds the 128 columns of a scale. The sixteen rows of a block share
// their weight scales (the launch sees to that).
template <int NT_, int CB_, int FB_, int KS_, bool GATED_>
struct Few {
  static constexpr int NT = NT_, CB = CB_, FB = FB_, KS = KS_, kThreads = 64 * FB * KS;
  static constexpr bool GATED = GATED_;
  static constexpr int OB = GATED ? 1 : CB, kCols = 16 * OB * FB, kRows = 16 * NT;
  static constexpr int kItems = (OB * NT + KS - 1) / KS;      // 16x16 blocks a wavefront finishes
  // stages whose loads are in flight together, as many as the registers hold
  static constexpr int kAhead = NT + CB <= (kThreads == 1024 ? 2 : 3) ? 4 : 2;
  static_assert(!GATED || CB == 2, "gate and up");
};

template <class S, bool F8>
__global__ __launch_bounds__(S::kThreads) void wb_linear_few_kernel(LinearArgs a, uint32_t tiles_n) {
  __shared__ f32x4 sums[S::FB * S::KS][S::CB * S::NT][64];
  __shared__ float tops[S::FB][S::kRows];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int fb = wave / S::KS, ks = wave % S::KS, l15 = lane & 15, quad = lane >> 4;
  RowTile rows;
  if (!find_rows(a, blockIdx.x / tiles_n, S::kRows, rows)) return;
  const int col0 = static_cast<int>(blockIdx.x % tiles_n) * S::kCols + fb * 16 * S::OB;
  const int64_t k_bytes = F8 ? int64_t(a.k) : 2 * int64_t(a.k);
  const int whole = static_cast<int>(k_bytes / kStageBytes), stages = static_cast<int>((k_bytes + kStageBytes - 1) / kStageBytes);

  const uint8_t *w[S::CB], *x[S::NT];
  const ConstFloat* sw[S::CB];
  const float* sx[S::NT];
#pragma unroll
  for (int c = 0; c < S::CB; ++c) {
    const int first = S::GATED ? c * a.n_out + min(col0, a.n_out - 1) : min(col0 + 16 * c, a.n - 1);
    const int last = S::GATED ? (c + 1) * a.n_out - 1 : a.n - 1;
    w[c] = a.weight + rows.expert * a.stride_w_bytes + int64_t(min(first + l15, last)) * a.ld_w_bytes + quad * 16;
    if constexpr (F8)
      sw[c] = (const ConstFloat*)(a.weight_scales + rows.expert * a.stride_ws + int64_t(first / kScaleBlock) * a.ld_ws);
  }
#pragma unroll
  for (int j = 0; j < S::NT; ++j) {
    const int64_t r = x_row(a, min(rows.first + j * 16 + l15, rows.end - 1));
    x[j] = a.x + r * a.ld_x_bytes + quad * 16;
    if constexpr (F8) sx[j] = a.x_scales + r * a.ld_xs;
  }

  f32x4 acc[S::CB][S::NT];
#pragma unroll
  for (int c = 0; c < S::CB; ++c)
#pragma unroll
    for (int j = 0; j < S::NT; ++j) acc[c][j] = f32x4{0, 0, 0, 0};

  struct Stage {
    u32x4 w[S::CB][2], x[S::NT][2];
    float sw[S::CB], sx[S::NT];
  };
  auto load = [&](Stage& t, int s) {
    const int64_t at = int64_t(s) * kStageBytes;
#pragma unroll
    for (int c = 0; c < S::CB; ++c) {
      t.w[c][0] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_a1*>(w[c] + at));
      t.w[c][1] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_a1*>(w[c] + at + 64));
      if constexpr (F8) t.sw[c] = sw[c][s];
    }
#pragma unroll
    for (int j = 0; j < S::NT; ++j) {
      t.x[j][0] = *reinterpret_cast<const u32x4_a1*>(x[j] + at);
      t.x[j][1] = *reinterpret_cast<const u32x4_a1*>(x[j] + at + 64);
      if constexpr (F8) t.sx[j] = sx[j][s];
    }
  };
  auto add = [&](const Stage& t) {
    Operand<F8> xo[S::NT];
#pragma unroll
    for (int j = 0; j < S::NT; ++j) xo[j] = Operand<F8>(__builtin_bit_cast(i32x4, t.x[j][0]), __builtin_bit_cast(i32x4, t.x[j][1]));
#pragma unroll
    for (int c = 0; c < S::CB; ++c) {
      const Operand<F8> wo(__builtin_bit_cast(i32x4, t.w[c][0]), __builtin_bit_cast(i32x4, t.w[c][1]));
#pragma unroll
      for (int j = 0; j < S::NT; ++j) {
        if constexpr (F8) {
          const f32x4 part = block_sum<F8>(wo, xo[j], f32x4{0, 0, 0, 0});
          const float both = t.sx[j] * t.sw[c];
          for (int r = 0; r < 4; ++r) acc[c][j][r] = __builtin_fmaf(part[r], both, acc[c][j][r]);
        } else {
          acc[c][j] = block_sum<F8>(wo, xo[j], acc[c][j]);
        }
      }
    }
  };
  int s = ks;
  for (; s + (S::kAhead - 1) * S::KS < whole; s += S::kAhead * S::KS) {
    Stage t[S::kAhead];
#pragma unroll
    for (int u = 0; u < S::kAhead; ++u) load(t[u], s + u * S::KS);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int u = 0; u < S::kAhead; ++u) add(t[u]);
  }
  for (; s < stages; s += S::KS) {
    Stage t;
    if (s < whole) {
      load(t, s);
    } else {  // the end of k
      const int64_t at = int64_t(s) * kStageBytes + quad * 16;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int c = 0; c < S::CB; ++c) t.w[c][h] = load_piece(w[c] - quad * 16, at + 64 * h, k_bytes);
#pragma unroll
        for (int j = 0; j < S::NT; ++j) t.x[j][h] = load_piece(x[j] - quad * 16, at + 64 * h, k_bytes);
      }
      if constexpr (F8) {
#pragma unroll
        for (int c = 0; c < S::CB; ++c) t.sw[c] = sw[c][s];
#pragma unroll
        for (int j = 0; j < S::NT; ++j) t.sx[j] = sx[j][s];
      }
    }
    add(t);
  }

#pragma unroll
  for (int c = 0; c < S::CB; ++c)
#pragma unroll
    for (int j = 0; j < S::NT; ++j) sums[wave][c * S::NT + j][lane] = acc[c][j];
  __syncthreads();
  auto total = [&](int c, int j, float(&v)[4]) {
    f32x4 t = sums[fb * S::KS][c * S::NT + j][lane];
    for (int i = 1; i < S::KS; ++i) {
      const f32x4 p = sums[fb * S::KS + i][c * S::NT + j][lane];
      for (int r = 0; r < 4; ++r) t[r] += p[r];
    }
    for (int r = 0; r < 4; ++r) v[r] = t[r];
  };
  float v[S::kItems][4];
#pragma unroll
  for (int i = 0; i < S::kItems; ++i) {
    const int item = ks + i * S::KS;
    if (item >= S::OB * S::NT) break;
    const int c = item / S::NT, j = item % S::NT, col = col0 + c * 16 + quad * 4;
    const int64_t m = rows.first + j * 16 + l15;
    const int in_row = m < rows.end ? a.n_out - col : 0;
    float u[4] = {1.0f, 1.0f, 1.0f, 1.0f};
    total(c, j, v[i]);
    if constexpr (S::GATED) total(1, j, u);
    finish(a, rows.expert, m, col, in_row, v[i], u);
    if (a.out_type != WB_F8E4M3) {
      if (in_row > 0) store_four(a.out, m * a.ld_out + col, a.out_type, in_row, v[i]);
      continue;
    }
    float top = largest(v[i], in_row, 0.0f);
    top = fmaxf(top, __shfl_xor(top, 16));
    top = fmaxf(top, __shfl_xor(top, 32));
    if (quad == 0) tops[fb][j * 16 + l15] = top;
  }
  if (a.out_type != WB_F8E4M3) return;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < S::kItems; ++i) {
    const int item = ks + i * S::KS;
    if (item >= S::OB * S::NT) break;
    const int j = item % S::NT, col = col0 + quad * 4;
    const int64_t m = rows.first + j * 16 + l15;
    const int in_row = m < rows.end ? a.n_out - col : 0;
    if (in_row <= 0) continue;
    float most = 0.0f;
    for (int f = 0; f < S::FB; ++f) most = fmaxf(most, tops[f][j * 16 + l15]);
    const RowScale q = row_scale(most);
    if (quad == 0 && fb == 0) a.out_scales[m * a.ld_os + col / kScaleBlock] = q.s;
    for (int r = 0; r < 4; ++r) v[i][r] = quotient(v[i][r], q);
    store_four(a.out, m * a.ld_out + col, WB_F8E4M3, in_row, v[i]);
  }
}

// Row tiles of `per` rows: each expert's last may be part of one, so there is
// at most one more per expert with rows.
int64_t row_tiles(const LinearArgs& a, int per) {
  if (!a.offsets) return (a.rows + per - 1) / per;
  return std::min<int64_t>(a.rows, a.rows / per + std::min<int64_t>(a.num_experts, a.rows));
}

template <class S>
hipError_t launch_few(const LinearArgs& a, hipStream_t st) {
  const int64_t tiles_n = (a.n_out + S::kCols - 1) / S::kCols, all = row_tiles(a, S::kRows) * tiles_n;
  if (all > 0x3fffff) return hipErrorInvalidConfiguration;
  const dim3 grid(static_cast<uint32_t>(all)), block(S::kThreads);
  if (a.in_type == WB_F8E4M3)
    hipLaunchKernelGGL((wb_linear_few_kernel<S, true>), grid, block, 0, st, a, static_cast<uint32_t>(tiles_n));
  else
    hipLaunchKernelGGL((wb_linear_few_kernel<S, false>), grid, block, 0, st, a, static_cast<uint32_t>(tiles_n));
  return hipGetLastError();
}

// NT * 16 tokens at a time.
template <int NT>
hipError_t launch_few_rows(const LinearArgs& a, hipStream_t st) {
  constexpr int kSplit = NT == 1 ? 2 : 1;  // of k, in the workgroups of eight groups
  if (a.out_type == WB_F8E4M3)
    return a.gated ? launch_few<Few<NT, 2, 8, kSplit, true>>(a, st) : launch_few<Few<NT, 1, 8, kSplit, false>>(a, st);
  return a.gated ? launch_few<Few<NT, 2, 1, 8, true>>(a, st) : launch_few<Few<NT, 1, 1, 8, false>>(a, st);
}

template <class S, bool F8, bool DIRECT>
hipError_t launch_tile(const LinearArgs& a, hipStream_t st) {
  const auto kernel = wb_linear_tile_kernel<S, F8, DIRECT>;
  const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, S::kLds);
  if (e != hipSuccess) return e;
  const int step = a.gated ? S::BN / 2 : S::BN;
  const int64_t tiles_n = (a.n_out + step - 1) / step;
  const int64_t all = row_tiles(a, S::BM) * tiles_n;
  if (all > 0x3fffff) return hipErrorInvalidConfiguration;
  hipLaunchKernelGGL(kernel, dim3(static_cast<uint32_t>(all)), dim3(S::kThreads), S::kLds, st, a,
                     static_cast<uint32_t>(tiles_n), 8u);
  return hipGetLastError();
}

template <class S>
hipError_t launch_shape(const LinearArgs& a, hipStream_t st) {
  if (a.in_type == WB_F8E4M3) return a.direct ? launch_tile<S, true, true>(a, st) : launch_tile<S, true, false>(a, st);
  return a.direct ? launch_tile<S, false, true>(a, st) : launch_tile<S, false, false>(a, st);
}

}  // namespace

int launch_linear(const LinearArgs& a, void* stream) {
  if (a.rows == 0) return hipSuccess;
  const auto st = static_cast<hipStream_t>(stream);
  const int64_t each = a.offsets ? a.rows / a.num_experts : a.rows;  // rows a weight meets
  const bool shared_scales = a.in_type != WB_F8E4M3 || !a.gated || a.n_out % 16 == 0;
  if (!shared_scales) return launch_shape<Shape<64, 256, 1, 4>>(a, st);
  if (each <= 16) return launch_few_rows<1>(a, st);
  if (each <= 32) return launch_few_rows<2>(a, st);
  if (each <= 64) return launch_few_rows<4>(a, st);
  return launch_shape<Shape<64, 256, 1, 4>>(a, st);
}

}  // namespace wb
