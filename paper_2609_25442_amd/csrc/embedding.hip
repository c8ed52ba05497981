// Lookup of token embeddings, and the gradient of the table by sorted tokens.
//   out_t = scale W[tok_t - first];   dW_v = scale sum_{t: tok_t - first = v} dout_t
//
// The lookup reads and writes a row per token: bandwidth bound, 16384 x 4096 bf16
// in 33 us, 8.1 TB/s with what the caches hold of the frequent rows. The gradient sorts the
// tokens (stably, so that the order of a row's sum follows from the tokens and not from
// which workgroup ran first: by ascending t within a chunk of sorted tokens, then the
// chunks' sums), sums runs of equal tokens, and writes every row of dW
// once, the ones without a token as zeros: 16384 tokens of 128256 in 247 us, of which
// the sort takes 24, its four launches' latency, and what sums and writes the 1.05 GB of dW
// 217 (210 without the non-temporal hint, but then the next lookup takes 47 us, not 32, for
// what it was left: a pass there and back on two sets of operands in turn 288 us, 277 with it).
#include <algorithm>

#include "ops_device.hpp"
#include "train.hpp"

namespace wb {
namespace {

constexpr int kThreads = 256;

// The row of a table of `rows` that token t names, or `rows` for none.
__device__ __forceinline__ uint32_t row_of(const void* tokens, int bytes, int64_t t, int64_t first, int64_t rows) {
  const int64_t id = bytes == 8 ? static_cast<const int64_t*>(tokens)[t] : int64_t(static_cast<const int32_t*>(tokens)[t]);
  const uint64_t at = static_cast<uint64_t>(id) - static_cast<uint64_t>(first);  // first <= 2^62: nothing wraps into the rows
  return static_cast<uint32_t>(at < static_cast<uint64_t>(rows) ? at : rows);
}

// ---- lookup ------------------------------------------------------------------

template <int V, bool NT>
__global__ __launch_bounds__(kThreads) void wb_embed_kernel(EmbedArgs a, int shift) {
  const int lanes = 1 << shift, lane = threadIdx.x & (lanes - 1);
  const int64_t row = int64_t(blockIdx.x) * (kThreads >> shift) + (threadIdx.x >> shift);
  if (row >= a.count) return;
  const uint32_t at = row_of(a.tokens, a.token_bytes, row, a.first, a.rows);
  const char* w = static_cast<const char*>(a.weight) + int64_t(at) * a.ld_weight * bytes_of(a.weight_type);
  char* out = static_cast<char*>(a.out) + row * a.ld_out * bytes_of(a.out_type);
  const bool there = at < a.rows;
  float v[V][8];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int64_t c = ((int64_t(blockIdx.y) * V + i) * lanes + lane) * 8;
    if (c >= a.cols) break;
    if (!there)
      for (int j = 0; j < 8; ++j) v[i][j] = 0.0f;
    else
      load_run(w, c, a.cols, a.weight_type, v[i]);
  }
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int64_t c = ((int64_t(blockIdx.y) * V + i) * lanes + lane) * 8;
    if (c >= a.cols) break;
    if (there)
      for (int j = 0; j < 8; ++j) v[i][j] *= a.scale;
    store_run<NT>(out, c, a.cols, a.out_type, v[i]);
  }
}

// ---- sort --------------------------------------------------------------------
// Least significant digits first, stable. Up to kOneBlock tokens one workgroup
// does every pass in LDS; above, a pass is two launches over blocks of tokens:
// the digits' counts, then places.

constexpr int kOneBlock = 8192, kOneThreads = 1024;
constexpr int kSortThreads = 256, kSortItems = 8, kMaxSortBlocks = 256;
constexpr int kMaxDigits = 512;

struct Passes {
  int count, bits;  // of digits of `bits`
};

Passes passes_of(int64_t rows) {  // keys 0..rows
  int bits = 1;
  while ((rows >> bits) != 0) ++bits;
  const int count = (bits + 8) / 9;
  return {count, (bits + count - 1) / count};
}

int64_t sort_block(int64_t count) {
  const int64_t per = (count + kMaxSortBlocks - 1) / kMaxSortBlocks;
  const int64_t tile = kSortThreads * (per >= kSortThreads * kSortItems ? kSortItems : 1);
  return (per + tile - 1) / tile * tile;
}

// The lanes below this one, and all, that hold the same digit.
__device__ __forceinline__ uint64_t same_digit(uint32_t digit, int bits, bool on) {
  uint64_t m = __ballot(on);
  for (int b = 0; b < bits; ++b) {
    const uint64_t with = __ballot((digit >> b) & 1);
    m &= ((digit >> b) & 1) ? with : ~with;
  }
  return m;
}

__device__ __forceinline__ int lanes_below(uint64_t m) {
  return __builtin_amdgcn_mbcnt_hi(static_cast<uint32_t>(m >> 32), __builtin_amdgcn_mbcnt_lo(static_cast<uint32_t>(m), 0));
}

// Exclusive sums over `n` digits of LDS counts, one or more to a thread; `wave` holds one entry per wavefront.
template <int THREADS>
__device__ __forceinline__ void exclusive(uint32_t* counts, int n, uint32_t* wave) {
  const int per = (n + THREADS - 1) / THREADS, tid = threadIdx.x;
  uint32_t sum = 0;
  for (int i = 0; i < per; ++i) sum += tid * per + i < n ? counts[tid * per + i] : 0;
  uint32_t upto = sum;
  for (int off = 1; off < 64; off <<= 1) {
    const uint32_t o = __shfl_up(upto, off);
    if ((tid & 63) >= off) upto += o;
  }
  if ((tid & 63) == 63) wave[tid >> 6] = upto;
  __syncthreads();
  uint32_t base = upto - sum;
  for (int w = 0; w < (tid >> 6); ++w) base += wave[w];
  for (int i = 0; i < per; ++i)
    if (tid * per + i < n) {
      const uint32_t c = counts[tid * per + i];
      counts[tid * per + i] = base;
      base += c;
    }
  __syncthreads();
}

// Up to kOneBlock tokens.
__global__ __launch_bounds__(kOneThreads) void wb_sort_few_kernel(EmbedGradArgs a, uint32_t* keys, int32_t* order, int passes,
                                                                  int bits) {
  constexpr int kWaves = kOneThreads / 64, kItems = kOneBlock / kOneThreads;
  __shared__ uint32_t key_at[kOneBlock];
  __shared__ uint16_t from_at[kOneBlock];
  __shared__ uint16_t seen[kWaves][kMaxDigits];  // per wavefront, of one digit; then where its next goes
  __shared__ uint32_t counts[kMaxDigits], wave_sums[kWaves];
  const int n = static_cast<int>(a.count), tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, digits = 1 << bits;
  // a wavefront has consecutive tokens, 64 at a time
  const int items = (n + kOneThreads - 1) / kOneThreads;
  uint32_t key[kItems], rank[kItems];
  uint32_t from[kItems];
#pragma unroll
  for (int i = 0; i < kItems; ++i) {
    if (i >= items) break;
    const int t = (wave * items + i) * 64 + lane;
    from[i] = t;
    key[i] = t < n ? row_of(a.tokens, a.token_bytes, t, a.first, a.rows) : 0xffffffffu;
  }
  for (int p = 0; p < passes; ++p) {
    for (int d = tid; d < kWaves * digits; d += kOneThreads) seen[d >> bits][d & (digits - 1)] = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      if (i >= items) break;
      const bool on = (wave * items + i) * 64 + lane < n;
      const uint32_t digit = (key[i] >> (p * bits)) & (digits - 1);
      const uint64_t same = same_digit(digit, bits, on);
      const uint32_t before = seen[wave][digit];
      rank[i] = before + lanes_below(same);
      order_lanes();
      if (on && lanes_below(same) == 0) seen[wave][digit] = static_cast<uint16_t>(before + __popcll(same));
      order_lanes();
    }
    __syncthreads();
    for (int d = tid; d < digits; d += kOneThreads) {
      uint32_t sum = 0;
      for (int w = 0; w < kWaves; ++w) {
        const uint32_t c = seen[w][d];
        seen[w][d] = static_cast<uint16_t>(sum);
        sum += c;
      }
      counts[d] = sum;
    }
    __syncthreads();
    exclusive<kOneThreads>(counts, digits, wave_sums);
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      if (i >= items || (wave * items + i) * 64 + lane >= n) continue;
      const uint32_t digit = (key[i] >> (p * bits)) & (digits - 1);
      const uint32_t to = counts[digit] + seen[wave][digit] + rank[i];
      key_at[to] = key[i];
      from_at[to] = static_cast<uint16_t>(from[i]);
    }
    __syncthreads();
    if (p + 1 < passes) {
#pragma unroll
      for (int i = 0; i < kItems; ++i) {
        if (i >= items) break;
        const int t = (wave * items + i) * 64 + lane;
        if (t < n) key[i] = key_at[t], from[i] = from_at[t];
      }
    }
  }
  for (int t = tid; t < n; t += kOneThreads) {
    keys[t] = key_at[t];
    order[t] = from_at[t];
  }
}

// Counts of a pass's digits by block, table[block][digit]. FIRST: the keys are
// made from the tokens.
template <bool FIRST>
__global__ __launch_bounds__(kSortThreads) void wb_sort_count_kernel(EmbedGradArgs a, const uint32_t* keys, uint32_t* table,
                                                                     int64_t per, int shift, int bits) {
  __shared__ uint32_t counts[kMaxDigits];
  const int digits = 1 << bits;
  for (int d = threadIdx.x; d < digits; d += kSortThreads) counts[d] = 0;
  __syncthreads();
  const int64_t begin = int64_t(blockIdx.x) * per, end = min(begin + per, a.count);
  for (int64_t t = begin + threadIdx.x; t < end; t += kSortThreads) {
    const uint32_t key = FIRST ? row_of(a.tokens, a.token_bytes, t, a.first, a.rows) : keys[t];
    atomicAdd(&counts[(key >> shift) & (digits - 1)], 1u);
  }
  __syncthreads();
  for (int d = threadIdx.x; d < digits; d += kSortThreads) table[blockIdx.x * digits + d] = counts[d];
}

// ITEMS: tokens of a thread at a time; one where there are few, for more blocks.
template <bool FIRST, int ITEMS>
__global__ __launch_bounds__(kSortThreads) void wb_sort_place_kernel(EmbedGradArgs a, const uint32_t* keys,
                                                                     const int32_t* order, const uint32_t* table,
                                                                     uint32_t* keys_to, int32_t* order_to, int64_t per,
                                                                     int shift, int bits) {
  constexpr int kWaves = kSortThreads / 64;
  __shared__ uint32_t next[kMaxDigits], mine[kMaxDigits], wave_sums[kWaves];
  __shared__ uint16_t seen[kWaves][kMaxDigits];
  const int digits = 1 << bits, tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, blocks = gridDim.x;
  // a digit's first place: those of the smaller digits, and of this one in the blocks before
  for (int d = tid; d < digits; d += kSortThreads) {
    uint32_t all = 0, before = 0;
#pragma unroll 32
    for (int b = 0; b < blocks; ++b) {
      const uint32_t c = table[b * digits + d];
      all += c;
      before += b < int(blockIdx.x) ? c : 0;
    }
    next[d] = all;
    mine[d] = before;
  }
  __syncthreads();
  exclusive<kSortThreads>(next, digits, wave_sums);
  for (int d = tid; d < digits; d += kSortThreads) next[d] += mine[d];
  __syncthreads();
  const int64_t begin = int64_t(blockIdx.x) * per, end = min(begin + per, a.count);
  for (int64_t tile = begin; tile < end; tile += kSortThreads * ITEMS) {
    for (int d = tid; d < kWaves * digits; d += kSortThreads) seen[d >> bits][d & (digits - 1)] = 0;
    __syncthreads();
    uint32_t key[ITEMS], rank[ITEMS];
    int32_t from[ITEMS];
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      const int64_t t = tile + (wave * ITEMS + i) * 64 + lane;
      if (t >= end) continue;
      key[i] = FIRST ? row_of(a.tokens, a.token_bytes, t, a.first, a.rows) : keys[t];
      from[i] = FIRST ? static_cast<int32_t>(t) : order[t];
    }
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      const bool on = tile + (wave * ITEMS + i) * 64 + lane < end;
      const uint32_t digit = on ? (key[i] >> shift) & (digits - 1) : 0;
      const uint64_t same = same_digit(digit, bits, on);
      const uint32_t before = seen[wave][digit];
      rank[i] = before + lanes_below(same);
      order_lanes();
      if (on && lanes_below(same) == 0) seen[wave][digit] = static_cast<uint16_t>(before + __popcll(same));
      order_lanes();
    }
    __syncthreads();
    for (int d = tid; d < digits; d += kSortThreads) {
      uint32_t sum = 0;
      for (int w = 0; w < kWaves; ++w) {
        const uint32_t c = seen[w][d];
        seen[w][d] = static_cast<uint16_t>(sum);
        sum += c;
      }
      mine[d] = sum;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      if (tile + (wave * ITEMS + i) * 64 + lane >= end) continue;
      const uint32_t digit = (key[i] >> shift) & (digits - 1);
      const uint32_t to = next[digit] + seen[wave][digit] + rank[i];
      keys_to[to] = key[i];
      order_to[to] = from[i];
    }
    __syncthreads();
    for (int d = tid; d < digits; d += kSortThreads) next[d] += mine[d];
    __syncthreads();
  }
}

// ---- sums --------------------------------------------------------------------
// Sorted tokens are taken in chunks. A run of equal tokens inside one chunk is
// summed and written; one that goes over an end leaves an fp32 row per chunk (0:
// the run that came in, 1: the one that goes on), which the second launch adds.

constexpr int kFillRows = 32;  // at most, to a workgroup
// Rows of a batch, their places fetched a batch ahead. Whole fp32 rows are under
// way together; a bf16 one is widened, and so waited for, before the next is asked
// for, inside load_eight's branch on the type.
constexpr int kBatch = 8;

struct Sorted {
  const uint32_t* keys;
  const int32_t* order;
  float* partial;  // [chunks][2][cols]
  int64_t chunks;
  int32_t chunk;  // tokens of one
  int32_t fill;   // rows of the table to a workgroup that looks for those without a token
};

__device__ __forceinline__ void store_scaled(const EmbedGradArgs& a, uint32_t v, int64_t c, float (&sum)[8]) {
  char* to = static_cast<char*>(a.d_weight) + int64_t(v) * a.ld_d_weight * bytes_of(a.d_weight_type);
  for (int j = 0; j < 8; ++j) sum[j] *= a.scale;
  store_run(to, c, a.cols, a.d_weight_type, sum);
}

// The first place of a key not below v, by all lanes of a wavefront: 64 places
// are looked at in a step, which takes three for 2^18 tokens where halves take
// eighteen, each a trip to memory.
__device__ __forceinline__ int64_t first_not_below(const uint32_t* keys, int64_t count, uint64_t v) {
  int64_t lo = 0, hi = count;  // keys before lo are below v, from hi on they are not
  while (lo < hi) {
    const int64_t step = (hi - lo + 63) >> 6, at = lo + (threadIdx.x & 63) * step;
    const int below = __popcll(__ballot(at < hi && keys[min(at, hi - 1)] < v));
    if (below == 0) break;
    hi = min(hi, lo + below * step);
    lo += (below - 1) * step + 1;
  }
  return lo;
}

// Zeros into the rows of a workgroup that no token names.
template <bool NT>
__device__ __forceinline__ void fill_rows(const EmbedGradArgs& a, const Sorted& s, int64_t v0, int shift) {
  __shared__ int named[kFillRows];
  if (threadIdx.x < kFillRows) named[threadIdx.x] = 0;
  __syncthreads();
  const int64_t at = first_not_below(s.keys, a.count, v0) + threadIdx.x;
  const uint32_t key = at < a.count ? s.keys[at] : ~0u;
  const bool mine = key < v0 + s.fill;
  if (mine) named[key - v0] = 1;
  if (__syncthreads_and(mine)) {  // their tokens go on past the workgroup's threads
    for (int r = threadIdx.x >> 6; r < s.fill; r += kThreads / 64) {
      const int64_t first = first_not_below(s.keys, a.count, v0 + r);
      if ((threadIdx.x & 63) == 0) named[r] = first < a.count && s.keys[first] == v0 + r;
    }
    __syncthreads();
  }
  const int lanes = 1 << shift, lane = threadIdx.x & (lanes - 1);
  const float none[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  for (int r = threadIdx.x >> shift; r < s.fill; r += kThreads >> shift) {
    const int64_t v = v0 + r;
    if (v >= a.rows || named[r]) continue;
    char* to = static_cast<char*>(a.d_weight) + v * a.ld_d_weight * bytes_of(a.d_weight_type);
    for (int64_t c = lane * 8; c < a.cols; c += lanes * 8) store_run<NT>(to, c, a.cols, a.d_weight_type, none);
  }
}

template <bool NT>
__global__ __launch_bounds__(kThreads) void wb_embed_sum_kernel(EmbedGradArgs a, Sorted s, int shift, int64_t sums, uint32_t slabs) {
  if (int64_t(blockIdx.x) >= sums) {
    fill_rows<NT>(a, s, (int64_t(blockIdx.x) - sums) * s.fill, shift);
    return;
  }
  const int lanes = 1 << shift, lane = threadIdx.x & (lanes - 1);
  const uint32_t block = blockIdx.x / slabs, slab = blockIdx.x - block * slabs;
  const int64_t chunk = int64_t(block) * (kThreads >> shift) + (threadIdx.x >> shift);
  if (chunk >= s.chunks) return;
  const int64_t c = (int64_t(slab) * lanes + lane) * 8;
  const int64_t begin = chunk * s.chunk, end = min(begin + s.chunk, a.count);
  const int db = a.d_out_type == WB_F32 ? 4 : 2;
  const int here = threadIdx.x & 63 & ~(lanes - 1);  // the wavefront's lane with this chunk's first token
  float sum[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  bool came = begin > 0 && s.keys[begin - 1] == s.keys[begin];  // the run began before this chunk
  // eight lanes have a batch's tokens and the ones after them, fetched a batch ahead
  uint32_t key_next, then_next;
  int32_t from_next;
  const auto fetch = [&](int64_t base) {
    const int64_t mine = min(base + (lane & (kBatch - 1)), end - 1);
    key_next = s.keys[mine], then_next = mine + 1 < a.count ? s.keys[mine + 1] : ~0u, from_next = s.order[mine];
  };
  fetch(begin);
  for (int64_t base = begin; base < end; base += kBatch) {
    const uint32_t key = key_next, then = then_next;
    const int32_t from = from_next;
    const int n = static_cast<int>(min(int64_t(kBatch), end - base));
    float x[kBatch][8];
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const char* row = static_cast<const char*>(a.d_out) + int64_t(__shfl(from, here + i)) * a.ld_d_out * db;
      if (c < a.cols) load_run<NT>(row, c, a.cols, a.d_out_type, x[i]);
    }
    fetch(base + kBatch);
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const uint32_t v = __shfl(key, here + i), next = __shfl(then, here + i);
      if (i >= n || v >= a.rows) continue;  // tokens of other rows are sorted last
      for (int j = 0; j < 8; ++j) sum[j] += x[i][j];
      const bool on = next == v;
      if (on && base + i + 1 < end) continue;
      if (c < a.cols) {
        if (came || on)
          store_run(reinterpret_cast<char*>(s.partial + (chunk * 2 + (came ? 0 : 1)) * a.cols), c, a.cols, WB_F32, sum);
        else
          store_scaled(a, v, c, sum);
      }
      for (int j = 0; j < 8; ++j) sum[j] = 0.0f;
      came = false;
    }
  }
}

// The runs that go over the end of the chunk they began in: a workgroup for
// each chunk's last run and 512 columns, its wavefronts over the chunks that the
// run goes on in.
constexpr int kJoinColumns = 512;

__global__ __launch_bounds__(kThreads) void wb_embed_join_kernel(EmbedGradArgs a, Sorted s, uint32_t slabs) {
  constexpr int kWaves = kThreads / 64;
  __shared__ float meet[kWaves][kJoinColumns];
  const int64_t chunk = blockIdx.x / slabs, slab = blockIdx.x - chunk * slabs, begin = chunk * s.chunk, end = begin + s.chunk;
  const uint32_t v = s.keys[end - 1];
  if (v >= a.rows || s.keys[end] != v) return;
  if (s.keys[begin] == v && begin > 0 && s.keys[begin - 1] == v) return;  // it began before
  // chunks that go on: all up to the first that begins with another token
  int64_t last = chunk + 1;
  for (bool all = true; all; last += kThreads) {
    const int64_t at = last + threadIdx.x;
    const bool on = at < s.chunks && s.keys[at * s.chunk] == v;
    all = __syncthreads_and(on);
    if (!all) {
      last += __syncthreads_count(on) - kThreads;
    }
  }
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int64_t c = slab * kJoinColumns + lane * 8;
  float sum[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  if (c < a.cols) {
    if (wave == 0) load_run(reinterpret_cast<const char*>(s.partial + (chunk * 2 + 1) * a.cols), c, a.cols, WB_F32, sum);
#pragma unroll 4
    for (int64_t next = chunk + 1 + wave; next < last; next += kWaves) {
      float x[8];
      load_run(reinterpret_cast<const char*>(s.partial + next * 2 * a.cols), c, a.cols, WB_F32, x);
      for (int j = 0; j < 8; ++j) sum[j] += x[j];
    }
  }
  for (int j = 0; j < 8; ++j) meet[wave][lane * 8 + j] = sum[j];
  __syncthreads();
  if (wave > 0 || c >= a.cols) return;
  for (int w = 1; w < kWaves; ++w)
    for (int j = 0; j < 8; ++j) sum[j] += meet[w][lane * 8 + j];
  store_scaled(a, v, c, sum);
}

// Short chunks give few tokens more workgroups (3001 x 1499 fp32: sums in 26 us with 16, 39 with 32), long ones leave many
// tokens' runs fewer rows to add (16384 x 4096 with a tenth padding: the join takes 6 us with 32, 9 with 16, 14 with 8).
int chunk_of(int64_t count) {
  int chunk = 16;
  while (chunk < 256 && count > int64_t(chunk) * 512) chunk *= 2;
  return chunk;
}

int64_t up16(int64_t n) { return (n + 15) / 16 * 16; }

// What of the workspace lies where, in bytes.
struct Layout {
  int64_t keys[2], order[2], table, partial, all;
};

Layout layout_of(int64_t count, int64_t rows, int64_t cols) {
  Layout l{};
  int64_t at = 0;
  const auto take = [&](int64_t bytes) {
    const int64_t here = at;
    at += up16(bytes);
    return here;
  };
  const bool few = count <= kOneBlock;
  for (int i = 0; i < (few ? 1 : 2); ++i) l.keys[i] = take(count * 4), l.order[i] = take(count * 4);
  if (!few) l.table = take((int64_t(4) << passes_of(rows).bits) * kMaxSortBlocks);
  const int64_t chunk = chunk_of(count);
  l.partial = take(count > chunk ? (count + chunk - 1) / chunk * 2 * cols * 4 : 0);
  l.all = at;
  return l;
}

// The launches after the sort: workgroups of the sums, of the rows without a
// token, and of the joins.
struct Grids {
  int shift;
  int32_t chunk, fill;
  int64_t chunks, slabs, sums, fills, joins;  // joins: to a chunk
  bool fit() const { return one_launch(sums + fills) && (chunks < 2 || one_launch((chunks - 1) * joins)); }
};

Grids grids_of(int64_t count, int64_t rows, int64_t cols) {
  Grids g;
  g.shift = row_shift(cols);
  g.chunk = chunk_of(count);
  g.chunks = (count + g.chunk - 1) / g.chunk;
  const int64_t per = kThreads >> g.shift;
  g.slabs = (cols + (int64_t(8) << g.shift) - 1) / (int64_t(8) << g.shift);
  // four rows, or as many as lie side by side: many workgroups, since each begins with a search (passes there
  // and back on two sets of operands in turn, 512 tokens of 32000 x 4096 bf16: 68 us against 70 with eight rows and 72 with
  // 32; 16384 of 128256: 277 against 290 and 285)
  g.fill = static_cast<int32_t>(std::max<int64_t>(4, per));
  g.sums = (g.chunks + per - 1) / per * g.slabs, g.fills = (rows + g.fill - 1) / g.fill;
  g.joins = (cols + kJoinColumns - 1) / kJoinColumns;
  return g;
}

}  // namespace

bool embed_grad_fits(int64_t count, int64_t rows, int64_t cols) { return grids_of(count, rows, cols).fit(); }

size_t embed_grad_workspace_bytes(int64_t count, int64_t rows, int64_t cols) {
  return static_cast<size_t>(layout_of(count, rows, cols).all);
}

int launch_embed(const EmbedArgs& a, void* stream) {
  if (a.count == 0) return hipSuccess;
  const auto st = static_cast<hipStream_t>(stream);
  const int shift = row_shift(a.cols);
  const int64_t per = kThreads >> shift, runs = (a.cols + 7) / 8;
  const int64_t lanes = int64_t(1) << shift;
  const auto go = [&](auto kernel, int v) {
    const int64_t x = (a.count + per - 1) / per, y = (runs + lanes * v - 1) / (lanes * v);
    if (!one_launch(x * y)) return hipErrorInvalidConfiguration;
    hipLaunchKernelGGL(kernel, dim3(static_cast<uint32_t>(x), static_cast<uint32_t>(y)), dim3(kThreads), 0, st, a, shift);
    return hipGetLastError();
  };
  const bool nt = a.count * a.cols * (bytes_of(a.weight_type) + bytes_of(a.out_type)) > kStreamBytes;
  if (runs <= lanes) return nt ? go(wb_embed_kernel<1, true>, 1) : go(wb_embed_kernel<1, false>, 1);
  return nt ? go(wb_embed_kernel<2, true>, 2) : go(wb_embed_kernel<2, false>, 2);
}

int launch_embed_grad(const EmbedGradArgs& a, void* stream) {
  const Grids g = grids_of(a.count, a.rows, a.cols);  // embed_grad_fits has said that they fit
  const auto st = static_cast<hipStream_t>(stream);
  char* ws = static_cast<char*>(a.workspace);
  const Layout l = layout_of(a.count, a.rows, a.cols);
  const Passes p = passes_of(a.rows);
  const auto keys = [&](int i) { return reinterpret_cast<uint32_t*>(ws + l.keys[i]); };
  const auto order = [&](int i) { return reinterpret_cast<int32_t*>(ws + l.order[i]); };
  int now = 0;
  if (a.count > 0 && a.count <= kOneBlock) {
    hipLaunchKernelGGL(wb_sort_few_kernel, dim3(1), dim3(kOneThreads), 0, st, a, keys(0), order(0), p.count, p.bits);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  } else if (a.count > 0) {
    const int64_t per = sort_block(a.count);
    const dim3 grid(static_cast<uint32_t>((a.count + per - 1) / per));
    auto* table = reinterpret_cast<uint32_t*>(ws + l.table);
    for (int i = 0; i < p.count; ++i) {
      const int from = now, to = i == 0 ? 0 : 1 - now, shift = i * p.bits;
      const auto pass = [&](auto counts, auto places) {
        hipLaunchKernelGGL(counts, grid, dim3(kSortThreads), 0, st, a, keys(from), table, per, shift, p.bits);
        hipLaunchKernelGGL(places, grid, dim3(kSortThreads), 0, st, a, keys(from), order(from), table, keys(to), order(to), per,
                           shift, p.bits);
      };
      const bool many = per % (kSortThreads * kSortItems) == 0;
      if (i == 0)
        pass(wb_sort_count_kernel<true>, many ? wb_sort_place_kernel<true, kSortItems> : wb_sort_place_kernel<true, 1>);
      else
        pass(wb_sort_count_kernel<false>, many ? wb_sort_place_kernel<false, kSortItems> : wb_sort_place_kernel<false, 1>);
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
      now = to;
    }
  }
  Sorted s{};
  s.keys = keys(now), s.order = order(now), s.partial = reinterpret_cast<float*>(ws + l.partial);
  s.chunk = g.chunk, s.chunks = g.chunks, s.fill = g.fill;
  if (g.sums + g.fills == 0) return hipSuccess;
  const bool nt = a.cols * (a.rows * bytes_of(a.d_weight_type) + a.count * bytes_of(a.d_out_type)) > kStreamBytes;
  hipLaunchKernelGGL(nt ? wb_embed_sum_kernel<true> : wb_embed_sum_kernel<false>, dim3(static_cast<uint32_t>(g.sums + g.fills)),
                     dim3(kThreads), 0, st, a, s, g.shift, g.sums, static_cast<uint32_t>(g.slabs));
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || g.chunks < 2) return e;
  hipLaunchKernelGGL(wb_embed_join_kernel, dim3(static_cast<uint32_t>((g.chunks - 1) * g.joins)), dim3(kThreads), 0, st, a, s,
                     static_cast<uint32_t>(g.joins));
  return hipGetLastError();
}

}  // namespace wb
