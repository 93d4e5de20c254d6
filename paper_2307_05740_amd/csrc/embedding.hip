// Embedding lookup with scaling, and its gradient by sorted tokens (include/arrow_embedding.h).
//
// Both are bound by the rows that they move.  The gradient is the product of a transposed one-hot matrix with dY: the tokens
// are sorted by id (a stable radix sort, so that a row's tokens keep their order), then each row of dW is the sum of its
// tokens' rows.  A few ids have a large part of all tokens: the sorted tokens are cut into chunks, rows that reach over a chunk's end
// are summed chunk by chunk into partial rows, which a last kernel adds up.  For few tokens one kernel does all of that, its workgroups by themselves.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "embedding_internal.h"

namespace arrow {
namespace {

// Eight (or four) columns, or one where a row has fewer.  Global memory is read and written 16 bytes at a time at any
// address, so rows need no alignment; the last piece of a row is moved back to end with it, and shares columns with the one before:
// both hold the same values for them.
template <typename T, int VEC> struct Columns { typedef T type __attribute__((ext_vector_type(VEC), aligned(sizeof(T)))); };
template <typename T> struct Columns<T, 1> { typedef T type; };

template <typename T, int VEC>
__device__ __forceinline__ void load(const T* p, float (&x)[VEC]) {
  if constexpr (VEC == 1) { x[0] = (float)*p; return; }
  else {
    const auto v = *(const typename Columns<T, VEC>::type*)p;
#pragma unroll
    for (int i = 0; i < VEC; ++i) x[i] = (float)v[i];
  }
}
template <typename T, int VEC>
__device__ __forceinline__ void store(T* p, const float (&x)[VEC]) {
  if constexpr (VEC == 1) { __builtin_nontemporal_store((T)x[0], p); return; }
  else if constexpr (sizeof(T) * VEC > 16) {
#pragma unroll
    for (int h = 0; h < VEC; h += 4) {
      typename Columns<T, 4>::type v;
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = (T)x[h + i];
      __builtin_nontemporal_store(v, (typename Columns<T, 4>::type*)(p + h));
    }
  } else {
    typename Columns<T, VEC>::type v;
#pragma unroll
    for (int i = 0; i < VEC; ++i) v[i] = (T)x[i];
    __builtin_nontemporal_store(v, (typename Columns<T, VEC>::type*)p);
  }
}

__device__ __forceinline__ int64_t id_at(const void* ids, int64_t t, int wide) { return wide ? ((const int64_t*)ids)[t] : ((const int32_t*)ids)[t]; }

// `lanes` (a power of two) threads share a row; 256 / lanes rows at a time, kRows times, whose ids and pieces are on their way together.  Bound by memory: 16,384 tokens of
// 32,000 x 4096, bfloat16, 32.5 us = 5.5 TB/s (a copy: 5.1; frequent rows come out of the caches).
constexpr int kRows = 4;

template <typename T, int VEC>
__global__ __launch_bounds__(256) void embedding_kernel(arrow_embedding_t e, const T* W, const void* ids, T* Y, int lanes_log, int pieces) {
  const int lane = threadIdx.x & ((1 << lanes_log) - 1), in = threadIdx.x >> lanes_log, abreast = 256 >> lanes_log;
  const int64_t first = (int64_t)blockIdx.x * abreast * kRows + in;
  int64_t id[kRows];
#pragma unroll
  for (int r = 0; r < kRows; ++r) {
    const int64_t t = first + r * abreast;
    id[r] = t < e.tokens ? id_at(ids, t, e.id_bytes == 8) : -1;
    if (id[r] >= e.rows) id[r] = -1;
  }
  for (int piece = lane; piece < pieces; piece += 1 << lanes_log) {
    const int c = VEC == 1 ? piece : min(piece * VEC, e.columns - VEC);
    float x[kRows][VEC];
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
#pragma unroll
      for (int i = 0; i < VEC; ++i) x[r][i] = 0.f;
      if (id[r] >= 0) load<T, VEC>(W + id[r] * e.w_stride + c, x[r]);
    }
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
      const int64_t t = first + r * abreast;
      if (t >= e.tokens) continue;
#pragma unroll
      for (int i = 0; i < VEC; ++i) x[r][i] = id[r] >= 0 ? x[r][i] * e.scale : 0.f;
      store<T, VEC>(Y + t * e.y_stride + c, x[r]);
    }
  }
}

// ---- sort by id: per digit, how often each value comes in each wavefront's tokens, the places these begin at, and the move ----

struct SortArgs {
  const void* ids;                 // first digit: the caller's
  int wide;
  const uint32_t *keys, *tokens;   // later ones: of the digit before
  uint32_t *to_keys, *to_tokens;
  uint32_t* counts;                // digit value x block; after the scan: where they begin
  int64_t n, block_tokens, blocks, rows;
  int shift, bits;
};

__device__ __forceinline__ uint32_t key_at(const SortArgs& s, int64_t t) {
  if (!s.ids) return s.keys[t];
  const int64_t id = id_at(s.ids, t, s.wide);
  return (uint32_t)(id < 0 || id >= s.rows ? s.rows : id);
}

__global__ __launch_bounds__(64) void sort_count_kernel(SortArgs s) {
  __shared__ uint32_t n[1 << kDigitBits];
  const int lane = threadIdx.x, values = 1 << s.bits;
  for (int i = lane; i < values; i += 64) n[i] = 0;
  __syncthreads();
  const int64_t begin = blockIdx.x * s.block_tokens, end = begin + s.block_tokens < s.n ? begin + s.block_tokens : s.n;
  for (int64_t t = begin + lane; t < end; t += 64) atomicAdd(&n[(key_at(s, t) >> s.shift) & (values - 1)], 1u);
  __syncthreads();
  for (int i = lane; i < values; i += 64) s.counts[i * s.blocks + blockIdx.x] = n[i];
}

// Exclusive sums of all counts, in place, one workgroup, each thread a stretch of its own: 131,072 tokens of 32,000 rows, 131,072 counts a digit, 218 us, twice, where the kernels before and
// after it take 5 and 8 and the sums 284.
__global__ __launch_bounds__(1024) void sort_scan_kernel(uint32_t* counts, int64_t n) {
  __shared__ uint32_t sums[16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t each = (n + 1023) / 1024, begin = threadIdx.x * each, end = begin + each < n ? begin + each : n;
  uint32_t own = 0;
  for (int64_t i = begin; i < end; ++i) own += counts[i];
  uint32_t upto = own;
  for (int m = 1; m < 64; m <<= 1) {
    const uint32_t x = __shfl_up(upto, m, 64);
    if (lane >= m) upto += x;
  }
  if (lane == 63) sums[wave] = upto;
  __syncthreads();
  uint32_t base = upto - own;
  for (int w = 0; w < wave; ++w) base += sums[w];
  for (int64_t i = begin; i < end; ++i) {
    const uint32_t x = counts[i];
    counts[i] = base;
    base += x;
  }
}

// A wavefront moves its tokens 64 at a time, in order; lanes with one digit value take places in the order of lanes.
__global__ __launch_bounds__(64) void sort_move_kernel(SortArgs s) {
  __shared__ uint32_t next[1 << kDigitBits];
  const int lane = threadIdx.x, values = 1 << s.bits;
  for (int i = lane; i < values; i += 64) next[i] = s.counts[i * s.blocks + blockIdx.x];
  __syncthreads();
  const int64_t begin = blockIdx.x * s.block_tokens, end = begin + s.block_tokens < s.n ? begin + s.block_tokens : s.n;
  for (int64_t t0 = begin; t0 < end; t0 += 64) {
    const int64_t t = t0 + lane;
    const bool in = t < end;
    const uint32_t key = in ? key_at(s, t) : 0, digit = (key >> s.shift) & (values - 1);
    uint64_t same = __ballot(in);
    for (int b = 0; b < s.bits; ++b) {
      const uint64_t set = __ballot(digit >> b & 1);
      same &= digit >> b & 1 ? set : ~set;
    }
    const int before = __popcll(same & (((uint64_t)1 << lane) - 1));
    const uint32_t at = in ? next[digit] + before : 0;
    __syncthreads();
    if (in && before == 0) next[digit] += __popcll(same);
    __syncthreads();
    if (in) {
      s.to_keys[at] = key;
      s.to_tokens[at] = s.tokens ? s.tokens[t] : (uint32_t)t;
    }
  }
}

// The sort of a digit in one launch, for few tokens: every workgroup counts all of them, those before its own ones in the upper half of
// a word, and so knows where its own go: block_tokens of them, whole wavefronts' and at most as many as it has threads.  16,384 tokens of 32,000
// rows: 17 us, of which the 32 Ki counts in LDS are about 6, where the three launches above take some 20, twice.
constexpr int kSortBlock = 1024;

__global__ __launch_bounds__(kSortBlock) void sort_few_kernel(SortArgs s, uint32_t* row_begin) {
  __shared__ __align__(16) uint32_t bins[1 << kWideDigitBits];
  __shared__ uint32_t sums[kSortBlock / 64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, values = 1 << s.bits, mask = values - 1;
  // four values to a place; threads that go through neighbouring places do not meet in a bank
  auto place = [](uint32_t b) { return b ^ ((b >> 6 & 7) << 2); };
  for (int i = 4 * threadIdx.x; i < values; i += 4 * kSortBlock) *(uint4*)&bins[i] = uint4{0, 0, 0, 0};
  const int n = (int)s.n, own = (int)(blockIdx.x * s.block_tokens), t = own + threadIdx.x;
  const bool in = threadIdx.x < s.block_tokens && t < n;
  uint32_t key = in ? key_at(s, t) : 0;
  constexpr int kBatch = 8;
  for (int begin = 0; begin < n; begin += kBatch * kSortBlock) {     // (as often for every thread: there is a barrier in it)
    const int t0 = begin + threadIdx.x;
    uint32_t x[kBatch];
#pragma unroll
    for (int r = 0; r < kBatch; ++r) x[r] = t0 + r * kSortBlock < n ? key_at(s, t0 + r * kSortBlock) : 0;
    if (begin == 0) __syncthreads();
#pragma unroll
    for (int r = 0; r < kBatch; ++r) {
      const int at = t0 + r * kSortBlock;
      if (at < n) atomicAdd(&bins[place((x[r] >> s.shift) & mask)], at < own ? 0x10001u : 1u);
    }
  }
  __syncthreads();
  // where each value begins: all tokens of smaller ones, and its own before this workgroup's
  const int each = (values + kSortBlock - 1) / kSortBlock, first = threadIdx.x * each;
  uint32_t count = 0;
  if (each < 4) {
    for (int i = first; i < first + each && i < values; ++i) count += bins[place(i)] & 0xffff;
  } else {
#pragma unroll 8
    for (int i = first; i < first + each; i += 4) {
      const uint4 x = *(const uint4*)&bins[place(i)];
      count += (x.x & 0xffff) + (x.y & 0xffff) + (x.z & 0xffff) + (x.w & 0xffff);
    }
  }
  uint32_t upto = count;
  for (int m = 1; m < 64; m <<= 1) {
    const uint32_t x = __shfl_up(upto, m, 64);
    if (lane >= m) upto += x;
  }
  if (lane == 63) sums[wave] = upto;
  __syncthreads();
  uint32_t base = lane < wave ? sums[lane] : 0;                      // (at most 15 wavefronts before)
  for (int m = 1; m < 16; m <<= 1) base += __shfl_xor(base, m, 64);
  base = __shfl(base, 0, 64) + upto - count;
  // the only digit: a value is a row; every workgroup notes a part of them
  const bool note = row_begin && threadIdx.x % gridDim.x == blockIdx.x;
  if (each < 4) {
    for (int i = first; i < first + each && i < values; ++i) {
      const uint32_t x = bins[place(i)];
      if (note && i <= s.rows) row_begin[i] = base;
      bins[place(i)] = base + (x >> 16);
      base += x & 0xffff;
    }
  } else {
#pragma unroll 8
    for (int i = first; i < first + each; i += 4) {
      const uint4 x = *(const uint4*)&bins[place(i)];
      const uint32_t a = base + (x.x & 0xffff), b = a + (x.y & 0xffff), c = b + (x.z & 0xffff);
      *(uint4*)&bins[place(i)] = uint4{base + (x.x >> 16), a + (x.y >> 16), b + (x.z >> 16), c + (x.w >> 16)};
      if (note && i <= s.rows) *(uint4*)&row_begin[i] = uint4{base, a, b, c};   // (there is room for the last four)
      base = c + (x.w & 0xffff);
    }
  }
  __syncthreads();
  // this workgroup's tokens, in order: the lanes of a wavefront with one value, one wavefront after the other
  const int waves = (int)(s.block_tokens + 63) / 64;
  if (waves == 1 && wave > 0) return;                                // (no barrier below is one of several wavefronts then)
  const uint32_t digit = (key >> s.shift) & mask;
  uint64_t same = __ballot(in);
  for (int b = 0; b < s.bits; ++b) {
    const uint64_t set = __ballot(digit >> b & 1);
    same &= digit >> b & 1 ? set : ~set;
  }
  const int before = __popcll(same & (((uint64_t)1 << lane) - 1));
  uint32_t at = 0;
  for (int w = 0; w < waves; ++w) {
    if (w == wave && in) {
      at = bins[place(digit)];
      if (before == 0) bins[place(digit)] = at + __popcll(same);
    }
    if (waves > 1) __syncthreads();
  }
  if (in) {
    s.to_keys[at + before] = key;
    s.to_tokens[at + before] = s.tokens ? s.tokens[t] : (uint32_t)t;
  }
}

// Where rows begin and end among the sorted tokens.
__global__ __launch_bounds__(256) void sort_rows_kernel(const uint32_t* keys, int64_t n, int64_t rows, uint32_t* begin, uint32_t* end) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= n) return;
  const uint32_t key = keys[i];
  if (key >= rows) return;
  if (i == 0 || keys[i - 1] != key) begin[key] = (uint32_t)i;
  if (i + 1 == n || keys[i + 1] != key) end[key] = (uint32_t)(i + 1);
}

// ---- sums ----

struct SumArgs {
  const uint32_t *keys, *tokens;   // sorted
  uint32_t *begin, *end;
  float* parts;
  int64_t n, chunk, padded, rows, w_stride, y_stride;
  float scale;
  int columns, pieces, lanes_log;
};

// One piece of columns of chunk `chunk` of the sorted tokens: a row whose tokens all lie in it goes to dW, the part of one that began
// before it to partial row 2 chunk, of one that begins in it and goes on to 2 chunk + 1.  Eight tokens' rows are on their way at a time, whichever
// rows of dW they belong to.
template <typename T, typename G, int VEC>
__device__ __forceinline__ void add_chunk(const SumArgs& a, const T* dY, G* dW, int64_t chunk, int piece) {
  constexpr int kAhead = 8;
  static_assert(kChunkTokens % kAhead == 0, "keys are read eight at a time");
  const int64_t lo = chunk * a.chunk, hi = lo + a.chunk < a.n ? lo + a.chunk : a.n;
  const int c = VEC == 1 ? piece : min(piece * VEC, a.columns - VEC);
  constexpr uint32_t kNone = 0xffffffffu;
  const uint32_t before = lo > 0 ? a.keys[lo - 1] : kNone, after = hi < a.n ? a.keys[hi] : kNone;
  struct Eight { uint4 lo, hi; };                                   // (the arrays have room for the last eight)
  auto eight = [](const uint32_t* p) { return Eight{*(const uint4*)p, *(const uint4*)(p + 4)}; };
  auto spread = [](const Eight& e, uint32_t (&x)[kAhead]) {
    x[0] = e.lo.x; x[1] = e.lo.y; x[2] = e.lo.z; x[3] = e.lo.w; x[4] = e.hi.x; x[5] = e.hi.y; x[6] = e.hi.z; x[7] = e.hi.w;
  };
  Eight keys = eight(a.keys + lo), tokens = eight(a.tokens + lo);
  bool began_before = keys.lo.x == before;
  float sum[VEC] = {};
  uint32_t key[kAhead], token[kAhead], now = kNone;
  for (int64_t i = lo; i < hi; i += kAhead) {
    spread(keys, key);
    spread(tokens, token);
    typename Columns<T, VEC>::type x[kAhead];
#pragma unroll
    for (int r = 0; r < kAhead; ++r)
      if (i + r < hi && key[r] < a.rows) x[r] = *(const typename Columns<T, VEC>::type*)(dY + (int64_t)token[r] * a.y_stride + c);
    const bool more = i + kAhead < hi;
    if (more) { keys = eight(a.keys + i + kAhead); tokens = eight(a.tokens + i + kAhead); }
#pragma unroll
    for (int r = 0; r < kAhead; ++r) {
      if (i + r >= hi || key[r] >= a.rows) continue;
      now = key[r];
      if constexpr (VEC == 1) sum[0] += (float)x[r];
      else {
#pragma unroll
        for (int j = 0; j < VEC; ++j) sum[j] += (float)x[r][j];
      }
      const uint32_t next = i + r + 1 == hi ? after : r + 1 < kAhead ? key[r + 1 < kAhead ? r + 1 : 0] : keys.lo.x;
      if (next == now) continue;
      if (began_before) {
#pragma unroll
        for (int j = 0; j < VEC; ++j) a.parts[2 * chunk * a.padded + piece * VEC + j] = sum[j];
      } else {
#pragma unroll
        for (int j = 0; j < VEC; ++j) sum[j] *= a.scale;
        store<G, VEC>(dW + (int64_t)now * a.w_stride + c, sum);
      }
      began_before = false;
#pragma unroll
      for (int j = 0; j < VEC; ++j) sum[j] = 0.f;
    }
  }
  if (after != kNone && now == after) {
#pragma unroll
    for (int j = 0; j < VEC; ++j) a.parts[(2 * chunk + !began_before) * a.padded + piece * VEC + j] = sum[j];
  }
}

constexpr int kTableRows = 8;      // rows of dW that a lane group looks over

// The first workgroups add up the chunks, `slices` of them per 256 >> lanes_log chunks; the others clear the rows of dW that have no tokens.
// kNoted: begin[] and end[] say which those are; otherwise they hold what they will for such rows, and a row has tokens only where the sorted ids say so.
// Bound by memory: 16,384 tokens of 32,000 x 4096, bfloat16, 78 us = 5.1 TB/s.
template <typename T, typename G, int VEC, bool kNoted>
__global__ __launch_bounds__(256) void embedding_rows_kernel(SumArgs a, const T* dY, G* dW, int64_t chunks, int chunk_blocks, int slices) {
  const int lane = threadIdx.x & ((1 << a.lanes_log) - 1), in = threadIdx.x >> a.lanes_log, abreast = 256 >> a.lanes_log;
  if ((int)blockIdx.x < chunk_blocks) {
    const int64_t chunk = (int64_t)(blockIdx.x / slices) * abreast + in;
    const int piece = (blockIdx.x % slices << a.lanes_log) + lane;
    if (chunk < chunks && piece < a.pieces) add_chunk<T, G, VEC>(a, dY, dW, chunk, piece);
    return;
  }
  __shared__ bool empty[256 * kTableRows];
  const int64_t row0 = (int64_t)(blockIdx.x - chunk_blocks) * abreast * kTableRows;
  for (int r = threadIdx.x; r < abreast * kTableRows; r += 256) {
    const int64_t row = row0 + r;
    bool none = row < a.rows;
    if (none && a.n > 0) {
      const uint32_t at = a.begin[row];
      none = kNoted ? at == a.end[row] : !(at < a.n && a.keys[at] == (uint32_t)row && (at == 0 || a.keys[at - 1] != (uint32_t)row));
    }
    empty[r] = none;
  }
  __syncthreads();
  const float zero[VEC] = {};
  for (int r = in; r < abreast * kTableRows; r += abreast)
    if (empty[r])
      for (int piece = lane; piece < a.pieces; piece += 1 << a.lanes_log)
        store<G, VEC>(dW + (row0 + r) * a.w_stride + (VEC == 1 ? piece : min(piece * VEC, a.columns - VEC)), zero);
}

// The rows that go over the end of a chunk, each by the end that it goes over first: their partial rows added up in order.
template <typename G, int VEC>
__global__ __launch_bounds__(64) void embedding_join_kernel(SumArgs a, G* dW) {
  const int64_t chunk = blockIdx.x, edge = (chunk + 1) * a.chunk;    // (there is a token at the edge)
  const uint32_t row = a.keys[edge];
  if (row >= a.rows || a.keys[edge - 1] != row) return;
  const int64_t lo = a.begin[row], last = (a.end[row] - 1) / a.chunk;
  if (lo < chunk * a.chunk) return;
  const int piece = blockIdx.y * 64 + threadIdx.x;
  if (piece >= a.pieces) return;
  const int c = VEC == 1 ? piece : min(piece * VEC, a.columns - VEC);
  float sum[VEC] = {};
  const float* from = a.parts + piece * VEC;
#pragma unroll
  for (int j = 0; j < VEC; ++j) sum[j] = from[(2 * chunk + 1) * a.padded + j];
#pragma unroll 8
  for (int64_t i = chunk + 1; i <= last; ++i)
#pragma unroll
    for (int j = 0; j < VEC; ++j) sum[j] += from[2 * i * a.padded + j];
#pragma unroll
  for (int j = 0; j < VEC; ++j) sum[j] *= a.scale;
  store<G, VEC>(dW + row * a.w_stride + c, sum);
}

// ---- the whole gradient in one launch, for few tokens ----

// A workgroup has one slice of the columns of every 2^step_log-th row of dW, at most kDirectRows of them (frequent ids often have numbers next to each
// other).  It goes through all ids for those that are its own, sorts them by row in LDS (each wavefront a quarter of the tokens, in
// order), and 16 groups of 16 lanes add up equal parts of what it found; rows that reach over a part's end are joined in LDS, in order.
//
// What bounds it: of few tokens, the launch and three loads that wait for each other; of large tables, the rows that are written.  Up to kDirectTokens it is
// faster than the launches it replaces (us, those -> this; ids as in text, of columns in bfloat16; "one": the same id for all):
//   128 tokens:   32,000 x 512 20 -> 10, 32,000 x 4096 65 -> 52, 1000 x 4096 12 -> 6, 50 x 64 11 -> 5
//   2048 tokens:  32,000 x 512 23 -> 14, 32,000 x 4096 67 -> 64, 1000 x 4096 18 -> 14, 50 x 64 13 -> 12; one: 40 -> 32, 87 -> 51, 35 -> 35, 28 -> 30
// and of rows shorter than a slice, which leave lanes idle, up to kDirectTable of them (512 tokens): 75,000 x 32 18 -> 8, 150,000 x 32 18 -> 12, 300,000 x 32 20 -> 19,
// 600,000 x 32 21 -> 32, 600,000 x 128 41 -> 33.  Beyond kDirectTokens:
//   4096 tokens:  32,000 x 512 24 -> 21, 32,000 x 4096 73 -> 126, 1000 x 4096 25 -> 23, 50 x 64 16 -> 19; one: 61 -> 57, 112 -> 88, 58 -> 71, 46 -> 56
constexpr int kDirectRows = 64, kDirectLanes = 16, kDirectBlocks = 1024;

template <typename T, typename G, int VEC>
__global__ __launch_bounds__(256) void embedding_direct_kernel(arrow_embedding_t e, const T* dY, const void* ids, G* dW, int step_log, int slices, int pieces) {
  constexpr int kSteps = kDirectTokens / 256, kGroups = 256 / kDirectLanes, kAhead = 8;
  constexpr uint32_t kNone = 0xffffffffu;
  static_assert(kDirectRows * 4 == 256 && kDirectTokens <= 65536, "a thread for every row and wavefront; tokens of 16 bits");
  __shared__ uint32_t next[kDirectRows * 4];       // per row and wavefront: its tokens, then where they go
  __shared__ uint32_t list[kDirectTokens];         // token, row << 16
  __shared__ uint32_t sums[4];
  __shared__ float parts[2 * kGroups][kDirectLanes * VEC];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, tokens = (int)e.tokens;
  const int slice = blockIdx.x % slices;
  const int64_t row0 = blockIdx.x / slices, step = (int64_t)1 << step_log;   // its rows: row0 + r step
  const int rows = (int)((e.rows - row0 + step - 1) >> step_log);
  next[threadIdx.x] = 0;
  const int steps = (tokens + 255) / 256, t0 = wave * steps * 64 + lane;
  uint32_t row[kSteps];
#pragma unroll
  for (int i = 0; i < kSteps; ++i) {
    const int t = t0 + 64 * i;
    const int64_t id = i < steps && t < tokens ? id_at(ids, t, e.id_bytes == 8) : -1;
    row[i] = id >= 0 && id < e.rows && (id & (step - 1)) == row0 ? (uint32_t)(id >> step_log) : kNone;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kSteps; ++i)
    if (row[i] != kNone) atomicAdd(&next[4 * row[i] + wave], 1u);
  __syncthreads();
  const uint32_t count = next[threadIdx.x];
  uint32_t upto = count;
  for (int m = 1; m < 64; m <<= 1) {
    const uint32_t x = __shfl_up(upto, m, 64);
    if (lane >= m) upto += x;
  }
  if (lane == 63) sums[wave] = upto;
  __syncthreads();
  uint32_t base = 0, all = 0;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    if (w < wave) base += sums[w];
    all += sums[w];
  }
  next[threadIdx.x] = base + upto - count;
  __syncthreads();
  // (a wavefront's places are its own: its steps go one after the other, and lanes with one row in the order of lanes)
  volatile uint32_t* place = next;
#pragma unroll
  for (int i = 0; i < kSteps; ++i) {
    const bool in = row[i] != kNone;
    uint64_t same = __ballot(in);
    if (same == 0) continue;
    for (int b = 0; b < 6; ++b) {
      const uint64_t set = __ballot(row[i] >> b & 1);
      same &= row[i] >> b & 1 ? set : ~set;
    }
    if (in) {
      const int before = __popcll(same & (((uint64_t)1 << lane) - 1));
      const uint32_t at = place[4 * row[i] + wave];
      if (before == 0) place[4 * row[i] + wave] = at + __popcll(same);
      list[at + before] = (uint32_t)(t0 + 64 * i) | row[i] << 16;
    }
  }
  __syncthreads();
  // now row r has the places from the end of the one before, next[4 r - 1], to next[4 r + 3]
  const int group = threadIdx.x / kDirectLanes, in = threadIdx.x % kDirectLanes, piece = slice * kDirectLanes + in;
  const bool there = piece < pieces;
  const int c = min(piece * VEC, e.columns - VEC);
  const float zero[VEC] = {};
  for (int r = group; r < rows; r += kGroups)
    if (there && next[4 * r + 3] == (r ? next[4 * r - 1] : 0)) store<G, VEC>(dW + (row0 + r * step) * e.w_stride + c, zero);
  const int n = (int)all, each = max(1, (n + kGroups - 1) / kGroups), lo = group * each, hi = min(n, lo + each);
  bool began_before = lo > 0 && lo < hi && list[lo] >> 16 == list[lo - 1] >> 16;
  float sum[VEC] = {};
  for (int i = lo; i < hi; i += kAhead) {
    uint32_t entry[kAhead + 1];
    typename Columns<T, VEC>::type x[kAhead];
#pragma unroll
    for (int r = 0; r <= kAhead; ++r) entry[r] = list[min(i + r, n - 1)];
#pragma unroll
    for (int r = 0; r < kAhead; ++r)                            // (without branches: some lanes load what they do not need)
      x[r] = *(const typename Columns<T, VEC>::type*)(dY + (int64_t)(entry[r] & 0xffff) * e.y_stride + c);
#pragma unroll
    for (int r = 0; r < kAhead; ++r) {
      if (i + r >= hi) continue;
      if constexpr (VEC == 1) sum[0] += (float)x[r];
      else {
#pragma unroll
        for (int j = 0; j < VEC; ++j) sum[j] += (float)x[r][j];
      }
      const bool goes_on = i + r + 1 < n && entry[r] >> 16 == entry[r + 1] >> 16;
      if (goes_on && i + r + 1 < hi) continue;
      if (began_before || goes_on) {
#pragma unroll
        for (int j = 0; j < VEC; ++j) parts[2 * group + !began_before][in * VEC + j] = sum[j];
      } else if (there) {
#pragma unroll
        for (int j = 0; j < VEC; ++j) sum[j] *= e.scale;
        store<G, VEC>(dW + (row0 + (entry[r] >> 16) * step) * e.w_stride + c, sum);
      }
      began_before = false;
#pragma unroll
      for (int j = 0; j < VEC; ++j) sum[j] = 0.f;
    }
  }
  __syncthreads();
  if (lo >= hi || hi >= n || !there) return;
  const int r = list[hi - 1] >> 16, begin = r ? next[4 * r - 1] : 0;
  if ((int)(list[hi] >> 16) != r || begin < lo) return;
  const int last = (int)(next[4 * r + 3] - 1) / each;
#pragma unroll
  for (int j = 0; j < VEC; ++j) sum[j] = parts[2 * group + 1][in * VEC + j];
  for (int g = group + 1; g <= last; ++g)
#pragma unroll
    for (int j = 0; j < VEC; ++j) sum[j] += parts[2 * g][in * VEC + j];
#pragma unroll
  for (int j = 0; j < VEC; ++j) sum[j] *= e.scale;
  store<G, VEC>(dW + (row0 + r * step) * e.w_stride + c, sum);
}

int log2_up(int64_t x, int most) {
  int r = 0;
  while (r < most && ((int64_t)1 << r) < x) ++r;
  return r;
}

template <typename T, int VEC>
int forward(const arrow_embedding_t& e, const void* W, const void* ids, void* Y, hipStream_t s) {
  const int pieces = (e.columns + VEC - 1) / VEC, lanes_log = log2_up(pieces, 8);
  const int64_t rows = (256 >> lanes_log) * kRows, blocks = (e.tokens + rows - 1) / rows;
  embedding_kernel<T, VEC><<<dim3((unsigned)blocks), dim3(256), 0, s>>>(e, (const T*)W, ids, (T*)Y, lanes_log, pieces);
  return (int)hipGetLastError();
}

template <typename T, typename G, int VEC>
int backward(const arrow_embedding_t& e, const EmbeddingPlan& p, const void* dY, const void* ids, void* dW, void* ws, hipStream_t s) {
  if (p.direct) {
    const int pieces = (e.columns + VEC - 1) / VEC, slices = (pieces + kDirectLanes - 1) / kDirectLanes;
    const int step_log = log2_up(std::max<int64_t>(kDirectBlocks / slices, (e.rows + kDirectRows - 1) / kDirectRows), 31);
    const int64_t blocks = std::min<int64_t>(e.rows, (int64_t)1 << step_log) * slices;
    if (blocks > 0x7fffffff) return (int)hipErrorInvalidConfiguration;
    embedding_direct_kernel<T, G, VEC><<<dim3((unsigned)blocks), dim3(256), 0, s>>>(e, (const T*)dY, ids, (G*)dW, step_log, slices, pieces);
    return (int)hipGetLastError();
  }
  auto at = [&](size_t offset) { return (uint32_t*)((char*)ws + offset); };
  int now = 0;
  const bool noted = p.few && p.passes == 1;
  for (int i = 0; i < p.passes && e.tokens; ++i) {
    SortArgs a{};
    a.ids = i == 0 ? ids : nullptr;
    a.wide = e.id_bytes == 8;
    a.keys = at(p.keys[now]);
    a.tokens = i == 0 ? nullptr : at(p.tokens[now]);
    now ^= 1;
    a.to_keys = at(p.keys[now]);
    a.to_tokens = at(p.tokens[now]);
    a.counts = at(p.counts);
    a.n = e.tokens; a.block_tokens = p.block_tokens; a.blocks = p.blocks; a.rows = e.rows;
    a.shift = i * p.bits; a.bits = p.bits;
    if (p.few) {
      a.block_tokens = 64 * ((e.tokens + 64 * 256 - 1) / (64 * 256));   // a workgroup for every compute unit
      a.blocks = (e.tokens + a.block_tokens - 1) / a.block_tokens;
      sort_few_kernel<<<dim3((unsigned)a.blocks), dim3(kSortBlock), 0, s>>>(a, noted ? at(p.begin) : nullptr);
      continue;
    }
    sort_count_kernel<<<dim3((unsigned)p.blocks), dim3(64), 0, s>>>(a);
    sort_scan_kernel<<<dim3(1), dim3(1024), 0, s>>>(a.counts, p.blocks << p.bits);
    sort_move_kernel<<<dim3((unsigned)p.blocks), dim3(64), 0, s>>>(a);
  }
  SumArgs a{};
  a.keys = at(p.keys[now]); a.tokens = at(p.tokens[now]);
  a.begin = at(p.begin); a.end = noted ? a.begin + 1 : at(p.end);
  a.parts = (float*)at(p.parts);
  a.n = e.tokens; a.chunk = p.chunk; a.padded = p.padded; a.rows = e.rows; a.w_stride = e.w_stride; a.y_stride = e.y_stride;
  a.scale = e.scale; a.columns = e.columns; a.pieces = (e.columns + VEC - 1) / VEC; a.lanes_log = log2_up(a.pieces, 8);
  if (e.tokens && !noted) sort_rows_kernel<<<dim3((unsigned)((e.tokens + 255) / 256)), dim3(256), 0, s>>>(a.keys, a.n, a.rows, a.begin, a.end);
  const int abreast = 256 >> a.lanes_log, slices = (a.pieces + (1 << a.lanes_log) - 1) >> a.lanes_log;
  const int64_t chunk_blocks = (p.chunks + abreast - 1) / abreast * slices;
  const int64_t rows = abreast * kTableRows, blocks = chunk_blocks + (e.rows + rows - 1) / rows;
  if (blocks > 0x7fffffff) return (int)hipErrorInvalidConfiguration;
  auto sums = [&](auto is_noted) {
    embedding_rows_kernel<T, G, VEC, decltype(is_noted)::value>
        <<<dim3((unsigned)blocks), dim3(256), 0, s>>>(a, (const T*)dY, (G*)dW, p.chunks, (int)chunk_blocks, slices);
  };
  if (noted) sums(std::true_type{}); else sums(std::false_type{});
  if (p.chunks > 1)
    embedding_join_kernel<G, VEC><<<dim3((unsigned)(p.chunks - 1), (unsigned)((a.pieces + 63) / 64)), dim3(64), 0, s>>>(a, (G*)dW);
  return (int)hipGetLastError();
}

template <typename T, typename G>
int backward_of(const arrow_embedding_t& e, const EmbeddingPlan& p, const void* dY, const void* ids, void* dW, void* ws, hipStream_t s) {
  constexpr int VEC = 16 / sizeof(T);
  return e.columns >= VEC ? backward<T, G, VEC>(e, p, dY, ids, dW, ws, s) : backward<T, G, 1>(e, p, dY, ids, dW, ws, s);
}

}  // namespace

int launch_embedding_forward(const arrow_embedding_t& e, const void* W, const void* ids, void* Y, void* stream) {
  hipStream_t s = (hipStream_t)stream;
  if (e.dtype == ARROW_F32) return e.columns >= 4 ? forward<float, 4>(e, W, ids, Y, s) : forward<float, 1>(e, W, ids, Y, s);
  if (e.dtype == ARROW_BF16) return e.columns >= 8 ? forward<__bf16, 8>(e, W, ids, Y, s) : forward<__bf16, 1>(e, W, ids, Y, s);
  return e.columns >= 8 ? forward<_Float16, 8>(e, W, ids, Y, s) : forward<_Float16, 1>(e, W, ids, Y, s);
}

int launch_embedding_backward(const arrow_embedding_t& e, const EmbeddingPlan& p, const void* dY, const void* ids, void* dW, void* ws, void* stream) {
  hipStream_t s = (hipStream_t)stream;
  if (e.dtype == ARROW_F32) return backward_of<float, float>(e, p, dY, ids, dW, ws, s);
  if (e.dtype == ARROW_BF16)
    return e.grad_dtype == ARROW_F32 ? backward_of<__bf16, float>(e, p, dY, ids, dW, ws, s) : backward_of<__bf16, __bf16>(e, p, dY, ids, dW, ws, s);
  return e.grad_dtype == ARROW_F32 ? backward_of<_Float16, float>(e, p, dY, ids, dW, ws, s) : backward_of<_Float16, _Float16>(e, p, dY, ids, dW, ws, s);
}

}  // namespace arrow
