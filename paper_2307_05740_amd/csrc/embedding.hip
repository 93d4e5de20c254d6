// Embedding lookup with scaling, and its gradient by sorted tokens (include/arrow_embedding.h).
//
// Both are bound by the rows that they move.  The gradient is the product of a transposed one-hot matrix with dY: the tokens
// are sorted by id (a stable radix sort, so that a row's tokens keep their order), then each row of dW is the sum of its
// tokens' rows.  A few ids have a large part of all tokens: the sorted tokens are cut into chunks, rows that reach over a chunk's end
// are summed chunk by chunk into partial rows, and a row's own workgroup adds those up.
#include <hip/hip_runtime.h>

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

// `lanes` (a power of two) threads share a row; 256 / lanes rows at a time, kRows times.
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

// Exclusive sums of all counts, in place, one workgroup.
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

// ---- sums ----

struct SumArgs {
  const uint32_t *keys, *tokens;   // sorted
  uint32_t *begin, *end;
  float* parts;
  int64_t n, chunk, padded, rows, w_stride, y_stride;
  float scale;
  int columns, pieces, lanes_log;
};

// Adds up the rows of dY of the sorted tokens lo .. hi - 1, one piece of columns; four rows on their way at a time.
template <typename T, int VEC>
__device__ __forceinline__ void add_rows(const SumArgs& a, const T* dY, int64_t lo, int64_t hi, int c, float (&sum)[VEC]) {
  int64_t i = lo;
  for (; i + 4 <= hi; i += 4) {
    float x[4][VEC];
#pragma unroll
    for (int r = 0; r < 4; ++r) load<T, VEC>(dY + a.tokens[i + r] * a.y_stride + c, x[r]);
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int j = 0; j < VEC; ++j) sum[j] += x[r][j];
  }
  for (; i < hi; ++i) {
    float x[VEC];
    load<T, VEC>(dY + a.tokens[i] * a.y_stride + c, x);
#pragma unroll
    for (int j = 0; j < VEC; ++j) sum[j] += x[j];
  }
}

// Chunk i, columns 256 VEC of it: notes where rows begin and end among the sorted tokens, and sums its part of rows that go on
// beyond it, one that began before it into partial row 2 i, one that begins in it into 2 i + 1.
template <typename T, int VEC>
__global__ __launch_bounds__(256) void embedding_chunk_kernel(SumArgs a, const T* dY) {
  const int64_t lo = blockIdx.x * a.chunk, hi = lo + a.chunk < a.n ? lo + a.chunk : a.n;
  if (blockIdx.y == 0)
    for (int64_t i = lo + threadIdx.x; i < hi; i += 256) {
      const uint32_t key = a.keys[i];
      if (key >= a.rows) continue;
      if (i == 0 || a.keys[i - 1] != key) a.begin[key] = (uint32_t)i;
      if (i + 1 == a.n || a.keys[i + 1] != key) a.end[key] = (uint32_t)(i + 1);
    }
  const uint32_t first = a.keys[lo], last = a.keys[hi - 1];
  const int piece = blockIdx.y * 256 + threadIdx.x;
  if (piece >= a.pieces) return;
  const int c = VEC == 1 ? piece : min(piece * VEC, a.columns - VEC);
  if (first < a.rows && lo > 0 && a.keys[lo - 1] == first) {        // began before: up to where it ends, or the chunk does
    int64_t to = hi;
    if (last != first) {                                             // first place of another key
      int64_t l = lo, h = hi - 1;
      while (l < h) { const int64_t m = (l + h) / 2; if (a.keys[m] == first) l = m + 1; else h = m; }
      to = l;
    }
    float sum[VEC] = {};
    add_rows<T, VEC>(a, dY, lo, to, c, sum);
#pragma unroll
    for (int j = 0; j < VEC; ++j) a.parts[(2 * (int64_t)blockIdx.x) * a.padded + piece * VEC + j] = sum[j];
  }
  const bool began_before = lo > 0 && a.keys[lo - 1] == last;
  if (last < a.rows && hi < a.n && a.keys[hi] == last && !began_before) {
    int64_t l = lo, h = hi - 1;                                      // its first place
    while (l < h) { const int64_t m = (l + h) / 2; if (a.keys[m] < last) l = m + 1; else h = m; }
    float sum[VEC] = {};
    add_rows<T, VEC>(a, dY, l, hi, c, sum);
#pragma unroll
    for (int j = 0; j < VEC; ++j) a.parts[(2 * (int64_t)blockIdx.x + 1) * a.padded + piece * VEC + j] = sum[j];
  }
}

constexpr int kTableRows = 8;      // rows of dW of a lane group

// Every row of dW: zero, the sum of its tokens' rows, or of its partial rows.  begin[] and end[] hold what they will for
// rows without tokens: a row has tokens only where the sorted ids say so.
template <typename T, typename G, int VEC>
__global__ __launch_bounds__(256) void embedding_rows_kernel(SumArgs a, const T* dY, G* dW) {
  __shared__ uint32_t begins[256 * kTableRows], ends[256 * kTableRows];
  const int lane = threadIdx.x & ((1 << a.lanes_log) - 1), in = threadIdx.x >> a.lanes_log, abreast = 256 >> a.lanes_log;
  const int64_t row0 = (int64_t)blockIdx.x * abreast * kTableRows;
  for (int r = threadIdx.x; r < abreast * kTableRows; r += 256) {
    const int64_t row = row0 + r;
    uint32_t lo = 0, hi = 0;
    if (row < a.rows && a.n > 0) {
      const uint32_t at = a.begin[row];
      if (at < a.n && a.keys[at] == (uint32_t)row && (at == 0 || a.keys[at - 1] != (uint32_t)row)) { lo = at; hi = a.end[row]; }
    }
    begins[r] = lo;
    ends[r] = hi;
  }
  __syncthreads();
  for (int r = in; r < abreast * kTableRows; r += abreast) {
    const int64_t row = row0 + r;
    if (row >= a.rows) return;
    const int64_t lo = begins[r], hi = ends[r], c0 = lo / a.chunk, c1 = hi > lo ? (hi - 1) / a.chunk : c0;
    for (int piece = lane; piece < a.pieces; piece += 1 << a.lanes_log) {
      const int c = VEC == 1 ? piece : min(piece * VEC, a.columns - VEC);
      float sum[VEC] = {};
      if (c0 == c1) {
        add_rows<T, VEC>(a, dY, lo, hi, c, sum);
      } else {
        for (int64_t i = c0; i <= c1; ++i) {
          const float* from = a.parts + (2 * i + (i == c0)) * a.padded + piece * VEC;
#pragma unroll
          for (int j = 0; j < VEC; ++j) sum[j] += from[j];
        }
      }
#pragma unroll
      for (int j = 0; j < VEC; ++j) sum[j] *= a.scale;
      store<G, VEC>(dW + row * a.w_stride + c, sum);
    }
  }
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
  auto at = [&](size_t offset) { return (uint32_t*)((char*)ws + offset); };
  int now = 0;
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
    sort_count_kernel<<<dim3((unsigned)p.blocks), dim3(64), 0, s>>>(a);
    sort_scan_kernel<<<dim3(1), dim3(1024), 0, s>>>(a.counts, p.blocks << p.bits);
    sort_move_kernel<<<dim3((unsigned)p.blocks), dim3(64), 0, s>>>(a);
  }
  SumArgs a{};
  a.keys = at(p.keys[now]); a.tokens = at(p.tokens[now]);
  a.begin = at(p.begin); a.end = at(p.end);
  a.parts = (float*)at(p.parts);
  a.n = e.tokens; a.chunk = p.chunk; a.padded = p.padded; a.rows = e.rows; a.w_stride = e.w_stride; a.y_stride = e.y_stride;
  a.scale = e.scale; a.columns = e.columns; a.pieces = (e.columns + VEC - 1) / VEC; a.lanes_log = log2_up(a.pieces, 8);
  if (e.tokens) embedding_chunk_kernel<T, VEC><<<dim3((unsigned)p.chunks, (unsigned)((a.pieces + 255) / 256)), dim3(256), 0, s>>>(a, (const T*)dY);
  const int64_t rows = (256 >> a.lanes_log) * kTableRows, blocks = (e.rows + rows - 1) / rows;
  embedding_rows_kernel<T, G, VEC><<<dim3((unsigned)blocks), dim3(256), 0, s>>>(a, (const T*)dY, (G*)dW);
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
