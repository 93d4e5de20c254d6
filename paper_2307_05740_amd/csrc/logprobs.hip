// Log probabilities of given tokens, entropies, most likely tokens, and the gradient (include/arrow_logprobs.h).
//
// What bounds it is memory: the logits are read once (backward: read and written).  A workgroup holds a part of a row in its registers, so that the
// maximum, the sums relative to it and the largest logits all come from one reading; a second kernel joins the parts of rows that were cut.
//
// The largest logits.  Value and index of a logit make one whole number, its key, so that no two are alike and the order is that of the results.  The value that comes `top`-th
// among the lanes' largest ones (a search by bits, counting lanes by ballots) is no larger than the `top`-th of all: the border.  The few pieces that reach it are read again, and their keys
// from it on go to a list in LDS, where each is placed by counting those before it.  If so many are alike that the list has no room, the border is found again as a key.
//
// Measured: 8192 rows of 32,000 in bfloat16 with the five best 112 us by itself, 4.7 TB/s of 524 MB, vector instructions in 83 % of the cycles, some twelve for a logit and a hundred for
// a row's border; 96 a call of several in a row, whose first workgroups fill what the last ones of the call before leave (5.5 TB/s: reads alone are faster than a copy, 5.1);
// 4095 of 50,257 without any, and their gradient: 110 and 135 us, 3.8 and 6.2 TB/s (the gradient's writes go on under the next forward call; forward calls alone 74), 243 together for 242 of
// the floor, in float32 145 and 296; 4 rows of 128,001 in float32 with the twenty best 7.3 us and 5.7 for the join, launches and barriers.  With a third or nine tenths of the
// logits masked by -infinity 4095 of 50,257 take 180 us and 8192 of 32,000 134, as every wavefront adds up its pieces again.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "attention_common.h"
#include "lanes.h"
#include "logprobs_internal.h"

namespace arrow {
namespace {

constexpr int kThreads = kScoreThreads, kWaves = kThreads / 64;
constexpr int kList = 1024;           // keys from the border on that a workgroup has room for
constexpr float kLeast = -256.f;      // exponents of two below this are 0, and so is their product with it

__device__ __forceinline__ uint32_t word_of(const u32x4& r, int i) { return i < 2 ? (i == 0 ? r[0] : r[1]) : i == 2 ? r[2] : r[3]; }

template <typename T> struct Piece;   // 16 bytes of a row; an element of it (`any` takes numbers that are no constants)
template <> struct Piece<float> {
  static constexpr int kEach = 4;
  static constexpr uint32_t kNothing = 0xff800000u;
  static __device__ __forceinline__ float any(const u32x4& r, int i) { return __uint_as_float(word_of(r, i)); }
  static __device__ __forceinline__ float get(const u32x4& r, int i) { return __uint_as_float(r[i]); }
};
template <> struct Piece<__bf16> {
  static constexpr int kEach = 8;
  static constexpr uint32_t kNothing = 0xff80ff80u;
  static __device__ __forceinline__ float any(const u32x4& r, int i) { return __uint_as_float(word_of(r, i >> 1) >> (16 * (i & 1)) << 16); }
  static __device__ __forceinline__ float get(const u32x4& r, int i) { return __uint_as_float(i & 1 ? r[i / 2] & 0xffff0000u : r[i / 2] << 16); }
};
template <> struct Piece<_Float16> {
  static constexpr int kEach = 8;
  static constexpr uint32_t kNothing = 0xfc00fc00u;
  static __device__ __forceinline__ float any(const u32x4& r, int i) {
    union { uint16_t u; _Float16 f; } x;
    x.u = (uint16_t)(word_of(r, i >> 1) >> (16 * (i & 1)));
    return (float)x.f;
  }
  static __device__ __forceinline__ float get(const u32x4& r, int i) {
    union { uint16_t u; _Float16 f; } x;
    x.u = (uint16_t)(i & 1 ? r[i / 2] >> 16 : r[i / 2]);
    return (float)x.f;
  }
};

// The scale for exponents of two.  (Finite: the largest logit's difference from itself times an infinity is no number.)
__device__ __forceinline__ float exponents(float scale) { return fminf(scale * kLog2e, 3.402823466e38f); }

// The larger of two; NaN where one is.
__device__ __forceinline__ float larger(float a, float b) { return __builtin_elementwise_maximum(a, b); }

// One element as a piece, for rows of so few that pieces of 16 bytes leave most lanes without any.
template <typename T> struct One : Piece<T> { static constexpr int kEach = 1; };

// A row's elements: those before the first address that is a multiple of 16, whole pieces, and the rest.
template <typename T, typename P = Piece<T>>
struct Row {
  const T* at;
  int head, pieces, rest;
  __device__ __forceinline__ Row(const T* row, int n) {
    constexpr int kEach = P::kEach;
    const int off = (int)(((uintptr_t)row & 15) / sizeof(T));
    at = row;
    head = kEach > 1 && off ? min(kEach - off, n) : 0;
    pieces = (n - head) / kEach;
    rest = (n - head) % kEach;
  }
  __device__ __forceinline__ const u32x4* piece(int i) const { return (const u32x4*)(at + head + (int64_t)i * P::kEach); }
  __device__ __forceinline__ u32x4 load(int i) const {
    if constexpr (P::kEach > 1) return *piece(i);
    else if constexpr (sizeof(T) == 4) return u32x4{((const uint32_t*)at)[i], 0, 0, 0};
    else return u32x4{((const uint16_t*)at)[i], 0, 0, 0};
  }
  __device__ __forceinline__ int index(int piece, int i) const { return head + piece * P::kEach + i; }
  // the element beside the pieces that lane `tid` of the first part has, -1: none
  __device__ __forceinline__ int edge(int tid, int n) const { return P::kEach == 1 ? -1 : tid < head ? tid : tid >= 8 && tid < 8 + rest ? n - rest + tid - 8 : -1; }
};

// Sums relative to a logit M near the largest: with d = (x - M) scale in exponents of two, s = sum 2^d, w = sum 2^d d.  (The difference comes before the product, so that
// logits of any size, the type's lowest ones among them, are as exact as they are near to each other.)
struct Sums {
  float M, s, w;
  __device__ __forceinline__ void raise(float to, float c) {       // (to >= M, or NaN)
    const float d = fmaxf((M - to) * c, kLeast), by = __builtin_amdgcn_exp2f(d);
    w = by * fmaf(s, d, w);
    s *= by;
    M = to;
  }
  __device__ __forceinline__ void add(Sums o, float c) {
    const float to = larger(M, o.M);
    raise(to, c);
    o.raise(to, c);
    s += o.s;
    w += o.w;
  }
};

// Results of a row from its sums.
struct Stats {
  float M, log, entropy;                                           // log: of sum exp(scale (x - M))
  __device__ __forceinline__ explicit Stats(const Sums& x) : M(x.M) {
    const bool empty = M == minus_infinity(), odd = !(M < __builtin_inff());
    const float two = __builtin_amdgcn_logf(x.s), nan = __builtin_nanf("");       // (base 2)
    log = empty ? 0.f : odd ? nan : two * kLn2;
    entropy = empty ? 0.f : odd ? nan : (two - x.w / x.s) * kLn2;
  }
  __device__ __forceinline__ float lse(float scale) const { return fmaf(M, scale, log); }
  __device__ __forceinline__ float of(float logit, float scale) const { return M == minus_infinity() ? M : fmaf(logit - M, scale, -log); }
};

// Larger logits have larger keys, and of equal ones those of lower indices; 0 is none's.
__device__ __forceinline__ uint64_t key_of(float x, int index) {
  uint32_t u = __float_as_uint(x + 0.f);                     // (-0 is 0)
  u = x != x ? 0xffffffffu : u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
  return (uint64_t)u << 32 | (uint32_t)~index;
}
__device__ __forceinline__ int index_of(uint64_t key) { return (int)~(uint32_t)key; }
__device__ __forceinline__ float value_of(uint64_t key) {
  const uint32_t u = (uint32_t)(key >> 32);
  return u == 0xffffffffu ? __builtin_nanf("") : __uint_as_float(u & 0x80000000u ? u ^ 0x80000000u : ~u);
}

// The largest number that `count` or more of these lanes' are at least, from bit `bits` - 1 on below `base`; or, where that many are, the first that is found with no
// more than these above it.  `lanes` and so the result may differ from lane to lane.
__device__ __forceinline__ uint32_t nth_of(uint32_t x, uint64_t lanes, int count, uint32_t base, int bits) {
  bool done = false;
  for (int b = bits - 1; b >= 0; --b) {
    const uint32_t more = base | 1u << b;
    // (lanes' own numbers are compared with their own group's)
    const int n = __popcll(__ballot(x >= more) & lanes);
    base = !done && n >= count ? more : base;
    done = done || n == count;
    if (__all(done)) break;
  }
  return base;
}

// The same over several numbers of each lane, of 32 bits.  Numbers that are all there have their highest bits alike, which are not searched then (kAll): 4372 rows of 20,450 with five
// tokens 44.4 -> 42.8 us, 64 of 32,000 with twenty 10.5 -> 10.3; parts of few pieces 0.2 to 0.4 us more; rows of a wavefront, which have more to do than to wait, 1 to 10 %.
template <bool kAll, int M>
__device__ __forceinline__ uint32_t nth_of_all(const uint32_t (&x)[M], int count) {
  uint32_t base = 0;
  int bits = 32;
  if constexpr (kAll) {
    uint32_t most = x[0], least = x[0];
#pragma unroll
    for (int i = 1; i < M; ++i) {
      most = max(most, x[i]);
      least = min(least, x[i]);
    }
    const auto over = [](uint32_t x, auto&& f) {
      return (uint32_t)__builtin_amdgcn_readfirstlane(
          __float_as_int(over_lanes(__uint_as_float(x), 6, [&](float a, float b) { return __uint_as_float(f(__float_as_uint(a), __float_as_uint(b))); })));
    };
    most = over(most, [](uint32_t a, uint32_t b) { return max(a, b); });
    least = over(least, [](uint32_t a, uint32_t b) { return min(a, b); });
    bits = most == least ? 0 : 32 - __clz((int)(most ^ least));
    base = bits > 31 ? 0 : most >> bits << bits;
  }
  for (int b = bits - 1; b >= 0; --b) {
    const uint32_t more = base | 1u << b;
    int n = 0;
#pragma unroll
    for (int i = 0; i < M; ++i) n += __popcll(__ballot(x[i] >= more));
    if (n >= count) base = more;
    if (n == count) break;
  }
  return base;
}

// A number that the `count`-th of the lanes' keys is at least, as near to it as is worth it; 0 where there are fewer.  Indices have `bits` bits.
__device__ __forceinline__ uint64_t nth_key(uint64_t key, uint64_t lanes, int count, int bits) {
  const uint32_t high = (uint32_t)(key >> 32), low = (uint32_t)key;
  const uint32_t value = nth_of(high, lanes, count, 0, 32);
  const int above = __popcll(__ballot(high >= value) & lanes);
  // (several lanes have the value that the count-th has: those of the lowest indices)
  uint32_t index = 0;
  if (__any(value && above > count)) {
    const uint64_t tied = __ballot(high == value) & lanes;
    index = nth_of(low, tied, count - (above - __popcll(tied)), ~0u << bits, bits);
    index = above > count ? index : 0;
  }
  return value ? (uint64_t)value << 32 | index : 0;
}

struct Chosen {
  uint64_t list[kList];               // (or a wavefront's in each quarter of it)
  uint32_t values[kThreads];
  int counts[kWaves];
  uint64_t border[kWaves];
  uint64_t most[kWaves];
  int count;
};

// The border from every lane's largest key (0: it has none); all threads of the workgroup.
__device__ __forceinline__ uint64_t border_of(uint64_t key, int top, int bits, Chosen& c) {
  if (threadIdx.x == 0) c.count = 0;
  const uint64_t mine = nth_key(key, ~(uint64_t)0, top, bits);
  if ((threadIdx.x & 63) == 0) c.border[threadIdx.x >> 6] = mine;
  __syncthreads();
  uint64_t b = c.border[0];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) b = c.border[w] > b ? c.border[w] : b;
  return b;
}

// Bits of an index.
__device__ __forceinline__ int index_bits(int vocabulary) { return 32 - __clz(vocabulary - 1 | 1); }

__device__ __forceinline__ void put(uint64_t key, uint64_t border, Chosen& c) {
  if (key == 0 || key < border) return;
  const int at = atomicAdd(&c.count, 1);                     // (the order in the list does not matter)
  if (at < kList) c.list[at] = key;
}

// The `top` largest keys to out(place, key); where there are fewer, the places behind them get 0.  Where the list has no room, the largest key below the last one is
// looked for `top` times: below(key) is this thread's largest one.
template <typename Out, typename Below>
__device__ __forceinline__ void place(int top, Chosen& c, Out&& out, Below&& below) {
  __syncthreads();
  const int n = c.count;
  if (n <= kList) {
    for (int i = threadIdx.x; i < max(n, top); i += kThreads) {
      if (i >= n) { out(i, (uint64_t)0); continue; }
      const uint64_t key = c.list[i];
      int before = 0;
#pragma unroll 8
      for (int j = 0; j < n; ++j) before += c.list[j] > key;
      if (before < top) out(before, key);
    }
    return;
  }
  uint64_t last = ~(uint64_t)0;
  for (int i = 0; i < top; ++i) {
    uint64_t mine = below(last);
    for (int m = 32; m; m >>= 1) {
      const uint64_t other = __shfl_xor((unsigned long long)mine, m, 64);
      mine = other > mine ? other : mine;
    }
    __syncthreads();
    if ((threadIdx.x & 63) == 0) c.most[threadIdx.x >> 6] = mine;
    __syncthreads();
    for (int w = 0; w < kWaves; ++w) mine = c.most[w] > mine ? c.most[w] : mine;
    if (threadIdx.x == 0) out(i, mine);
    last = mine;
  }
}

// The `top` largest keys of the wavefronts' quarters of the list to out(place, key), 0 where there are fewer; all threads, after a barrier.
template <typename Out>
__device__ __forceinline__ void rank_all(int top, const Chosen& chosen, Out&& out) {
  constexpr int kRoom = kList / kWaves;
  int counts[kWaves], n = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    counts[w] = __builtin_amdgcn_readfirstlane(chosen.counts[w]);
    n += counts[w];
  }
  for (int i = threadIdx.x; i < max(n, top); i += kThreads) {
    if (i >= n) { out(i, (uint64_t)0); continue; }
    int of = i, before = 0;
    const uint64_t* mine = chosen.list;
#pragma unroll
    for (int w = 0; w < kWaves - 1; ++w)
      if (mine == chosen.list + w * kRoom && of >= counts[w]) { of -= counts[w]; mine += kRoom; }
    const uint64_t key = mine[of];
#pragma unroll
    for (int w = 0; w < kWaves; ++w)
#pragma unroll 4
      for (int j = 0; j < counts[w]; ++j) before += chosen.list[w * kRoom + j] > key;
    if (before < top) out(before, key);
  }
}

__device__ __forceinline__ int64_t target_of(const ScoreArgs& p, int64_t row) {
  return p.a.target_bytes == 4 ? (int64_t)((const int32_t*)p.targets)[row] : ((const int64_t*)p.targets)[row];
}

// A row's target and its logit, looked up before the rest of the row is there.
struct Target {
  bool known;
  float logit;
  template <typename T>
  __device__ __forceinline__ Target(const ScoreArgs& p, int64_t row, const T*) {
    const int64_t t = target_of(p, row);
    known = t >= 0 && t < p.a.vocabulary;
    logit = (float)((const T*)p.logits)[row * p.a.stride + (known ? t : 0)];
  }
};

__device__ __forceinline__ void write_row(const ScoreArgs& p, int64_t row, const Stats& s, const Target& t) {
  p.lse[row] = s.lse(p.a.scale);
  p.entropy[row] = s.entropy;
  *(float2*)(p.stats + 2 * row) = {s.M, s.log};
  p.logp[row] = t.known ? s.of(t.logit, p.a.scale) : 0.f;
}

__device__ __forceinline__ void write_top(const ScoreArgs& p, int64_t row, int i, int id, float logit, const Stats& s) {
  p.top_ids[row * p.a.top + i] = id;
  p.top_logp[row * p.a.top + i] = s.of(logit, p.a.scale);
}
__device__ __forceinline__ void write_top(const ScoreArgs& p, int64_t row, int i, uint64_t key, const Stats& s) { write_top(p, row, i, index_of(key), value_of(key), s); }

// Sums of a lane's logits, as they come.  Relative to R = M c rounded, c = scale log2 e, a product and a sum are one instruction; what R is off by is taken out of
// the sums at the end.  M is raised when a piece exceeds it by 2^8.  A logit of -infinity makes w NaN, as 0 times an infinity is: then, and where others are not finite or
// too large, the wavefront goes through its pieces again, with exponents that are cut off.
struct LaneSums {
  float M = -__builtin_inff(), c, R = 0.f, s = 0.f, w = 0.f;
  __device__ __forceinline__ explicit LaneSums(float by) : c(by) {}
  __device__ __forceinline__ void start(float most) { M = most; R = M * c; }
  __device__ __forceinline__ void add(float x) {
    const float d = fmaf(x, c, -R), e = __builtin_amdgcn_exp2f(d);
    s += e;
    w = fmaf(e, d, w);
  }
  // (differences from M itself, for any M)
  __device__ __forceinline__ void add_any(float x) {
    const float d = fmaxf((x - M) * c, kLeast), e = __builtin_amdgcn_exp2f(d);
    s += e;
    w = fmaf(e, d, w);
  }
  __device__ __forceinline__ bool exceeded(float most) const { return fmaf(most, c, -R) > 8.f; }
  __device__ __forceinline__ void raise(float most) {
    const float before = R;
    start(most);
    const float d = before - R, by = __builtin_amdgcn_exp2f(d);
    w = by * fmaf(s, d, w);
    s *= by;
  }
  // whether the sums are not what they should be: a logit that is not finite, or so large that R is off by too much (here by less than 1/16)
  __device__ __forceinline__ bool failed() const { return !(fabsf(w) < __builtin_inff() && fabsf(R) < 1048576.f); }
  __device__ __forceinline__ Sums exact() const {
    const float off = M == minus_infinity() ? 0.f : fmaf(M, c, -R), by = __builtin_amdgcn_exp2f(-off);
    return {M, s * by, fmaf(-off, s, w) * by};
  }
};

// The same of many logits: what has been added up so far is put aside now and then, so that small terms are not lost in it one by one.
struct LongSums : LaneSums {
  float s_all = 0.f, w_all = 0.f;
  using LaneSums::LaneSums;
  __device__ __forceinline__ void aside() {
    s_all += s;
    w_all += w;
    s = w = 0.f;
  }
  __device__ __forceinline__ void raise(float most) {
    const float before = R;
    LaneSums::raise(most);
    const float d = before - R, by = __builtin_amdgcn_exp2f(d);
    w_all = by * fmaf(s_all, d, w_all);
    s_all *= by;
  }
};

// The sums of a wavefront, in all lanes.
__device__ __forceinline__ Sums of_wave(Sums x, float c) {
  x.raise(over_lanes(x.M, 6, larger), c);
  x.s = sum_of_lanes(x.s, 6);
  x.w = sum_of_lanes(x.w, 6);
  return x;
}

// Keys of any row, and of rows of at most 2^16 logits of a type of 16 bits: 16 bits of value and 16 of index.
struct LongKey {
  typedef uint64_t type;
  static constexpr int kIndexBits = 32;
  static __device__ __forceinline__ uint64_t of(float x, int index) { return key_of(x, index); }
  static __device__ __forceinline__ int index(uint64_t key) { return index_of(key); }
  static __device__ __forceinline__ float value(uint64_t key) { return value_of(key); }
};
template <typename T>
struct Key {
  typedef uint32_t type;
  static constexpr int kIndexBits = 16;
  static __device__ __forceinline__ uint32_t of(float x, int index) {
    union { T t; uint16_t u; } v;
    v.t = (T)(x + 0.f);                                      // (exact; -0 is 0)
    const uint32_t u = x != x ? 0xffffu : v.u & 0x8000u ? ~v.u & 0xffffu : v.u | 0x8000u;
    return u << 16 | (~index & 0xffff);
  }
  static __device__ __forceinline__ int index(uint32_t key) { return ~key & 0xffff; }
  static __device__ __forceinline__ float value(uint32_t key) {
    const uint32_t u = key >> 16;
    union { uint16_t u; T t; } v;
    v.u = (uint16_t)(u & 0x8000u ? u ^ 0x8000u : ~u);
    return u == 0xffffu ? __builtin_nanf("") : (float)v.t;
  }
};
template <>
struct Key<float> : LongKey {};

// Keys from the border on of a wavefront's lanes, to a list; how many they are (the list has the first of them).  `lanes` are those of this lane's row.  A lane holds the N pieces
// j * kStep + sub of `pieces`, the first of which is the row's piece `first`, knows the largest element of each (`most`), and may have one element beside
// them (`edge`).  It takes its pieces that reach the border one after the other, and of those their elements that do, so that a wavefront works on as many of either as the lane with
// most of them has.  They are counted off by ballots: nothing waits for LDS.
template <typename T, typename P, typename Of, int N, int kStep>
__device__ __forceinline__ int collect(typename Of::type border, const Row<T, P>& r, int first, int pieces, int sub, const u32x4 (&x)[N], const float (&most)[N],
                                       int edge, float beside, uint64_t lanes, typename Of::type* list, int room) {
  using K = typename Of::type;
  const uint64_t below = lanes & (((uint64_t)1 << (threadIdx.x & 63)) - 1);
  const float least = border >> Of::kIndexBits ? Of::value(border) : minus_infinity();
  int n = 0;
  auto keep = [&](bool has, float v, int index) {
    const K k = Of::of(v, index);
    const bool in = has && k >= border;
    const uint64_t all = __ballot(in);
    const int to = n + __popcll(all & below);
    if (in && to < room) list[to] = k;
    n += __popcll(all & lanes);
  };
  if (__any(edge >= 0)) keep(edge >= 0, beside, edge);
  uint32_t near = 0;
#pragma unroll
  for (int j = 0; j < N; ++j) near |= j * kStep + sub < pieces && !(most[j] < least) ? 1u << j : 0u;
  while (__any(near)) {
    const bool has = near;
    const int j = has ? __builtin_ctz(near) : 0, piece = j * kStep + sub;
    near &= near - 1;
    u32x4 v = x[0];
    if constexpr (N == 2) v = j ? x[1] : v;
    else if (N > 2 && has) v = r.load(first + piece);                    // (a choice of more registers costs more, and holds them)
    uint32_t bits = 0;
#pragma unroll
    for (int e = 0; e < P::kEach; ++e) bits |= !(P::get(v, e) < least) ? 1u << e : 0u;
    bits = has ? bits : 0;
    while (__any(bits)) {
      const int e = bits ? __builtin_ctz(bits) : 0;
      keep(bits, P::any(v, e), r.index(first + piece, e));
      bits &= bits - 1;
    }
  }
  return n;
}

// The key of a lane's largest element, 0: it has none.
template <typename T, typename P, typename Of, int N, int kStep>
__device__ __forceinline__ typename Of::type largest_key(const Row<T, P>& r, int first, int pieces, int sub, const float (&most)[N], float mine, int edge,
                                                         float beside) {
  auto alike = [](float a, float b) { return a == b || (a != a && b != b); };
  typename Of::type key = edge >= 0 ? Of::of(beside, edge) : 0;
  int found = -1;
#pragma unroll
  for (int j = N - 1; j >= 0; --j)
    if (j * kStep + sub < pieces && alike(most[j], mine)) found = j * kStep + sub;
  if (found >= 0) {
    const u32x4 piece = r.load(first + found);
    int e = 0;
#pragma unroll
    for (int i = P::kEach - 1; i >= 0; --i) e = alike(P::get(piece, i), mine) ? i : e;
    key = max(key, Of::of(mine, r.index(first + found, e)));
  }
  return key;
}

// A part of a row, of any length: a lane has four pieces on their way.  Six wavefronts to a SIMD; held to eight, it spills.
template <typename T>
__global__ __launch_bounds__(kThreads, 6) void score_sums_kernel(ScoreArgs p) {
  using P = Piece<T>;
  constexpr int kAhead = 4;
  __shared__ Sums waves[kWaves];
  const int tid = threadIdx.x, part = (int)(blockIdx.x % (unsigned)p.parts);
  const int64_t row = blockIdx.x / (unsigned)p.parts;
  const Row<T> r((const T*)p.logits + row * p.a.stride, p.a.vocabulary);
  const int first = part * p.vectors, pieces = min(p.vectors, r.pieces - first);      // (of this part; may be none)
  const u32x4* at = r.piece(first);
  const Target target(p, row, (const T*)nullptr);

  const int edge = part == 0 ? r.edge(tid, p.a.vocabulary) : -1;
  const float c = exponents(p.a.scale), beside = edge >= 0 ? (float)r.at[edge] : 0.f;
  LongSums lane(c);
  auto add = [&](const u32x4& v) {
    float most = P::get(v, 0);
#pragma unroll
    for (int e = 1; e < P::kEach; ++e) most = larger(most, P::get(v, e));
    if (lane.exceeded(most)) lane.raise(most);
#pragma unroll
    for (int e = 0; e < P::kEach; ++e) lane.add(P::get(v, e));
  };
  // rounds of all lanes: nothing but the sums branches, and loads beyond the last round read it again
  const int rounds = pieces / kThreads;
  if (rounds > 0) {
    auto load = [&](int j) { return at[min(j, rounds - 1) * kThreads + tid]; };
    u32x4 x[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) x[j] = load(j);
    lane.start(P::get(x[0], 0));
    int j = 0;
    for (; j + kAhead <= rounds; j += kAhead)
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        const u32x4 v = x[i];
        x[i] = load(j + i + kAhead);
        add(v);
        if (i == kAhead - 1 && (j & (kSumVectors - 1)) == kSumVectors - kAhead) lane.aside();
      }
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
      if (j + i < rounds) add(x[i]);
  }
  if (rounds * kThreads + tid < pieces) {
    const u32x4 v = at[rounds * kThreads + tid];
    if (rounds == 0) lane.start(P::get(v, 0));
    add(v);
  }
  if (edge >= 0) {
    if (tid >= pieces) lane.start(beside);
    else if (lane.exceeded(beside)) lane.raise(beside);
    lane.add(beside);
  }
  lane.aside();
  lane.s = lane.s_all;
  lane.w = lane.w_all;
  Sums lane_sums = lane.exact();
  if (__any(lane.failed())) {
    float most = edge >= 0 ? beside : minus_infinity();
    for (int i = tid; i < pieces; i += kThreads) {
      const u32x4 v = at[i];
#pragma unroll
      for (int e = 0; e < P::kEach; ++e) most = larger(most, P::get(v, e));
    }
    lane = LongSums(c);
    lane.M = most;
    if (edge >= 0) lane.add_any(beside);
    for (int i = tid; i < pieces; i += kThreads) {
      const u32x4 v = at[i];
#pragma unroll
      for (int e = 0; e < P::kEach; ++e) lane.add_any(P::get(v, e));
      if (i / kThreads % kSumVectors == kSumVectors - 1) lane.aside();
    }
    lane.aside();
    lane_sums = {lane.M, lane.s_all, lane.w_all};
  }
  const Sums wave_sums = of_wave(lane_sums, c);
  if ((tid & 63) == 0) waves[tid >> 6] = wave_sums;
  __syncthreads();
  if (tid) return;
  Sums sum = waves[0];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) sum.add(waves[w], c);
  if (p.parts > 1) *(f32x4*)(p.sums + (row * p.parts + part) * 4) = f32x4{sum.M, sum.s, sum.w, 0.f};
  else write_row(p, row, Stats(sum), target);
}

// The same with the largest logits: a lane holds its N pieces.
template <typename T, int N>
__global__ __launch_bounds__(kThreads) void score_kernel(ScoreArgs p) {
  using P = Piece<T>;
  __shared__ Sums waves[kWaves];
  __shared__ Chosen chosen;
  const int tid = threadIdx.x, part = (int)(blockIdx.x % (unsigned)p.parts);
  const int64_t row = blockIdx.x / (unsigned)p.parts;
  const Row<T> r((const T*)p.logits + row * p.a.stride, p.a.vocabulary);
  const int first = part * p.vectors, pieces = min(p.vectors, r.pieces - first);      // (of this part; may be none)
  const u32x4* at = r.piece(first);
  const Target target(p, row, (const T*)nullptr);

  u32x4 x[N];
#pragma unroll
  for (int j = 0; j < N; ++j) {
    x[j] = u32x4{P::kNothing, P::kNothing, P::kNothing, P::kNothing};
    if (j * kThreads + tid < pieces) x[j] = at[j * kThreads + tid];
  }
  const int edge = part == 0 ? r.edge(tid, p.a.vocabulary) : -1;
  const float beside = edge >= 0 ? (float)r.at[edge] : minus_infinity();

  // (the sums of a piece begin when it has come)
  const float c = exponents(p.a.scale);
  LaneSums lane(c);
  float most[N], mine = beside;
  if (edge >= 0) { lane.start(beside); lane.add(beside); }
#pragma unroll
  for (int j = 0; j < N; ++j) {
    most[j] = minus_infinity();
    if (j * kThreads + tid >= pieces) continue;
    most[j] = P::get(x[j], 0);
#pragma unroll
    for (int i = 1; i < P::kEach; ++i) most[j] = larger(most[j], P::get(x[j], i));
    mine = larger(mine, most[j]);
    if (j == 0 && edge < 0) lane.start(most[j]);
    else if (lane.exceeded(most[j])) lane.raise(most[j]);
#pragma unroll
    for (int i = 0; i < P::kEach; ++i) lane.add(P::get(x[j], i));
  }
  Sums lane_sums = lane.exact();
  if (__any(lane.failed())) {
    lane = LaneSums(c);
    lane.M = over_lanes(mine, 6, larger);
    lane.add_any(beside);
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const u32x4 again = here(x[j]);                     // (not kept as 32-bit numbers from above)
#pragma unroll
      for (int i = 0; i < P::kEach; ++i) lane.add_any(P::get(again, i));
    }
    lane_sums = {lane.M, lane.s, lane.w};
  }
  const Sums wave_sums = of_wave(lane_sums, c);
  if ((tid & 63) == 0) waves[tid >> 6] = wave_sums;
  chosen.values[tid] = edge >= 0 || tid < pieces ? (uint32_t)(key_of(mine, 0) >> 32) : 0;
  __syncthreads();
  Sums sum = waves[0];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) sum.add(waves[w], c);
  if (p.parts > 1 && tid == 0) *(f32x4*)(p.sums + (row * p.parts + part) * 4) = f32x4{sum.M, sum.s, sum.w, 0.f};
  const Stats s(sum);
  if (p.parts == 1 && tid == 0) write_row(p, row, s, target);
  auto out = [&](int i, uint64_t k) {
    if (p.parts > 1) p.keys[(row * p.parts + part) * p.a.top + i] = k;
    else write_top(p, row, i, k, s);
  };

  // Every wavefront looks for the border by itself, and has a quarter of the list.
  constexpr int kRoom = kList / kWaves;
  const int top = p.a.top, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  uint32_t values[kWaves];
#pragma unroll
  for (int w = 0; w < kWaves; ++w) values[w] = chosen.values[w * 64 + (tid & 63)];
  const uint64_t border = (uint64_t)nth_of_all<(N >= 8)>(values, top) << 32;
  const int count = collect<T, P, LongKey, N, kThreads>(border, r, first, pieces, tid, x, most, edge, beside, ~(uint64_t)0, chosen.list + wave * kRoom, kRoom);
  if ((tid & 63) == 0) chosen.counts[wave] = count;
  if (!__syncthreads_or(count > kRoom)) {
    rank_all(top, chosen, out);
    return;
  }
  // many are alike: the border is a value and an index, and all share the list
  const uint64_t key = largest_key<T, P, LongKey, N, kThreads>(r, first, pieces, tid, most, mine, edge, beside), exact = border_of(key, top, index_bits(p.a.vocabulary), chosen);
  if (edge >= 0) put(key_of(beside, edge), exact, chosen);
  for (int i = tid; i < pieces; i += kThreads) {
    const u32x4 v = at[i];
#pragma unroll
    for (int e = 0; e < P::kEach; ++e) put(key_of(P::get(v, e), r.index(first + i, e)), exact, chosen);
  }
  place(
      top, chosen, out,
      [&](uint64_t last) {
        uint64_t best = 0;
        auto next = [&](uint64_t k) { best = k < last && k > best ? k : best; };
        if (edge >= 0) next(key_of(beside, edge));
        for (int i = tid; i < pieces; i += kThreads) {
          const u32x4 v = at[i];
#pragma unroll
          for (int e = 0; e < P::kEach; ++e) next(key_of(P::get(v, e), r.index(first + i, e)));
        }
        return best;
      });
}

// Rows of few pieces: L lanes each, of which each holds N pieces; nothing is cut, and the rows of a wavefront have nothing to do with each other.
__device__ __forceinline__ uint32_t other_lane(uint32_t x, int m) { return (uint32_t)__shfl_xor((int)x, m, 64); }
__device__ __forceinline__ uint64_t other_lane(uint64_t x, int m) { return __shfl_xor((unsigned long long)x, m, 64); }

template <typename K, int L>
struct ChosenOfRows {
  static constexpr int kRows = kThreads / L, kRoom = kList / kRows;
  K list[kRows][kRoom];
};

template <typename T, int L, int N, bool kTop, typename P = Piece<T>>
__global__ __launch_bounds__(kThreads) void score_rows_kernel(ScoreArgs p) {
  constexpr int kLog = L == 16 ? 4 : L == 32 ? 5 : 6, kRows = kThreads / L;
  __shared__ std::conditional_t<kTop, ChosenOfRows<typename Key<T>::type, L>, int> chosen;
  const int sub = threadIdx.x & (L - 1), mine_of = threadIdx.x / L;
  const int64_t at_row = (int64_t)blockIdx.x * kRows + mine_of, row = min(at_row, p.a.rows - 1);     // (rows that are not there are the last one again)
  const bool there = at_row < p.a.rows;
  const uint64_t lanes = L == 64 ? ~(uint64_t)0 : (((uint64_t)1 << (L & 63)) - 1) << (threadIdx.x & (64 - L));
  const Row<T, P> r((const T*)p.logits + row * p.a.stride, p.a.vocabulary);
  const Target target(p, row, (const T*)nullptr);
  u32x4 x[N];
#pragma unroll
  for (int j = 0; j < N; ++j) {
    x[j] = u32x4{P::kNothing, P::kNothing, P::kNothing, P::kNothing};
    if (j * L + sub < r.pieces) x[j] = r.load(j * L + sub);
  }
  const int edge = r.edge(sub, p.a.vocabulary);
  const float beside = edge >= 0 ? (float)r.at[edge] : minus_infinity(), c = exponents(p.a.scale);
  LaneSums lane(c);
  float most[N], mine = beside;
  if (edge >= 0) { lane.start(beside); lane.add(beside); }
#pragma unroll
  for (int j = 0; j < N; ++j) {
    most[j] = minus_infinity();
    if (j * L + sub >= r.pieces) continue;
    most[j] = P::get(x[j], 0);
#pragma unroll
    for (int i = 1; i < P::kEach; ++i) most[j] = larger(most[j], P::get(x[j], i));
    mine = larger(mine, most[j]);
    if (j == 0 && edge < 0) lane.start(most[j]);
    else if (lane.exceeded(most[j])) lane.raise(most[j]);
#pragma unroll
    for (int i = 0; i < P::kEach; ++i) lane.add(P::get(x[j], i));
  }
  Sums lane_sums = lane.exact();
  const bool failed = (__ballot(lane.failed()) & lanes) != 0;
  if (failed) {
    lane = LaneSums(c);
    lane.M = over_lanes(mine, kLog, larger);               // (all lanes of a row are here)
    lane.add_any(beside);
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const u32x4 again = here(x[j]);
#pragma unroll
      for (int i = 0; i < P::kEach; ++i) lane.add_any(P::get(again, i));
    }
    lane_sums = {lane.M, lane.s, lane.w};
  }
  Sums sum = lane_sums;
  sum.raise(over_lanes(sum.M, kLog, larger), c);
  sum.s = sum_of_lanes(sum.s, kLog);
  sum.w = sum_of_lanes(sum.w, kLog);
  const Stats s(sum);
  if (there && sub == 0) write_row(p, row, s, target);

  if constexpr (kTop) {
    using Of = Key<T>;
    using K = typename Of::type;
    constexpr int kRoom = ChosenOfRows<K, L>::kRoom;
    const int top = p.a.top;
    K* list = chosen.list[mine_of];
    auto reach = [&](K border) {
      const int n = collect<T, P, Of, N, L>(border, r, 0, r.pieces, sub, x, most, edge, beside, lanes, list, kRoom);
      // (a wavefront's own accesses of LDS keep their order)
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
      return n;
    };
    // As many lanes as there are tokens have a value from the border on.
    const uint32_t value = edge >= 0 || sub < r.pieces ? (uint32_t)(Of::of(mine, 0) >> Of::kIndexBits) : 0;
    int n = reach((K)nth_of(value, lanes, top, 0, Of::kIndexBits) << Of::kIndexBits);
    if (__any(n > kRoom)) {
      // many are alike: the border is a value and an index
      const K key = largest_key<T, P, Of, N, L>(r, 0, r.pieces, sub, most, mine, edge, beside);
      if constexpr (sizeof(K) == 4) n = reach(nth_of(key, lanes, top, 0, 32));
      else n = reach(nth_key(key, lanes, top, index_bits(p.a.vocabulary)));
    }
    if (L == 64 && n > 64 && n <= kRoom) {
      // (a few lanes have many of them: those from the list's own `top`-th on, by the first 32 bits of their keys)
      constexpr int kEach = kRoom / 64;
      K k[kEach];
      uint32_t high[kEach];
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        k[i] = 64 * i + sub < n ? list[64 * i + sub] : 0;
        high[i] = (uint32_t)(k[i] >> (8 * sizeof(K) - 32));
      }
      const uint32_t border = nth_of_all<false>(high, top);
      n = 0;
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        const bool in = k[i] && high[i] >= border;
        const uint64_t all = __ballot(in);
        if (in) list[n + __popcll(all & (((uint64_t)1 << sub) - 1))] = k[i];
        n += __popcll(all);
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
    if (n <= kRoom) {
      for (int i = sub; i < n; i += L) {
        const K k = list[i];
        int before = 0;
#pragma unroll 8
        for (int j = 0; j < n; ++j) before += list[j] > k;
        if (there && before < top) write_top(p, row, before, Of::index(k), Of::value(k), s);
      }
    } else {
      // no room: the largest key below the last one, `top` times
      K last = ~(K)0;
      for (int i = 0; i < top; ++i) {
        K best = 0;
        auto next = [&](K k) { best = k < last && k > best ? k : best; };
        if (edge >= 0) next(Of::of(beside, edge));
        for (int j = sub; j < r.pieces; j += L) {
          const u32x4 v = r.load(j);
#pragma unroll
          for (int e = 0; e < P::kEach; ++e) next(Of::of(P::get(v, e), r.index(j, e)));
        }
        for (int m = L / 2; m; m >>= 1) best = max(best, other_lane(best, m));
        if (there && sub == 0) write_top(p, row, i, Of::index(best), Of::value(best), s);
        last = best;
      }
    }
  }
}

// The parts of a row.  All loads that others do not wait for come first.  Of up to 2048 keys each thread holds some, and the border comes from the threads' largest ones, as above;
// of more, from those of the parts.
template <typename T>
__global__ __launch_bounds__(kThreads) void score_join_kernel(ScoreArgs p) {
  constexpr int kHeld = 8, kRoom = kList / kWaves;
  __shared__ Sums waves[kWaves];
  __shared__ Chosen chosen;
  const int tid = threadIdx.x, top = p.a.top, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int64_t row = blockIdx.x, n = (int64_t)p.parts * top;
  const float c = exponents(p.a.scale);
  const uint64_t* keys = p.keys + row * n;
  uint64_t held[kHeld], most = 0;
#pragma unroll
  for (int i = 0; i < kHeld; ++i) held[i] = i * kThreads + tid < n ? keys[i * kThreads + tid] : 0;
  const Target target(p, row, (const T*)nullptr);
  Sums sum{minus_infinity(), 0.f, 0.f};
  for (int i = tid; i < p.parts; i += kThreads) {
    const f32x4 v = *(const f32x4*)(p.sums + (row * p.parts + i) * 4);
    sum.add({v[0], v[1], v[2]}, c);
  }
  sum = of_wave(sum, c);
  if ((tid & 63) == 0) waves[wave] = sum;
#pragma unroll
  for (int i = 0; i < kHeld; ++i) most = max(most, held[i]);
  chosen.values[tid] = (uint32_t)(most >> 32);
  __syncthreads();
  sum = waves[0];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) sum.add(waves[w], c);
  const Stats s(sum);
  if (tid == 0) write_row(p, row, s, target);
  if (top == 0) return;
  auto out = [&](int i, uint64_t k) { write_top(p, row, i, k, s); };
  if (n <= kHeld * kThreads) {
    uint32_t values[kWaves];
#pragma unroll
    for (int w = 0; w < kWaves; ++w) values[w] = chosen.values[w * 64 + (tid & 63)];
    const uint64_t border = (uint64_t)nth_of_all<false>(values, top) << 32, below = ((uint64_t)1 << (tid & 63)) - 1;
    int count = 0;
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
      const uint64_t all = __ballot(held[i] && held[i] >= border);
      const int to = count + __popcll(all & below);
      if (held[i] && held[i] >= border && to < kRoom) chosen.list[wave * kRoom + to] = held[i];
      count += __popcll(all);
    }
    if ((tid & 63) == 0) chosen.counts[wave] = count;
    if (!__syncthreads_or(count > kRoom)) {
      rank_all(top, chosen, out);
      return;
    }
  }
  // more keys, or many of one value
  uint64_t key = 0;
  for (int i = tid; i < p.parts; i += kThreads) key = max(key, keys[(int64_t)i * top]);
  const uint64_t border = border_of(key, top, index_bits(p.a.vocabulary), chosen);
  for (int64_t i = tid; i < n; i += kThreads) put(keys[i], border, chosen);
  place(top, chosen, out, [&](uint64_t last) {
    uint64_t best = 0;
    for (int64_t i = tid; i < n; i += kThreads) best = keys[i] < last && keys[i] > best ? keys[i] : best;
    return best;
  });
}

// The same without tokens, of few parts: a row to a lane.
template <typename T>
__global__ __launch_bounds__(kThreads) void score_join_rows_kernel(ScoreArgs p) {
  const int64_t row = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  if (row >= p.a.rows) return;
  const float c = exponents(p.a.scale);
  const Target target(p, row, (const T*)nullptr);
  Sums sum{minus_infinity(), 0.f, 0.f};
  for (int i = 0; i < p.parts; ++i) {
    const f32x4 v = *(const f32x4*)(p.sums + (row * p.parts + i) * 4);
    sum.add({v[0], v[1], v[2]}, c);
  }
  write_row(p, row, Stats(sum), target);
}

template <typename T>
__device__ __forceinline__ void put_value(u32x4& r, int i, float x) {
  if constexpr (sizeof(T) == 4) {
    r[i] = __float_as_uint(x);
  } else {
    union { T t; uint16_t u; } v;
    v.t = (T)x;
    r[i / 2] = i & 1 ? (r[i / 2] & 0xffffu) | (uint32_t)v.u << 16 : v.u;
  }
}

constexpr int kGradPieces = 4;        // of a lane

// Gradients: L lanes have four pieces each of a row.
template <typename T, int L>
__global__ __launch_bounds__(kThreads) void score_grad_kernel(ScoreArgs p, int chunks) {
  using P = Piece<T>;
  const int lane = threadIdx.x & (L - 1);
  const int64_t id = (int64_t)blockIdx.x * (kThreads / L) + (L == 64 ? wave_id() : (int)(threadIdx.x / L));
  const int64_t row = id / chunks;
  const int chunk = (int)(id - row * chunks);
  if (row >= p.a.rows) return;
  const T* in = (const T*)p.logits + row * p.a.stride;
  T* out = (T*)p.d_logits + row * p.a.d_stride;
  const int64_t target = target_of(p, row);
  const bool known = target >= 0 && target < p.a.vocabulary;
  const int t = known ? (int)target : -1;
  const float2 stats = *(const float2*)(p.stats + 2 * row);
  const float most = stats.x, log = stats.y, scale = p.a.scale, g = known && p.d_logp ? p.d_logp[row] * scale : 0.f;
  const float h = p.d_entropy ? p.d_entropy[row] * scale : 0.f, entropy = p.d_entropy ? p.entropy_in[row] : 0.f;
  const bool empty = most == minus_infinity();
  auto grad = [&](float x, int index) {
    const float d = fmaf(x - most, scale, -log), e = __builtin_amdgcn_exp2f(d * kLog2e);
    const float y = fmaf(-e, fmaf(h, fmaxf(d, kLeast) + entropy, g), index == t ? g : 0.f);
    return empty ? 0.f : y;
  };
  const Row<T> r(in, p.a.vocabulary);
  // (pieces of both where the two rows lie alike)
  const bool alike = (((uintptr_t)in ^ (uintptr_t)out) & 15) == 0;
  const int first = chunk * L * kGradPieces;
  u32x4 x[kGradPieces];
#pragma unroll
  for (int j = 0; j < kGradPieces; ++j) {
    const int i = first + j * L + lane;
    if (i < r.pieces) x[j] = *r.piece(i);
  }
  if (chunk == 0) {
    const int edge = r.edge(lane, p.a.vocabulary);
    if (edge >= 0) out[edge] = (T)grad((float)in[edge], edge);
  }
#pragma unroll
  for (int j = 0; j < kGradPieces; ++j) {
    const int i = first + j * L + lane;
    if (i >= r.pieces) break;
    u32x4 y = {0, 0, 0, 0};
#pragma unroll
    for (int e = 0; e < P::kEach; ++e) put_value<T>(y, e, grad(P::get(x[j], e), r.index(i, e)));
    T* to = out + r.index(i, 0);
    if (alike) {
      *(u32x4*)to = y;
    } else {
#pragma unroll
      for (int e = 0; e < P::kEach; ++e) to[e] = (T)P::get(y, e);
    }
  }
}

constexpr int64_t kMostBlocks = 0xffffffff / kThreads;      // (a launch has less than 2^32 threads)

template <typename T, bool kTop>
int rows(const ScoreArgs& p, hipStream_t s) {
  const int lanes = p.lanes, n = p.vectors / lanes;
  const int64_t blocks = (p.a.rows + kThreads / lanes - 1) / (kThreads / lanes);
  const dim3 grid((unsigned)blocks), block(kThreads);
  if (lanes == 16) {
    if (n <= 1) score_rows_kernel<T, 16, 1, kTop><<<grid, block, 0, s>>>(p);
    else if (n <= 2) score_rows_kernel<T, 16, 2, kTop><<<grid, block, 0, s>>>(p);
    else if (n <= 4) score_rows_kernel<T, 16, 4, kTop><<<grid, block, 0, s>>>(p);
    else score_rows_kernel<T, 16, 8, kTop><<<grid, block, 0, s>>>(p);
  } else if (lanes == 32) {
    if (n <= 1) score_rows_kernel<T, 32, 1, kTop><<<grid, block, 0, s>>>(p);
    else if (n <= 2) score_rows_kernel<T, 32, 2, kTop><<<grid, block, 0, s>>>(p);
    else score_rows_kernel<T, 32, 4, kTop><<<grid, block, 0, s>>>(p);
  } else if (kTop && p.single) {
    if (n <= 2) score_rows_kernel<T, 64, 2, true, One<T>><<<grid, block, 0, s>>>(p);
    else if (n <= 4) score_rows_kernel<T, 64, 4, true, One<T>><<<grid, block, 0, s>>>(p);
    else score_rows_kernel<T, 64, 8, true, One<T>><<<grid, block, 0, s>>>(p);
  } else {
    if (n <= 2) score_rows_kernel<T, 64, 2, kTop><<<grid, block, 0, s>>>(p);
    else if (n <= 4) score_rows_kernel<T, 64, 4, kTop><<<grid, block, 0, s>>>(p);
    else if (n <= 8) score_rows_kernel<T, 64, 8, kTop><<<grid, block, 0, s>>>(p);
    else score_rows_kernel<T, 64, 16, kTop><<<grid, block, 0, s>>>(p);
  }
  return (int)hipGetLastError();
}

template <typename T>
int forward(const ScoreArgs& p, hipStream_t s) {
  if (p.lanes) return p.a.top ? rows<T, true>(p, s) : rows<T, false>(p, s);
  const int64_t blocks = p.a.rows * p.parts;
  const dim3 grid((unsigned)blocks), block(kThreads);
  const int n = p.vectors / kThreads;
  if (p.a.top == 0) score_sums_kernel<T><<<grid, block, 0, s>>>(p);
  else if (n <= 1) score_kernel<T, 1><<<grid, block, 0, s>>>(p);
  else if (n <= 2) score_kernel<T, 2><<<grid, block, 0, s>>>(p);
  else if (n <= 4) score_kernel<T, 4><<<grid, block, 0, s>>>(p);
  else if (n <= 8) score_kernel<T, 8><<<grid, block, 0, s>>>(p);
  else if (n <= 16) score_kernel<T, 16><<<grid, block, 0, s>>>(p);
  else if (n <= 24) score_kernel<T, 24><<<grid, block, 0, s>>>(p);
  else score_kernel<T, 32><<<grid, block, 0, s>>>(p);
  if (p.parts > 1 && p.parts <= 8 && p.a.top == 0) score_join_rows_kernel<T><<<dim3((unsigned)((p.a.rows + kThreads - 1) / kThreads)), block, 0, s>>>(p);
  else if (p.parts > 1) score_join_kernel<T><<<dim3((unsigned)p.a.rows), block, 0, s>>>(p);
  return (int)hipGetLastError();
}

// Gradients: 16 lanes where rows have up to 64 pieces, and 64; workgroups' worth of pieces to a row.
template <typename T>
int grad_lanes(const ScoreArgs& p) { return p.a.vocabulary / Piece<T>::kEach <= 16 * kGradPieces ? 16 : 64; }
template <typename T>
int64_t grad_chunks(const ScoreArgs& p) {
  const int64_t each = grad_lanes<T>(p) * kGradPieces;
  return std::max<int64_t>(1, (p.a.vocabulary / Piece<T>::kEach + each - 1) / each);
}
template <typename T, int L>
int backward(const ScoreArgs& p, hipStream_t s) {
  const int64_t chunks = grad_chunks<T>(p), blocks = (p.a.rows * chunks + kThreads / L - 1) / (kThreads / L);
  score_grad_kernel<T, L><<<dim3((unsigned)blocks), dim3(kThreads), 0, s>>>(p, (int)chunks);
  return (int)hipGetLastError();
}

// A call's rows from one on.
ScoreArgs rows_from(const ScoreArgs& p, int64_t first, int64_t rows, int64_t size) {
  ScoreArgs q = p;
  const auto by = [&](auto*& at, int64_t each) { at = at ? at + first * each : at; };
  const auto bytes = [&](auto* at, int64_t each) { return at ? decltype(at)((uintptr_t)at + first * each) : at; };
  q.a.rows = rows;
  q.logits = bytes(p.logits, p.a.stride * size);
  q.targets = bytes(p.targets, p.a.target_bytes);
  q.d_logits = bytes(p.d_logits, p.a.d_stride * size);
  by(q.d_logp, 1); by(q.d_entropy, 1); by(q.entropy_in, 1);
  by(q.logp, 1); by(q.entropy, 1); by(q.lse, 1); by(q.stats, 2);
  by(q.top_logp, p.a.top); by(q.top_ids, p.a.top);
  by(q.sums, 4 * p.parts); by(q.keys, (int64_t)p.parts * p.a.top);
  return q;
}

// In as many launches as have `most` rows each: nearly always one.
template <typename F>
int in_turn(const ScoreArgs& p, int64_t most, int64_t size, F&& f) {
  if (p.a.rows <= most) return f(p);
  for (int64_t first = 0; first < p.a.rows; first += most)
    if (int rc = f(rows_from(p, first, std::min(most, p.a.rows - first), size))) return rc;
  return 0;
}

template <typename T>
int forward_all(const ScoreArgs& p, void* stream) {
  return in_turn(p, p.lanes ? kMostBlocks * (kThreads / p.lanes) : kMostBlocks / p.parts, sizeof(T), [&](const ScoreArgs& q) { return forward<T>(q, (hipStream_t)stream); });
}
template <typename T>
int backward_all(const ScoreArgs& p, void* stream) {
  const int lanes = grad_lanes<T>(p);
  return in_turn(p, kMostBlocks * (kThreads / lanes) / grad_chunks<T>(p), sizeof(T), [&](const ScoreArgs& q) {
    return lanes == 16 ? backward<T, 16>(q, (hipStream_t)stream) : backward<T, 64>(q, (hipStream_t)stream);
  });
}

}  // namespace

int launch_score_forward(const ScoreArgs& p, void* stream) {
  return p.a.dtype == ARROW_F32 ? forward_all<float>(p, stream) : p.a.dtype == ARROW_BF16 ? forward_all<__bf16>(p, stream) : forward_all<_Float16>(p, stream);
}

int launch_score_backward(const ScoreArgs& p, void* stream) {
  return p.a.dtype == ARROW_F32 ? backward_all<float>(p, stream) : p.a.dtype == ARROW_BF16 ? backward_all<__bf16>(p, stream) : backward_all<_Float16>(p, stream);
}

}  // namespace arrow
