// A cache of keys and values in 4 bits: writes, reads, and the attention of one new token per sequence over it (include/arrow_packed.h).
//
// What bounds the attention is the cache: every visible key and value is read once, for all query heads that share it.  A workgroup takes the up to 16
// query heads of a key head and a stretch of the visible keys; its wavefronts take tiles of 32 keys in turn, each with a running maximum and sum of its
// own, and are joined in LDS; long caches are cut into several stretches, whose results a second kernel joins (attention_decode.hip's).
//
// Everything stays in registers.  Scores are computed transposed, keys by heads: a lane holds a quarter of a key's row, whose order within the product is
// free, so that its 16 bytes are one load.  Of the result a lane holds four keys of a head in each half of a tile, and the products with the values take these
// eight as they are: the values of four tokens lie together in the cache so that a lane finds its four tokens' eight columns (heads of 128) in 16 bytes, and two
// permutations of bytes turn two tokens' pairs of columns into two columns' pairs of tokens.
//
// Measured: 32 rows of up to 16,000 keys, 32/8 heads of 128, 366 MB in 80 us, 4.6 TB/s (a 1 GiB copy: 5.1), matrix units busy in 16 % of the cycles and vector
// instructions, most of them conversions and the softmax of 16 columns of which 4 are heads, in 49 %, and 5 us for the join, which mostly goes on beside the next call; 64 rows under a window of
// 4096, 16/4 heads of 64, 18.7 us on changing inputs, 3.9 TB/s, where a wavefront has 16 tiles in all, one of two on its SIMD: some 170 vector and 65 scalar instructions each, and the
// waits between them; one row of 1000 keys 5.5 us and 3.1 for the join, which are launches and four loads that wait for each other.  A new token's key and value are written by a launch of
// their own, 3.8 us more of any of these.  Tried for the window: four blocks of 16 keys to a tile, whose four heads fill the 16 columns, for a quarter of the softmax
// (22 us, and spills with heads of 128); tiles of 64 keys (24, spills); twice as many tiles on their way (22).
#include <algorithm>

#include "attention_common.h"
#include "packed_internal.h"

namespace arrow {
namespace {

template <int N> struct Words;
template <> struct Words<1> { typedef uint32_t type; };
template <> struct Words<2> { typedef u32x2 type; };
template <> struct Words<4> { typedef u32x4 type; };
template <int N> using words = typename Words<N>::type;
__device__ __forceinline__ uint32_t word(uint32_t w, int) { return w; }
__device__ __forceinline__ uint32_t word(const u32x2& w, int i) { return w[i]; }
__device__ __forceinline__ uint32_t word(const u32x4& w, int i) { return w[i]; }

// The two elements of byte B of a word, times a power of two.
template <int B> __device__ __forceinline__ uint32_t pair_of(uint32_t w, float scale, __bf16) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, B));
}
template <int B> __device__ __forceinline__ uint32_t pair_of(uint32_t w, float scale, _Float16) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, B));
}
template <typename T>
__device__ __forceinline__ uint32_t pair_at(uint32_t w, float scale, int byte) {       // (a constant, once loops are unrolled)
  switch (byte) {
    case 0: return pair_of<0>(w, scale, T{});
    case 1: return pair_of<1>(w, scale, T{});
    case 2: return pair_of<2>(w, scale, T{});
    default: return pair_of<3>(w, scale, T{});
  }
}
template <typename T>
__device__ __forceinline__ x8<T> eight_of(uint32_t w, float scale) {
  union { uint32_t u[4]; x8<T> all; } r;
  r.u[0] = pair_of<0>(w, scale, T{});
  r.u[1] = pair_of<1>(w, scale, T{});
  r.u[2] = pair_of<2>(w, scale, T{});
  r.u[3] = pair_of<3>(w, scale, T{});
  return r.all;
}

// Two floats as one word, and its two as floats.  (The word is what they are read from: otherwise each is rounded for itself once more.)
template <typename T>
__device__ __forceinline__ uint32_t rounded_pair(float a, float b) {
  uint32_t w = __builtin_bit_cast(uint32_t, x2<T>{(T)a, (T)b});
  asm("" : "+v"(w));
  return w;
}
template <typename T>
__device__ __forceinline__ float2 pair_wide(uint32_t w) {
  if constexpr (std::is_same<T, __bf16>::value) {
    return {__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)};
  } else {
    const x2<T> x = __builtin_bit_cast(x2<T>, w);
    return {(float)x[0], (float)x[1]};
  }
}

// A scale's byte as a float: 2^(e - 127), and infinity for 255, which makes NaN of the elements.
__device__ __forceinline__ float scale_of(uint32_t e) { return __uint_as_float(e << 23); }

// Of a block: where codes and scales begin.
__device__ __forceinline__ int64_t values_at(int page, int dim) { return (int64_t)page * (dim / 2); }
__device__ __forceinline__ int64_t key_scales_at(int page, int dim) { return (int64_t)page * dim; }
__device__ __forceinline__ int64_t value_scales_at(int page, int dim) { return (int64_t)page * (dim + dim / 32); }

// ---- writes and reads ----
// Eight elements a lane, four lanes to a scale.  Four tokens of a head lie in neighbouring lanes, so that what a wavefront writes are whole runs of bytes.  Bound by memory:
// 16,384 tokens of 8 heads of 128 are written in 16.9 us, 5.2 TB/s, and read in 15.3, 5.8.
struct Place {
  int64_t row, slot;                  // slot -1: none
  int head, piece;
  bool in;
};
__device__ __forceinline__ Place place_of(const PackedArgs& p, int64_t id) {
  const arrow_packed_t& c = p.c;
  const int pieces = c.dim / 8;
  Place at;
  at.piece = (int)(id & (pieces - 1));
  id /= pieces;
  const int t = (int)(id & 3);
  id >>= 2;
  at.head = (int)(id % c.kv_heads);
  at.row = id / c.kv_heads * 4 + t;
  at.in = at.row < p.tokens;
  at.slot = -1;
  if (!at.in) return at;
  if (p.slots) {
    at.slot = p.slots[at.row];
  } else {                            // the last place of a sequence
    const int64_t j = (int64_t)c.lengths[at.row] - 1, column = j >> p.page_log;
    if (j < 0 || column >= c.columns) return at;
    const int page = c.table[at.row * c.columns + column];
    at.slot = page < 0 ? -1 : ((int64_t)page << p.page_log) + (j & (c.page - 1));
  }
  if (at.slot < 0 || at.slot >> p.page_log >= c.pages) at.slot = -1;
  return at;
}

__device__ __forceinline__ uint32_t codes_of(const x8<__bf16>& x, float scale) {
  uint32_t r = 0;
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, x2<__bf16>{x[0], x[1]}, scale, 0);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, x2<__bf16>{x[2], x[3]}, scale, 1);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, x2<__bf16>{x[4], x[5]}, scale, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, x2<__bf16>{x[6], x[7]}, scale, 3);
}
__device__ __forceinline__ uint32_t codes_of(const x8<_Float16>& x, float scale) {
  uint32_t r = 0;
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(r, x2<_Float16>{x[0], x[1]}, scale, 0);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(r, x2<_Float16>{x[2], x[3]}, scale, 1);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(r, x2<_Float16>{x[4], x[5]}, scale, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(r, x2<_Float16>{x[6], x[7]}, scale, 3);
}

// Codes of a lane's eight elements and the scale of the 32 ones that its four lanes have.
template <typename T>
__device__ __forceinline__ uint32_t pack8(const x8<T>& x, uint32_t* scale) {
  uint32_t most = 0;                  // (sizes of floats are in the order of their bits, those of NaN last)
#pragma unroll
  for (int i = 0; i < 8; ++i) most = max(most, __float_as_uint((float)x[i]) & 0x7fffffffu);
  most = max(most, (uint32_t)__shfl_xor((int)most, 1, 64));
  most = max(most, (uint32_t)__shfl_xor((int)most, 2, 64));
  // 1.m 2^(E - 127) <= 7 2^(e - 127): e = E - 2 where 1.m is up to 7/4
  const int E = (int)(most >> 23), e = E - 2 + ((most & 0x7fffffu) > 0x600000u), limit = std::is_same<T, _Float16>::value ? 140 : 252;
  *scale = E == 255 ? 255u : (uint32_t)min(max(e, 1), limit);
  return E == 255 ? 0u : codes_of(x, scale_of(*scale));
}

// Codes of a token's elements 8 piece .. + 7 to their place among the values.
template <int D>
__device__ __forceinline__ void store_values(char* block, int t, int piece, uint32_t codes) {
  char* at = block + (t >> 2) * (2 * D);
  if (D == 128) {
    *(uint32_t*)(at + piece * 16 + (t & 3) * 4) = codes;
  } else if (D == 64) {
#pragma unroll
    for (int i = 0; i < 2; ++i) *(uint16_t*)(at + (2 * piece + i) * 8 + (t & 3) * 2) = (uint16_t)(codes >> (16 * i));
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) *(uint8_t*)(at + (4 * piece + i) * 4 + (t & 3)) = (uint8_t)(codes >> (8 * i));
  }
}
template <int D>
__device__ __forceinline__ uint32_t load_values(const char* block, int t, int piece) {
  const char* at = block + (t >> 2) * (2 * D);
  uint32_t codes = 0;
  if (D == 128) {
    codes = *(const uint32_t*)(at + piece * 16 + (t & 3) * 4);
  } else if (D == 64) {
#pragma unroll
    for (int i = 0; i < 2; ++i) codes |= (uint32_t)*(const uint16_t*)(at + (2 * piece + i) * 8 + (t & 3) * 2) << (16 * i);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) codes |= (uint32_t)*(const uint8_t*)(at + (4 * piece + i) * 4 + (t & 3)) << (8 * i);
  }
  return codes;
}

template <typename T, int D>
__global__ __launch_bounds__(256) void packed_append_kernel(PackedArgs p) {
  const arrow_packed_t& c = p.c;
  const Place at = place_of(p, (int64_t)blockIdx.x * 256 + threadIdx.x);
  if (at.slot < 0) return;            // (the four lanes of a scale have one row)
  const x8<T> k = *(const x8<T>*)((const T*)p.k.at + at.row * p.k.token + at.head * p.k.head + at.piece * 8);
  const x8<T> v = *(const x8<T>*)((const T*)p.v.at + at.row * p.v.token + at.head * p.v.head + at.piece * 8);
  const int t = (int)(at.slot & (c.page - 1)), of = at.piece >> 2;
  char* block = (char*)p.pool + (at.slot >> p.page_log) * c.page_step + at.head * c.head_step;
  uint32_t ks, vs;
  const uint32_t kc = pack8<T>(k, &ks), vc = pack8<T>(v, &vs);
  *(uint32_t*)(block + (int64_t)t * (D / 2) + at.piece * 4) = kc;
  store_values<D>(block + values_at(c.page, D), t, at.piece, vc);
  if ((at.piece & 3) == 0) {
    *(uint8_t*)(block + key_scales_at(c.page, D) + t * (D / 32) + of) = (uint8_t)ks;
    *(uint8_t*)(block + value_scales_at(c.page, D) + ((t >> 2) * (D / 32) + of) * 4 + (t & 3)) = (uint8_t)vs;
  }
}

template <typename T, int D>
__global__ __launch_bounds__(256) void packed_read_kernel(PackedArgs p) {
  const arrow_packed_t& c = p.c;
  const Place at = place_of(p, (int64_t)blockIdx.x * 256 + threadIdx.x);
  if (!at.in) return;
  x8<T> k = {}, v = {};
  if (at.slot >= 0) {
    const int t = (int)(at.slot & (c.page - 1)), of = at.piece >> 2;
    const char* block = (const char*)p.pool + (at.slot >> p.page_log) * c.page_step + at.head * c.head_step;
    const uint32_t ks = *(const uint8_t*)(block + key_scales_at(c.page, D) + t * (D / 32) + of);
    const uint32_t vs = *(const uint8_t*)(block + value_scales_at(c.page, D) + ((t >> 2) * (D / 32) + of) * 4 + (t & 3));
    k = eight_of<T>(*(const uint32_t*)(block + (int64_t)t * (D / 2) + at.piece * 4), scale_of(ks));
    v = eight_of<T>(load_values<D>(block + values_at(c.page, D), t, at.piece), scale_of(vs));
  }
  *(x8<T>*)((T*)const_cast<void*>(p.k.at) + at.row * p.k.token + at.head * p.k.head + at.piece * 8) = k;
  *(x8<T>*)((T*)const_cast<void*>(p.v.at) + at.row * p.v.token + at.head * p.v.head + at.piece * 8) = v;
}

// ---- attention ----
// max / sum over the four lanes that have one l % 16
__device__ __forceinline__ float max_quarters(float x) {
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return max_halves(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}
__device__ __forceinline__ float add_quarters(float x) {
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return add_halves(__uint_as_float(r[0]) + __uint_as_float(r[1]));
}

// A tile on its way: of each half, the lane's quarter of key l % 16's row with its scale, and tokens 4 (l / 16) + 0..3 of its columns with theirs.
template <int D>
struct Codes {
  words<D / 32> k[2], v[2];
  uint32_t ks[2], vs[2];
  uint32_t visible;                   // keys, the same in all lanes
};

template <typename T, int D, int kWaves, bool kPairs>
__global__ __launch_bounds__(64 * kWaves, 4) void packed_decode_kernel(PackedArgs a) {
  constexpr int kSteps = D / 32;      // of the scores' inner dimension
  constexpr int kColumns = D / 16;    // columns of a lane
  constexpr int kAhead = D == 128 ? 1 : 2;   // tiles on their way
  __shared__ __align__(16) float smem[kWaves * 16 * D + kWaves * 2 * 16];
  const int lane = threadIdx.x & 63, wave = wave_id(), quarter = lane >> 4, col = lane & 15;
  const arrow_packed_t& c = a.c;
  int id = blockIdx.x;
  const int kv = id % c.kv_heads; id /= c.kv_heads;
  const int split = id % a.splits; id /= a.splits;
  const int head_tiles = (a.group + kHeadTile - 1) / kHeadTile;
  const int head_tile = id % head_tiles, b = id / head_tiles;
  const int head0 = head_tile * kHeadTile, heads = min(a.group - head0, kHeadTile);
  // (columns << page_log is at most 2^26.  All that follows to the first load is the same in all lanes, and said to be so where the compiler loses sight of it.)
  const int length = __builtin_amdgcn_readfirstlane(max(0, min(c.lengths[b], c.columns << a.page_log)));
  const int begin = c.window ? max(0, length - c.window) : 0;
  // groups of 16 keys, or of 32 (within a page), those that only hide between the first ones and the window left out; tiles of 32 keys, stretches of whole rounds of the wavefronts
  constexpr int kLog = kPairs ? 5 : 4, kGroups = kPairs ? 1 : 2, kKeys = 1 << kLog;
  const int rest = begin >> kLog, lead = min((min(c.sinks, begin) + kKeys - 1) >> kLog, rest), groups = lead + ((length + kKeys - 1) >> kLog) - rest;
  const int tiles = (groups + kGroups - 1) / kGroups, rounds = (tiles + kWaves - 1) / kWaves;
  const int tile0 = kWaves * (int)((int64_t)rounds * split / a.splits), tile1 = min(tiles, kWaves * (int)((int64_t)rounds * (split + 1) / a.splits));
  const int32_t* table = c.table + (int64_t)b * c.columns;
  const char* pool = (const char*)a.pool + kv * c.head_step;

  // the queries in the order of the keys' quarters
  x8<T> qf[kSteps];
#pragma unroll
  for (int s = 0; s < kSteps; ++s) {
    const x8<T> z = {};
    qf[s] = col < heads ? *(const x8<T>*)((const T*)a.q.at + b * a.q.sequence + (int64_t)(kv * a.group + head0 + col) * a.q.head + quarter * (D / 4) + 8 * s) : z;
  }

  // (nothing here branches: the loads of one tile are to be on their way while another's are waited for; a page that is not there is read as the first one)
  auto group_at = [&](int g) { return g < lead ? g : g - lead + rest; };
  auto page_of = [&](int g) { return table[group_at(min(g, groups - 1)) >> (a.page_log - kLog)]; };
  int page[kGroups] = {};             // of the tile that is loaded next, looked up a tile ahead
  auto find_pages = [&](int tile) {
#pragma unroll
    for (int h = 0; h < kGroups; ++h) page[h] = page_of(kGroups * tile + h);
  };
  // (what a lane adds to its wavefront's addresses: of its quarter of key l % 16, of tokens 4 (l / 16) + 0..3, and of their scales)
  const uint32_t of_key = col * (D / 2) + quarter * (D / 8), of_value = (quarter * 16 + col) * (D / 8);
  const uint32_t of_key_scale = col * (D / 32) + quarter * (D / 4) / 32, of_value_scale = (quarter * (D / 32) + col * kColumns / 32) * 4;
  auto load = [&](int tile, int after) {
    Codes<D> x;
    x.visible = 0;
#pragma unroll
    for (int h = 0; h < kGroups; ++h) {
      const int g = kGroups * tile + h, key0 = kKeys * group_at(g), slot0 = key0 & (c.page - 1);
      const bool in = g < groups && (uint32_t)page[h] < (uint32_t)c.pages;
      const char* block = pool + (uint32_t)__builtin_amdgcn_readfirstlane(in ? page[h] : 0) * c.page_step;
      const char *codes = block + slot0 * (D / 2), *scales = block + c.page * D + slot0 * (D / 32);
      const char *values = codes + c.page * (D / 2), *value_scales = scales + c.page * (D / 32);
#pragma unroll
      for (int i = h; i < h + 2 / kGroups; ++i) {           // (sixteen keys are 8 D bytes of codes and D / 2 of scales further)
        const int of = i - h;
        x.k[i] = *(const words<kSteps>*)(codes + of * 8 * D + of_key);
        x.ks[i] = *(const uint8_t*)(scales + of * (D / 2) + of_key_scale);
        x.v[i] = *(const words<kSteps>*)(values + of * 8 * D + of_value);
        x.vs[i] = *(const uint32_t*)(value_scales + of * (D / 2) + of_value_scale);
      }
      constexpr uint32_t kAll = kPairs ? 0xffffffffu : 0xffffu;
      uint32_t mask = kAll;
      if (key0 < begin || key0 + kKeys > length) {          // at an edge of what is seen
        const auto below = [](int n) { return n >= 32 ? ~0u : (1u << max(0, n)) - 1; };
        mask = below(length - key0) & (~below(begin - key0) | below(c.sinks - key0)) & kAll;
      }
      x.visible |= (in ? mask : 0u) << (16 * h);
    }
    find_pages(after);
    return x;
  };

  f32x4 acc[kColumns];
#pragma unroll
  for (int m = 0; m < kColumns; ++m) acc[m] = (f32x4)(0.f);
  const float scale = c.scale * kLog2e;
  float top = minus_infinity(), total = 0.f;

  auto work = [&](const Codes<D>& x) {
    f32x4 s[2] = {(f32x4)(0.f), (f32x4)(0.f)};
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const float ks = scale_of(x.ks[h]);
#pragma unroll
      for (int i = 0; i < kSteps; ++i) s[h] = mma16(eight_of<T>(word(x.k[h], i), ks), qf[i], s[h]);
    }
    float vs[2][4];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      vs[h][0] = __uint_as_float(x.vs[h] << 23 & 0x7f800000u);
      vs[h][1] = __uint_as_float(x.vs[h] << 15 & 0x7f800000u);
      vs[h][2] = __uint_as_float(x.vs[h] << 7 & 0x7f800000u);
      vs[h][3] = __uint_as_float(x.vs[h] >> 1 & 0x7f800000u);
    }
    if (x.visible != 0xffffffffu) {   // what is not seen does not count, whatever its scale
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const bool seen = x.visible >> (16 * h + 4 * quarter + i) & 1;
          s[h][i] = seen ? s[h][i] : minus_infinity();
          vs[h][i] = seen ? vs[h][i] : 1.f;
        }
    }
    float most = minus_infinity();
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < 4; ++i) most = fmaxf(most, s[h][i]);
    most = max_quarters(most) * scale;
    const float raised = fmaxf(top, most), off = raised == minus_infinity() ? 0.f : raised;
    if (__any(raised > top)) {
      const float by = __builtin_amdgcn_exp2f(top - off);
      total *= by;
#pragma unroll
      for (int m = 0; m < kColumns; ++m) acc[m] = acc[m] * by;
      top = raised;
    }
    // Probabilities as the sum of two numbers of the operands' type, the second what the first's rounding left: off by 2^-16 (float16: 2^-22) of themselves, not by 2^-8 (2^-11), which
    // made the results' error a fifth larger.  (16 vector instructions and twice the products with the values: 79.2 -> 81.1 us of long caches, 18.9 -> 19.8 under a window.)
    union { uint32_t u[4]; x8<T> all; } pf, rest;
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      const float one = __builtin_amdgcn_exp2f(fmaf(s[i / 4][i % 4], scale, -off)), two = __builtin_amdgcn_exp2f(fmaf(s[i / 4][i % 4 + 1], scale, -off));
      total += one;
      total += two;
      pf.u[i / 2] = rounded_pair<T>(one, two);
      const float2 near = pair_wide<T>(pf.u[i / 2]);
      rest.u[i / 2] = rounded_pair<T>(one - near.x, two - near.y);
    }
#pragma unroll
    for (int j = 0; j < kColumns / 2; ++j) {
      union { uint32_t u[4]; x8<T> all; } lo, hi;
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int t = 0; t < 4; t += 2) {
          const int i = t * (D / 32) + j, n = (t + 1) * (D / 32) + j;          // the bytes of the two tokens
          const uint32_t one = pair_at<T>(word(x.v[h], i / 4), vs[h][t], i % 4), two = pair_at<T>(word(x.v[h], n / 4), vs[h][t + 1], n % 4);
          lo.u[2 * h + t / 2] = __builtin_amdgcn_perm(two, one, 0x05040100u);
          hi.u[2 * h + t / 2] = __builtin_amdgcn_perm(two, one, 0x07060302u);
        }
      acc[2 * j] = mma16(lo.all, pf.all, acc[2 * j]);
      acc[2 * j + 1] = mma16(hi.all, pf.all, acc[2 * j + 1]);
      acc[2 * j] = mma16(lo.all, rest.all, acc[2 * j]);
      acc[2 * j + 1] = mma16(hi.all, rest.all, acc[2 * j + 1]);
    }
  };
  // (tiles beyond the last one are the last one again: loads that are always there can be told apart when one of them is waited for)
  int tile = tile0 + wave;
  if (tile < tile1) {
    const int last = tile + (tile1 - 1 - tile) / kWaves * kWaves;
    Codes<D> next[kAhead];
    find_pages(tile);
#pragma unroll
    for (int u = 0; u < kAhead; ++u) next[u] = load(min(tile + u * kWaves, last), min(tile + (u + 1) * kWaves, last));
    while (tile <= last) {
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const Codes<D> x = next[u];
        next[u] = load(min(tile + kAhead * kWaves, last), min(tile + (kAhead + 1) * kWaves, last));
        if (tile <= last) work(x);
        tile += kWaves;
      }
    }
  }
  total = add_quarters(total);

  // the wavefronts' results: column d of head h at [d][h], 16 floats to a row
  float* mine = smem + wave * 16 * D;
  float *tops = smem + kWaves * 16 * D, *totals = tops + kWaves * 16;
#pragma unroll
  for (int m = 0; m < kColumns; ++m)
#pragma unroll
    for (int i = 0; i < 4; ++i) mine[((4 * quarter + i) * kColumns + m) * 16 + col] = acc[m][i];
  if (quarter == 0) { tops[wave * 16 + col] = top; totals[wave * 16 + col] = total; }
  __syncthreads();
  for (int e = threadIdx.x; e < heads * D; e += 64 * kWaves) {
    const int h = e / D, d = e % D;
    float all = tops[h];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) all = fmaxf(all, tops[w * 16 + h]);
    const float off = all == minus_infinity() ? 0.f : all;
    float sum = 0.f, weight = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float by = __builtin_amdgcn_exp2f(tops[w * 16 + h] - off);
      sum = fmaf(by, smem[(w * D + d) * 16 + h], sum);
      weight = fmaf(by, totals[w * 16 + h], weight);
    }
    const int head = kv * a.group + head0 + h;
    if (a.splits == 1) {
      ((T*)const_cast<void*>(a.o.at))[b * a.o.sequence + head * a.o.head + d] = (T)(weight > 0.f || weight != weight ? sum / weight : 0.f);
    } else {
      float* part = a.parts + ((int64_t)(b * c.q_heads + head) * a.splits + split) * (D + 2);
      part[d] = sum;
      if (d == 0) { part[D] = all; part[D + 1] = weight; }
    }
  }
}

template <typename T, int D>
int decode(const PackedArgs& a, hipStream_t s) {
  const arrow_packed_t& c = a.c;
  const int64_t blocks = (int64_t)c.batch * c.kv_heads * a.splits * ((a.group + kHeadTile - 1) / kHeadTile), rows = (int64_t)c.batch * c.q_heads;
  // Pages of 32 tokens or more have a tile in one of them: half the work on addresses and edges, which is scalar but takes turns with the rest (64 rows under a window of 4096, heads of 64
  // 20.9 us as for pages of 16, 19.1; 54 rows of up to 12,700 keys, 6/2 heads of 128, 35.2 and 32.2).
  const auto launch = [&](auto* kernel) { kernel<<<dim3((unsigned)blocks), dim3(64 * a.waves), 0, s>>>(a); };
  if (a.waves == 4) launch(c.page >= 32 ? packed_decode_kernel<T, D, 4, true> : packed_decode_kernel<T, D, 4, false>);
  else launch(c.page >= 32 ? packed_decode_kernel<T, D, 8, true> : packed_decode_kernel<T, D, 8, false>);
  if (a.splits > 1) return launch_attention_decode_join({a.o, a.parts, a.splits, c.q_heads, c.dim}, c.dtype, rows, s);
  return (int)hipGetLastError();
}

template <typename F>
int of_kind(const arrow_packed_t& c, F&& f) {
  if (c.dtype == ARROW_BF16) return c.dim == 128 ? f.template operator()<__bf16, 128>() : c.dim == 64 ? f.template operator()<__bf16, 64>() : f.template operator()<__bf16, 32>();
  return c.dim == 128 ? f.template operator()<_Float16, 128>() : c.dim == 64 ? f.template operator()<_Float16, 64>() : f.template operator()<_Float16, 32>();
}

// Writes and reads, in as many launches as it takes: nearly always one.
template <typename F>
int in_turn(const PackedArgs& p, F&& launch) {
  const int64_t pieces = (int64_t)p.c.kv_heads * (p.c.dim / 8), most = kMostBlocks * 256 / pieces / 4 * 4;
  for (int64_t first = 0; first < p.tokens; first += most) {
    PackedArgs q = p;
    q.tokens = std::min(most, p.tokens - first);
    q.slots = p.slots ? p.slots + first : nullptr;           // (the last places of sequences are fewer than a launch has)
    q.k.at = (const char*)p.k.at + first * p.k.token * 2;
    q.v.at = (const char*)p.v.at + first * p.v.token * 2;
    launch(q, dim3((unsigned)(((q.tokens + 3) / 4 * 4 * pieces + 255) / 256)));
    if (const hipError_t rc = hipGetLastError()) return (int)rc;
  }
  return 0;
}

struct Append {
  const PackedArgs& p;
  hipStream_t s;
  template <typename T, int D> int operator()() const {
    return in_turn(p, [&](const PackedArgs& q, dim3 grid) { packed_append_kernel<T, D><<<grid, dim3(256), 0, s>>>(q); });
  }
};
struct Read {
  const PackedArgs& p;
  hipStream_t s;
  template <typename T, int D> int operator()() const {
    return in_turn(p, [&](const PackedArgs& q, dim3 grid) { packed_read_kernel<T, D><<<grid, dim3(256), 0, s>>>(q); });
  }
};
struct Decode {
  const PackedArgs& p;
  hipStream_t s;
  template <typename T, int D> int operator()() const { return decode<T, D>(p, s); }
};

}  // namespace

int launch_packed_append(const PackedArgs& p, void* stream) { return of_kind(p.c, Append{p, (hipStream_t)stream}); }
int launch_packed_read(const PackedArgs& p, void* stream) { return of_kind(p.c, Read{p, (hipStream_t)stream}); }
int launch_packed_decode(const PackedArgs& p, void* stream) { return of_kind(p.c, Decode{p, (hipStream_t)stream}); }

}  // namespace arrow
