// Attention of one new token per sequence over a cache in pages, and writes into it (include/arrow_attention.h).
//
// What bounds it is the cache: every visible key and value is read once, for all query heads that share it.  A workgroup takes
// the up to 16 query heads of a key head and a stretch of the visible keys; its wavefronts take tiles of 16 keys in turn, each with
// a running maximum and sum of its own, and are joined in LDS.  Long caches are cut into several stretches; their results go to the
// workspace and a second kernel joins them.
//
// 32 sequences of 4000 to 16,000 tokens, 32/8 heads of 128: 265 us in the first kernel, 5.2 TB/s (a copy: 5.1), 5 us in the second.  One sequence of 1000, 8/2 heads: 6
// and 3 us, launches and loads that wait for each other.  Tiles of 16 keys are what a wavefront can have on its way in registers beside the one that it
// works on, four wavefronts to a SIMD; with sixteen wavefronts to a stretch short caches took longer, and loads past the caches cost 10 %.
//
// Visible keys are counted without the gap between the first ones and the window, so that stretches are of one length.
#include "attention_common.h"

namespace arrow {
namespace {

constexpr int kWaves = 4;
constexpr int kKeys = 16;    // keys of a tile

// Scores: 16 x 16 with 32 inner steps; lane l holds row / column l % 16 at inner steps 8 (l / 16) + 0..7; of C and D column l % 16, rows
// 4 (l / 16) + 0..3.  Values: 16 x 16 with 16 inner steps, 4 (l / 16) + 0..3 in lane l: a result's rows as they come.
__device__ __forceinline__ f32x4 mma_values(i16x4 a, x4<__bf16> b, f32x4 c) {
  union { x4<__bf16> t; i16x4 i; } u;
  u.t = b;
  return __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(a, u.i, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mma_values(i16x4 a, x4<_Float16> b, f32x4 c) {
  union { x4<_Float16> t; i16x4 i; } u;
  u.i = a;
  return __builtin_amdgcn_mfma_f32_16x16x16f16(u.t, b, c, 0, 0, 0);
}

// max / sum over the four lanes that have one l % 16
__device__ __forceinline__ float max_quarters(float x) {
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return max_halves(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}
__device__ __forceinline__ float add_quarters(float x) {
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return add_halves(__uint_as_float(r[0]) + __uint_as_float(r[1]));
}

struct Row {
  const char *k, *v;    // null: not visible
  int64_t to_k, to_v;   // where the new token's go in the pools, -1: nowhere
};

template <typename T, int D>
__global__ __launch_bounds__(64 * kWaves, 4) void attention_decode_kernel(CacheArgs a) {
  using Tl = Tile<D>;
  constexpr int kPer = D / 32;                                   // pieces of 16 bytes of a row that a lane loads
  constexpr int kRoom = 16 * D * 4;                              // of a wavefront: its sums, and before them a tile of values
  static_assert(kKeys * Tl::kRowBytes <= kRoom, "room for a tile of values");
  __shared__ __align__(1024) unsigned char smem[kWaves * kRoom + kWaves * 2 * 16 * 4];
  const int lane = threadIdx.x & 63, wave = wave_id(), quarter = lane >> 4, col = lane & 15;
  const arrow_cache_t& c = a.c;
  int id = blockIdx.x;
  const int kv = id % c.kv_heads; id /= c.kv_heads;
  const int split = id % a.splits; id /= a.splits;
  const int head_tiles = (a.group + kHeadTile - 1) / kHeadTile;
  const int head_tile = id % head_tiles, b = id / head_tiles;
  const int head0 = head_tile * kHeadTile, heads = min(a.group - head0, kHeadTile);
  const int64_t room = (int64_t)c.columns << a.page_log;
  const int tokens = c.lengths[b], length = (int)max((int64_t)0, min((int64_t)tokens, room));
  const int begin = c.window ? max(0, length - c.window) : 0, lead = min(c.sinks, begin);
  const int seen = lead + length - begin;
  // stretches of whole tiles, as many for each wavefront
  const int tiles = (seen + kKeys - 1) / kKeys, rounds = (tiles + kWaves - 1) / kWaves;
  const int tile0 = kWaves * (int)((int64_t)rounds * split / a.splits), tile1 = min(tiles, kWaves * (int)((int64_t)rounds * (split + 1) / a.splits));
  const int32_t* table = c.table + (int64_t)b * c.columns;
  const char* k_pool = (const char*)a.k_pool + 2 * kv * c.k_head;
  const char* v_pool = (const char*)a.v_pool + 2 * kv * c.v_head;
  const bool fresh = a.k.at != nullptr && tokens <= room;        // (a new token beyond the table has no place: the last one is another's)
  const char* k_new = (const char*)a.k.at + 2 * (b * a.k.sequence + kv * a.k.head);
  const char* v_new = (const char*)a.v.at + 2 * (b * a.v.sequence + kv * a.v.head);

  x8<T> qf[kPer];
#pragma unroll
  for (int s = 0; s < kPer; ++s) {
    const int d = 32 * s + 8 * quarter;
    const x8<T> z = {};
    qf[s] = col < heads && d < c.dim
                ? *(const x8<T>*)((const char*)a.q.at + 2 * (b * a.q.sequence + (int64_t)(kv * a.group + head0 + col) * a.q.head + d)) : z;
  }

  // the new token to its place, by the last stretch
  if (fresh && head_tile == 0 && split == a.splits - 1 && wave == kWaves - 1 && length > 0) {
    const int page = table[(length - 1) >> a.page_log], slot = (length - 1) & (c.page - 1), d = 8 * lane;
    if (page >= 0 && page < c.pages && d < c.dim) {
      *(x8<T>*)((char*)k_pool + 2 * (page * c.k_page + slot * c.k_token + d)) = *(const x8<T>*)(k_new + 2 * d);
      *(x8<T>*)((char*)v_pool + 2 * (page * c.v_page + slot * c.v_token + d)) = *(const x8<T>*)(v_new + 2 * d);
    }
  }

  // A tile on its way: of key col, the pieces 4 s + quarter of its row.  Nothing here branches: the loads of one tile are to be on their way while
  // another's are waited for.  Pieces beyond the row are read as its last one, and cleared or meet unused sums below; keys that are not
  // visible as q, whose scores are masked and whose values are cleared below.
  x8<T> kf[kPer], vf[kPer];
  uint32_t visible = 0;                                          // of the tile's keys, the same in all lanes
  int offset[kPer];
#pragma unroll
  for (int s = 0; s < kPer; ++s) offset[s] = min(64 * s + 16 * quarter, 2 * c.dim - 16);
  const char* nothing = (const char*)a.q.at + 2 * (b * a.q.sequence + (int64_t)kv * a.group * a.q.head);
  auto key_of = [&](int i) { return i < lead ? i : i - lead + begin; };
  auto page_of = [&](int tile) { return table[key_of(min(tile * kKeys + col, seen - 1)) >> a.page_log]; };
  int page = 0;                                                  // of the tile that is loaded next, looked up a tile ahead
  auto load = [&](int tile) {
    const int i = tile * kKeys + col, j = key_of(i), slot = j & (c.page - 1);
    const bool in = i < seen && page >= 0 && page < c.pages, newest = fresh && j == length - 1;
    const char* k = !in ? nothing : newest ? k_new : k_pool + 2 * (page * c.k_page + slot * c.k_token);
    const char* v = !in ? nothing : newest ? v_new : v_pool + 2 * (page * c.v_page + slot * c.v_token);
    visible = (uint32_t)__ballot(in) & 0xffff;
    page = page_of(tile + kWaves);
#pragma unroll
    for (int s = 0; s < kPer; ++s) kf[s] = *(const x8<T>*)(k + offset[s]);
#pragma unroll
    for (int s = 0; s < kPer; ++s) vf[s] = *(const x8<T>*)(v + offset[s]);
  };

  f32x4 acc[D / 16];
#pragma unroll
  for (int m = 0; m < D / 16; ++m) acc[m] = (f32x4)(0.f);
  const float scale = c.scale * kLog2e;
  float top = minus_infinity(), total = 0.f;
  lds_byte* vt = (lds_byte*)smem + wave * kRoom;
  lds_byte* to = vt + col * Tl::kRowBytes;
  const int turn = Tl::turn(col);
  // the transposed read: rows 4 quarter + 0..3, columns 16 m + col
  const int row = 4 * quarter + (col >> 2), row_turn = Tl::turn(row), piece = (col & 3) >> 1;
  const lds_byte* from = vt + row * Tl::kRowBytes + ((col & 1) << 3);

  int tile = tile0 + wave;
  if (tile < tile1) {
    page = page_of(tile);
    load(tile);
  }
  while (tile < tile1) {
    f32x4 s = (f32x4)(0.f);
    if (c.dim < D) {                                             // (zeros of q times an infinity are none)
      const x8<T> z = {};
#pragma unroll
      for (int i = 0; i < kPer; ++i) kf[i] = 32 * i + 8 * quarter < c.dim ? kf[i] : z;
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) s = mma16(kf[i], qf[i], s);
    if (visible != 0xffff) {
      const x8<T> z = {};
#pragma unroll
      for (int i = 0; i < kPer; ++i) vf[i] = visible >> col & 1 ? vf[i] : z;
    }
    // (the tile is this wavefront's own: no barrier)
#pragma unroll
    for (int i = 0; i < kPer; ++i) *(__attribute__((address_space(3))) x8<T>*)(to + (((4 * i + quarter) ^ turn) << 4)) = vf[i];
    const uint32_t now = visible >> (4 * quarter);
    tile += kWaves;
    if (tile < tile1) load(tile);

    float most = minus_infinity();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      s[i] = now >> i & 1 ? s[i] : minus_infinity();
      most = fmaxf(most, s[i]);
    }
    most = max_quarters(most) * scale;
    const float next = fmaxf(top, most), off = next == minus_infinity() ? 0.f : next;
    const float by = __builtin_amdgcn_exp2f(top - off);
    top = next;
    total *= by;
    x4<T> pf;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      s[i] = __builtin_amdgcn_exp2f(fmaf(s[i], scale, -off));
      total += s[i];
      pf[i] = (T)s[i];
    }
#pragma unroll
    for (int m = 0; m < D / 16; ++m) acc[m] = mma_values(lds_transposed(from + (((2 * m + piece) ^ row_turn) << 4)), pf, acc[m] * by);
    reads_ahead<D / 16, D / 16, 1>();
  }
  total = add_quarters(total);

  // the wavefronts' results: column d of head h at [d][h], 16 floats to a row (the tiles are done with)
  __syncthreads();
  float* mine = (float*)(smem + wave * kRoom);
  float *tops = (float*)(smem + kWaves * kRoom), *totals = tops + kWaves * 16;
#pragma unroll
  for (int m = 0; m < D / 16; ++m)
#pragma unroll
    for (int i = 0; i < 4; ++i) mine[(16 * m + 4 * quarter + i) * 16 + col] = acc[m][i];
  if (quarter == 0) { tops[wave * 16 + col] = top; totals[wave * 16 + col] = total; }
  __syncthreads();
  for (int e = threadIdx.x; e < heads * c.dim; e += 64 * kWaves) {
    const int h = e / c.dim, d = e % c.dim;
    float all = tops[h];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) all = fmaxf(all, tops[w * 16 + h]);
    const float off = all == minus_infinity() ? 0.f : all;
    float sum = 0.f, weight = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float by = __builtin_amdgcn_exp2f(tops[w * 16 + h] - off);
      sum = fmaf(by, ((const float*)(smem + w * kRoom))[d * 16 + h], sum);
      weight = fmaf(by, totals[w * 16 + h], weight);
    }
    const int head = kv * a.group + head0 + h;
    if (a.splits == 1) {
      ((T*)a.o.at)[b * a.o.sequence + head * a.o.head + d] = (T)(weight > 0.f || weight != weight ? sum / weight : 0.f);
    } else {
      float* part = a.parts + ((int64_t)(b * c.q_heads + head) * a.splits + split) * (c.dim + 2);
      part[d] = sum;
      if (d == 0) { part[c.dim] = all; part[c.dim + 1] = weight; }
    }
  }
}

// The results of the stretches of one query head, joined: two columns per lane, every fourth stretch per wavefront.  3 to 5 us, most of it the launch.
template <typename T>
__global__ __launch_bounds__(64 * kWaves) void attention_decode_join_kernel(DecodeJoinArgs a) {
  constexpr int kAhead = 4;
  __shared__ float weights[kMostSplits];
  __shared__ float2 sums[kWaves][64];
  const int row = blockIdx.x, b = row / a.q_heads, head = row % a.q_heads, step = a.dim + 2, lane = threadIdx.x & 63, wave = wave_id(), d = 2 * lane;
  const float* from = a.parts + (int64_t)row * a.splits * step;
  // (all maxima and totals, and the columns of the first stretches, are on their way before one of them is waited for)
  float2 stats[kMostSplits / 64], ahead[kAhead];
#pragma unroll
  for (int k = 0; k < kMostSplits / 64; ++k) {
    const int i = lane + 64 * k;
    stats[k] = float2{minus_infinity(), 0.f};
    if (i < a.splits) stats[k] = *(const float2*)(from + (int64_t)i * step + a.dim);
  }
#pragma unroll
  for (int k = 0; k < kAhead; ++k) {
    const int i = wave + k * kWaves;
    ahead[k] = i < a.splits && d < a.dim ? *(const float2*)(from + (int64_t)i * step + d) : float2{0.f, 0.f};
  }
  float all = minus_infinity();
#pragma unroll
  for (int k = 0; k < kMostSplits / 64; ++k) all = fmaxf(all, stats[k].x);
  for (int m = 32; m; m >>= 1) all = fmaxf(all, __shfl_xor(all, m, 64));
  const float off = all == minus_infinity() ? 0.f : all;
  float total = 0.f;
#pragma unroll
  for (int k = 0; k < kMostSplits / 64; ++k) {
    const int i = lane + 64 * k;
    if (i >= a.splits) break;
    const float by = __builtin_amdgcn_exp2f(stats[k].x - off);
    if (wave == 0) weights[i] = by;
    total = fmaf(by, stats[k].y, total);
  }
  for (int m = 32; m; m >>= 1) total += __shfl_xor(total, m, 64);
  __syncthreads();
  float2 sum = {0.f, 0.f};
#pragma unroll
  for (int k = 0; k < kAhead; ++k) {
    const int i = wave + k * kWaves;
    if (i >= a.splits) break;
    sum.x = fmaf(weights[i], ahead[k].x, sum.x);
    sum.y = fmaf(weights[i], ahead[k].y, sum.y);
  }
#pragma unroll 4
  for (int i = wave + kAhead * kWaves; i < a.splits; i += kWaves) {
    const float2 x = d < a.dim ? *(const float2*)(from + (int64_t)i * step + d) : float2{0.f, 0.f};
    sum.x = fmaf(weights[i], x.x, sum.x);
    sum.y = fmaf(weights[i], x.y, sum.y);
  }
  sums[wave][lane] = sum;
  __syncthreads();
  if (wave > 0 || d >= a.dim) return;
#pragma unroll
  for (int w = 1; w < kWaves; ++w) { sum.x += sums[w][lane].x; sum.y += sums[w][lane].y; }
  const float over = total > 0.f || total != total ? 1.f / total : 0.f;
  x2<T> r;
  r[0] = (T)(sum.x * over);
  r[1] = (T)(sum.y * over);
  *(x2<T>*)((T*)a.o.at + b * a.o.sequence + head * a.o.head + d) = r;
}

// One piece of 16 bytes per thread.  Bound by memory: 8 prompts of 2048 tokens, 8 heads of 128, 22 us = 6.2 TB/s (what was just written comes out of the caches; a copy: 5.1).
template <typename T>
__global__ __launch_bounds__(256) void cache_append_kernel(CacheArgs a) {
  const arrow_cache_t& c = a.c;
  const int pieces = c.dim / 8;
  int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int piece = (int)(id % pieces); id /= pieces;
  const int kv = (int)(id % c.kv_heads); id /= c.kv_heads;
  const int t = (int)(id % a.tokens);
  const int64_t b = id / a.tokens;
  if (b >= c.batch) return;
  const int64_t j = (int64_t)c.lengths[b] - a.tokens + t;
  if (j < 0 || j >= ((int64_t)c.columns << a.page_log)) return;
  const int page = c.table[b * c.columns + (j >> a.page_log)], slot = (int)(j & (c.page - 1));
  if (page < 0 || page >= c.pages) return;
  *(x8<T>*)((T*)a.k_pool + page * c.k_page + slot * c.k_token + kv * c.k_head + piece * 8) =
      *(const x8<T>*)((const T*)a.k.at + b * a.k.sequence + t * a.k.token + kv * a.k.head + piece * 8);
  *(x8<T>*)((T*)a.v_pool + page * c.v_page + slot * c.v_token + kv * c.v_head + piece * 8) =
      *(const x8<T>*)((const T*)a.v.at + b * a.v.sequence + t * a.v.token + kv * a.v.head + piece * 8);
}

template <typename T>
int decode(const CacheArgs& a, void* stream) {
  const arrow_cache_t& c = a.c;
  const int64_t blocks = (int64_t)c.batch * c.kv_heads * a.splits * ((a.group + kHeadTile - 1) / kHeadTile), rows = (int64_t)c.batch * c.q_heads;
  if (blocks > 0x7fffffff || rows > 0x7fffffff) return (int)hipErrorInvalidConfiguration;
  hipStream_t s = (hipStream_t)stream;
  if (c.dim <= 64) attention_decode_kernel<T, 64><<<dim3((unsigned)blocks), dim3(64 * kWaves), 0, s>>>(a);
  else attention_decode_kernel<T, 128><<<dim3((unsigned)blocks), dim3(64 * kWaves), 0, s>>>(a);
  if (a.splits > 1) attention_decode_join_kernel<T><<<dim3((unsigned)rows), dim3(64 * kWaves), 0, s>>>({a.o, a.parts, a.splits, c.q_heads, c.dim});
  return (int)hipGetLastError();
}

}  // namespace

int launch_attention_decode(const CacheArgs& a, void* stream) { return a.c.dtype == ARROW_BF16 ? decode<__bf16>(a, stream) : decode<_Float16>(a, stream); }

int launch_attention_decode_join(const DecodeJoinArgs& a, int32_t dtype, int64_t rows, void* stream) {
  const dim3 grid((unsigned)rows), threads(64 * kWaves);
  if (dtype == ARROW_BF16) attention_decode_join_kernel<__bf16><<<grid, threads, 0, (hipStream_t)stream>>>(a);
  else attention_decode_join_kernel<_Float16><<<grid, threads, 0, (hipStream_t)stream>>>(a);
  return (int)hipGetLastError();
}

int launch_cache_append(const CacheArgs& a, void* stream) {
  const int64_t blocks = ((int64_t)a.c.batch * a.tokens * a.c.kv_heads * (a.c.dim / 8) + 255) / 256;
  if (blocks > 0x7fffffff) return (int)hipErrorInvalidConfiguration;
  hipStream_t s = (hipStream_t)stream;
  if (a.c.dtype == ARROW_BF16) cache_append_kernel<__bf16><<<dim3((unsigned)blocks), dim3(256), 0, s>>>(a);
  else cache_append_kernel<_Float16><<<dim3((unsigned)blocks), dim3(256), 0, s>>>(a);
  return (int)hipGetLastError();
}

}  // namespace arrow
