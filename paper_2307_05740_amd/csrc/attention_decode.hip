// Attention of one new token per sequence over a cache in pages, and writes into it (include/arrow_attention.h).
//
// What bounds it is the cache: every visible key and value is read once, for all query heads that share it.  A workgroup takes
// the up to 16 query heads of a key head and a stretch of the visible keys; its wavefronts take tiles of 32 keys in turn, each with
// a running maximum and sum of its own, and are joined in LDS.  Long caches are cut into several stretches; their results go to the
// workspace and a second kernel joins them.
//
// Visible keys are counted without the gap between the first ones and the window, so that stretches are of one length.
#include "attention_common.h"

namespace arrow {
namespace {

constexpr int kWaves = 4;
constexpr int kKeys = 32;    // keys of a tile

// 16 x 16 with 32 inner steps: lane l holds row / column l % 16 at inner steps 8 (l / 16) + 0..7; of C and D column l % 16, rows 4 (l / 16) + 0..3.

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
__global__ __launch_bounds__(64 * kWaves, 2) void attention_decode_kernel(CacheArgs a) {
  using Tl = Tile<D>;
  constexpr int kPer = D / 32;                                   // pieces of 16 bytes of a row that a lane loads
  __shared__ __align__(1024) unsigned char smem[kWaves][kKeys * Tl::kRowBytes];
  __shared__ float tops[kWaves][16], totals[kWaves][16];
  const int lane = threadIdx.x & 63, wave = wave_id(), quarter = lane >> 4, col = lane & 15;
  const arrow_cache_t& c = a.c;
  int id = blockIdx.x;
  const int kv = id % c.kv_heads; id /= c.kv_heads;
  const int split = id % a.splits; id /= a.splits;
  const int head_tiles = (a.group + kHeadTile - 1) / kHeadTile;
  const int head_tile = id % head_tiles, b = id / head_tiles;
  const int head0 = head_tile * kHeadTile, heads = min(a.group - head0, kHeadTile);
  const int64_t room = (int64_t)c.columns << a.page_log;
  const int length = (int)max((int64_t)0, min((int64_t)c.lengths[b], room));
  const int begin = c.window ? max(0, length - c.window) : 0, lead = min(c.sinks, begin);
  const int seen = lead + length - begin;
  // stretches of whole tiles
  const int tiles = (seen + kKeys - 1) / kKeys;
  const int tile0 = (int)((int64_t)tiles * split / a.splits), tile1 = (int)((int64_t)tiles * (split + 1) / a.splits);
  const int32_t* table = c.table + (int64_t)b * c.columns;
  const char* k_pool = (const char*)a.k_pool + 2 * kv * c.k_head;
  const char* v_pool = (const char*)a.v_pool + 2 * kv * c.v_head;
  const bool fresh = a.k.at != nullptr;
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

  auto row_of = [&](int i) {
    Row r{nullptr, nullptr, -1, -1};
    if (i >= seen) return r;
    const int j = i < lead ? i : i - lead + begin;
    const int page = table[j >> a.page_log];
    if (page < 0 || page >= c.pages) return r;
    const int slot = j & (c.page - 1);
    const int64_t at_k = page * c.k_page + slot * c.k_token, at_v = page * c.v_page + slot * c.v_token;
    r.k = k_pool + 2 * at_k;
    r.v = v_pool + 2 * at_v;
    if (fresh && j == length - 1) { r.to_k = at_k; r.to_v = at_v; r.k = k_new; r.v = v_new; }
    return r;
  };
  // A tile on its way: of rows col and 16 + col, the pieces 4 s + quarter
  x8<T> kf[2][kPer], vf[2][kPer];
  uint32_t visible = 0;                                          // of the tile's keys, the same in all lanes
  auto load = [&](int tile) {
    const Row r[2] = {row_of(tile * kKeys + col), row_of(tile * kKeys + 16 + col)};
    visible = (uint32_t)(__ballot(r[0].k != nullptr) & 0xffff) | (uint32_t)(__ballot(r[1].k != nullptr) & 0xffff) << 16;
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int s = 0; s < kPer; ++s) {
        const int d = 32 * s + 8 * quarter;
        const x8<T> z = {};
        const bool in = r[n].k != nullptr && d < c.dim;
        kf[n][s] = in ? *(const x8<T>*)(r[n].k + 2 * d) : z;
        vf[n][s] = in ? *(const x8<T>*)(r[n].v + 2 * d) : z;
      }
    if (fresh && head_tile == 0) {
#pragma unroll
      for (int n = 0; n < 2; ++n)
        if (r[n].to_k >= 0) {
#pragma unroll
          for (int s = 0; s < kPer; ++s) {
            const int d = 32 * s + 8 * quarter;
            if (d < c.dim) {
              *(x8<T>*)((char*)k_pool + 2 * (r[n].to_k + d)) = kf[n][s];
              *(x8<T>*)((char*)v_pool + 2 * (r[n].to_v + d)) = vf[n][s];
            }
          }
        }
    }
  };

  f32x4 acc[D / 16];
#pragma unroll
  for (int m = 0; m < D / 16; ++m) acc[m] = (f32x4)(0.f);
  const float scale = c.scale * kLog2e;
  float top = minus_infinity(), total = 0.f;
  lds_byte* vt = (lds_byte*)smem[wave];
  // the transposed read: rows 16 u + 4 quarter + 0..3, columns 16 m + col
  const int tr_row = 4 * quarter + (col >> 2), tr_turn = Tl::turn(tr_row), tr_byte = tr_row * Tl::kRowBytes + ((col & 1) << 3), tr_piece = (col & 3) >> 1;

  int tile = tile0 + wave;
  if (tile < tile1) load(tile);
  while (tile < tile1) {
    f32x4 s[2];
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      s[n] = (f32x4)(0.f);
#pragma unroll
      for (int i = 0; i < kPer; ++i) s[n] = mma16(kf[n][i], qf[i], s[n]);
    }
    // (the tile is this wavefront's own: no barrier)
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int i = 0; i < kPer; ++i)
        *(__attribute__((address_space(3))) x8<T>*)(vt + (16 * n + col) * Tl::kRowBytes + (((4 * i + quarter) ^ Tl::turn(16 * n + col)) << 4)) = vf[n][i];
    const uint32_t now = visible;
    tile += kWaves;
    if (tile < tile1) load(tile);

    float most = minus_infinity();
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        s[n][i] = now >> (16 * n + 4 * quarter + i) & 1 ? s[n][i] : minus_infinity();
        most = fmaxf(most, s[n][i]);
      }
    most = max_quarters(most) * scale;
    const float next = fmaxf(top, most), off = next == minus_infinity() ? 0.f : next;
    const float by = __builtin_amdgcn_exp2f(top - off);
    top = next;
    total *= by;
#pragma unroll
    for (int m = 0; m < D / 16; ++m) acc[m] *= by;
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        s[n][i] = __builtin_amdgcn_exp2f(fmaf(s[n][i], scale, -off));
        total += s[n][i];
      }
    const x8<T> pf = round8<T>(s[0][0], s[0][1], s[0][2], s[0][3], s[1][0], s[1][1], s[1][2], s[1][3]);
#pragma unroll
    for (int m = 0; m < D / 16; ++m) {
      const lds_byte* at = vt + tr_byte + (((2 * m + tr_piece) ^ tr_turn) << 4);
      union { i16x4 half[2]; x8<T> all; } vr;
      vr.half[0] = lds_transposed(at);
      vr.half[1] = lds_transposed(at + 16 * Tl::kRowBytes);
      acc[m] = mma16(vr.all, pf, acc[m]);
    }
  }
  total = add_quarters(total);

  // the wavefronts' results, sums first: column d of head h at [d][h], 16 floats to a row (the tiles are done with)
  __syncthreads();
  float* mine = (float*)smem[wave];
  static_assert(kKeys * Tl::kRowBytes >= 16 * D * 4, "room for a wavefront's sums");
#pragma unroll
  for (int m = 0; m < D / 16; ++m)
#pragma unroll
    for (int i = 0; i < 4; ++i) mine[(16 * m + 4 * quarter + i) * 16 + col] = acc[m][i];
  if (quarter == 0) { tops[wave][col] = top; totals[wave][col] = total; }
  __syncthreads();
  for (int e = threadIdx.x; e < heads * c.dim; e += 64 * kWaves) {
    const int h = e / c.dim, d = e % c.dim;
    float all = tops[0][h];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) all = fmaxf(all, tops[w][h]);
    const float off = all == minus_infinity() ? 0.f : all;
    float sum = 0.f, weight = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float by = __builtin_amdgcn_exp2f(tops[w][h] - off);
      sum = fmaf(by, ((const float*)smem[w])[d * 16 + h], sum);
      weight = fmaf(by, totals[w][h], weight);
    }
    const int head = kv * a.group + head0 + h;
    if (a.splits == 1) {
      ((T*)a.o.at)[b * a.o.sequence + head * a.o.head + d] = (T)(weight > 0.f || weight != weight ? sum / weight : 0.f);
    } else {
      float* to = a.parts + ((int64_t)(b * c.q_heads + head) * a.splits + split) * (c.dim + 2);
      to[d] = sum;
      if (d == 0) { to[c.dim] = all; to[c.dim + 1] = weight; }
    }
  }
}

// The results of the stretches of one query head, joined: a wavefront, two columns per lane.
template <typename T>
__global__ __launch_bounds__(64) void attention_decode_join_kernel(CacheArgs a) {
  const arrow_cache_t& c = a.c;
  const int row = blockIdx.x, b = row / c.q_heads, head = row % c.q_heads, step = c.dim + 2, lane = threadIdx.x, d = 2 * lane;
  const float* from = a.parts + (int64_t)row * a.splits * step;
  float all = minus_infinity();
  for (int i = lane; i < a.splits; i += 64) all = fmaxf(all, from[(int64_t)i * step + c.dim]);
  for (int m = 32; m; m >>= 1) all = fmaxf(all, __shfl_xor(all, m, 64));
  const float off = all == minus_infinity() ? 0.f : all;
  float s0 = 0.f, s1 = 0.f, weight = 0.f;
  for (int i = 0; i < a.splits; ++i, from += step) {
    const float by = __builtin_amdgcn_exp2f(from[c.dim] - off);
    weight = fmaf(by, from[c.dim + 1], weight);
    if (d < c.dim) {
      const float2 x = *(const float2*)(from + d);
      s0 = fmaf(by, x.x, s0);
      s1 = fmaf(by, x.y, s1);
    }
  }
  const float over = weight > 0.f || weight != weight ? 1.f / weight : 0.f;
  if (d < c.dim) {
    T* to = (T*)a.o.at + b * a.o.sequence + head * a.o.head + d;
    to[0] = (T)(s0 * over);
    to[1] = (T)(s1 * over);
  }
}

// One piece of 16 bytes per thread.
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
  if (a.splits > 1) attention_decode_join_kernel<T><<<dim3((unsigned)rows), dim3(64), 0, s>>>(a);
  return (int)hipGetLastError();
}

}  // namespace

int launch_attention_decode(const CacheArgs& a, void* stream) { return a.c.dtype == ARROW_BF16 ? decode<__bf16>(a, stream) : decode<_Float16>(a, stream); }

int launch_cache_append(const CacheArgs& a, void* stream) {
  const int64_t blocks = ((int64_t)a.c.batch * a.tokens * a.c.kv_heads * (a.c.dim / 8) + 255) / 256;
  if (blocks > 0x7fffffff) return (int)hipErrorInvalidConfiguration;
  hipStream_t s = (hipStream_t)stream;
  if (a.c.dtype == ARROW_BF16) cache_append_kernel<__bf16><<<dim3((unsigned)blocks), dim3(256), 0, s>>>(a);
  else cache_append_kernel<_Float16><<<dim3((unsigned)blocks), dim3(256), 0, s>>>(a);
  return (int)hipGetLastError();
}

}  // namespace arrow
