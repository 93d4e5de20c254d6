// Attention under an arrow-shaped mask, gradients (include/arrow_attention.h).
//
// The probabilities are computed anew from the scores and the saved log-sums.  Two kernels, each with its sums in registers from
// the first tile to the last, so that no gradient is added up in memory: one over queries for dq (three products), one over keys for dk
// and dv (four).  That is seven products where five would do; the five would take an addition in memory for every tile's dq, whose
// order either changes from run to run or has to be enforced.
#include "attention_common.h"

namespace arrow {
namespace {

constexpr int kStep = 64;   // keys of a tile (dq)

// dq, and <do_i, o_i> for the other kernel.  As the forward kernel: a wavefront holds 32 queries, scores and their gradients are
// transposed, dS^T is at once the B operand of dQ^T += K^T dS^T.
template <typename T, int D>
__global__ __launch_bounds__(256, 2) void attention_dq_kernel(AttentionArgs a, int tiles) {
  using Tl = Tile<D>;
  __shared__ __align__(1024) unsigned char smem[4][kStep * Tl::kRowBytes];
  const int lane = threadIdx.x & 63, wave = wave_id(), half = lane >> 5;
  int id = blockIdx.x;
  const int g = id % a.group; id /= a.group;
  const int tile = tiles - 1 - id % tiles; id /= tiles;
  const int kv = id % a.kv_heads, b = id / a.kv_heads, head = kv * a.group + g;
  const bool ragged = a.q_offsets != nullptr;
  const Span sq = span_of(a.q_offsets, b, a.q_tokens, a.q_len), sk = span_of(a.k_offsets, b, a.k_tokens, a.k_len);
  const int first = tile * kQueryTile;
  if (first >= sq.count) return;
  const int shift = sk.count - sq.count;
  const int row = first + wave * 32 + (lane & 31);
  const bool there = row < sq.count;
  const int p = row + shift;
  const char* q = rows_of(a.q, ragged, b, sq.first, head);
  const char* k = rows_of(a.k, ragged, b, sk.first, kv);
  const char* v = rows_of(a.v, ragged, b, sk.first, kv);
  const char* o = rows_of(a.o, ragged, b, sq.first, head);
  const char* d_o = rows_of(a.d_o, ragged, b, sq.first, head);

  x8<T> qf[D / 16], df[D / 16];
  float delta = 0.f;
#pragma unroll
  for (int s = 0; s < D / 16; ++s) {
    const int d = 16 * s + 8 * half;
    const x8<T> z = {};
    const bool in = there && d < a.dim;
    qf[s] = in ? *(const x8<T>*)(q + 2 * ((int64_t)row * a.q.token + d)) : z;
    df[s] = in ? *(const x8<T>*)(d_o + 2 * ((int64_t)row * a.d_o.token + d)) : z;
    const x8<T> of = in ? *(const x8<T>*)(o + 2 * ((int64_t)row * a.o.token + d)) : z;
#pragma unroll
    for (int i = 0; i < 8; ++i) delta = fmaf((float)df[s][i], (float)of[i], delta);
  }
  delta = add_halves(delta);
  const int64_t stat = ragged ? head * a.q_tokens + sq.first + row : ((int64_t)b * a.q_heads + head) * a.q_len + row;
  if (there && half == 0) a.delta[stat] = delta;
  // of a row that sees nothing, -infinity: its probabilities are masked
  const float lse = there ? a.lse_in[stat] * kLog2e : 0.f;

  const int last = min(first + kQueryTile, sq.count) - 1 + shift;
  const SeenTiles seen = seen_tiles<kStep>(max(first + shift, 0), last, a.window, a.sinks);
  const int low = first + wave * 32 + shift, high = min(low + 31, sk.count - 1);
  f32x16 acc[D / 32];
#pragma unroll
  for (int m = 0; m < D / 32; ++m) acc[m] = (f32x16)(0.f);
  const float c = a.scale * kLog2e;

  const Loader<D, kStep, 4> lk(wave, lane, a.k.token, a.dim), lv(wave, lane, a.v.token, a.dim);
  lds_byte* base = (lds_byte*)smem;
  auto load = [&](int t, int to) {
    const int k0 = seen.at(t) * kStep;
    lk.load(k + 2 * (int64_t)k0 * a.k.token, sk.count - k0, base + (2 * to) * (kStep * Tl::kRowBytes), wave);
    lv.load(v + 2 * (int64_t)k0 * a.v.token, sk.count - k0, base + (2 * to + 1) * (kStep * Tl::kRowBytes), wave);
  };
  if (seen.total > 0) load(0, 0);
  for (int t = 0; t < seen.total; ++t) {
    wait_for_tiles();
    if (t + 1 < seen.total) load(t + 1, (t + 1) & 1);
    const lds_byte* kt = base + (2 * (t & 1)) * (kStep * Tl::kRowBytes);
    const lds_byte* vt = kt + kStep * Tl::kRowBytes;
    const int k0 = seen.at(t) * kStep;
    if (k0 > high || (a.window && k0 >= a.sinks && k0 + kStep - 1 <= low - a.window)) continue;
    const bool whole = k0 + kStep - 1 <= low && (!a.window || k0 > low + 31 - a.window || k0 + kStep <= a.sinks);
    const int ago = p - k0 - 4 * half, sinks = min(a.sinks - k0 - 4 * half, ago + 1);
    const uint32_t window = a.window ? (uint32_t)a.window : 0x80000000u;
#pragma unroll
    for (int n = 0; n < kStep / 32; ++n) {
      f32x16 s = (f32x16)(0.f), e = (f32x16)(0.f);
#pragma unroll
      for (int i = 0; i < D / 16; ++i) {
        s = mma32(lds_rows<T>(kt + n * 32 * Tl::kRowBytes + Tl::rows_at(lane, i)), qf[i], s);
        e = mma32(lds_rows<T>(vt + n * 32 * Tl::kRowBytes + Tl::rows_at(lane, i)), df[i], e);
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = __builtin_amdgcn_exp2f(fmaf(s[i], c, -lse)) * (e[i] - delta);
      if (!whole) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int j = n * 32 + 8 * (i / 4) + i % 4;
          const bool visible = ((uint32_t)(ago - j) < window) | (j < sinks);   // (without branches)
          s[i] = visible ? s[i] : 0.f;
        }
      }
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const x8<T> ds = round8<T>(s[8 * u], s[8 * u + 1], s[8 * u + 2], s[8 * u + 3], s[8 * u + 4], s[8 * u + 5], s[8 * u + 6], s[8 * u + 7]);
        const lds_byte* at = kt + (n * 32 + 16 * u) * Tl::kRowBytes;
#pragma unroll
        for (int m = 0; m < D / 32; ++m)
          acc[m] = mma32(lds_columns<T>(at + Tl::columns_at(lane, m, 0), at + Tl::columns_at(lane, m, 1)), ds, acc[m]);
      }
    }
  }

  T* dq = (T*)rows_of(a.dq, ragged, b, sq.first, head) + (int64_t)row * a.dq.token;
#pragma unroll
  for (int m = 0; m < D / 32; ++m) acc[m] *= a.scale;
  if (there) store_columns<T, D>(acc, dq, half, a.dim);
}

// dk and dv of 128 keys, 32 per wavefront, over the queries of all heads that share them.  Scores are not transposed here: a lane
// has one key's, P and dS are at once the B operands of dV^T += dO^T P and dK^T += Q^T dS.
//
// Parts: part i of n takes the steps (64 queries of one head) from i / n to (i + 1) / n of the tile's; with n > 1 their sums go
// to the workspace and attention_join_kernel adds them up in order.
template <typename T, int D>
__global__ __launch_bounds__(256, 1) void attention_dkv_kernel(AttentionArgs a, int tiles) {
  using Tl = Tile<D>;
  constexpr int kBytes = kQueryStep * Tl::kRowBytes;
  __shared__ __align__(1024) unsigned char smem[4][kBytes];      // q and do, two tiles each
  __shared__ float stats[2][2][kQueryStep];                      // lse and delta
  const int lane = threadIdx.x & 63, wave = wave_id(), half = lane >> 5;
  int id = blockIdx.x;
  const int per_head = a.sink_tiles * a.sink_parts + (tiles - a.sink_tiles) * a.tile_parts;
  const int item = id % per_head; id /= per_head;
  const int kv = id % a.kv_heads, b = id / a.kv_heads;
  const int sink_items = a.sink_tiles * a.sink_parts;
  const int parts = item < sink_items ? a.sink_parts : a.tile_parts;
  const int tile = item < sink_items ? item / parts : a.sink_tiles + (item - sink_items) / parts;
  const int part = (item < sink_items ? item : item - sink_items) % parts;
  const bool ragged = a.q_offsets != nullptr;
  const Span sq = span_of(a.q_offsets, b, a.q_tokens, a.q_len), sk = span_of(a.k_offsets, b, a.k_tokens, a.k_len);
  const int first = tile * kKeyTile;
  if (first >= sk.count) return;
  const int shift = sk.count - sq.count;
  const int key = first + wave * 32 + (lane & 31);
  const bool there = key < sk.count;
  const char* k = rows_of(a.k, ragged, b, sk.first, kv);
  const char* v = rows_of(a.v, ragged, b, sk.first, kv);
  x8<T> kf[D / 16], vf[D / 16];
#pragma unroll
  for (int s = 0; s < D / 16; ++s) {
    const int d = 16 * s + 8 * half;
    const x8<T> z = {};
    const bool in = there && d < a.dim;
    kf[s] = in ? *(const x8<T>*)(k + 2 * ((int64_t)key * a.k.token + d)) : z;
    vf[s] = in ? *(const x8<T>*)(v + 2 * ((int64_t)key * a.v.token + d)) : z;
  }
  f32x16 dk[D / 32], dv[D / 32];
#pragma unroll
  for (int m = 0; m < D / 32; ++m) { dk[m] = (f32x16)(0.f); dv[m] = (f32x16)(0.f); }

  // queries that see one of the tile's keys: positions first .. end
  const int tile_end = min(first + kKeyTile, sk.count) - 1;
  int end = sk.count - 1;
  if (a.window && first >= a.sinks) end = (int)min((int64_t)end, (int64_t)tile_end + a.window - 1);
  const int q_begin = max(first - shift, 0) / kQueryStep;
  const int q_steps = end - shift < 0 || first - shift >= sq.count ? 0 : (end - shift) / kQueryStep + 1 - q_begin;
  const int steps = max(q_steps, 0) * a.group;
  const int step0 = (int)((int64_t)steps * part / parts), step1 = (int)((int64_t)steps * (part + 1) / parts);
  const float c = a.scale * kLog2e;

  const Loader<D, kQueryStep, 4> lq(wave, lane, a.q.token, a.dim), ld(wave, lane, a.d_o.token, a.dim);
  lds_byte* base = (lds_byte*)smem;
  float held = 0.f;                                              // lse or delta on its way to LDS, threads 0..127
  auto load = [&](int t, int to) {
    const int head = kv * a.group + t / q_steps, q0 = (q_begin + t % q_steps) * kQueryStep;
    const char* q = rows_of(a.q, ragged, b, sq.first, head);
    const char* d_o = rows_of(a.d_o, ragged, b, sq.first, head);
    lq.load(q + 2 * (int64_t)q0 * a.q.token, sq.count - q0, base + (2 * to) * kBytes, wave);
    ld.load(d_o + 2 * (int64_t)q0 * a.d_o.token, sq.count - q0, base + (2 * to + 1) * kBytes, wave);
    const int64_t stat = ragged ? head * a.q_tokens + sq.first + q0 : ((int64_t)b * a.q_heads + head) * a.q_len + q0;
    const int i = threadIdx.x & 63;
    if (wave < 2) held = q0 + i < sq.count ? (wave == 0 ? a.lse_in : a.delta)[stat + i] : 0.f;
  };
  if (step0 < step1) load(step0, 0);
  for (int t = step0; t < step1; ++t) {
    const int now = (t - step0) & 1;
    if (wave < 2) stats[now][wave][threadIdx.x & 63] = wave == 0 ? held * kLog2e : held;
    wait_for_tiles();
    if (t + 1 < step1) load(t + 1, now ^ 1);
    const lds_byte* qt = base + (2 * now) * kBytes;
    const lds_byte* dt = qt + kBytes;
    const int q0 = (q_begin + t % q_steps) * kQueryStep;
    const int low = first + wave * 32, high = min(low + 31, sk.count - 1);   // this wavefront's keys
#pragma unroll
    for (int n = 0; n < kQueryStep / 32; ++n) {
      const int p0 = q0 + n * 32 + shift;                        // position of the first of 32 queries
      if (q0 + n * 32 >= sq.count || p0 + 31 < low || (a.window && low >= a.sinks && p0 - a.window >= high)) continue;
      f32x16 s = (f32x16)(0.f), e = (f32x16)(0.f);
#pragma unroll
      for (int i = 0; i < D / 16; ++i) {
        s = mma32(lds_rows<T>(qt + n * 32 * Tl::kRowBytes + Tl::rows_at(lane, i)), kf[i], s);
        e = mma32(lds_rows<T>(dt + n * 32 * Tl::kRowBytes + Tl::rows_at(lane, i)), vf[i], e);
      }
      const bool whole = p0 >= low + 31 && q0 + n * 32 + 32 <= sq.count && (!a.window || p0 + 31 - a.window < low || low + 32 <= a.sinks);
      const int ahead = p0 + 4 * half - key;                     // how far the first of this lane's queries is ahead of its key
      const uint32_t window = a.window && key >= a.sinks ? (uint32_t)a.window : 0x80000000u;
#pragma unroll
      for (int i = 0; i < 16; i += 4) {
        const f32x4 lse = *(const f32x4*)&stats[now][0][n * 32 + 2 * i + 4 * half], delta = *(const f32x4*)&stats[now][1][n * 32 + 2 * i + 4 * half];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          float x = __builtin_amdgcn_exp2f(fmaf(s[i + j], c, -lse[j])), y = x * (e[i + j] - delta[j]);
          if (!whole) {
            const bool visible = (uint32_t)(ahead + 2 * i + j) < window && q0 + n * 32 + 2 * i + 4 * half + j < sq.count;
            x = visible ? x : 0.f;
            y = visible ? y : 0.f;
          }
          s[i + j] = x;
          e[i + j] = y;
        }
      }
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const x8<T> pf = round8<T>(s[8 * u], s[8 * u + 1], s[8 * u + 2], s[8 * u + 3], s[8 * u + 4], s[8 * u + 5], s[8 * u + 6], s[8 * u + 7]);
        const x8<T> ds = round8<T>(e[8 * u], e[8 * u + 1], e[8 * u + 2], e[8 * u + 3], e[8 * u + 4], e[8 * u + 5], e[8 * u + 6], e[8 * u + 7]);
        const lds_byte* at = dt + (n * 32 + 16 * u) * Tl::kRowBytes;
        const lds_byte* qat = qt + (n * 32 + 16 * u) * Tl::kRowBytes;
#pragma unroll
        for (int m = 0; m < D / 32; ++m) {
          dv[m] = mma32(lds_columns<T>(at + Tl::columns_at(lane, m, 0), at + Tl::columns_at(lane, m, 1)), pf, dv[m]);
          dk[m] = mma32(lds_columns<T>(qat + Tl::columns_at(lane, m, 0), qat + Tl::columns_at(lane, m, 1)), ds, dk[m]);
        }
      }
    }
  }

#pragma unroll
  for (int m = 0; m < D / 32; ++m) dk[m] *= a.scale;
  if (parts == 1) {
    if (!there) return;
    store_columns<T, D>(dk, (T*)rows_of(a.dk, ragged, b, sk.first, kv) + (int64_t)key * a.dk.token, half, a.dim);
    store_columns<T, D>(dv, (T*)rows_of(a.dv, ragged, b, sk.first, kv) + (int64_t)key * a.dv.token, half, a.dim);
    return;
  }
  // parts in the workspace: [sequence, head][item][dk, dv][key][dim]; items of tiles in one part have no place there
  const int64_t pair = part_place(a, tiles, ((int64_t)b * a.kv_heads + kv), tile, part);
  float* to = a.parts + pair * 2 * kKeyTile * a.dim + (int64_t)(wave * 32 + (lane & 31)) * a.dim;
#pragma unroll
  for (int m = 0; m < D / 32; ++m)
#pragma unroll
    for (int i = 0; i < 16; i += 4) {
      const int d = 32 * m + 2 * i + 4 * half;
      if (d < a.dim) {
        *(f32x4*)(to + d) = f32x4{dk[m][i], dk[m][i + 1], dk[m][i + 2], dk[m][i + 3]};
        *(f32x4*)(to + kKeyTile * a.dim + d) = f32x4{dv[m][i], dv[m][i + 1], dv[m][i + 2], dv[m][i + 3]};
      }
    }
}

// Adds up the parts of tiles that were cut, eight columns of a key per thread, dk and dv.
template <typename T>
__global__ __launch_bounds__(256) void attention_join_kernel(AttentionArgs a, int tiles, int cut_tiles, int first_cut) {
  const int pieces = a.dim / 8;
  const int64_t per_tile = (int64_t)kKeyTile * pieces * 2;
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x, place = id / per_tile;
  const int64_t unit = place / cut_tiles;                        // sequence and key head
  if (unit >= (int64_t)a.batch * a.kv_heads) return;
  const int tile = first_cut + (int)(place % cut_tiles), in = (int)(id % per_tile);
  const int piece = in % pieces, key_in = in / pieces % kKeyTile, value = in / pieces / kKeyTile;
  const int b = (int)(unit / a.kv_heads), kv = (int)(unit % a.kv_heads);
  const bool ragged = a.q_offsets != nullptr;
  const Span sk = span_of(a.k_offsets, b, a.k_tokens, a.k_len);
  const int key = tile * kKeyTile + key_in;
  if (key >= sk.count) return;
  const int parts = tile < a.sink_tiles ? a.sink_parts : a.tile_parts;
  float sum[8] = {};
  const float* from = a.parts + part_place(a, tiles, unit, tile, 0) * 2 * kKeyTile * a.dim + ((int64_t)value * kKeyTile + key_in) * a.dim + piece * 8;
  for (int i = 0; i < parts; ++i, from += 2 * kKeyTile * a.dim) {
    const f32x4 lo = *(const f32x4*)from, hi = *(const f32x4*)(from + 4);
#pragma unroll
    for (int j = 0; j < 4; ++j) { sum[j] += lo[j]; sum[4 + j] += hi[j]; }
  }
  const Operand& to = value ? a.dv : a.dk;
  *(x8<T>*)((T*)rows_of(to, ragged, b, sk.first, kv) + (int64_t)key * to.token + piece * 8) =
      round8<T>(sum[0], sum[1], sum[2], sum[3], sum[4], sum[5], sum[6], sum[7]);
}

template <typename T, int D>
int backward(const AttentionArgs& a, void* stream) {
  const int64_t q_tiles = (a.q_len + (int64_t)kQueryTile - 1) / kQueryTile, q_blocks = q_tiles * a.q_heads * a.batch;
  const int64_t k_tiles = (a.k_len + (int64_t)kKeyTile - 1) / kKeyTile;
  const int64_t k_blocks = (a.sink_tiles * (int64_t)a.sink_parts + (k_tiles - a.sink_tiles) * a.tile_parts) * a.kv_heads * a.batch;
  const int first_cut = a.sink_parts > 1 ? 0 : a.sink_tiles, cut = (int)((a.tile_parts > 1 ? k_tiles : a.sink_tiles) - first_cut);
  const int64_t join_blocks = cut > 0 ? ((int64_t)cut * a.kv_heads * a.batch * kKeyTile * (a.dim / 8) * 2 + 255) / 256 : 0;
  if (q_blocks > 0x7fffffff || k_blocks > 0x7fffffff || join_blocks > 0x7fffffff) return (int)hipErrorInvalidConfiguration;
  hipStream_t s = (hipStream_t)stream;
  if (q_blocks) attention_dq_kernel<T, D><<<dim3((unsigned)q_blocks), dim3(256), 0, s>>>(a, (int)q_tiles);
  if (k_blocks) attention_dkv_kernel<T, D><<<dim3((unsigned)k_blocks), dim3(256), 0, s>>>(a, (int)k_tiles);
  if (join_blocks) attention_join_kernel<T><<<dim3((unsigned)join_blocks), dim3(256), 0, s>>>(a, (int)k_tiles, cut, first_cut);
  return (int)hipGetLastError();
}

}  // namespace

int launch_attention_backward(const AttentionArgs& a, int32_t dtype, void* stream) {
  if (dtype == ARROW_BF16) return a.dim <= 64 ? backward<__bf16, 64>(a, stream) : backward<__bf16, 128>(a, stream);
  return a.dim <= 64 ? backward<_Float16, 64>(a, stream) : backward<_Float16, 128>(a, stream);
}

}  // namespace arrow
