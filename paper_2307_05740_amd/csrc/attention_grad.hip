// Attention under an arrow-shaped mask, gradients (include/arrow_attention.h).
//
// The probabilities are computed anew from the scores and the saved log-sums.  Two kernels, each with its sums in registers from
// the first tile to the last, so that no gradient is added up in memory: one over queries for dq (three products, and a fourth that puts it right), one over keys for dk
// and dv (four).  That is seven products where five would do; the five would take an addition in memory for every tile's dq, whose
// order either changes from run to run or has to be enforced.
#include <type_traits>

#include "attention_common.h"

namespace arrow {
namespace {

// float16 holds nothing below 2^-24, and whole numbers of 2^-24 below 2^-14, which the P and dS of long rows and small gradients do not stay above.  So dS (and P
// in the dk, dv kernel) are rounded as multiples of a power of two, by the size of d_o: of a row in the dq kernel, of all rows that a key tile's
// queries are among in the other one, which takes those from the dq kernel's notes, one for 32 queries.
template <typename T> constexpr bool kScaled = std::is_same<T, _Float16>::value;
__device__ __forceinline__ float finite_size(float x) { return fabsf(x) < __builtin_inff() ? fabsf(x) : 0.f; }
// The power of two that brings x into [1, 2), 1 for 0.
__device__ __forceinline__ float unit_of(float x) { return x > 0.f ? __uint_as_float((254u << 23) - (__float_as_uint(x) & 0x7f800000u)) : 1.f; }
// Where the notes of a sequence and head begin.
__device__ __forceinline__ int64_t groups_at(const AttentionArgs& a, bool ragged, int b, int64_t head, int64_t first) {
  return ragged ? head * (a.q_tokens / 32 + a.batch) + first / 32 + b : ((int64_t)b * a.q_heads + head) * ((a.q_len + 31) / 32);
}

// dq, and D_i = sum_j P(i,j) <do_i, v_j> for the other kernel.  As the forward kernel: a wavefront holds 32 queries, scores and their gradients
// are transposed, dS^T is at once the B operand of dQ^T += K^T dS^T.
//
// D is <do_i, o_i> as well, but o has been rounded, and where a row has one large probability dS is a small difference of <do_i, v_j>
// and D.  dS is formed with <do_i, o_i>; the error -sum_j dS(i,j) of that comes out with the row, in 32 bits.  dq is put right with one
// product more, sum_j P(i,j) k_j times that sum.  Workgroups whose wavefronts share queries, where all sequences of up to 64 keys are, take the
// sum of the dS as they were rounded for their product: the weights then add up to nothing, as the true gradient's do, which a row of few keys notices
// (dq of 5 keys off by 1.55 times what rounding dq alone does, and 1.4 so; for long rows the same, and 15 % of the kernel's time).
//
// What bounds it: matrix instructions (four products) and the vector instructions between them, at the clock that the power leaves: 8192 tokens, 32/8 heads of
// 128, window of 2048, 470 us = 1030 TFLOP/s with the product P K, matrix units busy 55 % of the cycles.  Heads of more than 64 leave no registers for the queries, which
// are read from LDS again and again, and tiles of 32 keys; of 64, 4 x 2048 tokens, window of 512: 57 us.
//
// kGroups: as in the forward kernel, how many groups of 32 queries the four wavefronts have.
template <typename T, int C, int kGroups>
__global__ __launch_bounds__(256, kGroups > 1 ? 2 : 1) void attention_dq_kernel(AttentionArgs a, int tiles) {
  constexpr int D = columns_of_tile(C);
  using Tl = Tile<D>;
  constexpr bool kShare = kGroups > 1;                           // tiles
  constexpr bool kQueriesInLds = D > 64;                         // no registers are left for them
  constexpr int kMine = kQueriesInLds || kGroups < 4 ? 32 : 64;  // keys of a tile that a wavefront takes
  constexpr int kStep = kGroups == 2 ? 64 : kMine, kBytes = kStep * Tl::kRowBytes;   // keys of a tile
  constexpr int kTurns = kShare ? 1 : 4, kRows = 32 * kGroups, kParts = 4 / kGroups;
  // k and v, two tiles each, of all wavefronts or of each one, or their sums to be joined; the queries, afterwards the sums of dS to be joined
  constexpr int kQueriesAt = 4 * kTurns * kBytes, kQueriesBytes = kQueriesInLds ? kRows * Tl::kRowBytes : 0;
  constexpr int kRestBytes = kParts == 1 ? 0 : 2 * 4 * 64 * 4 + 4 * 8;
  static_assert(kParts == 1 || kQueriesAt >= 4 * C * 32 * 4, "room for the sums");
  __shared__ __align__(1024) unsigned char smem[kQueriesAt + (kQueriesBytes > kRestBytes ? kQueriesBytes : kRestBytes)];
  const int lane = threadIdx.x & 63, wave = wave_id(), half = lane >> 5;
  const int units = a.kv_heads * a.batch, unit = blockIdx.x % units, item = blockIdx.x / units;   // as in the forward kernel
  const int g = item % a.group, tile = tiles - 1 - item / a.group;
  const int kv = unit % a.kv_heads, b = unit / a.kv_heads, head = kv * a.group + g;
  const bool ragged = a.q_offsets != nullptr;
  const Span sq = span_of(a.q_offsets, b, a.q_tokens, a.q_len), sk = span_of(a.k_offsets, b, a.k_tokens, a.k_len);
  const int first = tile * kRows;
  if (first >= sq.count) return;
  const int shift = sk.count - sq.count;
  const int group = wave % kGroups, split = wave / kGroups;
  const int mine = first + group * 32;
  const int row = mine + (lane & 31);
  const bool there = row < sq.count;
  const int p = row + shift;
  const char* q = rows_of(a.q, ragged, b, sq.first, head);
  const char* k = rows_of(a.k, ragged, b, sk.first, kv);
  const char* v = rows_of(a.v, ragged, b, sk.first, kv);
  const char* o = rows_of(a.o, ragged, b, sq.first, head);
  const char* d_o = rows_of(a.d_o, ragged, b, sq.first, head);
  lds_byte *room = (lds_byte*)smem, *base = room + (kShare ? 0 : wave * 4 * kBytes);

  x8<T> qf[kQueriesInLds ? 1 : C / 16], df[C / 16];
  if constexpr (kQueriesInLds)                                   // (waited for with the first tiles)
    Loader<D, kRows, 4>(wave, lane, a.q.token, a.dim).load(q + 2 * (int64_t)first * a.q.token, sq.count - first, room + kQueriesAt, wave);
  float delta = 0.f, most = 0.f;
#pragma unroll
  for (int s = 0; s < C / 16; ++s) {
    const int d = 16 * s + 8 * half;
    const x8<T> z = {};
    const bool in = there && d < a.dim;
    if constexpr (!kQueriesInLds) qf[s] = in ? *(const x8<T>*)(q + 2 * ((int64_t)row * a.q.token + d)) : z;
    df[s] = in ? *(const x8<T>*)(d_o + 2 * ((int64_t)row * a.d_o.token + d)) : z;
    const x8<T> of = in ? *(const x8<T>*)(o + 2 * ((int64_t)row * a.o.token + d)) : z;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      delta = fmaf((float)df[s][i], (float)of[i], delta);
      if constexpr (kScaled<T>) most = fmaxf(most, finite_size((float)df[s][i]));
    }
  }
  delta = add_halves(delta);
  float larger = 1.f;                                            // that d_o of this row is multiplied by, and taken out of the result again
  if constexpr (kScaled<T>) {
    most = max_halves(most);
    larger = unit_of(most);
    delta *= larger;
#pragma unroll
    for (int s = 0; s < C / 16; ++s)
#pragma unroll
      for (int i = 0; i < 8; ++i) df[s][i] = (T)((float)df[s][i] * larger);
    for (int m = 16; m; m >>= 1) most = fmaxf(most, __shfl_xor(most, m, 64));
    if (lane == 0 && split == 0 && mine < sq.count) a.most[groups_at(a, ragged, b, head, sq.first) + mine / 32] = most;
  }
  const int64_t stat = ragged ? head * a.q_tokens + sq.first + row : ((int64_t)b * a.q_heads + head) * a.q_len + row;
  // of a row that sees nothing, infinity: its probabilities are masked
  const float off = there ? -a.lse_in[stat] / a.scale : 0.f;

  const int last = min(first + kRows, sq.count) - 1 + shift;
  const SeenTiles seen = seen_tiles<kStep>(max(first + shift, 0), last, a.window, a.sinks);
  const int low = mine + shift, high = min(low + 31, sk.count - 1);
  const float c = a.scale * kLog2e;

  const int sharer = kShare ? wave : 0;
  const Loader<D, kStep, 4 / kTurns> lk(sharer, lane, a.k.token, a.dim), lv(sharer, lane, a.v.token, a.dim);
  const TileReads<D> my(lane);
  auto load = [&](int t, int to) {
    const int k0 = seen.at(t) * kStep;
    lk.load(k + 2 * (int64_t)k0 * a.k.token, sk.count - k0, base + (2 * to) * kBytes, sharer);
    lv.load(v + 2 * (int64_t)k0 * a.v.token, sk.count - k0, base + (2 * to + 1) * kBytes, sharer);
  };
  f32x16 acc[C / 32], pk[C / 32];                             // dS K and P K
#pragma unroll
  for (int m = 0; m < C / 32; ++m) { acc[m] = (f32x16)(0.f); pk[m] = (f32x16)(0.f); }
  float rest = 0.f, kept = 0.f;                               // sums of dS of this lane's keys, before and after they are rounded
  const int t0 = kShare ? 0 : wave;
  if (t0 < seen.total) load(t0, 0);
  if constexpr (!kShare && kQueriesInLds) wait_for_tiles();     // (all wavefronts' queries)
  for (int t = t0, now = 0; t < seen.total; t += kTurns, now ^= 1) {
    if constexpr (kShare) wait_for_tiles();
    else wait_for_own_tiles();
    if (t + kTurns < seen.total) load(t + kTurns, now ^ 1);
    const int skip = kMine < kStep ? split * kMine : 0;
    const uint32_t kt = lds_address(base) + 2 * now * kBytes + skip * Tl::kRowBytes, vt = kt + kBytes;
    const uint32_t qt = kQueriesInLds ? here(lds_address(room) + kQueriesAt + group * 32 * Tl::kRowBytes + my.rows) : 0;
    const int k0 = seen.at(t) * kStep + skip;
    if (k0 > high || (a.window && k0 >= a.sinks && k0 + kMine - 1 <= low - a.window)) continue;
    const bool whole = k0 + kMine - 1 <= low && (!a.window || k0 > low + 31 - a.window || k0 + kMine <= a.sinks);
    const int ago = p - k0 - 4 * half, sinks = min(a.sinks - k0 - 4 * half, ago + 1);
    const uint32_t window = a.window ? (uint32_t)a.window : 0x80000000u;
#pragma unroll
    for (int n = 0; n < kMine / 32; ++n) {
      // the products begin with what is taken off them (which is in one register each, not in 16 ready for that, where those are needed)
      f32x16 s = (f32x16)(kQueriesInLds ? here(off) : off), e = (f32x16)(kQueriesInLds ? here(-delta) : -delta);
#pragma unroll
      for (int i = 0; i < C / 16; ++i)
        s = mma32(read_rows<T>(kt + my.rows, i, n * 32 * Tl::kRowBytes), kQueriesInLds ? read_rows<T>(qt, i, 0) : qf[kQueriesInLds ? 0 : i], s);
#pragma unroll
      for (int i = 0; i < C / 16; ++i) e = mma32(read_rows<T>(vt + my.rows, i, n * 32 * Tl::kRowBytes), df[i], e);
      reads_ahead<4, C / 16, kQueriesInLds ? 2 : 1, C / 16, 1>();
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = __builtin_amdgcn_exp2f(s[i] * c);
      if (!whole) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int j = n * 32 + 8 * (i / 4) + i % 4;
          const bool visible = ((uint32_t)(ago - j) < window) | (j < sinks);   // (without branches)
          s[i] = visible ? s[i] : 0.f;
          e[i] = visible ? e[i] : 0.f;
        }
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        e[i] *= s[i];
        rest += e[i];
      }
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const x8<T> pf = round8<T>(s[8 * u], s[8 * u + 1], s[8 * u + 2], s[8 * u + 3], s[8 * u + 4], s[8 * u + 5], s[8 * u + 6], s[8 * u + 7]);
        const x8<T> ds = round8<T>(e[8 * u], e[8 * u + 1], e[8 * u + 2], e[8 * u + 3], e[8 * u + 4], e[8 * u + 5], e[8 * u + 6], e[8 * u + 7]);
        if constexpr (kParts > 1) kept = add8(ds, kept);
#pragma unroll
        for (int m = 0; m < C / 32; ++m) {
          const x8<T> kf = read_columns<T, D>(kt + my.columns, m, (n * 32 + 16 * u) * Tl::kRowBytes);
          acc[m] = mma32(kf, ds, acc[m]);
          pk[m] = mma32(kf, pf, pk[m]);
        }
      }
      reads_ahead<4, 4 * (C / 32), 1>();
    }
  }

  rest = add_halves(rest);
  kept = kParts == 1 ? rest : add_halves(kept);
  T* dq = (T*)rows_of(a.dq, ragged, b, sq.first, head) + (int64_t)row * a.dq.token;
  // Rows to be done in plain steps, as in the forward kernel: with a result that is not finite, though what they see may be
  auto odd_rows = [&](float test) {
    const uint64_t odd = __ballot(there && off == off && delta == delta && test != test);
    return (odd | odd >> 32) & 0xffffffffu;
  };
  auto plain_rows = [&](uint64_t odd) {
    const int d = 2 * lane;
    const bool in = d < a.dim;
    while (odd) {
      const int r = __builtin_ctzll(odd), at = mine + r, pr = at + shift;
      odd &= odd - 1;
      const T *qr = (const T*)q + (int64_t)at * a.q.token + d, *gr = (const T*)d_o + (int64_t)at * a.d_o.token + d;
      const float q0 = in ? (float)qr[0] : 0.f, q1 = in ? (float)qr[1] : 0.f, g0 = in ? (float)gr[0] : 0.f, g1 = in ? (float)gr[1] : 0.f;
      const float plus = __shfl(off, r, 64), by = __shfl(larger, r, 64), less = __shfl(delta + rest, r, 64);
      float x0 = 0.f, x1 = 0.f;
      for (int j = 0; j <= pr; ++j) {
        if (a.window && j >= a.sinks && j <= pr - a.window) { j = pr - a.window; continue; }
        const T *kj = (const T*)k + (int64_t)j * a.k.token + d, *vj = (const T*)v + (int64_t)j * a.v.token + d;
        const float k0 = in ? (float)kj[0] : 0.f, k1 = in ? (float)kj[1] : 0.f;
        float s = q0 * k0 + q1 * k1, e = in ? g0 * (float)vj[0] + g1 * (float)vj[1] : 0.f;
        for (int m = 32; m; m >>= 1) { s += __shfl_xor(s, m, 64); e += __shfl_xor(e, m, 64); }
        const float ds = exp2f((s + plus) * c) * (e * by - less);
        x0 = fmaf(ds, k0, x0);
        x1 = fmaf(ds, k1, x1);
      }
      T* to = (T*)rows_of(a.dq, ragged, b, sq.first, head) + (int64_t)at * a.dq.token + d;
      if (in) { to[0] = (T)(a.scale / by * x0); to[1] = (T)(a.scale / by * x1); }
    }
  };
  float test = 0.f;                                           // NaN where a result is not finite
  uint64_t* odds = (uint64_t*)(smem + kQueriesAt + 2 * 4 * 64 * 4);
  if constexpr (kParts > 1) {
    float* rests = (float*)(smem + kQueriesAt);
    wait_for_tiles();                                           // the tiles and queries are done with, or there and not needed
    rests[wave * 64 + lane] = rest;
    rests[(4 + wave) * 64 + lane] = kept;
    __syncthreads();
    rest = kept = 0.f;
#pragma unroll
    for (int w = 0; w < kParts; ++w) {
      rest += rests[(group + kGroups * w) * 64 + lane];
      kept += rests[(4 + group + kGroups * w) * 64 + lane];
    }
  }
  if (there && half == 0 && split == 0) {
    a.off[stat] = off;
    a.delta[stat] = -(delta + rest) / larger;
  }
  const float by = a.scale / larger;
#pragma unroll
  for (int m = 0; m < C / 32; ++m)
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[m][i] = by * fmaf(-kept, pk[m][i], acc[m][i]);
  if constexpr (kParts == 1) {
#pragma unroll
    for (int m = 0; m < C / 32; ++m)
#pragma unroll
      for (int i = 0; i < 16; ++i) test = fmaf(acc[m][i], 0.f, test);
    const uint64_t odd = odd_rows(test);
    if (there && !(odd >> (lane & 31) & 1)) store_columns<T, C>(acc, dq, half, a.dim);
    plain_rows(odd);
  } else {
    float* sums = (float*)smem;
    constexpr int kBlocks = C / 32, kJoined = (kBlocks + kParts - 1) / kParts;
#pragma unroll
    for (int m = 0; m < kBlocks; ++m)
#pragma unroll
      for (int i = 0; i < 16; ++i) sums[((wave * kBlocks + m) * 16 + i) * 64 + lane] = acc[m][i];
    __syncthreads();
    f32x16 r[kJoined];                                          // a wavefront joins every kParts-th block of 32 columns
#pragma unroll
    for (int n = 0; n < kJoined; ++n) {
      const int m = split + n * kParts;
      r[n] = (f32x16)(0.f);
      if (m >= kBlocks) continue;
#pragma unroll
      for (int w = 0; w < kParts; ++w)
#pragma unroll
        for (int i = 0; i < 16; ++i) r[n][i] += sums[(((group + kGroups * w) * kBlocks + m) * 16 + i) * 64 + lane];
#pragma unroll
      for (int i = 0; i < 16; ++i) test = fmaf(r[n][i], 0.f, test);
    }
    uint64_t odd = odd_rows(test);
    if (lane == 0) odds[wave] = odd;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kParts; ++w) odd |= odds[group + kGroups * w];
#pragma unroll
    for (int n = 0; n < kJoined; ++n) {
      const int m = split + n * kParts;
      if (m < kBlocks && there && !(odd >> (lane & 31) & 1)) store_block<T>(r[n], m, dq, half, a.dim);
    }
    if (split == 0) plain_rows(odd);
  }
}

// dk and dv of 128 keys, 32 per wavefront, over the queries of all heads that share them.  Scores are not transposed here: a lane
// has one key's, P and dS are at once the B operands of dV^T += dO^T P and dK^T += Q^T dS.
//
// Parts: part i of n takes the steps (64 queries of one head) from i / n to (i + 1) / n of the tile's; with n > 1 their sums go
// to the workspace and attention_join_kernel adds them up in order.
//
// kShare: wavefronts of 32 keys each share steps, or have the same 32 and every fourth step; tiles are in one part then.
//
// What bounds it: as the dq kernel; of 256 registers 128 are sums (heads of 128), so the keys are read from LDS as the queries are there.  8192 tokens, as above: 530 us = 910
// TFLOP/s, matrix units busy 45 %, LDS 34 % of the cycles; 4 x 2048: 61 us.  The queries come from behind the L2 (1.6 GB); another order of them, in which
// workgroups of a die read the same ones, took as long.
template <typename T, int C, bool kShare>
__global__ __launch_bounds__(256, kShare ? (C <= 64 ? 3 : 2) : 1) void attention_dkv_kernel(AttentionArgs a, int tiles) {
  constexpr int D = columns_of_tile(C);
  using Tl = Tile<D>;
  constexpr bool kKeysInLds = D > 64;
  constexpr int kQ = kKeysInLds || !kShare ? 32 : 64, kBytes = kQ * Tl::kRowBytes;   // queries of a step
  constexpr int kTurns = kShare ? 1 : 4, kKeys = kShare ? kKeyTile : 32;
  // q and do, two tiles each, of all wavefronts or of each one, or their sums to be joined; the keys; what the dq kernel noted of each query, two steps'
  constexpr int kKeysAt = 4 * kTurns * kBytes, kStatsAt = kKeysAt + (kKeysInLds ? kKeys * Tl::kRowBytes : 0), kStatsBytes = 2 * 2 * 4 * kQ;
  static_assert(kShare || kKeysAt >= 4 * 2 * D * 32 * 4, "room for the sums");
  __shared__ __align__(1024) unsigned char smem[kStatsAt + kTurns * kStatsBytes];
  const int lane = threadIdx.x & 63, wave = wave_id(), half = lane >> 5;
  // an item of every head and sequence in turn; the longest first, and last the small parts of keys that all queries see
  const int units = a.kv_heads * a.batch, unit = blockIdx.x % units, item = blockIdx.x / units;
  const int kv = unit % a.kv_heads, b = unit / a.kv_heads;
  const int usual = (tiles - a.sink_tiles) * a.tile_parts;
  const bool sink = item >= usual;
  const int parts = sink ? a.sink_parts : a.tile_parts;
  const int tile = sink ? (item - usual) / parts : a.sink_tiles + item / parts;
  const int part = (sink ? item - usual : item) % parts;
  const bool ragged = a.q_offsets != nullptr;
  const Span sq = span_of(a.q_offsets, b, a.q_tokens, a.q_len), sk = span_of(a.k_offsets, b, a.k_tokens, a.k_len);
  const int first = tile * kKeys;
  if (first >= sk.count) return;
  const int shift = sk.count - sq.count;
  const int mine = first + (kShare ? wave * 32 : 0);
  const int key = mine + (lane & 31);
  const bool there = key < sk.count;
  const char* k = rows_of(a.k, ragged, b, sk.first, kv);
  const char* v = rows_of(a.v, ragged, b, sk.first, kv);
  x8<T> kf[kKeysInLds ? 1 : C / 16], vf[C / 16];
  if constexpr (kKeysInLds)                                      // (waited for with the first step's tiles)
    Loader<D, kKeys, 4>(wave, lane, a.k.token, a.dim).load(k + 2 * (int64_t)first * a.k.token, sk.count - first, (lds_byte*)smem + kKeysAt, wave);
#pragma unroll
  for (int s = 0; s < C / 16; ++s) {
    const int d = 16 * s + 8 * half;
    const x8<T> z = {};
    const bool in = there && d < a.dim;
    if constexpr (!kKeysInLds) kf[s] = in ? *(const x8<T>*)(k + 2 * ((int64_t)key * a.k.token + d)) : z;
    vf[s] = in ? *(const x8<T>*)(v + 2 * ((int64_t)key * a.v.token + d)) : z;
  }
  f32x16 dk[C / 32], dv[C / 32];
#pragma unroll
  for (int m = 0; m < C / 32; ++m) { dk[m] = (f32x16)(0.f); dv[m] = (f32x16)(0.f); }

  // queries that see one of the tile's keys: positions first .. end
  const int tile_end = min(first + kKeys, sk.count) - 1;
  int end = sk.count - 1;
  if (a.window && first >= a.sinks) end = (int)min((int64_t)end, (int64_t)tile_end + a.window - 1);
  const int q_begin = max(first - shift, 0) / kQ;
  const int q_steps = end - shift < 0 || first - shift >= sq.count ? 0 : (end - shift) / kQ + 1 - q_begin;
  const int steps = max(q_steps, 0) * a.group;
  const int step0 = (int)((int64_t)steps * part / parts), step1 = (int)((int64_t)steps * (part + 1) / parts);
  float up = 0.f;                                                // P and dS are rounded 2^up times as large
  if constexpr (kScaled<T>) {
    const int from = q_begin * kQ / 32, groups = min((q_begin + max(q_steps, 0)) * (kQ / 32), (sq.count + 31) / 32) - from;
    float most = 0.f;
    for (int i = lane; i < groups * a.group; i += 64)
      most = fmaxf(most, a.most[groups_at(a, ragged, b, kv * a.group + i / groups, sq.first) + from + i % groups]);
    for (int m = 32; m; m >>= 1) most = fmaxf(most, __shfl_xor(most, m, 64));
    up = __builtin_amdgcn_readfirstlane(min(max(127 - (int)(__float_as_uint(most) >> 23), 0), most > 0.f ? 15 : 0));
  }
  const float c = a.scale * kLog2e;

  const int sharer = kShare ? wave : 0;
  const Loader<D, kQ, 4 / kTurns> lq(sharer, lane, a.q.token, a.dim), ld(sharer, lane, a.d_o.token, a.dim);
  lds_byte *room = (lds_byte*)smem, *base = room + (kShare ? 0 : wave * 4 * kBytes);
  lds_byte* stats = room + kStatsAt + (kShare ? 0 : wave * kStatsBytes);
  const TileReads<D> my(lane);
  // the step that is loaded next: a head's queries from q_next on, and where they lie
  const int64_t q_step = 2 * kQ * a.q.token, d_step = 2 * kQ * a.d_o.token;
  int head = kv * a.group, q_next = 0;
  const char *q_at = nullptr, *d_at = nullptr;
  int64_t stat_at = 0;
  auto begin = [&](int from) {
    q_next = from * kQ;
    q_at = rows_of(a.q, ragged, b, sq.first, head) + from * q_step;
    d_at = rows_of(a.d_o, ragged, b, sq.first, head) + from * d_step;
    stat_at = (ragged ? head * a.q_tokens + sq.first : ((int64_t)b * a.q_heads + head) * a.q_len) + q_next;
  };
  auto load_stats = [&](const float* from, lds_byte* at) {
    auto rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(from), 0, 4 * min(max(sq.count - q_next, 0), kQ), 0x00020000);
    if (lane < kQ) __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (lds_void*)at, 4, 4 * lane, 0, 0, 0);
  };
  auto load = [&](int to) {
    lq.load(q_at, sq.count - q_next, base + (2 * to) * kBytes, sharer);
    ld.load(d_at, sq.count - q_next, base + (2 * to + 1) * kBytes, sharer);
    if (!kShare || wave == 0) load_stats(a.off + stat_at, stats + 2 * to * 4 * kQ);
    if (!kShare || wave == 1) load_stats(a.delta + stat_at, stats + (2 * to + 1) * 4 * kQ);
    if constexpr (kShare) {
      q_next += kQ;
      if (q_next < (q_begin + q_steps) * kQ) {
        q_at += q_step;
        d_at += d_step;
        stat_at += kQ;
      } else if (++head < (kv + 1) * a.group) {
        begin(q_begin);
      }
    } else {
      int from = q_next / kQ + kTurns;
      while (from >= q_begin + q_steps) { from -= q_steps; ++head; }
      if (head < (kv + 1) * a.group) begin(from);
    }
  };
  const int mine0 = step0 + (kShare ? 0 : wave);                 // this wavefront's first step
  int q_loaded = 0;
  if (mine0 < step1) {
    head += mine0 / q_steps;
    begin(q_begin + mine0 % q_steps);
    q_loaded = q_next;
    load(0);
  }
  if constexpr (!kShare) wait_for_tiles();                       // (all wavefronts' keys)
  for (int t = mine0, now = 0; t < step1; t += kTurns, now ^= 1) {
    if constexpr (kShare) wait_for_tiles();
    else wait_for_own_tiles();
    const int q_now = q_loaded;
    if (t + kTurns < step1) { q_loaded = q_next; load(now ^ 1); }
    const uint32_t qt = lds_address(base) + (2 * now) * kBytes;
    const uint32_t kt = lds_address(room) + kKeysAt + sharer * 32 * Tl::kRowBytes + my.rows;
    const uint32_t stat = lds_address(stats) + now * (2 * 4 * kQ) + 16 * half;
    const int low = mine, high = min(low + 31, sk.count - 1);   // this wavefront's keys
#pragma unroll
    for (int n = 0; n < kQ / 32; ++n) {
      const int p0 = q_now + n * 32 + shift;                     // position of the first of 32 queries
      if (q_now + n * 32 >= sq.count || p0 + 31 < low || (a.window && low >= a.sinks && p0 - a.window >= high)) continue;
      f32x16 s, e;                                               // the products begin with what is taken off them
#pragma unroll
      for (int i = 0; i < 16; i += 4) {
        const f32x4 x = lds_read4(stat + 4 * (n * 32 + 2 * i)), y = lds_read4(stat + 4 * (kQ + n * 32 + 2 * i));
#pragma unroll
        for (int j = 0; j < 4; ++j) { s[i + j] = x[j]; e[i + j] = y[j]; }
      }
#pragma unroll
      for (int i = 0; i < C / 16; ++i)
        s = mma32(read_rows<T>(qt + my.rows, i, n * 32 * Tl::kRowBytes), kKeysInLds ? read_rows<T>(kt, i, 0) : kf[kKeysInLds ? 0 : i], s);
#pragma unroll
      for (int i = 0; i < C / 16; ++i) e = mma32(read_rows<T>(qt + my.rows, i, kBytes + n * 32 * Tl::kRowBytes), vf[i], e);
      reads_ahead<kKeysInLds ? 16 : 12, C / 16, kKeysInLds ? 2 : 1, C / 16, 1>();   // (eight of those ahead: what the products begin with)
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = __builtin_amdgcn_exp2f(kScaled<T> ? fmaf(s[i], c, up) : s[i] * c);
      const bool whole = p0 >= low + 31 && q_now + n * 32 + 32 <= sq.count && (!a.window || p0 + 31 - a.window < low || low + 32 <= a.sinks);
      if (!whole) {
        const int ahead = p0 + 4 * half - key;                   // how far the first of this lane's queries is ahead of its key
        const int left = sq.count - (q_now + n * 32 + 4 * half);
        const uint32_t window = a.window && key >= a.sinks ? (uint32_t)a.window : 0x80000000u;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int j = 8 * (i / 4) + i % 4;
          const bool visible = ((uint32_t)(ahead + j) < window) & (j < left);
          s[i] = visible ? s[i] : 0.f;
          e[i] = visible ? e[i] : 0.f;
        }
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) e[i] *= s[i];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const x8<T> pf = round8<T>(s[8 * u], s[8 * u + 1], s[8 * u + 2], s[8 * u + 3], s[8 * u + 4], s[8 * u + 5], s[8 * u + 6], s[8 * u + 7]);
        const x8<T> ds = round8<T>(e[8 * u], e[8 * u + 1], e[8 * u + 2], e[8 * u + 3], e[8 * u + 4], e[8 * u + 5], e[8 * u + 6], e[8 * u + 7]);
#pragma unroll
        for (int m = 0; m < C / 32; ++m) {
          dv[m] = mma32(read_columns<T, D>(qt + my.columns, m, kBytes + (n * 32 + 16 * u) * Tl::kRowBytes), pf, dv[m]);
          dk[m] = mma32(read_columns<T, D>(qt + my.columns, m, (n * 32 + 16 * u) * Tl::kRowBytes), ds, dk[m]);
        }
      }
      reads_ahead<kKeysInLds ? 8 : 4, 4 * (C / 32), 2>();
    }
  }

  T *dk_to = (T*)rows_of(a.dk, ragged, b, sk.first, kv), *dv_to = (T*)rows_of(a.dv, ragged, b, sk.first, kv);
  // parts in the workspace: [sequence, head][item][dk, dv][key][dim]; items of tiles in one part have no place there
  float* part_to = nullptr;
  if (parts > 1) part_to = a.parts + part_place(a, tiles, ((int64_t)b * a.kv_heads + kv), tile, part) * 2 * kKeyTile * a.dim + (int64_t)(mine - first) * a.dim;
  // Keys to be done in plain steps, as rows in the forward kernel: with a result that is not finite, which may come from a query that does
  // not see them.  A key whose gradients are NaN throughout is done.
  auto odd_keys = [&](float test) {
    const uint64_t odd = __ballot(there && test != test);
    return (odd | odd >> 32) & 0xffffffffu;
  };
  auto plain_keys = [&](uint64_t odd) {
    const int d = 2 * lane;
    const bool in = d < a.dim;
    while (odd) {
      const int r = __builtin_ctzll(odd), j = mine + r;
      odd &= odd - 1;
      const T *kj = (const T*)k + (int64_t)j * a.k.token + d, *vj = (const T*)v + (int64_t)j * a.v.token + d;
      const float k0 = in ? (float)kj[0] : 0.f, k1 = in ? (float)kj[1] : 0.f, v0 = in ? (float)vj[0] : 0.f, v1 = in ? (float)vj[1] : 0.f;
      float x0 = 0.f, x1 = 0.f, y0 = 0.f, y1 = 0.f;
      bool done = false;
      for (int t = step0; t < step1 && !done; ++t) {
        const int from = (q_begin + t % q_steps) * kQ, h = kv * a.group + t / q_steps;
        const T *qh = (const T*)rows_of(a.q, ragged, b, sq.first, h) + d, *gh = (const T*)rows_of(a.d_o, ragged, b, sq.first, h) + d;
        const int64_t stat = ragged ? h * a.q_tokens + sq.first : ((int64_t)b * a.q_heads + h) * a.q_len;
        for (int i = from; i < min(from + kQ, sq.count) && !done; ++i) {
          const int p = i + shift;
          if (j > p || (a.window && j >= a.sinks && j <= p - a.window)) continue;
          const T *qi = qh + (int64_t)i * a.q.token, *gi = gh + (int64_t)i * a.d_o.token;
          const float q0 = in ? (float)qi[0] : 0.f, q1 = in ? (float)qi[1] : 0.f, g0 = in ? (float)gi[0] : 0.f, g1 = in ? (float)gi[1] : 0.f;
          float s = q0 * k0 + q1 * k1, e = g0 * v0 + g1 * v1;
          for (int m = 32; m; m >>= 1) { s += __shfl_xor(s, m, 64); e += __shfl_xor(e, m, 64); }
          const float w = exp2f((s + a.off[stat + i]) * c), ds = w * (e + a.delta[stat + i]);
          x0 = fmaf(ds, q0, x0);
          x1 = fmaf(ds, q1, x1);
          y0 = fmaf(w, g0, y0);
          y1 = fmaf(w, g1, y1);
          done = __all(!in || (x0 != x0 && x1 != x1 && y0 != y0 && y1 != y1));
        }
      }
      if (in && parts > 1) {
        float* to = part_to + (int64_t)r * a.dim + d;
        to[0] = a.scale * x0;
        to[1] = a.scale * x1;
        to[kKeyTile * a.dim] = y0;
        to[kKeyTile * a.dim + 1] = y1;
      } else if (in) {
        T *x = dk_to + (int64_t)j * a.dk.token + d, *y = dv_to + (int64_t)j * a.dv.token + d;
        x[0] = (T)(a.scale * x0);
        x[1] = (T)(a.scale * x1);
        y[0] = (T)y0;
        y[1] = (T)y1;
      }
    }
  };
  const float back = kScaled<T> ? __builtin_amdgcn_exp2f(-up) : 1.f;
  float test = 0.f;                                              // NaN where a result is not finite
  if constexpr (!kShare) {
    float* sums = (float*)smem;
    uint64_t* odds = (uint64_t*)(smem + kStatsAt);
    __syncthreads();                                             // the tiles are done with
#pragma unroll
    for (int m = 0; m < C / 32; ++m)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        sums[((wave * (C / 32) + m) * 32 + i) * 64 + lane] = dk[m][i];
        sums[((wave * (C / 32) + m) * 32 + 16 + i) * 64 + lane] = dv[m][i];
      }
    __syncthreads();
    f32x16 x = (f32x16)(0.f), y = (f32x16)(0.f);                 // a wavefront joins 32 columns
    if (wave < C / 32) {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          x[i] += sums[((w * (C / 32) + wave) * 32 + i) * 64 + lane];
          y[i] += sums[((w * (C / 32) + wave) * 32 + 16 + i) * 64 + lane];
        }
        x[i] *= a.scale * back;
        y[i] *= back;
        test = fmaf(x[i], 0.f, fmaf(y[i], 0.f, test));
      }
    }
    uint64_t odd = odd_keys(test);
    if (lane == 0) odds[wave] = odd;
    __syncthreads();
    odd = odds[0] | odds[1] | odds[2] | odds[3];
    if (wave < C / 32 && there && !(odd >> (lane & 31) & 1)) {
      store_block<T>(x, wave, dk_to + (int64_t)key * a.dk.token, half, a.dim);
      store_block<T>(y, wave, dv_to + (int64_t)key * a.dv.token, half, a.dim);
    }
    if (wave == 0) plain_keys(odd);
    return;
  }
#pragma unroll
  for (int m = 0; m < C / 32; ++m) {
    dk[m] *= a.scale * back;
    if constexpr (kScaled<T>) dv[m] *= back;
#pragma unroll
    for (int i = 0; i < 16; ++i) test = fmaf(dk[m][i], 0.f, fmaf(dv[m][i], 0.f, test));
  }
  const uint64_t odd = odd_keys(test);
  if (parts == 1) {
    if (there && !(odd >> (lane & 31) & 1)) {
      store_columns<T, C>(dk, dk_to + (int64_t)key * a.dk.token, half, a.dim);
      store_columns<T, C>(dv, dv_to + (int64_t)key * a.dv.token, half, a.dim);
    }
  } else if (!(odd >> (lane & 31) & 1)) {
    float* to = part_to + (int64_t)(lane & 31) * a.dim;
#pragma unroll
    for (int m = 0; m < C / 32; ++m)
#pragma unroll
      for (int i = 0; i < 16; i += 4) {
        const int d = 32 * m + 2 * i + 4 * half;
        if (d < a.dim) {
          *(f32x4*)(to + d) = f32x4{dk[m][i], dk[m][i + 1], dk[m][i + 2], dk[m][i + 3]};
          *(f32x4*)(to + kKeyTile * a.dim + d) = f32x4{dv[m][i], dv[m][i + 1], dv[m][i + 2], dv[m][i + 3]};
        }
      }
  }
  plain_keys(odd);
}

// Adds up the parts of tiles that were cut, eight columns of a key per thread, dk and dv.  Bound by the parts: 47 MB in 9 us (2 x 1531 tokens, 12/2 heads of 96).
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

// How many groups of 32 queries a workgroup of the dq kernel has, by `blocks`, the workgroups of four groups that there would be: as in the forward kernel, with other
// limits (all three kernels' us, of one / two / four groups):
//   heads of 64:   64 blocks, window 256, 28.1 / 29.1 / 33.0, no window, 2048 keys, 49.4 / 54.8 / 65.4;  128 blocks 37.9 / 36.0 / 40.1, 60.0 / 62.7 / 72.3
//                  256 blocks 53.4 / 46.0 / 46.8, 85.6 / 77.7 / 83.2;  384 blocks 63.5 / 53.4 / 52.5, 109 / 92.5 / 98.2;  512 blocks 73.5 / 61.5 / 57.5, 124 / 104 / 102
//   heads of 128:  64 blocks 37.4 / 38.4 / 44.6, 71.3 / 77.4 / 103;  128 blocks 61.1 / 51.3 / 57.4, 91.7 / 89.2 / 113;  256 blocks 92.6 / 63.7 / 64.0,
//                  154 / 119 / 137;  384 blocks 118 / 76.8 / 76.6, 211 / 150 / 160;  512 blocks 160 / 105 / 98, 254 / 177 / 175
// Up to 64 keys two, which are all queries of such a sequence as a rule, for what the kernel says of rows of few keys.  Up to 64 queries never fill four (300
// keys, 2048 blocks of 20 queries, 75.0 / 71.1 / 76.2, 156 / 120 / 134).
int query_groups(int64_t blocks, const AttentionArgs& a) {
  if (a.k_len <= 64) return 2;
  if (blocks <= 64) return 1;
  return a.q_len <= 64 || blocks <= (a.window == 0 && a.k_len >= 1000 ? 384 : 256) ? 2 : 4;
}

template <typename T, int C>
int backward(const AttentionArgs& a, void* stream) {
  const int64_t q_heads = (int64_t)a.q_heads * a.batch, kv_heads = (int64_t)a.kv_heads * a.batch;
  auto tiles_of = [](int64_t n, int64_t of) { return (n + of - 1) / of; };
  const int groups = query_groups(tiles_of(a.q_len, kQueryTile) * q_heads, a);
  const int64_t q_tiles = tiles_of(a.q_len, 32 * groups), k_tiles = tiles_of(a.k_len, a.few_keys ? 32 : kKeyTile);
  const int64_t q_blocks = q_tiles * q_heads, k_blocks = (a.sink_tiles * (int64_t)a.sink_parts + (k_tiles - a.sink_tiles) * a.tile_parts) * kv_heads;
  const int first_cut = a.sink_parts > 1 ? 0 : a.sink_tiles, cut = (int)((a.tile_parts > 1 ? k_tiles : a.sink_tiles) - first_cut);
  const int64_t join_blocks = cut > 0 ? (cut * kv_heads * kKeyTile * (a.dim / 8) * 2 + 255) / 256 : 0;
  if (q_blocks > 0x7fffffff || k_blocks > 0x7fffffff || join_blocks > 0x7fffffff) return (int)hipErrorInvalidConfiguration;
  hipStream_t s = (hipStream_t)stream;
  const dim3 q_grid((unsigned)q_blocks), k_grid((unsigned)k_blocks), block(256);
  if (q_blocks && groups == 4) attention_dq_kernel<T, C, 4><<<q_grid, block, 0, s>>>(a, (int)q_tiles);
  else if (q_blocks && groups == 2) attention_dq_kernel<T, C, 2><<<q_grid, block, 0, s>>>(a, (int)q_tiles);
  else if (q_blocks) attention_dq_kernel<T, C, 1><<<q_grid, block, 0, s>>>(a, (int)q_tiles);
  if (k_blocks && !a.few_keys) attention_dkv_kernel<T, C, true><<<k_grid, block, 0, s>>>(a, (int)k_tiles);
  else if (k_blocks) attention_dkv_kernel<T, C, false><<<k_grid, block, 0, s>>>(a, (int)k_tiles);
  if (join_blocks) attention_join_kernel<T><<<dim3((unsigned)join_blocks), block, 0, s>>>(a, (int)k_tiles, cut, first_cut);
  return (int)hipGetLastError();
}

template <typename T>
int by_columns(const AttentionArgs& a, void* stream) {
  return a.dim <= 64 ? backward<T, 64>(a, stream) : a.dim <= 96 ? backward<T, 96>(a, stream) : backward<T, 128>(a, stream);
}

}  // namespace

int launch_attention_backward(const AttentionArgs& a, int32_t dtype, void* stream) {
  if (dtype == ARROW_BF16) return by_columns<__bf16>(a, stream);
  return by_columns<_Float16>(a, stream);
}

}  // namespace arrow
