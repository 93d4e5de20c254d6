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
// in the dk, dv kernel) are rounded as multiples of a power of two, by the size of d_o where that is below 1: of a row in the dq kernel, of all rows that a key tile's
// queries are among in the other one, which takes those from the dq kernel's notes, one for 32 queries.
template <typename T> constexpr bool kScaled = std::is_same<T, _Float16>::value;
__device__ __forceinline__ float finite_size(float x) { return fabsf(x) < __builtin_inff() ? fabsf(x) : 0.f; }
// The power of two that brings x into [1, 2), 1 for 0.
__device__ __forceinline__ float unit_of(float x) { return x > 0.f ? __uint_as_float((254u << 23) - (__float_as_uint(x) & 0x7f800000u)) : 1.f; }
// Values of a row or key (this lane's, and those of the lane 32 further on), made smaller by a power of two where they do not fit float16; by which.
__device__ __forceinline__ float fit(f32x16& x) {
  float most = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) most = fmaxf(most, finite_size(x[i]));
  most = max_halves(most);
  const float less = most > 0x1p15f ? 0x1p14f * unit_of(most) : 1.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) x[i] *= less;
  return less;
}
// A kernel's arguments, read from memory from here on.
__device__ __forceinline__ const AttentionArgs& arguments() {
  auto at = (const __attribute__((address_space(4))) AttentionArgs*)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(at));
  return *(const AttentionArgs*)at;
}
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
// 128, window of 2048, 445 us = 1090 TFLOP/s with the product P K, matrix units busy 55 % of the cycles.  Heads of more than 64 leave no registers for the queries, which
// are read from LDS again and again, and tiles of 32 keys; of 64, 4 x 2048 tokens, window of 512: 52 us, 1.5 wavefronts to a SIMD.
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
  constexpr int kSumBytes = 2 * 4 * 64 * 4, kRestBytes = kParts == 1 ? 0 : kSumBytes + 16, kFlagBytes = kParts == 1 ? 16 : 0;
  static_assert(kParts == 1 || kQueriesAt >= 4 * C * 32 * 4, "room for the sums");
  constexpr int kEnd = kQueriesAt + (kQueriesBytes > kRestBytes ? kQueriesBytes : kRestBytes);
  __shared__ __align__(1024) unsigned char smem[kEnd + kFlagBytes];
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
    larger = fmaxf(unit_of(most), 1.f);                          // (never less: what is small beside the largest may be all that counts)
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
  // a wavefront joins every kParts-th block of 32 columns
  constexpr int kBlocks = C / 32, kJoined = (kBlocks + kParts - 1) / kParts;
  f32x16 r[kJoined];
  float row_rest;

  // Twice where a result is not finite though what the row sees may be, as in the forward kernel: the second time elements of keys that are not finite are taken out of the
  // product, and make NaN of their column for those who see them.  In float16 results are not finite where dS passes 65,504 either: it is rounded as many times smaller there as
  // it takes.
  auto pass = [&](auto is_careful) -> bool {
    constexpr bool kCareful = decltype(is_careful)::value;
    constexpr int kNow = kCareful ? 32 : kMine;               // keys at a time
    if constexpr (kQueriesInLds)                              // (waited for with the first tiles)
      Loader<D, kRows, 4>(wave, lane, a.q.token, a.dim).load(q + 2 * (int64_t)first * a.q.token, sq.count - first, room + kQueriesAt, wave);
    f32x16 acc[C / 32], pk[C / 32];                           // dS K and P K
#pragma unroll
    for (int m = 0; m < C / 32; ++m) { acc[m] = (f32x16)(0.f); pk[m] = (f32x16)(0.f); }
    float rest = 0.f, kept = 0.f;                             // sums of dS of this lane's keys, before and after they are rounded
    const int t0 = kShare ? 0 : wave;
    if (t0 < seen.total) load(t0, 0);
    if constexpr (!kShare && kQueriesInLds) wait_for_tiles(); // (all wavefronts' queries)
    for (int t = t0, now = 0; t < seen.total; t += kTurns, now ^= 1) {
      if constexpr (kShare) wait_for_tiles();
      else wait_for_own_tiles();
      if (t + kTurns < seen.total) load(t + kTurns, now ^ 1);
#pragma unroll 1
      for (int in = 0; in < kMine; in += kNow) {
        const int skip = (kMine < kStep ? split * kMine : 0) + in;
        const uint32_t kt = lds_address(base) + 2 * now * kBytes + skip * Tl::kRowBytes, vt = kt + kBytes;
        const uint32_t qt = kQueriesInLds ? here(lds_address(room) + kQueriesAt + group * 32 * Tl::kRowBytes + my.rows) : 0;
        const int k0 = seen.at(t) * kStep + skip;
        if (k0 > high || (a.window && k0 >= a.sinks && k0 + kNow - 1 <= low - a.window)) continue;
        const bool whole = k0 + kNow - 1 <= low && (!a.window || k0 > low + 31 - a.window || k0 + kNow <= a.sinks);
        const int ago = p - k0 - 4 * half, sinks = min(a.sinks - k0 - 4 * half, ago + 1);
        const uint32_t window = a.window ? (uint32_t)a.window : 0x80000000u;
        auto sees = [&](int j, int ago, int sinks) { return bool(((uint32_t)(ago - j) < window) | (j < sinks)); };   // (without branches)
#pragma unroll
        for (int n = 0; n < kNow / 32; ++n) {
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
              const bool visible = sees(n * 32 + 8 * (i / 4) + i % 4, ago, sinks);
              s[i] = visible ? s[i] : 0.f;
              e[i] = visible ? e[i] : 0.f;
            }
          }
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            e[i] *= s[i];
            rest += e[i];
          }
          const float less = kCareful && kScaled<T> ? fit(e) : 1.f;
          x8<T> pf[2], ds[2];
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            pf[u] = round8<T>(s[8 * u], s[8 * u + 1], s[8 * u + 2], s[8 * u + 3], s[8 * u + 4], s[8 * u + 5], s[8 * u + 6], s[8 * u + 7]);
            ds[u] = round8<T>(e[8 * u], e[8 * u + 1], e[8 * u + 2], e[8 * u + 3], e[8 * u + 4], e[8 * u + 5], e[8 * u + 6], e[8 * u + 7]);
            if constexpr (kParts > 1) kept = kCareful && kScaled<T> ? fmaf(add8(ds[u], 0.f), 1.f / less, kept) : add8(ds[u], kept);
          }
          if constexpr (kCareful) {
            auto seen_of = [&](int u, int i) { return sees(16 * u + 8 * (i / 4) + i % 4, here(ago), here(sinks)); };
#pragma unroll
            for (int m = 0; m < C / 32; ++m) add_finite<T, D, 2>(pk[m], kt + my.columns, m, pf);
#pragma unroll
            for (int m = 0; m < C / 32; ++m) {
              if constexpr (kScaled<T>) {
                f32x16 x = (f32x16)(0.f);
                add_finite<T, D, 2>(x, kt + my.columns, m, ds);
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[m][i] = fmaf(x[i], 1.f / less, acc[m][i]);
              } else {
                add_finite<T, D, 2>(acc[m], kt + my.columns, m, ds);
              }
              add_others<T, D, 2, false>(acc[m], kt + my.columns, m, seen_of);
            }
            continue;
          }
#pragma unroll
          for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int m = 0; m < C / 32; ++m) {
              const x8<T> kf = read_columns<T, D>(kt + my.columns, m, (n * 32 + 16 * u) * Tl::kRowBytes);
              acc[m] = mma32(kf, ds[u], acc[m]);
              pk[m] = mma32(kf, pf[u], pk[m]);
            }
          reads_ahead<4, 4 * (C / 32), 1>();
        }
      }
    }

    rest = add_halves(rest);
    kept = kParts == 1 ? rest : add_halves(kept);
    if constexpr (kParts > 1) {
      float* rests = (float*)(smem + kQueriesAt);
      wait_for_tiles();                                       // the tiles and queries are done with, or there and not needed
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
    row_rest = rest;
    const float by = a.scale / larger;
#pragma unroll
    for (int m = 0; m < C / 32; ++m)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[m][i] = by * fmaf(-kept, pk[m][i], acc[m][i]);
    if constexpr (kParts == 1) {
#pragma unroll
      for (int m = 0; m < kBlocks; ++m) r[m] = acc[m];
    } else {
      float* sums = (float*)smem;
#pragma unroll
      for (int m = 0; m < kBlocks; ++m)
#pragma unroll
        for (int i = 0; i < 16; ++i) sums[((wave * kBlocks + m) * 16 + i) * 64 + lane] = acc[m][i];
      __syncthreads();
#pragma unroll
      for (int n = 0; n < kJoined; ++n) {
        const int m = split + n * kParts;
        r[n] = (f32x16)(0.f);
        if (m >= kBlocks) continue;
#pragma unroll
        for (int w = 0; w < kParts; ++w)
#pragma unroll
          for (int i = 0; i < 16; ++i) r[n][i] += sums[(((group + kGroups * w) * kBlocks + m) * 16 + i) * 64 + lane];
      }
    }
    float test = 0.f;                                         // NaN where a result is not finite
#pragma unroll
    for (int n = 0; n < kJoined; ++n)
#pragma unroll
      for (int i = 0; i < 16; ++i) test = fmaf(r[n][i], 0.f, test);
    return there && off == off && delta == delta && test != test;
  };
  auto store = [&] {
    if (there && half == 0 && split == 0) {
      a.off[stat] = off;
      a.delta[stat] = -(delta + row_rest) / larger;
    }
    T* dq = (T*)rows_of(a.dq, ragged, b, sq.first, head) + (int64_t)row * a.dq.token;
#pragma unroll
    for (int n = 0; n < kJoined; ++n) {
      const int m = split + n * kParts;
      if (m < kBlocks && there) store_block<T>(r[n], m, dq, half, a.dim);
    }
  };
  const bool again = pass(std::false_type{});
  store();
  if (__builtin_expect(any_wave(again, room + (kParts == 1 ? kEnd : kQueriesAt + kSumBytes)), 0)) {
    pass(std::true_type{});
    store();
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
// What bounds it: as the dq kernel; of 256 registers 128 are sums (heads of 128), so the keys are read from LDS as the queries are there.  8192 tokens, as above: 490 us = 980
// TFLOP/s, matrix units busy 45 %, LDS 34 % of the cycles; 4 x 2048: 55 us, 1.8 wavefronts to a SIMD.  The queries come from behind the L2 (1.7 GB); another order of them, in which
// workgroups of a die read the same ones, took as long.
//
// Twice where a result is not finite, as in the dq kernel: the second time (kCareful) elements of queries and of gradients that are not finite are taken out of the products and
// count for the keys that their queries see.  All gradients, 4096 tokens, 8 heads of 64, no window: 135 us, 496 with an infinity in one gradient of o; 8192 tokens, as above, in
// float16: 1010 and 4050.
template <int C, bool kShare>
struct KeyRoom {                                                 // in LDS
  static constexpr int D = columns_of_tile(C);
  static constexpr bool kKeysInLds = D > 64;
  static constexpr int kQ = kKeysInLds || !kShare ? 32 : 64, kBytes = kQ * Tile<D>::kRowBytes;   // queries of a step
  static constexpr int kTurns = kShare ? 1 : 4, kKeys = kShare ? kKeyTile : 32;
  // q and do, two tiles each, of all wavefronts or of each one, or their sums to be joined; the keys; what the dq kernel noted of each query, two steps'
  static constexpr int kKeysAt = 4 * kTurns * kBytes, kStatsAt = kKeysAt + (kKeysInLds ? kKeys * Tile<D>::kRowBytes : 0), kStatsBytes = 2 * 2 * 4 * kQ;
  static constexpr int kFlagsAt = kStatsAt + kTurns * kStatsBytes, kAll = kFlagsAt + 16;
  static_assert(kShare || kKeysAt >= 4 * 2 * D * 32 * 4, "room for the sums");
};

// Whether a result of this lane's is not finite.
template <typename T, int C, bool kShare, bool kCareful>
__device__ __forceinline__ bool dkv_pass(const AttentionArgs& a, int tiles, unsigned char* smem, int thread) {
  using Room = KeyRoom<C, kShare>;
  constexpr int D = Room::D, kQ = Room::kQ, kBytes = Room::kBytes, kTurns = Room::kTurns, kKeys = Room::kKeys, kKeysAt = Room::kKeysAt;
  constexpr bool kKeysInLds = Room::kKeysInLds;
  using Tl = Tile<D>;
  const int lane = thread & 63, wave = __builtin_amdgcn_readfirstlane(thread >> 6), half = lane >> 5;
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
  if (first >= sk.count) return false;
  const int shift = sk.count - sq.count;
  const int mine = first + (kShare ? wave * 32 : 0);
  const int key = mine + (lane & 31);
  const bool there = key < sk.count;
  const char* k = rows_of(a.k, ragged, b, sk.first, kv);
  const char* v = rows_of(a.v, ragged, b, sk.first, kv);
  if constexpr (kKeysInLds)                                      // (waited for with the first step's tiles)
    Loader<D, kKeys, 4>(wave, lane, a.k.token, a.dim).load(k + 2 * (int64_t)first * a.k.token, sk.count - first, (lds_byte*)smem + kKeysAt, wave);
  // this lane's key and value, columns 16 s + 8 half and on: in registers, or (kCareful) read again and again
  const char *k_at = k + 2 * ((int64_t)key * a.k.token + 8 * half), *v_at = v + 2 * ((int64_t)key * a.v.token + 8 * half);
  auto piece = [&](const char* at, int s) {
    const x8<T> z = {};
    return there && 16 * s + 8 * half < a.dim ? *(const x8<T>*)(at + 32 * s) : z;
  };
  x8<T> kf[kKeysInLds || kCareful ? 1 : C / 16], vf[kCareful ? 1 : C / 16];
  if constexpr (!kCareful)
#pragma unroll
    for (int s = 0; s < C / 16; ++s) {
      if constexpr (!kKeysInLds) kf[s] = piece(k_at, s);
      vf[s] = piece(v_at, s);
    }
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
    const AttentionArgs& z = arguments();                        // (what only this needs is in no register later)
    const float* notes = z.most + groups_at(z, ragged, b, kv * z.group, sq.first) + from;
    const int64_t step = groups_at(z, ragged, 0, 1, 0) - groups_at(z, ragged, 0, 0, 0);
    for (int h = 0; h < z.group; ++h, notes += step)
      for (int i = lane; i < groups; i += 64) most = fmaxf(most, notes[i]);
    for (int m = 32; m; m >>= 1) most = fmaxf(most, __shfl_xor(most, m, 64));
    up = __builtin_amdgcn_readfirstlane(min(max(127 - (int)(__float_as_uint(most) >> 23), 0), most > 0.f ? 15 : 0));
  }
  const float c = a.scale * kLog2e;

  const int sharer = kShare ? wave : 0;
  const Loader<D, kQ, 4 / kTurns> lq(sharer, lane, a.q.token, a.dim), ld(sharer, lane, a.d_o.token, a.dim);
  lds_byte *room = (lds_byte*)smem, *base = room + (kShare ? 0 : wave * 4 * kBytes);
  lds_byte* stats = room + Room::kStatsAt + (kShare ? 0 : wave * Room::kStatsBytes);
  const TileReads<D> my(lane);
  const int64_t q_step = 2 * kQ * a.q.token, d_step = 2 * kQ * a.d_o.token;
  constexpr int kNow = kCareful ? 32 : kQ;                       // queries at a time
  f32x16 dk[C / 32], dv[C / 32];
#pragma unroll
  for (int m = 0; m < C / 32; ++m) { dk[m] = (f32x16)(0.f); dv[m] = (f32x16)(0.f); }
  // the step that is loaded next: a head's queries from q_next on, and where they lie
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
  const int mine0 = step0 + (kShare ? 0 : wave);              // this wavefront's first step
  int q_loaded = 0;
  if (mine0 < step1) {
    head += mine0 / q_steps;
    begin(q_begin + mine0 % q_steps);
    q_loaded = q_next;
    load(0);
  }
  if constexpr (!kShare) wait_for_tiles();                    // (all wavefronts' keys)
  for (int t = mine0, now = 0; t < step1; t += kTurns, now ^= 1) {
    if constexpr (kShare) wait_for_tiles();
    else wait_for_own_tiles();
    const int q_now = q_loaded;
    if (t + kTurns < step1) { q_loaded = q_next; load(now ^ 1); }
    const uint32_t kt = lds_address(room) + kKeysAt + sharer * 32 * Tl::kRowBytes + my.rows;
    auto key_of = [&](int i) {
      if constexpr (kKeysInLds) return read_rows<T>(kCareful ? here(kt) : kt, i, 0);
      else if constexpr (kCareful) return piece(here(k_at), i);
      else return kf[i];
    };
    auto value_of = [&](int i) {
      if constexpr (kCareful) return piece(here(v_at), i);
      else return vf[i];
    };
    const int low = mine, high = min(low + 31, sk.count - 1); // this wavefront's keys
#pragma unroll 1
    for (int in = 0; in < kQ; in += kNow) {
      const uint32_t qt = lds_address(base) + (2 * now) * kBytes + in * Tl::kRowBytes;
      const uint32_t stat = lds_address(stats) + now * (2 * 4 * kQ) + 16 * half + 4 * in;
#pragma unroll
      for (int n = 0; n < kNow / 32; ++n) {
        const int first_q = q_now + in + n * 32, p0 = first_q + shift;   // the first of 32 queries, and its position
        if (first_q >= sq.count || p0 + 31 < low || (a.window && low >= a.sinks && p0 - a.window >= high)) continue;
        f32x16 s, e;                                          // the products begin with what is taken off them
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
          const f32x4 x = lds_read4(stat + 4 * (n * 32 + 2 * i)), y = lds_read4(stat + 4 * (kQ + n * 32 + 2 * i));
#pragma unroll
          for (int j = 0; j < 4; ++j) { s[i + j] = x[j]; e[i + j] = y[j]; }
        }
#pragma unroll
        for (int i = 0; i < C / 16; ++i) {
          s = mma32(read_rows<T>(qt + my.rows, i, n * 32 * Tl::kRowBytes), key_of(i), s);
          if constexpr (kCareful) one_by_one(s);
        }
#pragma unroll
        for (int i = 0; i < C / 16; ++i) {
          e = mma32(read_rows<T>(qt + my.rows, i, kBytes + n * 32 * Tl::kRowBytes), value_of(i), e);
          if constexpr (kCareful) one_by_one(e);
        }
        if constexpr (!kCareful) reads_ahead<kKeysInLds ? 16 : 12, C / 16, kKeysInLds ? 2 : 1, C / 16, 1>();   // (eight of those ahead: what the products begin with)
        const float lift = kScaled<T> ? here(up) : 0.f;          // (in a scalar register otherwise)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = __builtin_amdgcn_exp2f(kScaled<T> ? fmaf(s[i], c, lift) : s[i] * c);
        const bool whole = p0 >= low + 31 && first_q + 32 <= sq.count && (!a.window || p0 + 31 - a.window < low || low + 32 <= a.sinks);
        const int ahead = p0 + 4 * half - key;                // how far the first of this lane's queries is ahead of its key
        const int left = sq.count - (first_q + 4 * half);
        const uint32_t window = a.window && key >= a.sinks ? (uint32_t)a.window : 0x80000000u;
        auto seen = [&](int j, int ahead) { return bool(((uint32_t)(ahead + j) < window) & (j < left)); };
        if (!whole) {
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const bool visible = seen(8 * (i / 4) + i % 4, ahead);
            s[i] = visible ? s[i] : 0.f;
            e[i] = visible ? e[i] : 0.f;
          }
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) e[i] *= s[i];
        const float less = kCareful && kScaled<T> ? fit(e) : 1.f;
        x8<T> pf[2], ds[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          pf[u] = round8<T>(s[8 * u], s[8 * u + 1], s[8 * u + 2], s[8 * u + 3], s[8 * u + 4], s[8 * u + 5], s[8 * u + 6], s[8 * u + 7]);
          ds[u] = round8<T>(e[8 * u], e[8 * u + 1], e[8 * u + 2], e[8 * u + 3], e[8 * u + 4], e[8 * u + 5], e[8 * u + 6], e[8 * u + 7]);
        }
        if constexpr (kCareful) {
          auto seen_of = [&](int u, int i) { return seen(16 * u + 8 * (i / 4) + i % 4, here(ahead)); };
          const uint32_t q_tile = qt + my.columns, d_tile = q_tile + kBytes;
#pragma unroll
          for (int m = 0; m < C / 32; ++m) {
            add_finite<T, D, 2>(dv[m], d_tile, m, pf);
            add_others<T, D, 2, true>(dv[m], d_tile, m, seen_of);
          }
#pragma unroll
          for (int m = 0; m < C / 32; ++m) {
            if constexpr (kScaled<T>) {
              f32x16 x = (f32x16)(0.f);
              add_finite<T, D, 2>(x, q_tile, m, ds);
#pragma unroll
              for (int i = 0; i < 16; ++i) dk[m][i] = fmaf(x[i], 1.f / less, dk[m][i]);
            } else {
              add_finite<T, D, 2>(dk[m], q_tile, m, ds);
            }
            add_others<T, D, 2, false>(dk[m], q_tile, m, seen_of);
          }
          continue;
        }
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int m = 0; m < C / 32; ++m) {
            dv[m] = mma32(read_columns<T, D>(qt + my.columns, m, kBytes + (n * 32 + 16 * u) * Tl::kRowBytes), pf[u], dv[m]);
            dk[m] = mma32(read_columns<T, D>(qt + my.columns, m, (n * 32 + 16 * u) * Tl::kRowBytes), ds[u], dk[m]);
          }
        reads_ahead<kKeysInLds ? 8 : 4, 4 * (C / 32), 2>();
      }
    }
  }

  // what this wavefront has in the end: all columns, or 32 of them of what the four have together
  constexpr int kBlocks = kShare ? C / 32 : 1;
  f32x16 dk_sum[kBlocks], dv_sum[kBlocks];
  if constexpr (kShare) {
#pragma unroll
    for (int m = 0; m < C / 32; ++m) { dk_sum[m] = dk[m]; dv_sum[m] = dv[m]; }
  } else {
    float* sums = (float*)smem;
    __syncthreads();                                          // the tiles are done with
#pragma unroll
    for (int m = 0; m < C / 32; ++m)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        sums[((wave * (C / 32) + m) * 32 + i) * 64 + lane] = dk[m][i];
        sums[((wave * (C / 32) + m) * 32 + 16 + i) * 64 + lane] = dv[m][i];
      }
    __syncthreads();
    f32x16 x = (f32x16)(0.f), y = (f32x16)(0.f);              // a wavefront joins 32 columns
    if (wave < C / 32) {
#pragma unroll
      for (int i = 0; i < 16; ++i)
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          x[i] += sums[((w * (C / 32) + wave) * 32 + i) * 64 + lane];
          y[i] += sums[((w * (C / 32) + wave) * 32 + 16 + i) * 64 + lane];
        }
    }
    dk_sum[0] = x;
    dv_sum[0] = y;
  }
  const float back = kScaled<T> ? __builtin_amdgcn_exp2f(-up) : 1.f;
  float test = 0.f;                                           // NaN where a result is not finite
#pragma unroll
  for (int m = 0; m < kBlocks; ++m) {
    dk_sum[m] *= a.scale * back;
    if constexpr (kScaled<T>) dv_sum[m] *= back;
#pragma unroll
    for (int i = 0; i < 16; ++i) test = fmaf(dk_sum[m][i], 0.f, fmaf(dv_sum[m][i], 0.f, test));
  }
  T* dk_to = (T*)rows_of(a.dk, ragged, b, sk.first, kv) + (int64_t)key * a.dk.token;
  T* dv_to = (T*)rows_of(a.dv, ragged, b, sk.first, kv) + (int64_t)key * a.dv.token;
  if constexpr (!kShare) {
    if (wave < C / 32 && there) {
      store_block<T>(dk_sum[0], wave, dk_to, half, a.dim);
      store_block<T>(dv_sum[0], wave, dv_to, half, a.dim);
    }
  } else if (parts == 1) {
    if (there) {
      store_columns<T, C>(dk_sum, dk_to, half, a.dim);
      store_columns<T, C>(dv_sum, dv_to, half, a.dim);
    }
  } else {
    // parts in the workspace: [sequence, head][item][dk, dv][key][dim]; items of tiles in one part have no place there
    float* to = a.parts + part_place(a, tiles, ((int64_t)b * a.kv_heads + kv), tile, part) * 2 * kKeyTile * a.dim + (int64_t)(key - first) * a.dim;
#pragma unroll
    for (int m = 0; m < C / 32; ++m)
#pragma unroll
      for (int i = 0; i < 16; i += 4) {
        const int d = 32 * m + 2 * i + 4 * half;
        if (d < a.dim) {
          *(f32x4*)(to + d) = f32x4{dk_sum[m][i], dk_sum[m][i + 1], dk_sum[m][i + 2], dk_sum[m][i + 3]};
          *(f32x4*)(to + kKeyTile * a.dim + d) = f32x4{dv_sum[m][i], dv_sum[m][i + 1], dv_sum[m][i + 2], dv_sum[m][i + 3]};
        }
      }
  }
  return there && test != test;
}

template <typename T, int C, bool kShare>
__global__ __launch_bounds__(256, kShare ? (C <= 64 ? 3 : 2) : 1) void attention_dkv_kernel(AttentionArgs a, int tiles) {
  using Room = KeyRoom<C, kShare>;
  __shared__ __align__(1024) unsigned char smem[Room::kAll];
  const bool again = dkv_pass<T, C, kShare, false>(a, tiles, smem, threadIdx.x);
  if (__builtin_expect(any_wave(again, (lds_byte*)smem + Room::kFlagsAt), 0)) {
    dkv_pass<T, C, kShare, true>(arguments(), tiles, smem, here((int)threadIdx.x));   // (nothing is kept in registers for this)
  }
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
