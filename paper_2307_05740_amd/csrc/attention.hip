// Attention under an arrow-shaped mask, forward (include/arrow_attention.h).
//
// A wavefront holds 32 queries and goes through tiles of 64 keys.  It computes the scores transposed, S^T = K Q^T, so that a
// lane has one query's scores in its registers: the running maximum and sum of the softmax need one exchange, between lane halves, and
// the probabilities are at once the B operand of O^T += V^T P^T.
//
// Four wavefronts share the tiles and have 128 queries together.  Where that gives too few workgroups to fill the chip, they have 64 queries, half of every tile
// each, or the same 32 queries and every fourth tile, of 32 keys and its own, and join their results in LDS.
//
// What bounds it: with heads of 128, matrix instructions and the vector instructions between them (one exponential, one addition, one maximum, one
// multiply-add and half a conversion per score), at the clock that the card's power leaves: 16,384 tokens, 16/2 heads, window of 4096, 490 us = 985 TFLOP/s,
// where a large matrix product reaches 1312.  With heads of 64 how few wavefronts have work: 4 x 2048, 16 heads, window of 512, 30 us = 500 TFLOP/s, 2.3 wavefronts to a SIMD, whose
// chains of products, maximum, exponentials and products cover each other so far that vector instructions issue in 46 % of the cycles and matrix units run in 20 %.  Tiles
// of 64 keys, because two of keys and two of values (64 KiB) leave room for two workgroups on a compute unit, and each wavefront then has two
// independent chains of products; 32 queries to a wavefront, because scores, sums and queries of 64 would not fit 256 registers.
#include <algorithm>

#include "attention_common.h"

namespace arrow {
namespace {

// How many groups of 32 queries a workgroup has, by `blocks`, the workgroups of four groups that there would be.  One up to 64 of those, 128 for small heads, and
// twice as many where a row sees 2000 keys or more; two up to 256 of them, 384 without a window, whose workgroups are half as long on average, and 512 for
// small heads (us, of one / two / four groups):
//   heads of 64:   128 blocks, window 256, 8.9 / 9.1 / 12.1, no window, 2048 keys, 19.0 / 25.0 / 32.5;  256 blocks 15.9 / 11.0 / 12.6, 27.1 / 26.1 / 33.1
//                  512 blocks 27.2 / 16.8 / 16.7, 46.2 / 30.2 / 34.6;  768 blocks 40.3 / 23.2 / 22.5, 70.5 / 44.3 / 41.2
//   heads of 128:  64 blocks 9.6 / 11.4 / 14.6, 21.2 / 31.1 / 40.1;  128 blocks 17.4 / 11.8 / 15.3, 28.9 / 33.1 / 41.2;  256 blocks 32.6 / 16.2 / 16.4,
//                  52.6 / 36.1 / 42.3;  384 blocks 49.3 / 25.4 / 23.2, 76.6 / 42.1 / 46.0;  512 blocks 62.9 / 31.0 / 24.8, 100 / 53.0 / 49.9
// A tile of keys has nothing to be shared out: 64 keys, 1024 blocks of 64 queries, 19.3 / 9.0 / 8.7, 42.8 / 16.8 / 14.5.  Up to 64 queries never fill four
// groups, and of up to 32 there are as many workgroups of one group as of four (heads of 64 and of 128, of 20 queries):
//   300 keys, 256 blocks 7.7 / 7.9 / 8.8, 9.2 / 10.0 / 10.9, 2048 blocks 32.5 / 24.8 / 27.6, 70.4 / 55.9 / 56.4
//   2000 keys, 256 blocks 17.9 / 25.1 / 33.5, 23.0 / 33.6 / 42.4
int query_groups(int64_t blocks, int64_t heads, const AttentionArgs& a) {
  if (a.k_len <= 64) return 4;
  const int64_t seen = a.window ? std::min<int64_t>((int64_t)a.window + a.sinks, a.k_len) : a.k_len;
  const bool twice = seen >= 2000 && (a.dim <= 64 || a.q_len > 64);
  const int64_t ones = a.q_len <= 64 ? ((int64_t)a.q_len + 31) / 32 * heads : 4 * blocks;
  if (ones <= (a.dim <= 64 ? 512 : 256) * (twice ? 2 : 1)) return 1;
  if (a.q_len <= 64) return 2;
  return blocks <= (a.dim <= 64 ? 512 : a.window == 0 && seen >= 1000 ? 384 : 256) ? 2 : 4;
}

// kGroups: how many groups of 32 queries the four wavefronts have.  (Four workgroups to a compute unit for heads of 64, 128 registers: so many the first pass takes.)
template <typename T, int C, int kGroups>
__global__ __launch_bounds__(256, kGroups > 1 ? (C <= 64 ? 4 : 2) : 1) void attention_forward_kernel(AttentionArgs a, int tiles) {
  constexpr int D = columns_of_tile(C);
  using Tl = Tile<D>;
  constexpr bool kShare = kGroups > 1;                        // tiles
  constexpr int kStep = kShare ? 64 : 32, kTurns = kShare ? 1 : 4;   // keys of a tile; a wavefront has every kTurns-th tile
  constexpr int kMine = kGroups == 4 ? 64 : 32;               // and so many of its keys
  constexpr int kParts = 4 / kGroups;                         // wavefronts with the same queries
  constexpr int kBytes = kStep * Tl::kRowBytes;
  // keys and values, two tiles each, of all wavefronts or of each one; joined afterwards: the sums of each, its maxima and totals
  constexpr int kRoom = 4 * kTurns * kBytes;
  static_assert(kParts == 1 || kRoom >= 4 * C * 32 * 4, "room for the sums");
  __shared__ __align__(1024) unsigned char smem[kRoom + (kParts == 1 ? 0 : 4 * 2 * 64 * 4) + 16];
  const int lane = threadIdx.x & 63, wave = wave_id(), half = lane >> 5;
  // Workgroups next to each other go to different dies: an item of every sequence and key head in turn, so that a die has the same keys again
  // and again (8192 queries, 32/8 heads of 128: 300 -> 270 us); of one, the longest rows of a triangle first.
  const int units = a.kv_heads * a.batch, unit = blockIdx.x % units;
  int item = blockIdx.x / units, split = 0;
  if constexpr (kGroups == 1) { split = item % a.splits; item /= a.splits; }
  const int g = item % a.group, tile = tiles - 1 - item / a.group;
  const int kv = unit % a.kv_heads, b = unit / a.kv_heads, head = kv * a.group + g;
  const bool ragged = a.q_offsets != nullptr;
  const Span sq = span_of(a.q_offsets, b, a.q_tokens, a.q_len), sk = span_of(a.k_offsets, b, a.k_tokens, a.k_len);
  constexpr int kRows = 32 * kGroups;
  const int first = tile * kRows;
  if (first >= sq.count) return;
  const int group = wave % kGroups, part = wave / kGroups;
  const int mine = first + group * 32;                        // the first of this wavefront's queries
  const int shift = sk.count - sq.count;                      // position of query 0
  const int row = mine + (lane & 31);                         // this lane's query
  const bool there = row < sq.count;
  const int p = row + shift;
  const char* q = rows_of(a.q, ragged, b, sq.first, head);
  const char* k = rows_of(a.k, ragged, b, sk.first, kv);
  const char* v = rows_of(a.v, ragged, b, sk.first, kv);

  x8<T> qf[C / 16];
#pragma unroll
  for (int s = 0; s < C / 16; ++s) {
    const int d = 16 * s + 8 * half;
    x8<T> z = {};
    qf[s] = there && d < a.dim ? *(const x8<T>*)(q + 2 * ((int64_t)row * a.q.token + d)) : z;
  }

  const int last = min(first + kRows, sq.count) - 1 + shift;
  const SeenTiles seen = seen_tiles<kStep>(max(first + shift, 0), last, a.window, a.sinks);
  int begin = 0, end = seen.total;                            // tiles of this workgroup: whole rounds of its wavefronts
  if constexpr (kGroups == 1) {
    const int rounds = (seen.total + 3) / 4;
    begin = 4 * (int)((int64_t)rounds * split / a.splits);
    end = min(seen.total, 4 * (int)((int64_t)rounds * (split + 1) / a.splits));
  }
  // of this wavefront's queries
  const int low = mine + shift, high = min(low + 31, sk.count - 1);

  const float c = a.scale * kLog2e;
  const int sharer = kShare ? wave : 0;
  const Loader<D, kStep, 4 / kTurns> lk(sharer, lane, a.k.token, a.dim), lv(sharer, lane, a.v.token, a.dim);
  lds_byte* base = (lds_byte*)smem + (kShare ? 0 : wave * 4 * kBytes);
  const TileReads<D> my(lane);
  auto load = [&](int t, int to) {
    const int k0 = seen.at(t) * kStep;
    lk.load(k + 2 * (int64_t)k0 * a.k.token, sk.count - k0, base + 2 * to * kBytes, sharer);
    lv.load(v + 2 * (int64_t)k0 * a.v.token, sk.count - k0, base + (2 * to + 1) * kBytes, sharer);
  };
  // a wavefront joins every kParts-th block of 32 columns; joined_here: the row's keys are all this workgroup's
  constexpr int kBlocks = C / 32, kJoined = (kBlocks + kParts - 1) / kParts;
  const bool joined_here = kGroups > 1 || a.splits == 1;
  f32x16 r[kJoined];
  float row_top, row_total, row_lse;

  // Matrix instructions multiply what a query does not see by a probability of 0, and that is no zero where a value there is infinite or NaN.  Where a result is not finite though
  // its row's sum is (so the pass says), the workgroup goes through its tiles again, with care: such values count for those who see them alone.  16,384 tokens, 16/2 heads of
  // 128, window of 4096: 490 us with finite values, 1780 with an infinity that a quarter of the rows see, 3280 where all see one.
  auto pass = [&](auto is_careful) -> bool {
    constexpr bool kCareful = decltype(is_careful)::value;
    constexpr int kNow = kCareful ? 32 : kMine;                 // keys at a time
    f32x16 acc[C / 32];
#pragma unroll
    for (int m = 0; m < C / 32; ++m) acc[m] = (f32x16)(0.f);
    float top = minus_infinity(), total = 0.f;                  // of c times the scores; of this lane's keys
    const int t0 = begin + (kShare ? 0 : wave);
    if (t0 < end) load(t0, 0);
    for (int t = t0, now = 0; t < end; t += kTurns, now ^= 1) {
      if constexpr (kShare) wait_for_tiles();
      else wait_for_own_tiles();
      if (t + kTurns < end) load(t + kTurns, now ^ 1);
#pragma unroll 1
      for (int in = 0; in < kMine; in += kNow) {
        const int skip = (kMine < kStep ? part * kMine : 0) + in; // (keys of the tile that are another wavefront's)
        const uint32_t kt = lds_address(base) + 2 * now * kBytes + skip * Tl::kRowBytes, vt = kt + kBytes;
        const int k0 = seen.at(t) * kStep + skip;
        // no query of this wavefront sees the tile
        if (k0 > high || (a.window && k0 >= a.sinks && k0 + kNow - 1 <= low - a.window)) continue;

        f32x16 s[kNow / 32];
#pragma unroll
        for (int n = 0; n < kNow / 32; ++n) s[n] = (f32x16)(0.f);
#pragma unroll
        for (int i = 0; i < C / 16; ++i)                          // (in turn: a product waits for the last one on the same sums)
#pragma unroll
          for (int n = 0; n < kNow / 32; ++n) s[n] = mma32(read_rows<T>(kt + my.rows, i, n * 32 * Tl::kRowBytes), qf[i], s[n]);
        reads_ahead<6, (kNow / 32) * (C / 16), 1>();
        // every query sees every key: nothing to mask
        const bool whole = k0 + kNow - 1 <= low && (!a.window || k0 > low + 31 - a.window || k0 + kNow <= a.sinks);
        const int ago = p - k0 - 4 * half, sinks = min(a.sinks - k0 - 4 * half, ago + 1);
        const uint32_t window = a.window ? (uint32_t)a.window : 0x80000000u;
        auto sees = [&](int j, int ago, int sinks) { return bool(((uint32_t)(ago - j) < window) | (j < sinks)); };   // (without branches)
        if (!whole) {
#pragma unroll
          for (int n = 0; n < kNow / 32; ++n)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const bool visible = sees(n * 32 + 8 * (i / 4) + i % 4, ago, sinks);
              s[n][i] = visible ? s[n][i] : minus_infinity();
            }
        }
        float most = s[0][0];
#pragma unroll
        for (int n = 0; n < kNow / 32; ++n)
#pragma unroll
          for (int i = 0; i < 16; ++i) most = fmaxf(most, s[n][i]);
        most = max_halves(most) * c;
        // The maximum is only raised where a score is more than 2^8 times the terms' scale: until then they stay within what the sums and
        // both types hold, and the sums are left as they are.
        if (__any(most > top + 8.f)) {
          const float now = most > top + 8.f ? most : top;
          const float by = now == top ? 1.f : __builtin_amdgcn_exp2f(top - now);
          top = now;
          total *= by;
#pragma unroll
          for (int m = 0; m < C / 32; ++m) acc[m] *= by;
        }
        const float off = top == minus_infinity() ? 0.f : top;
        x8<T> pf[kNow / 16];
#pragma unroll
        for (int n = 0; n < kNow / 32; ++n) {
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            s[n][i] = __builtin_amdgcn_exp2f(fmaf(s[n][i], c, -off));
            total += s[n][i];
          }
#pragma unroll
          for (int u = 0; u < 2; ++u)
            pf[2 * n + u] = round8<T>(s[n][8 * u], s[n][8 * u + 1], s[n][8 * u + 2], s[n][8 * u + 3], s[n][8 * u + 4], s[n][8 * u + 5],
                                      s[n][8 * u + 6], s[n][8 * u + 7]);
        }
        if constexpr (kCareful) {
#pragma unroll
          for (int m = 0; m < C / 32; ++m) {
            add_finite<T, D, kNow / 16>(acc[m], vt + my.columns, m, pf);
            add_others<T, D, kNow / 16, true>(acc[m], vt + my.columns, m,
                                              [&](int u, int i) { return sees(16 * u + 8 * (i / 4) + i % 4, here(ago), here(sinks)); });
          }
          continue;
        }
#pragma unroll
        for (int u = 0; u < kNow / 16; ++u)
#pragma unroll
          for (int m = 0; m < C / 32; ++m)
            acc[m] = mma32(read_columns<T, D>(vt + my.columns, m, 16 * u * Tl::kRowBytes), pf[u], acc[m]);
        reads_ahead<8, (kNow / 16) * (C / 32), 2>();
      }
    }

    total = add_halves(total);
    if constexpr (kParts == 1) {
      row_top = top;
      row_total = total;
#pragma unroll
      for (int m = 0; m < C / 32; ++m) r[m] = acc[m];
    } else {
      float *sums = (float*)smem, *tops = (float*)(smem + kRoom), *totals = tops + 4 * 64;
      __syncthreads();                                          // the tiles are done with
#pragma unroll
      for (int m = 0; m < C / 32; ++m)
#pragma unroll
        for (int i = 0; i < 16; ++i) sums[((wave * (C / 32) + m) * 16 + i) * 64 + lane] = acc[m][i];
      tops[wave * 64 + lane] = top;
      totals[wave * 64 + lane] = total;
      __syncthreads();
      float all = minus_infinity(), share[kParts];
#pragma unroll
      for (int w = 0; w < kParts; ++w) all = fmaxf(all, tops[(group + kGroups * w) * 64 + lane]);
      const float off = all == minus_infinity() ? 0.f : all;
      row_top = all;
      row_total = 0.f;
#pragma unroll
      for (int w = 0; w < kParts; ++w) {
        share[w] = __builtin_amdgcn_exp2f(tops[(group + kGroups * w) * 64 + lane] - off);
        row_total = fmaf(share[w], totals[(group + kGroups * w) * 64 + lane], row_total);
      }
#pragma unroll
      for (int n = 0; n < kJoined; ++n) {
        const int m = part + n * kParts;
        r[n] = (f32x16)(0.f);
        if (m >= kBlocks) continue;
#pragma unroll
        for (int w = 0; w < kParts; ++w)
#pragma unroll
          for (int i = 0; i < 16; ++i) r[n][i] = fmaf(share[w], sums[(((group + kGroups * w) * kBlocks + m) * 16 + i) * 64 + lane], r[n][i]);
      }
    }
    // 1 / total, 0 for a row that sees nothing; parts of rows are left as they are
    const float by = !joined_here ? 1.f : row_total > 0.f || row_total != row_total ? 1.f / row_total : 0.f;
    row_lse = row_total == 0.f ? minus_infinity() : (row_top + __log2f(row_total)) * kLn2;
    float test = 0.f;                                           // NaN where a result is not finite
#pragma unroll
    for (int n = 0; n < kJoined; ++n)
#pragma unroll
      for (int i = 0; i < 16; ++i) { r[n][i] *= by; test = fmaf(r[n][i], 0.f, test); }
    return there && row_lse < -minus_infinity() && test != test;
  };
  auto store = [&] {
    if (!joined_here) {
      const int64_t rows = (int64_t)a.batch * a.q_heads * a.q_len, place = (((int64_t)b * a.q_heads + head) * a.q_len + row) * a.splits + split;
      if (there && half == 0 && part == 0) {
        float* to = a.parts + rows * a.splits * a.dim + 2 * place;
        to[0] = row_top;
        to[1] = row_total;
      }
#pragma unroll
      for (int n = 0; n < kJoined; ++n)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
          const int m = part + n * kParts, d = 32 * m + 2 * i + 4 * half;
          if (m < kBlocks && there && d < a.dim) *(f32x4*)(a.parts + place * a.dim + d) = f32x4{r[n][i], r[n][i + 1], r[n][i + 2], r[n][i + 3]};
        }
      return;
    }
    const int64_t stat = ragged ? head * a.q_tokens + sq.first + row : ((int64_t)b * a.q_heads + head) * a.q_len + row;
    if (a.lse && there && half == 0 && part == 0) a.lse[stat] = row_lse;
    T* o = (T*)rows_of(a.o, ragged, b, sq.first, head) + (int64_t)row * a.o.token;
#pragma unroll
    for (int n = 0; n < kJoined; ++n) {
      const int m = part + n * kParts;
      // (all lanes take part in the exchange; whether a row is stored is the same in both halves)
      if (m < kBlocks && there) store_block<T>(r[n], m, o, half, a.dim);
    }
  };
  const bool again = pass(std::false_type{});
  store();
  if (__builtin_expect(any_wave(again, (lds_byte*)smem + sizeof smem - 16), 0)) {
    pass(std::true_type{});
    store();
  }
}

// The parts of one row joined, by a wavefront, two columns per lane.
template <typename T>
__global__ __launch_bounds__(64) void attention_forward_join_kernel(AttentionArgs a) {
  const int64_t id = blockIdx.x, unit = id / a.q_len, rows = (int64_t)a.batch * a.q_heads * a.q_len;
  const int row = (int)(id % a.q_len), head = (int)(unit % a.q_heads), b = (int)(unit / a.q_heads), lane = threadIdx.x, d = 2 * lane;
  const bool ragged = a.q_offsets != nullptr;
  const Span sq = span_of(a.q_offsets, b, a.q_tokens, a.q_len);
  if (row >= sq.count) return;
  const bool mine = d < a.dim;
  const float *from = a.parts + id * a.splits * a.dim + d, *stats = a.parts + rows * a.splits * a.dim + 2 * id * a.splits;
  const float top = lane < a.splits ? stats[2 * lane] : minus_infinity();
  float all = top;
  for (int m = 32; m; m >>= 1) all = fmaxf(all, __shfl_xor(all, m, 64));
  const float share = __builtin_amdgcn_exp2f(top - (all == minus_infinity() ? 0.f : all));
  float total = lane < a.splits ? share * stats[2 * lane + 1] : 0.f;
  for (int m = 32; m; m >>= 1) total += __shfl_xor(total, m, 64);
  float x0 = 0.f, x1 = 0.f;
  for (int i = 0; i < a.splits; i += 8) {
    float2 x[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = mine && i + j < a.splits ? *(const float2*)(from + (int64_t)(i + j) * a.dim) : float2{0.f, 0.f};
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float by = __shfl(share, i + j, 64);
      x0 = fmaf(by, x[j].x, x0);
      x1 = fmaf(by, x[j].y, x1);
    }
  }
  const float by = total > 0.f || total != total ? 1.f / total : 0.f, lse = total == 0.f ? minus_infinity() : (all + __log2f(total)) * kLn2;
  x0 *= by;
  x1 *= by;
  T* o = (T*)rows_of(a.o, ragged, b, sq.first, head) + (int64_t)row * a.o.token;
  if (a.lse && lane == 0) a.lse[ragged ? head * a.q_tokens + sq.first + row : id] = lse;
  if (mine) {
    o[d] = (T)x0;
    o[d + 1] = (T)x1;
  }
}

template <typename T, int C>
int forward(const AttentionArgs& a, void* stream) {
  const int64_t heads = (int64_t)a.q_heads * a.batch, tiles = ((int64_t)a.q_len + kQueryTile - 1) / kQueryTile;
  const int groups = query_groups(tiles * heads, heads, a);
  const int64_t rows = ((int64_t)a.q_len + 32 * groups - 1) / (32 * groups), blocks = rows * heads * (groups == 1 ? a.splits : 1);
  if (blocks > 0x7fffffff) return (int)hipErrorInvalidConfiguration;
  const dim3 grid((unsigned)blocks), block(256);
  if (groups == 4) attention_forward_kernel<T, C, 4><<<grid, block, 0, (hipStream_t)stream>>>(a, (int)rows);
  else if (groups == 2) attention_forward_kernel<T, C, 2><<<grid, block, 0, (hipStream_t)stream>>>(a, (int)rows);
  else attention_forward_kernel<T, C, 1><<<grid, block, 0, (hipStream_t)stream>>>(a, (int)rows);
  if (groups == 1 && a.splits > 1) attention_forward_join_kernel<T><<<dim3((unsigned)(heads * a.q_len)), dim3(64), 0, (hipStream_t)stream>>>(a);
  return (int)hipGetLastError();
}

template <typename T>
int by_columns(const AttentionArgs& a, void* stream) {
  return a.dim <= 64 ? forward<T, 64>(a, stream) : a.dim <= 96 ? forward<T, 96>(a, stream) : forward<T, 128>(a, stream);
}

}  // namespace

// Keys are cut where workgroups of 32 queries leave the chip empty: as many parts as fill it, of at least four rounds of their wavefronts each (128 keys
// a round, some 0.8 us).  The join takes 4 us and more with more rows, so that there have to be some keys (us, whole -> cut, heads of 64 and of 128):
//   16 queries, 4 heads: 1000 keys 10.8 -> 10.9, 13.2 -> 12.7, 1500 13.8 -> 11.1, 17.9 -> 12.9, 5000 33.9 -> 11.6, 41.4 -> 13.4
//   256 queries, 16 heads: 1500 keys 14.4 -> 15.9, 18.1 -> 19.0, 2000 17.2 -> 16.3, 21.7 -> 21.3, 5000 34.9 -> 22.7, 43.4 -> 31.9
//   1000 queries, 8 heads of 64: 2000 keys 18.0 -> 20.3, 3000 24.5 -> 24.1, 8000 52.1 -> 42.1
int attention_forward_splits(const AttentionArgs& a) {
  const int64_t heads = (int64_t)a.q_heads * a.batch, tiles = ((int64_t)a.q_len + kQueryTile - 1) / kQueryTile;
  if (heads == 0 || a.q_len == 0 || query_groups(tiles * heads, heads, a) != 1) return 1;
  const int64_t seen = a.window ? std::min<int64_t>((int64_t)a.window + a.sinks, a.k_len) : a.k_len;
  const int64_t rows = a.q_len * heads;
  if (seen < (rows <= 2048 ? 1500 : rows <= 4096 ? 2000 : 3000)) return 1;
  const int64_t ones = ((int64_t)a.q_len + 31) / 32 * heads, fill = (a.dim <= 64 ? 512 : 256) / ones;
  return (int)std::max<int64_t>(1, std::min<int64_t>({kMostRowSplits, fill, (seen + 127) / 128 / 4}));
}

int launch_attention_forward(const AttentionArgs& a, int32_t dtype, void* stream) {
  if (dtype == ARROW_BF16) return by_columns<__bf16>(a, stream);
  return by_columns<_Float16>(a, stream);
}

}  // namespace arrow
