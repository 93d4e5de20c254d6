// Page tables and slot maps from lengths (include/arrow_pages.h).
//
// What a step has to touch is little: the entries of columns that change, a page of the list for each, and the slots.  What is needed of a row of the table is two
// runs of columns, the first ones and those of the window, so that what changes are up to three runs, found from the two lengths without looking at the table.
// Small steps, such as that of a token for each sequence, are one launch of one workgroup, bound by the loads and barriers that follow each other (64 sequences, 3.6 us there and 4.5 back, the
// launch with them); of more new tokens a second launch takes the pages and writes the slots; steps of large tables count, give back and take in a launch each (256 prompts of up to
// 16,000 tokens: 2.8, 3.7 and 12.0 us, of which the slots' 20 MB are 4; and 2.8 and 3.7 for their end).  The rules are with their numbers in pages_internal.h.
#include <hip/hip_runtime.h>

#include <cstdint>

#include "pages_internal.h"

namespace arrow {
namespace {

// Columns that a sequence of `length` tokens needs: 0 .. lead - 1 and rest .. end - 1.
struct Needed {
  int lead, rest, end;
  __device__ __forceinline__ Needed(const PagesArgs& p, int length) {
    length = max(0, min(length, p.a.columns << p.page_log));
    end = (length + p.a.page - 1) >> p.page_log;
    rest = p.a.window ? max(0, length - p.a.window) >> p.page_log : 0;
    lead = min((int)(((int64_t)p.a.sinks + p.a.page - 1) >> p.page_log), rest);
  }
};

// Columns that are in `a` and not in `b`, from `least` on, as three runs in rising order.  (A first run that is shorter than the other's ends where its window begins, so
// that what the other has beyond is either in that window or behind its end.)
struct Runs {
  int from[3], count[3];
  __device__ __forceinline__ Runs(const Needed& a, const Needed& b, int least) {
    set(0, b.lead < a.lead ? b.end : a.lead, a.lead, least);
    set(1, max(a.rest, b.lead), min(a.end, b.rest), least);
    set(2, max(a.rest, b.end), a.end, least);
  }
  __device__ __forceinline__ void set(int i, int begin, int end, int least) {
    from[i] = max(begin, least);
    count[i] = max(0, end - from[i]);
  }
  __device__ __forceinline__ int total() const { return count[0] + count[1] + count[2]; }
  __device__ __forceinline__ int column(int i) const {
    if (i < count[0]) return from[0] + i;
    i -= count[0];
    return i < count[1] ? from[1] + i : from[2] + i - count[1];
  }
  // which of the columns c is, -1: none
  __device__ __forceinline__ int place(int c) const {
    int at = 0;
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      if (c >= from[i] && c < from[i] + count[i]) return at + c - from[i];
      at += count[i];
    }
    return -1;
  }
};

// New tokens of a sequence: rows first .. first + count - 1 of the slots, positions from `position` on.
struct Fresh {
  int64_t first;
  int count, position;
  __device__ __forceinline__ Fresh(const PagesArgs& p, int b, int now) : Fresh(p, b, now, p.a.offsets ? p.a.offsets + b : nullptr) {}
  // (offsets: this sequence's and the next one's)
  __device__ __forceinline__ Fresh(const PagesArgs& p, int b, int now, const int* offsets) {
    if (p.a.offsets) {
      first = max((int64_t)0, min((int64_t)offsets[0], p.rows));
      count = (int)(max(first, min((int64_t)offsets[1], p.rows)) - first);
    } else {
      first = (int64_t)b * p.a.tokens;
      count = p.a.tokens;
    }
    position = (int)max((int64_t)-0x80000000ll, (int64_t)now - count);
  }
  __device__ __forceinline__ int column(const PagesArgs& p) const { return (max(0, min(position, 1 << 30)) + p.a.page - 1) >> p.page_log; }   // the first that begins with one
};

// (lengths of before and now)
__device__ __forceinline__ Runs given_of(const PagesArgs& p, int before, int now) { return Runs(Needed(p, before), Needed(p, now), 0); }
__device__ __forceinline__ Runs taken_of(const PagesArgs& p, const Fresh& f, int before, int now) { return Runs(Needed(p, now), Needed(p, before), f.column(p)); }
__device__ __forceinline__ Runs taken_of(const PagesArgs& p, int b, int before, int now) { return taken_of(p, Fresh(p, b, now), before, now); }
__device__ __forceinline__ int list_size(const PagesArgs& p) { return max(0, min(p.list[0], (int)p.a.pages)); }

// Columns first .. end - 1 of those that change.
struct Part {
  int first, end;
  __device__ __forceinline__ Part(const Runs& r) : first(0), end(r.total()) {}
  __device__ __forceinline__ Part(const PagesArgs& p, const Runs& r, int chunk) : first(chunk * p.chunk), end(min(r.total(), first + p.chunk)) {}
  __device__ __forceinline__ int count() const { return max(0, end - first); }
};

// f(column, page or -1) for some columns of runs, 64 at a time, four of those on their way together; a wavefront.
template <typename F>
__device__ __forceinline__ void each_entry(const PagesArgs& p, int b, const Runs& r, const Part& part, F&& f) {
  const int lane = threadIdx.x & 63, n = part.end;
  const int32_t* row = p.table + (int64_t)b * p.a.columns;
  for (int i0 = part.first; i0 < n; i0 += 256) {
    int page[4], column[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int i = i0 + 64 * j + lane;
      column[j] = i < n ? r.column(i) : -1;
      page[j] = i < n ? row[column[j]] : -1;
      if (page[j] < 0 || page[j] >= p.a.pages) page[j] = -1;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (i0 + 64 * j < n) f(column[j], page[j]);
  }
}

__device__ __forceinline__ int count_given(const PagesArgs& p, int b, const Runs& r, const Part& part) {
  int n = 0;
  each_entry(p, b, r, part, [&](int, int page) { n += __popcll(__ballot(page >= 0)); });
  return n;
}

// Pages of a sequence to the list: `first` have gone there before them, the last of all to place `size`.
__device__ __forceinline__ void give(const PagesArgs& p, int b, const Runs& r, const Part& part, int first, int size, int all) {
  const uint64_t below = ((uint64_t)1 << (threadIdx.x & 63)) - 1;
  each_entry(p, b, r, part, [&](int column, int page) {
    const uint64_t there = __ballot(page >= 0);
    const int at = size + all - 1 - first - __popcll(there & below);
    first += __popcll(there);
    if (page >= 0 && at < p.a.pages) p.list[1 + at] = page;
    if (column >= 0) p.table[(int64_t)b * p.a.columns + column] = -1;
  });
}

// The i-th page that is taken from a list of `size`.
__device__ __forceinline__ int page_taken(const PagesArgs& p, int i, int size) { return i < size ? p.list[size - i] : -1; }

__device__ __forceinline__ void take(const PagesArgs& p, int b, const Runs& r, const Part& part, int first, int size) {
  for (int i = part.first + (threadIdx.x & 63); i < part.end; i += 64) p.table[(int64_t)b * p.a.columns + r.column(i)] = page_taken(p, first + i - part.first, size);
}

// A slot from its position and its column's page.
__device__ __forceinline__ int64_t slot_of(const PagesArgs& p, int position, int page) {
  return position < 0 || page < 0 || page >= p.a.pages ? -1 : ((int64_t)page << p.page_log) + (position & (p.a.page - 1));
}

// The slot of row `row`, one of sequence b's: from the list, or from the table where its column is no new one.
__device__ __forceinline__ int64_t slot_at(const PagesArgs& p, const Fresh& f, int b, int64_t row, int before, int now, int first, int size) {
  if (row < f.first || row >= f.first + f.count) return -1;
  const int position = f.position + (int)(row - f.first), column = position >> p.page_log;
  if (position < 0 || column >= p.a.columns) return -1;
  const int at = taken_of(p, f, before, now).place(column);
  return slot_of(p, position, at >= 0 ? page_taken(p, first + at, size) : p.table[(int64_t)b * p.a.columns + column]);
}

// Sums of x over the threads before this one, and over all of them: two numbers in one.
template <int kThreads>
__device__ __forceinline__ uint64_t before_me(uint64_t x, uint64_t* all, uint64_t* room) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint64_t sum = x;
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) {
    const uint64_t y = __shfl_up((unsigned long long)sum, m, 64);
    if (lane >= m) sum += y;
  }
  __syncthreads();
  if (lane == 63) room[wave] = sum;
  __syncthreads();
  uint64_t first = 0, total = 0;
#pragma unroll
  for (int w = 0; w < kThreads / 64; ++w) {
    const uint64_t y = room[w];
    if (w < wave) first += y;
    total += y;
  }
  *all = total;
  return first + sum - x;
}

// The last of n rising numbers that is at most x, of those from `low` on (which is).
__device__ __forceinline__ int last_upto(const int* numbers, int low, int n, int x) {
  int high = n - 1;
  while (low < high) {
    const int mid = (low + high + 1) >> 1;
    if (numbers[mid] <= x) low = mid;
    else high = mid - 1;
  }
  return low;
}

// A step in one workgroup.  Columns that change are numbered through all sequences, so that the threads share them evenly; a page that is given back is read
// once and put where it goes if all the others are there, too, which is nearly always so.  Where some are not, they are counted first.
template <int kThreads>
__global__ __launch_bounds__(kThreads) void pages_step_kernel(PagesArgs p) {
  constexpr int kAhead = 4, kWaves = kThreads / 64;
  __shared__ int before[kPagesBatch], now[kPagesBatch], given[kPagesBatch], taken[kPagesBatch], offsets[kPagesBatch + 1];
  __shared__ uint64_t room[kWaves];
  const int tid = threadIdx.x, batch = p.a.batch, columns = p.a.columns;
  const int size0 = list_size(p);
  // (one sequence a thread, or several one after the other)
  const int each = (batch + kThreads - 1) / kThreads, b0 = min(batch, tid * each), b1 = min(batch, b0 + each);
  if (p.a.offsets)
    for (int b = tid; b <= batch; b += kThreads) offsets[b] = p.a.offsets[b];
  uint64_t mine = 0, all;
  for (int b = b0; b < b1; ++b) {
    const int held = p.held[b], length = p.lengths[b];
    before[b] = held;
    now[b] = length;
    given[b] = given_of(p, held, length).total();
    taken[b] = taken_of(p, b, held, length).total();
    mine += (uint64_t)given[b] << 32 | (uint32_t)taken[b];
  }
  uint64_t first = before_me<kThreads>(mine, &all, room);
  for (int b = b0; b < b1; ++b) {
    const uint64_t x = (uint64_t)given[b] << 32 | (uint32_t)taken[b];
    given[b] = (int)(first >> 32);
    taken[b] = (int)first;
    first += x;
  }
  __syncthreads();
  int gives = (int)(all >> 32);
  const int takes = (int)all, columns_given = gives;
  // f(i, its sequence, its column) for the i-th columns that give their pages back, i0 + 64 j; most often they are all of one sequence
  const auto some_given = [&](int i0, auto&& f) {
    const int low = last_upto(given, 0, batch, i0), high = last_upto(given, low, batch, min(i0 + 64 * kAhead, columns_given) - 1), lane = tid & 63;
    if (low == high) {
      const int b = __builtin_amdgcn_readfirstlane(low);
      const Runs r = given_of(p, before[b], now[b]);
#pragma unroll
      for (int j = 0; j < kAhead; ++j) f(j, i0 + 64 * j + lane, b, r.column(i0 + 64 * j + lane - given[b]));
    } else {
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        const int i = min(i0 + 64 * j + lane, columns_given - 1), b = last_upto(given, low, high + 1, i);
        f(j, i0 + 64 * j + lane, b, given_of(p, before[b], now[b]).column(i - given[b]));
      }
    }
  };
  const int wave0 = __builtin_amdgcn_readfirstlane(tid >> 6) * (64 * kAhead);
  const bool many = columns_given > kAhead * kThreads;
  if (gives) {
    bool hole = false;
    if (many) {
      for (int i0 = wave0; i0 < columns_given; i0 += kAhead * kThreads) {
        int page[kAhead];
        some_given(i0, [&](int j, int i, int b, int column) { page[j] = i < columns_given ? p.table[(int64_t)b * columns + column] : 0; });
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
          const int i = i0 + 64 * j + (tid & 63), at = size0 + gives - 1 - i;
          if (i >= columns_given) continue;
          hole = hole || page[j] < 0 || page[j] >= p.a.pages;
          if (at < p.a.pages) p.list[1 + at] = page[j];
        }
      }
    }
    for (int i0 = many ? columns_given : tid; i0 < columns_given; i0 += kAhead * kThreads) {
      int page[kAhead];
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        const int i = i0 + j * kThreads;
        if (i >= columns_given) continue;
        const int b = last_upto(given, 0, batch, i);
        page[j] = p.table[(int64_t)b * columns + given_of(p, before[b], now[b]).column(i - given[b])];
      }
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        const int i = i0 + j * kThreads, at = size0 + gives - 1 - i;
        if (i >= columns_given) continue;
        hole = hole || page[j] < 0 || page[j] >= p.a.pages;
        if (at < p.a.pages) p.list[1 + at] = page[j];            // (behind the list's end until it is said to be longer)
      }
    }
    if (__syncthreads_or(hole)) {
      const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
      for (int b = wave; b < batch; b += kWaves) {
        const Runs r = given_of(p, before[b], now[b]);
        const int n = count_given(p, b, r, r);
        if ((tid & 63) == 0) given[b] = n;
      }
      __syncthreads();
      mine = 0;
      for (int b = b0; b < b1; ++b) mine += given[b];
      first = before_me<kThreads>(mine, &all, room);
      for (int b = b0; b < b1; ++b) {
        const int n = given[b];
        given[b] = (int)first;
        first += n;
      }
      gives = (int)all;
      __syncthreads();
      for (int b = wave; b < batch; b += kWaves) {
        const Runs r = given_of(p, before[b], now[b]);
        give(p, b, r, r, given[b], size0, gives);
      }
    } else {
      if (many)
        for (int i0 = wave0; i0 < columns_given; i0 += kAhead * kThreads)
          some_given(i0, [&](int, int i, int b, int column) { if (i < columns_given) p.table[(int64_t)b * columns + column] = -1; });
      for (int i = many ? columns_given : tid; i < columns_given; i += kThreads) {
        const int b = last_upto(given, 0, batch, i);
        p.table[(int64_t)b * columns + given_of(p, before[b], now[b]).column(i - given[b])] = -1;
      }
    }
    __syncthreads();
  }
  const int size = min(size0 + gives, (int)p.a.pages);
  if (p.two) {
    // (what is taken, and the slots, are another kernel's)
    for (int b = b0; b < b1; ++b) {
      p.before[b] = before[b];
      p.taken[b] = taken[b];
      p.held[b] = now[b];
    }
    if (tid == 0) {
      p.sizes[0] = size0;
      p.sizes[1] = gives;
      p.sizes[2] = takes;
      p.list[0] = max(0, size - takes);
    }
    return;
  }
  for (int i = tid; i < takes; i += kThreads) {
    const int b = last_upto(taken, 0, batch, i);
    p.table[(int64_t)b * columns + taken_of(p, b, before[b], now[b]).column(i - taken[b])] = page_taken(p, i, size);
  }
  // (a slot's page is looked for in the list where it is a new one: nothing here waits for the table)
  for (int row = tid; row < p.rows; row += kThreads) {
    int b;
    if (p.a.offsets) b = batch == 0 || offsets[0] > row ? -1 : last_upto(offsets, 0, batch, row);
    else b = row / p.a.tokens;
    p.slots[row] = b < 0 ? -1 : slot_at(p, Fresh(p, b, now[b], offsets + b), b, row, before[b], now[b], taken[b], size);
  }
  for (int b = b0; b < b1; ++b) p.held[b] = now[b];
  if (tid == 0) p.list[0] = max(0, size - takes);
}

// ---- larger steps ----
// A unit of the work is up to p.chunk of the columns that change of a sequence, for a wavefront.
struct Unit {
  int at, b, chunk;
  bool in;
  __device__ __forceinline__ explicit Unit(const PagesArgs& p) {
    at = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    b = p.chunks == 1 ? at : (uint32_t)at / (uint32_t)p.chunks;
    chunk = at - b * p.chunks;
    in = b < p.a.batch;
  }
};

__global__ __launch_bounds__(256) void pages_count_kernel(PagesArgs p) {
  if (blockIdx.x == 0 && threadIdx.x == 0) p.sizes[0] = list_size(p);
  const Unit u(p);
  if (!u.in) return;
  const int before = p.held[u.b], now = p.lengths[u.b];
  const Runs given = given_of(p, before, now);
  const int n = count_given(p, u.b, given, Part(p, given, u.chunk));
  if (threadIdx.x & 63) return;
  if (u.chunk == 0) p.before[u.b] = before;
  p.given[u.at] = n;
  p.taken[u.at] = Part(p, taken_of(p, u.b, before, now), u.chunk).count();
}

// What is given back and taken in all, and before each unit.  Of up to kPagesBatch units every workgroup that gives back adds them up for itself, into LDS, and the first one
// writes them down for what follows; of more one has done so, in place.
struct Sums {
  const int *given, *taken;
  int size0, gives, takes;
  __device__ __forceinline__ int size(const PagesArgs& p) const { return min(size0 + gives, (int)p.a.pages); }
};

template <int kThreads>
__device__ __forceinline__ Sums add_up(const PagesArgs& p, int* given, int* taken, uint64_t* room) {
  const int units = p.a.batch * p.chunks, each = (units + kThreads - 1) / kThreads, b0 = min(units, (int)threadIdx.x * each), b1 = min(units, b0 + each);
  uint64_t mine = 0, all;
  for (int b = b0; b < b1; ++b) mine += (uint64_t)p.given[b] << 32 | (uint32_t)p.taken[b];
  uint64_t first = before_me<kThreads>(mine, &all, room);
  for (int b = b0; b < b1; ++b) {
    const uint64_t x = (uint64_t)p.given[b] << 32 | (uint32_t)p.taken[b];
    given[b] = (int)(first >> 32);
    taken[b] = (int)first;
    first += x;
  }
  __syncthreads();
  return {given, taken, p.sizes[0], (int)(all >> 32), (int)all};
}

constexpr int kSumThreads = 1024;

__global__ __launch_bounds__(kSumThreads) void pages_sum_kernel(PagesArgs p) {
  __shared__ uint64_t room[kSumThreads / 64];
  const Sums s = add_up<kSumThreads>(p, p.given, p.taken, room);
  if (threadIdx.x) return;
  p.sizes[1] = s.gives;
  p.sizes[2] = s.takes;
}

struct Room {
  int given[kPagesBatch], taken[kPagesBatch];
  uint64_t sums[4];
};

// The state after the step, by the last kernel's first workgroups.
__device__ __forceinline__ void finish(const PagesArgs& p, const Sums& s, int block, int blocks) {
  for (int b = block * 256 + threadIdx.x; b < p.a.batch; b += blocks * 256) p.held[b] = p.lengths[b];
  if (block == 0 && threadIdx.x == 0) p.list[0] = max(0, s.size(p) - s.takes);
}

__global__ __launch_bounds__(256) void pages_give_kernel(PagesArgs p, bool last) {
  __shared__ Room room;
  const int units = p.a.batch * p.chunks;
  const bool few = units <= kPagesBatch;
  const Sums s = few ? add_up<256>(p, room.given, room.taken, room.sums) : Sums{p.given, p.taken, p.sizes[0], p.sizes[1], p.sizes[2]};
  if (few && !last && blockIdx.x == 0) {
    for (int i = threadIdx.x; i < units; i += 256) p.first[i] = s.taken[i];
    if (threadIdx.x == 0) { p.sizes[1] = s.gives; p.sizes[2] = s.takes; }
  }
  const Unit u(p);
  if (u.in) {
    const Runs r = given_of(p, p.before[u.b], p.lengths[u.b]);
    give(p, u.b, r, Part(p, r, u.chunk), s.given[u.at], s.size0, s.gives);
  }
  if (last) finish(p, s, blockIdx.x, gridDim.x);
}

// Takes and slots: neither waits for the other, as a slot's page is found in the list where it is a new one.  What bounds it is a wavefront's chain of loads (offsets, the
// sequence's lengths, the list or table: 6.6 us of the 12.0 above); eight rows of a lane share it.
constexpr int kRowsEach = 8;

__global__ __launch_bounds__(256) void pages_take_kernel(PagesArgs p, int take_blocks) {
  __shared__ int counts[2][4];
  const int tid = threadIdx.x, batch = p.a.batch;
  const int* first = p.a.batch * p.chunks <= kPagesBatch && !p.two ? p.first : p.taken;
  const int64_t row0 = (int64_t)((int)blockIdx.x - take_blocks) * (256 * kRowsEach), last = min(row0 + 256 * kRowsEach, p.rows) - 1;
  int low = 0, high = 0;                     // the sequences that the first and the last row may be of: those of this wavefront's that begin up to there
  if (p.a.offsets)
    for (int b0 = 0; b0 < batch; b0 += 256) {
      const int begin = b0 + tid < batch ? p.a.offsets[b0 + tid] : 0x7fffffff;
      low += __popcll(__ballot(begin <= row0));
      high += __popcll(__ballot(begin <= last));
    }
  const Sums s{nullptr, nullptr, p.sizes[0], p.sizes[1], p.sizes[2]};
  const int size = s.size(p);
  if ((int)blockIdx.x < take_blocks) {
    const Unit u(p);
    if (u.in) {
      const Runs r = taken_of(p, u.b, p.before[u.b], p.lengths[u.b]);
      take(p, u.b, r, Part(p, r, u.chunk), first[u.at], size);
    }
    if (!p.two) finish(p, s, blockIdx.x, take_blocks);
    return;
  }
  if (p.a.offsets) {
    if ((tid & 63) == 0) { counts[0][tid >> 6] = low; counts[1][tid >> 6] = high; }
    __syncthreads();
    low = __builtin_amdgcn_readfirstlane(counts[0][0] + counts[0][1] + counts[0][2] + counts[0][3]) - 1;
    high = __builtin_amdgcn_readfirstlane(counts[1][0] + counts[1][1] + counts[1][2] + counts[1][3]) - 1;
  } else {
    low = (int)(row0 / p.a.tokens);
    high = (int)(last / p.a.tokens);
  }
  if (high - low <= 4) {
    // few sequences: one after the other, with what they have in common worked out once
    int64_t done = row0;                     // (rows up to there are written)
    for (int b = max(low, 0); b <= high; ++b) {
      const int now = p.lengths[b], before = p.before[b], taken = first[b * p.chunks];
      const Fresh f(p, b, now);
      const Runs runs = taken_of(p, f, before, now);
      const int64_t begin = max(done, f.first), end = min(last + 1, f.first + f.count);
      for (int64_t row = done + tid; row < min(begin, last + 1); row += 256) p.slots[row] = -1;
      int page[kRowsEach], position[kRowsEach];
#pragma unroll
      for (int j = 0; j < kRowsEach; ++j) {
        const int64_t row = begin + j * 256 + tid;
        page[j] = position[j] = -1;
        if (row >= end) continue;
        position[j] = f.position + (int)(row - f.first);
        const int column = position[j] >> p.page_log;
        if (position[j] < 0 || column >= p.a.columns) continue;
        const int at = runs.place(column);
        const int32_t* where = at < 0 ? p.table + (int64_t)b * p.a.columns + column : taken + at < size ? p.list + size - taken - at : nullptr;
        if (where) page[j] = *where;
      }
#pragma unroll
      for (int j = 0; j < kRowsEach; ++j) {
        const int64_t row = begin + j * 256 + tid;
        if (row < end) p.slots[row] = slot_of(p, position[j], page[j]);
      }
      done = max(done, end);
    }
    for (int64_t row = done + tid; row <= last; row += 256) p.slots[row] = -1;
    return;
  }
  for (int64_t row = row0 + tid; row <= last; row += 256) {
    int b;
    if (!p.a.offsets) b = (int)(row / p.a.tokens);
    else b = low < 0 && p.a.offsets[0] > row ? -1 : last_upto(p.a.offsets, max(0, low), high + 1, (int)row);
    p.slots[row] = b < 0 ? -1 : slot_at(p, Fresh(p, b, p.lengths[b]), b, row, p.before[b], p.lengths[b], first[b * p.chunks], size);
  }
}

}  // namespace

int launch_pages_step(const PagesArgs& p, void* stream) {
  hipStream_t s = (hipStream_t)stream;
  if (p.one) {
    // Fewer threads wait less for each other: four new tokens and back, us a pass with 256 and 1024 threads, 4 sequences 8.2, 8.5, 32 8.1, 9.0, 256 10.7, 9.7.  Where all pages of a table
    // go they take longer: prompts and back, the way back with 256 and 1024, 4 sequences of 4000 pages 21 18, of 16,000 40 26, 64 of 4000 33 23, of 16,000 58 30.  So steps without new
    // tokens have 1024.
    if (p.rows > 0 && p.a.batch <= 128 && p.rows <= 2048 && (int64_t)p.a.batch * p.a.columns <= 16384) pages_step_kernel<256><<<dim3(1), dim3(256), 0, s>>>(p);
    else pages_step_kernel<1024><<<dim3(1), dim3(1024), 0, s>>>(p);
    return (int)hipGetLastError();
  }
  const unsigned fours = (unsigned)(((int64_t)p.a.batch * p.chunks + 3) / 4), rows = (unsigned)((p.rows + 256 * kRowsEach - 1) / (256 * kRowsEach));
  if (p.two) {
    pages_step_kernel<1024><<<dim3(1), dim3(1024), 0, s>>>(p);
    pages_take_kernel<<<dim3(fours + rows), dim3(256), 0, s>>>(p, (int)fours);
    return (int)hipGetLastError();
  }
  if (fours) pages_count_kernel<<<dim3(fours), dim3(256), 0, s>>>(p);
  if ((int64_t)p.a.batch * p.chunks > kPagesBatch) pages_sum_kernel<<<dim3(1), dim3(kSumThreads), 0, s>>>(p);
  if (fours) pages_give_kernel<<<dim3(fours), dim3(256), 0, s>>>(p, rows == 0);
  // (without new tokens nothing is taken)
  if (rows) pages_take_kernel<<<dim3(fours + rows), dim3(256), 0, s>>>(p, (int)fours);
  return (int)hipGetLastError();
}

}  // namespace arrow
