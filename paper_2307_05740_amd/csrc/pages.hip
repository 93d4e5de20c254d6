// Page tables and slot maps from lengths (include/arrow_pages.h).
//
// What a step has to touch is little: the entries of columns that change, a page of the list for each, and the slots.  What is needed of a row of the table is two
// runs of columns, the first ones and those of the window, so that what changes are up to three runs, found from the two lengths without looking at the table.
// Small steps, such as that of a token for each sequence, are one launch of one workgroup, bound by the loads and barriers that follow each other; larger ones
// four: count, add up, give back, take.
#include <hip/hip_runtime.h>

#include <cstdint>

#include "pages_internal.h"

namespace arrow {
namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;

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
  __device__ __forceinline__ Fresh(const PagesArgs& p, int b) {
    if (p.a.offsets) {
      first = max((int64_t)0, min((int64_t)p.a.offsets[b], p.rows));
      count = (int)(max(first, min((int64_t)p.a.offsets[b + 1], p.rows)) - first);
    } else {
      first = (int64_t)b * p.a.tokens;
      count = p.a.tokens;
    }
    position = (int)max((int64_t)-0x40000000, (int64_t)p.lengths[b] - count);
  }
  __device__ __forceinline__ int column(const PagesArgs& p) const { return (max(0, min(position, 1 << 30)) + p.a.page - 1) >> p.page_log; }   // the first that begins with one
};

__device__ __forceinline__ Runs given_of(const PagesArgs& p, int b, int before) { return Runs(Needed(p, before), Needed(p, p.lengths[b]), 0); }
__device__ __forceinline__ Runs taken_of(const PagesArgs& p, int b, int before) {
  return Runs(Needed(p, p.lengths[b]), Needed(p, before), Fresh(p, b).column(p));
}
__device__ __forceinline__ int list_size(const PagesArgs& p) { return max(0, min(p.list[0], (int)p.a.pages)); }

// f(column, page or -1) for the columns of runs, 64 at a time, four of those on their way together; a wavefront.
template <typename F>
__device__ __forceinline__ void each_entry(const PagesArgs& p, int b, const Runs& r, F&& f) {
  const int lane = threadIdx.x & 63, n = r.total();
  const int32_t* row = p.table + (int64_t)b * p.a.columns;
  for (int i0 = 0; i0 < n; i0 += 256) {
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

__device__ __forceinline__ int count_given(const PagesArgs& p, int b, const Runs& r) {
  int n = 0;
  each_entry(p, b, r, [&](int, int page) { n += __popcll(__ballot(page >= 0)); });
  return n;
}

// The pages of a sequence to the list: `first` have gone there before it, the last of all to place `size`.
__device__ __forceinline__ void give(const PagesArgs& p, int b, const Runs& r, int first, int size, int all) {
  const uint64_t below = ((uint64_t)1 << (threadIdx.x & 63)) - 1;
  each_entry(p, b, r, [&](int column, int page) {
    const uint64_t there = __ballot(page >= 0);
    const int at = size + all - 1 - first - __popcll(there & below);
    first += __popcll(there);
    if (page >= 0 && at < p.a.pages) p.list[1 + at] = page;
    if (column >= 0) p.table[(int64_t)b * p.a.columns + column] = -1;
  });
}

// The i-th page that is taken from a list of `size`.
__device__ __forceinline__ int page_taken(const PagesArgs& p, int i, int size) { return i < size ? p.list[size - i] : -1; }

__device__ __forceinline__ void take(const PagesArgs& p, int b, const Runs& r, int first, int size) {
  const int n = r.total();
  for (int i = threadIdx.x & 63; i < n; i += 64) p.table[(int64_t)b * p.a.columns + r.column(i)] = page_taken(p, first + i, size);
}

// A slot from its position and its column's page.
__device__ __forceinline__ int64_t slot_of(const PagesArgs& p, int position, int page) {
  return position < 0 || page < 0 || page >= p.a.pages ? -1 : ((int64_t)page << p.page_log) + (position & (p.a.page - 1));
}

// Sums of x over the threads before this one, and over all of them.
__device__ __forceinline__ int before_me(int x, int* all, int* room) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int sum = x;
  for (int m = 1; m < 64; m <<= 1) {
    const int y = __shfl_up(sum, m, 64);
    if (lane >= m) sum += y;
  }
  __syncthreads();
  if (lane == 63) room[wave] = sum;
  __syncthreads();
  int first = 0, total = 0;
  for (int w = 0; w < kWaves; ++w) {
    if (w < wave) first += room[w];
    total += room[w];
  }
  *all = total;
  return first + sum - x;
}

__global__ __launch_bounds__(kThreads) void pages_step_kernel(PagesArgs p) {
  __shared__ int given[kPagesBatch], taken[kPagesBatch], room[kWaves];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), batch = p.a.batch;
  const int size0 = list_size(p);
  for (int b = wave; b < batch; b += kWaves) {
    const int before = p.held[b], n = count_given(p, b, given_of(p, b, before));
    if ((tid & 63) == 0) { given[b] = n; taken[b] = taken_of(p, b, before).total(); }
  }
  __syncthreads();
  int gives = 0, takes = 0;
  const int mine = tid < batch ? given[tid] : 0, mine_too = tid < batch ? taken[tid] : 0;
  const int first = before_me(mine, &gives, room), first_too = before_me(mine_too, &takes, room);
  if (tid < batch) { given[tid] = first; taken[tid] = first_too; }
  __syncthreads();
  const int size = min(size0 + gives, (int)p.a.pages);
  if (gives) {
    for (int b = wave; b < batch; b += kWaves) give(p, b, given_of(p, b, p.held[b]), given[b], size0, gives);
    __syncthreads();
  }
  if (takes) {
    for (int b = wave; b < batch; b += kWaves) take(p, b, taken_of(p, b, p.held[b]), taken[b], size);
    __syncthreads();
  }
  if (p.a.offsets) {                        // what no sequence has, then what one has
    for (int64_t i = tid; i < p.rows; i += kThreads) p.slots[i] = -1;
    __syncthreads();
  }
  for (int b = p.rows ? wave : batch; b < batch; b += kWaves) {
    const Fresh f(p, b);
    for (int i = tid & 63; i < f.count; i += 64) {
      const int position = f.position + i, column = position >> p.page_log;
      p.slots[f.first + i] = slot_of(p, position, position >= 0 && column < p.a.columns ? p.table[(int64_t)b * p.a.columns + column] : -1);
    }
  }
  for (int b = tid; b < batch; b += kThreads) p.held[b] = p.lengths[b];
  if (tid == 0) p.list[0] = max(0, size - takes);
}

// ---- larger steps ----
__global__ __launch_bounds__(256) void pages_count_kernel(PagesArgs p) {
  const int b = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  if (b >= p.a.batch) return;
  const int before = p.held[b], n = count_given(p, b, given_of(p, b, before));
  if (threadIdx.x & 63) return;
  p.before[b] = before;
  p.given[b] = n;
  p.taken[b] = taken_of(p, b, before).total();
}

__global__ __launch_bounds__(kThreads) void pages_sum_kernel(PagesArgs p) {
  __shared__ int room[kWaves];
  int gives = 0, takes = 0;
  for (int b0 = 0; b0 < p.a.batch; b0 += kThreads) {
    const int b = b0 + threadIdx.x;
    int all, all_too;
    const int first = before_me(b < p.a.batch ? p.given[b] : 0, &all, room), first_too = before_me(b < p.a.batch ? p.taken[b] : 0, &all_too, room);
    if (b < p.a.batch) {
      p.given[b] = gives + first;
      p.taken[b] = takes + first_too;
      p.held[b] = p.lengths[b];
    }
    gives += all;
    takes += all_too;
  }
  if (threadIdx.x) return;
  const int size0 = list_size(p), size = min(size0 + gives, (int)p.a.pages);
  p.sizes[0] = size0;
  p.sizes[1] = gives;
  p.sizes[2] = size;
  p.list[0] = max(0, size - takes);
}

__global__ __launch_bounds__(256) void pages_give_kernel(PagesArgs p) {
  const int b = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  if (b >= p.a.batch) return;
  give(p, b, given_of(p, b, p.before[b]), p.given[b], p.sizes[0], p.sizes[1]);
}

// Takes and slots: neither waits for the other, as a slot's page is found in the list where it is a new one.
__global__ __launch_bounds__(256) void pages_take_kernel(PagesArgs p, int take_blocks) {
  const int size = p.sizes[2];
  if ((int)blockIdx.x < take_blocks) {
    const int b = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    if (b < p.a.batch) take(p, b, taken_of(p, b, p.before[b]), p.taken[b], size);
    return;
  }
  const int64_t row = (int64_t)(blockIdx.x - take_blocks) * 256 + threadIdx.x;
  if (row >= p.rows) return;
  int b;
  if (p.a.offsets) {                        // the last sequence that begins at or before the row
    int low = 0, high = p.a.batch;
    while (low < high) {
      const int mid = (low + high) >> 1;
      if (p.a.offsets[mid] <= row) low = mid + 1;
      else high = mid;
    }
    b = low - 1;
  } else {
    b = (int)(row / p.a.tokens);
  }
  int64_t slot = -1;
  if (b >= 0) {
    const Fresh f(p, b);
    if (row >= f.first && row < f.first + f.count) {
      const int position = f.position + (int)(row - f.first), column = position >> p.page_log;
      if (position >= 0 && column < p.a.columns) {
        const int at = taken_of(p, b, p.before[b]).place(column);
        slot = slot_of(p, position, at >= 0 ? page_taken(p, p.taken[b] + at, size) : p.table[(int64_t)b * p.a.columns + column]);
      }
    }
  }
  p.slots[row] = slot;
}

}  // namespace

int launch_pages_step(const PagesArgs& p, void* stream) {
  hipStream_t s = (hipStream_t)stream;
  if (p.one) {
    pages_step_kernel<<<dim3(1), dim3(kThreads), 0, s>>>(p);
    return (int)hipGetLastError();
  }
  const unsigned fours = (unsigned)((p.a.batch + 3) / 4), rows = (unsigned)((p.rows + 255) / 256);
  if (fours) pages_count_kernel<<<dim3(fours), dim3(256), 0, s>>>(p);
  pages_sum_kernel<<<dim3(1), dim3(kThreads), 0, s>>>(p);
  if (fours) pages_give_kernel<<<dim3(fours), dim3(256), 0, s>>>(p);
  if (fours + rows) pages_take_kernel<<<dim3(fours + rows), dim3(256), 0, s>>>(p, (int)fours);
  return (int)hipGetLastError();
}

}  // namespace arrow
