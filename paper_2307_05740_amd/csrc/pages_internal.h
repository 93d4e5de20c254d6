// What the entry of arrow_pages.h hands to its kernels.
#pragma once

#include <cstddef>
#include <cstdint>

#include "arrow_pages.h"

namespace arrow {

// A step in one launch, of one workgroup, has at most so many sequences, new tokens and entries of the table; entries where it has no new tokens, so that it most often gives back.
// Where little changes it is faster (four new tokens and back: 8 to 10 us, several launches 19; 8 and 11 where only the way back takes several), where all pages of a
// table go it is not (prompts and back, us, with the way back in one launch and in two; 4 sequences, and 256):
//   4096 entries 18 21, 26 23;  16,384: 24 22, 38 23;  32,768: 34 23, 53 21;  65,536: 48 24, 83 21
constexpr int kPagesBatch = 1024;
constexpr int64_t kPagesRows = 8192;
constexpr int64_t kPagesEntries = 65536;
constexpr int64_t kPagesBack = 16384;
// More new tokens: two launches, the first as above, or three.  (Prompts and back, us; 4 sequences, 32, 256.  1024 entries: 15 19, 21 23, 24 25;  2048: 18 19, 22 22, 28 24;  4096: 23 21, 27 20, 35 23;
// 65,536: 182 24, 221 24, 267 21)
constexpr int64_t kPagesFew = 2048;

struct PagesArgs {
  arrow_pages_t a;
  const int32_t* lengths;
  int32_t *held, *table, *list;
  int64_t* slots;
  int64_t rows;                            // of slots
  int32_t page_log;
  bool one, two;                           // launches; of two, the first is of one workgroup
  int32_t chunk, chunks;                   // several launches: columns that change, of a unit of the work, and units of a sequence
  // per sequence the length before; per unit how many pages are given back and taken, then by how many before it; and the list's size before, what
  // is given back in all, and what is taken
  int32_t *before, *given, *taken, *first, *sizes;   // first: what is taken before each, where `taken` stays as it was
};

// Launchers: 0 or a hipError_t.
int launch_pages_step(const PagesArgs& p, void* stream);

}  // namespace arrow
