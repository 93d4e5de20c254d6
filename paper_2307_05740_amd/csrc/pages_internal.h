// What the entry of arrow_pages.h hands to its kernels.
#pragma once

#include <cstddef>
#include <cstdint>

#include "arrow_pages.h"

namespace arrow {

constexpr int kPagesBatch = 1024;          // sequences of a step in one launch, at most
constexpr int64_t kPagesRows = 8192;       // new tokens of one, at most
constexpr int64_t kPagesEntries = 65536;   // and entries of the table

struct PagesArgs {
  arrow_pages_t a;
  const int32_t* lengths;
  int32_t *held, *table, *list;
  int64_t* slots;
  int64_t rows;                            // of slots
  int32_t page_log;
  bool one, two;                           // launches; of two, the first is of one workgroup
  // several launches: per sequence the length before, and how many pages are given back and taken, then by how many before it; and the list's size
  // before, what is given back in all, and what is taken
  int32_t *before, *given, *taken, *first, *sizes;   // first: what is taken before each, where `taken` stays as it was
};

// Launchers: 0 or a hipError_t.
int launch_pages_step(const PagesArgs& p, void* stream);

}  // namespace arrow
