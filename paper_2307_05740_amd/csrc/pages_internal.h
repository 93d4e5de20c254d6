// What the entry of arrow_pages.h hands to its kernels.
#pragma once

#include <cstddef>
#include <cstdint>

#include "arrow_pages.h"

namespace arrow {

constexpr int kPagesBatch = 1024;          // sequences of a step in one launch, at most
constexpr int64_t kPagesRows = 8192;       // new tokens of one, at most
constexpr int64_t kPagesEntries = 65536;   // and entries of its table

struct PagesArgs {
  arrow_pages_t a;
  const int32_t* lengths;
  int32_t *held, *table, *list;
  int64_t* slots;
  int64_t rows;                            // of slots
  int32_t page_log;
  bool one;                                // launch
  // several launches: per sequence the length before, and how many pages are given back and taken, then by how many before it; and the list's size before
  // and after what is given back
  int32_t *before, *given, *taken, *sizes;
};

// Launchers: 0 or a hipError_t.
int launch_pages_step(const PagesArgs& p, void* stream);

}  // namespace arrow
