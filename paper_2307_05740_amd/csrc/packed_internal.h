// What the entries of arrow_packed.h hand to their kernels.
#pragma once

#include <cstddef>
#include <cstdint>

#include "arrow_packed.h"
#include "attention_internal.h"

namespace arrow {

constexpr int64_t kMostBlocks = 0xffffffff / 256;    // workgroups of 256: a launch has less than 2^32 threads

struct PackedArgs {
  arrow_packed_t c;
  Operand q, k, v, o;
  void* pool;
  const int64_t* slots;      // null: the last places of the sequences, by table and lengths
  int64_t tokens;
  int32_t group, splits, page_log;
  int32_t waves;             // of a workgroup: 4 or 8
  float* parts;              // splits x batch x q_heads x (dim + 2)
};

// Launchers: 0 or a hipError_t.
int launch_packed_append(const PackedArgs& p, void* stream);
int launch_packed_read(const PackedArgs& p, void* stream);
int launch_packed_decode(const PackedArgs& p, void* stream);

}  // namespace arrow
