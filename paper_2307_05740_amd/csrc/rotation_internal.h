// What the entries of arrow_rotation.h hand to their kernels.
#pragma once

#include <cstddef>
#include <cstdint>

#include "arrow_rotation.h"

namespace arrow {

constexpr int kRotationThreads = 256;
constexpr int kRotationAngles = 4096;     // of a workgroup at a time, at most: tokens x rotary / 2
constexpr int kRotationTokens = 64;       // and tokens
constexpr int kRotationBlocks = 1024;     // workgroups of a gradient, at most: four to a compute unit; each leaves a sum of a weight's gradient

// Tokens that a workgroup has at a time, such tiles of a sequence, and of all.
struct RotationTiles {
  int32_t per, tiles, all;
};

struct RotationArgs {
  arrow_rotation_t a;
  const void *q, *k, *wq, *wk;            // the forward call's
  const void *gq, *gk;                    // gradients of its results
  void *yq, *yk;                          // its results, or the gradients of q and k
  arrow_strides_t q_to, k_to;             // steps of these
  void *dwq, *dwk;
  float* parts;                           // blocks x dim sums of the weights' gradients
  int32_t sequences, length;              // and tokens of each: one of all where sequences follow each other
  RotationTiles tiles[2];                 // forward: [0]; of a gradient, those of queries and of keys
  int32_t blocks, q_blocks;               // workgroups; of a gradient, those that have queries: the first ones
  int32_t lanes_log;                      // lanes of a head: a power of two, each has 16 elements
  bool whole;                             // all of them have them
  float share;                            // 1 / dim
};

// Launchers: 0 or a hipError_t.
int launch_rotation(const RotationArgs& p, bool backward, void* stream);

}  // namespace arrow
