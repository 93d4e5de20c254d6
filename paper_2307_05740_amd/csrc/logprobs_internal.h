// What the entries of arrow_logprobs.h hand to their kernels.
#pragma once

#include <cstddef>
#include <cstdint>

#include "arrow_logprobs.h"

namespace arrow {

constexpr int kScoreThreads = 256;
constexpr int kMostTop = 32;
constexpr int kMostVectors = 32;       // pieces of 16 bytes of a whole row that a lane of a workgroup holds
constexpr int kPartVectors = 16;       // and of a part of one
// A lane's sums have no more than so many steps, which is what they are as exact as: up to 256 logits one after the other, and of these sums up to 128.
constexpr int kSumVectors = 32;        // pieces, of a part that is not held, to a sum
constexpr int kMostSums = 128;         // and sums of a part

struct ScoreArgs {
  arrow_logprobs_t a;
  const void *logits, *targets;
  const float *d_logp, *d_entropy, *entropy_in;
  float *logp, *entropy, *lse, *stats, *top_logp;
  int64_t* top_ids;
  void* d_logits;
  int32_t parts;                       // that a row is cut into
  int32_t vectors;                     // pieces of 16 bytes of a part: parts x vectors cover a row whatever its first address
  int32_t lanes;                       // that have a row: 16, 32 or 64, or 0 for workgroups, which parts have
  bool single;                         // of 64 lanes: a logit is a piece
  float* sums;                         // rows x parts x 4: the largest logit, the sums relative to it, 0; where rows are cut
  uint64_t* keys;                      // rows x parts x top, falling
};

// How a row is cut: set in `p` from p.a.
void plan_score(ScoreArgs& p);

// Launchers: 0 or a hipError_t.
int launch_score_forward(const ScoreArgs& p, void* stream);
int launch_score_backward(const ScoreArgs& p, void* stream);

}  // namespace arrow
