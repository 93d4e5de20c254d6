// What the entries of arrow_attention.h hand to their kernels.
#pragma once

#include <cstddef>
#include <cstdint>

#include "arrow_attention.h"

namespace arrow {

// Sets the calling thread's arrow_last_error() text and returns `code` (abi.cpp).
int fail_text(int code, const char* text);

struct Operand {
  const void* at;
  int64_t sequence, token, head;   // steps in elements
};

struct AttentionArgs {
  Operand q, k, v, o, d_o, dq, dk, dv;
  const float* lse_in;             // backward
  float* lse;                      // forward, may be null
  float *off, *delta;              // backward, laid out as lse: -lse_i / scale and -sum_j P(i,j) <do_i, v_j>
  float* most;                     // backward, float16: the largest |d_o| of every 32 queries, finite ones
  float* parts;                    // backward: sums of the parts of a key tile, dk then dv of each; forward: of the parts of a row, and after them its
                                   // maximum and total, batch x q_heads x q_len x splits of each
  int32_t splits;                  // forward: parts that a row's keys are cut into
  const int32_t *q_offsets, *k_offsets;
  int64_t q_tokens, k_tokens;
  int32_t batch, q_heads, kv_heads, group, dim, q_len, k_len, window, sinks;
  float scale;
  // backward, keys: tiles of keys that some query sees for good (the first ones, with a window), and into how many parts
  // the work of those and of the others is cut
  int32_t sink_tiles, sink_parts, tile_parts;
  bool few_keys;                   // workgroups of 32 keys, not 128; no tile is cut
};

struct CacheArgs {
  arrow_cache_t c;
  Operand q, k, v, o;              // the new token's (k, v may be null)
  void *k_pool, *v_pool;
  int32_t group, splits, page_log, tokens;
  float* parts;                    // splits x batch x q_heads x (dim + 2)
};

// Into how many parts the forward call cuts a row's keys where it has a workspace, 1 to kMostRowSplits.
int attention_forward_splits(const AttentionArgs& a);

// Launchers: 0 or a hipError_t.
int launch_attention_forward(const AttentionArgs& a, int32_t dtype, void* stream);
int launch_attention_backward(const AttentionArgs& a, int32_t dtype, void* stream);
int launch_cache_append(const CacheArgs& a, void* stream);
int launch_attention_decode(const CacheArgs& a, void* stream);

constexpr int kQueryTile = 128;    // queries of a workgroup, forward and dq
constexpr int kKeyTile = 128;      // keys of a workgroup, dk and dv
constexpr int kQueryStep = 64;     // queries that it goes through at a time
constexpr int kMostSplits = 256;   // stretches of a cache
constexpr int kMostRowSplits = 32; // parts of a row's keys, forward
constexpr int kHeadTile = 16;      // query heads of a workgroup, single tokens

}  // namespace arrow
