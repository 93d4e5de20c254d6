// What the entries of arrow_embedding.h hand to their kernels.
#pragma once

#include <cstddef>
#include <cstdint>

#include "arrow_embedding.h"

namespace arrow {

constexpr int kDigitBits = 9;        // of the sort by id of many tokens, at most
constexpr int kSortTokens = 256;     // of a wavefront of it, at least
constexpr int kWideDigitBits = 15;   // of the sort of few tokens, at most
constexpr int kFewTokens = 65535;    // they are counted in 16 bits
constexpr int kDirectTokens = 2048;  // of a gradient in one launch, at most
constexpr int kDirectTable = 1 << 18;   // rows of one whose columns fill no slice of 256 bytes, at most
constexpr int kChunkTokens = 8;      // sorted tokens that a lane group of the sums goes through, a multiple of this: a row's load or two for few
                                     // tokens, and four where there are enough to fill the chip

// How the gradient of a call is carried out, and where its workspace keeps what.
struct EmbeddingPlan {
  bool direct;                     // one launch does it all; the rest is not used
  bool few;                        // tokens: each workgroup of the sort counts them all
  int32_t passes, bits;            // of the sort by id: digits, and bits of each
  int64_t blocks, block_tokens;    // its workgroups, and the tokens of each
  int64_t chunk, chunks;           // sorted tokens of a workgroup of the sums, and how many of those
  int64_t padded;                  // columns of a row of partial sums
  size_t keys[2], tokens[2];       // sorted ids and the tokens they stand at, two of each
  size_t counts;                   // digits x blocks
  size_t begin, end;               // per row of the table, its sorted tokens: begin up to the next row's after a sort of one digit; after others both,
                                   // and nothing for rows without any
  size_t parts;                    // two rows of partial sums per chunk
  size_t bytes;
};
EmbeddingPlan plan_embedding(const arrow_embedding_t& e);

// Launchers: 0 or a hipError_t.
int launch_embedding_forward(const arrow_embedding_t& e, const void* W, const void* ids, void* Y, void* stream);
int launch_embedding_backward(const arrow_embedding_t& e, const EmbeddingPlan& p, const void* dY, const void* ids, void* dW, void* ws, void* stream);

int fail_text(int code, const char* text);   // abi.cpp

}  // namespace arrow
