// C boundary of the entries of include/arrow_logprobs.h: checks of the arguments, the plan of a call.
#include <algorithm>
#include <cmath>

#include "checks.h"
#include "logprobs_internal.h"

namespace arrow {

void plan_score(ScoreArgs& p) {
  // Pieces of 16 bytes that a row reaches into, at any address.
  const int64_t each = 16 / size_of(p.a.dtype), pieces = ceil_div((int64_t)p.a.vocabulary, each) + 1;
  // Rows of few pieces have 16 lanes, 32 or a wavefront each.  (Tokens on top are looked for among those that lanes have as their largest: there have to be some more lanes than
  // tokens.)  A wavefront and a workgroup, us, bfloat16: rows of 5675 with the 20 best, 2048 of them 12.2 24.3, 20,000 57.8 140; of 8100 with 5, one 7.7 11.8 (in two launches), 9668 35.2 58.0;
  // without any, of 5675, 4096 12.0 12.0, 20,000 41.4 52.6, of 8100, 2048 10.5 9.0, 20,000 59.0 60.0.
  // 16 lanes, 32, and 64, 65,536 rows: of 472 without tokens 12.5 14.2 19.8, with 5 25.2 31.9 41.2, with 12 37.1 37.8 44.5, with 20 - 47.5 48.1; of 952 21.7 20.8 25.4, 33.7 38.5 45.9,
  // 47.8 46.0 51.7, - 58.0 58.6;  of 232 with 20 - 39.6 52.5.
  p.parts = 1;
  if (p.a.top <= 8 && pieces <= 128) p.lanes = 16;
  else if ((p.a.top <= 16 && pieces >= 24 && pieces <= 128) || (p.a.top <= 20 && pieces >= 28 && pieces <= 64)) p.lanes = 32;
  else p.lanes = pieces <= 64 * (p.a.top ? 16 : p.a.rows >= 4096 ? 12 : 8) ? 64 : 0;
  // More tokens than there are lanes with pieces, or nearly as many, leave no border to look for: lanes have single logits then.  (65,536 rows, pieces and logits: of 40 with 20 70.8 33.5;
  // of 150 with 12 51.6 41.3, with 32 91.6 48.8; of 200 with 12 31.5 42.6, with 20 55.8 46.0.)
  if (p.a.top > 8 && (pieces < 24 || 2 * pieces < 3 * p.a.top)) {
    p.single = true;
    p.lanes = 64;
    p.vectors = (int32_t)(ceil_div(p.a.vocabulary, 64) * 64);
    return;
  }
  if (p.lanes) {
    p.vectors = (int32_t)(ceil_div(pieces, p.lanes) * p.lanes);
    return;
  }
  // With most likely tokens a workgroup holds its pieces in registers, up to 32 to a lane.  Longer rows are cut, into parts of up to 16 to a lane, and where there are few of them, so
  // are rows without tokens that would take longer than the second launch that joins parts.  One part and several, us, bfloat16:
  //   6 rows of 18,065 without tokens 5.3 8.3, with 5 8.6 11.8, with 32 9.4 20.9; of 65,000 without any 7.2 8.1; of 110,000 10.1 9.1; of 157,065 13.3 9.1
  //   with 5, 85 rows of 33,000 10.7 14.7, 4000 60 85; 85 of 50,257 12.0 16.0, 4000 98.6 102.9; 85 of 65,000 13.7 16.3, 4000 115.2 114.7; 48 to a lane, 300 of 66,000 28.4 22.5
  //   parts of 16 and 32 to a lane, 2000 rows of 128,001 with 5 114 126
  // 512 workgroups in all: 24 rows of 110,000 with 5, parts for 64, 128, ... 2048 workgroups, 16.6, 16.1, 15.5, 15.1, 15.2, 16.7; 93 of 500,000 without any 47, 47, 28, 20, 21, 21.
  const int64_t one = kScoreThreads * (p.a.top ? kMostVectors : 48);
  const int64_t least = ceil_div(pieces, kScoreThreads * (p.a.top ? kPartVectors : kSumVectors * kMostSums)), most = ceil_div(pieces, kScoreThreads);
  const int64_t limit = p.a.top ? 64 : 128;       // (of lists that are joined)
  const int64_t wanted = pieces <= one ? 1 : std::max<int64_t>(least, std::min<int64_t>({most, limit, 512 / std::max<int64_t>(1, p.a.rows)}));
  const int64_t rounds = ceil_div(pieces, wanted * kScoreThreads);           // pieces per lane
  p.parts = (int32_t)ceil_div(pieces, rounds * kScoreThreads);
  p.vectors = (int32_t)(rounds * kScoreThreads);
}

}  // namespace arrow

namespace {

using namespace arrow;

int check(const arrow_logprobs_t* a, bool grad) {
  if (!a) return refuse(ARROW_EINVAL, "NULL arguments");
  if (!is_dtype(a->dtype)) return refuse(ARROW_EINVAL, "dtype %d", a->dtype);
  if (a->target_bytes != 4 && a->target_bytes != 8) return refuse(ARROW_EINVAL, "target_bytes = %d is neither 4 nor 8", a->target_bytes);
  if (a->vocabulary < 1 || a->vocabulary > (1 << 30)) return refuse(ARROW_EINVAL, "vocabulary = %d: 1 .. 2^30", a->vocabulary);
  if (a->top < 0 || a->top > kMostTop || a->top > a->vocabulary) return refuse(ARROW_EINVAL, "top = %d: 0 .. %d, at most vocabulary = %d", a->top, kMostTop, a->vocabulary);
  if (a->rows < 0 || a->rows > 0x7fffffff) return refuse(ARROW_EINVAL, "rows = %lld: 0 .. 2^31 - 1", (long long)a->rows);
  if (a->stride < a->vocabulary || (grad && a->d_stride < a->vocabulary))
    return refuse(ARROW_EINVAL, "rows %lld and %lld elements apart, of %d", (long long)a->stride, (long long)a->d_stride, a->vocabulary);
  if (!(a->scale > 0.f) || !std::isfinite(a->scale)) return refuse(ARROW_EINVAL, "scale = %g is not positive and finite", a->scale);
  return ARROW_OK;
}

size_t sums_bytes(const ScoreArgs& p) { return align_up((size_t)p.a.rows * p.parts * 16); }
size_t bytes_of(const ScoreArgs& p) { return p.parts == 1 ? 0 : sums_bytes(p) + align_up((size_t)p.a.rows * p.parts * p.a.top * 8); }

int64_t extent(const arrow_logprobs_t* a, int64_t stride) { return a->rows ? ((a->rows - 1) * stride + a->vocabulary) * size_of(a->dtype) : 0; }

}  // namespace

extern "C" {

size_t arrow_logprobs_workspace_bytes(const arrow_logprobs_t* a) {
  if (check(a, false)) return 0;
  ScoreArgs p{};
  p.a = *a;
  plan_score(p);
  return bytes_of(p);
}

int arrow_logprobs_forward(const arrow_logprobs_t* a, const void* logits, const void* targets, float* logp, float* entropy, float* lse, float* stats, float* top_logp,
                           int64_t* top_ids, void* ws, size_t ws_bytes, void* stream) {
  if (int rc = check(a, false)) return rc;
  if (a->rows == 0) return ARROW_OK;
  if (int rc = check_pointer("logits", logits, size_of(a->dtype))) return rc;
  if (int rc = check_pointer("targets", targets, a->target_bytes)) return rc;
  const struct { const char* name; const void* at; int64_t each; } out[] = {{"logp", logp, 4}, {"entropy", entropy, 4}, {"lse", lse, 4}, {"stats", stats, 8},
                                                                           {"top_logp", top_logp, 4 * a->top}, {"top_ids", top_ids, 8 * a->top}};
  for (auto& o : out) {
    if (o.each == 0) continue;
    if (int rc = check_pointer(o.name, o.at, (o.at == top_ids || o.at == stats) ? 8 : 4)) return rc;
    if (overlap(o.at, o.each * a->rows, logits, extent(a, a->stride)) || overlap(o.at, o.each * a->rows, targets, a->rows * a->target_bytes))
      return refuse(ARROW_EINVAL, "%s overlaps an input", o.name);
    for (auto& other : out)
      if (&other != &o && overlap(o.at, o.each * a->rows, other.at, other.each * a->rows)) return refuse(ARROW_EINVAL, "%s and %s overlap", o.name, other.name);
  }
  ScoreArgs p{};
  p.a = *a;
  plan_score(p);
  if (int rc = check_workspace(ws, ws_bytes, bytes_of(p))) return rc;
  p.logits = logits; p.targets = targets;
  p.logp = logp; p.entropy = entropy; p.lse = lse; p.stats = stats; p.top_logp = top_logp; p.top_ids = top_ids;
  p.sums = (float*)ws;
  p.keys = (uint64_t*)((char*)ws + sums_bytes(p));
  return launched("logprobs forward", launch_score_forward(p, stream));
}

int arrow_logprobs_backward(const arrow_logprobs_t* a, const float* d_logp, const float* d_entropy, const void* logits, const void* targets, const float* stats,
                            const float* entropy, void* d_logits, void* stream) {
  if (int rc = check(a, true)) return rc;
  if (a->rows == 0) return ARROW_OK;
  const int size = size_of(a->dtype);
  if (int rc = check_pointer("logits", logits, size)) return rc;
  if (int rc = check_pointer("targets", targets, a->target_bytes)) return rc;
  if (int rc = check_pointer("stats", stats, 8)) return rc;
  if (d_entropy)
    if (int rc = check_pointer("entropy", entropy, 4)) return rc;
  if ((uintptr_t)d_logp % 4 || (uintptr_t)d_entropy % 4) return refuse(ARROW_EINVAL, "d_logp or d_entropy is not 4-byte aligned");
  if (int rc = check_pointer("d_logits", d_logits, size)) return rc;
  const int64_t bytes = extent(a, a->d_stride);
  if (d_logits == logits ? a->stride != a->d_stride : overlap(d_logits, bytes, logits, extent(a, a->stride)))
    return refuse(ARROW_EINVAL, "d_logits overlaps logits and is not the same");
  const struct { const void* at; int64_t bytes; } in[] = {{targets, a->rows * a->target_bytes}, {stats, 8 * a->rows}, {entropy, 4 * a->rows}, {d_logp, 4 * a->rows},
                                                          {d_entropy, 4 * a->rows}};
  for (auto& m : in)
    if (m.at && overlap(d_logits, bytes, m.at, m.bytes)) return refuse(ARROW_EINVAL, "d_logits overlaps an input");
  ScoreArgs p{};
  p.a = *a;
  p.logits = logits; p.targets = targets; p.d_logp = d_logp; p.d_entropy = d_entropy; p.stats = const_cast<float*>(stats); p.entropy_in = entropy;
  p.d_logits = d_logits;
  return launched("logprobs backward", launch_score_backward(p, stream));
}

}  // extern "C"
