// C boundary of the rotation entries (include/arrow_rotation.h): checks of the arguments, the plan of a call.
#include <algorithm>
#include <cmath>
#include <numeric>

#include "checks.h"
#include "rotation_internal.h"

namespace {

using namespace arrow;

int check(const arrow_rotation_t* a) {
  if (!a) return refuse(ARROW_EINVAL, "NULL arguments");
  if (!is_dtype(a->dtype)) return refuse(ARROW_EINVAL, "dtype %d", a->dtype);
  if (a->weight_dtype != a->dtype && a->weight_dtype != ARROW_F32) return refuse(ARROW_EINVAL, "weight_dtype %d is neither dtype nor ARROW_F32", a->weight_dtype);
  if (a->batch < 0 || a->tokens < 0 || (int64_t)a->batch * a->tokens > 0x7fffffff) return refuse(ARROW_EINVAL, "batch = %d of tokens = %d", a->batch, a->tokens);
  if (a->q_heads < 1 || a->kv_heads < 1 || a->q_heads > 65536 || a->kv_heads > 65536)
    return refuse(ARROW_EINVAL, "q_heads = %d, kv_heads = %d: 1 .. 65536", a->q_heads, a->kv_heads);
  if (a->dim < 8 || a->dim > 256 || a->dim % 8) return refuse(ARROW_EINVAL, "dim = %d is none of 8, 16, ..., 256", a->dim);
  if (a->rotary < 0 || a->rotary > a->dim || a->rotary % 16) return refuse(ARROW_EINVAL, "rotary = %d is none of 0, 16, 32, ... up to dim = %d", a->rotary, a->dim);
  if (a->interleaved != 0 && a->interleaved != 1) return refuse(ARROW_EINVAL, "interleaved = %d", a->interleaved);
  if (!(a->eps >= 0.f) || !std::isfinite(a->eps)) return refuse(ARROW_EINVAL, "eps = %g is negative or not finite", a->eps);
  if (a->positions) {
    if (a->position_bytes != 4 && a->position_bytes != 8) return refuse(ARROW_EINVAL, "position_bytes = %d is neither 4 nor 8", a->position_bytes);
    if (int rc = check_pointer("positions", a->positions, a->position_bytes)) return rc;
  }
  if (a->shift < -((int64_t)1 << 52) || a->shift > (int64_t)1 << 52) return refuse(ARROW_EINVAL, "shift = %lld: within 2^52 of 0", (long long)a->shift);
  if (a->rotary)
    if (int rc = check_pointer("turns", a->turns, 8)) return rc;
  return ARROW_OK;
}

Rows rows_of(const arrow_rotation_t* a, const void* at, const arrow_strides_t& s, int32_t heads) {
  const int64_t size = size_of(a->dtype);
  return {at, a->dim * size, {a->batch, s.sequence * size}, {a->tokens, s.token * size}, {heads, s.head * size}};
}

int check_heads(const arrow_rotation_t* a, const char* name, const void* at, const arrow_strides_t& s, int32_t heads, bool written) {
  if (int rc = check_pointer(name, at, 16)) return rc;
  const int step = 16 / size_of(a->dtype);
  if (s.sequence % step || s.token % step || s.head % step || s.sequence < 0 || s.token < 0 || s.head < 0)
    return refuse(ARROW_EINVAL, "%s: steps of %lld, %lld, %lld elements: multiples of %d, not negative", name, (long long)s.sequence, (long long)s.token,
                  (long long)s.head, step);
  for (int64_t step : {s.sequence, s.token, s.head})
    if (step > (int64_t)1 << 56) return refuse(ARROW_EINVAL, "%s: a step of %lld elements", name, (long long)step);
  if (written && !rows_of(a, at, s, heads).distinct()) return refuse(ARROW_EINVAL, "%s is written, and its rows overlap", name);
  return ARROW_OK;
}

bool same(const arrow_strides_t& a, const arrow_strides_t& b) { return a.sequence == b.sequence && a.token == b.token && a.head == b.head; }

int check_weights(const arrow_rotation_t* a, const char* name, const void* q, const void* k) {
  if (!q != !k) return refuse(ARROW_EINVAL, "%s of queries and of keys: both or neither", name);
  const int size = size_of(a->weight_dtype);
  if ((uintptr_t)q % size || (uintptr_t)k % size) return refuse(ARROW_EINVAL, "%s are not %d-byte aligned", name, size);
  return ARROW_OK;
}

Rows weights_of(const arrow_rotation_t* a, const void* at) { return {at, (int64_t)a->dim * size_of(a->weight_dtype)}; }
Rows positions_of(const arrow_rotation_t* a) { return {a->positions, a->batch * (int64_t)a->tokens * a->position_bytes}; }
Rows turns_of(const arrow_rotation_t* a) { return {a->rotary ? a->turns : nullptr, (int64_t)a->rotary * 4}; }

bool follow(const arrow_rotation_t* a, const arrow_strides_t& s) { return a->batch <= 1 || s.sequence == a->tokens * s.token; }

// Tokens of a workgroup at a time, which share its angles: up to eight rounds of its groups of lanes, as even a share of all as that leaves, but enough for one round, and where a
// round is of whole tokens, a multiple of them.  At most 4096 angles, 32 KiB; us for 1.3e8 elements (gradients: 0.67e8, with the forward call):
//   up to 8 tokens, and 1024 angles: heads 32/8 of 128 110 (148), 8/2 of 64 128 (268), 4/1 of 128 140 (297), 2/1 of 256 147 (257)
//   2048 angles: 109 (142), 107 (163), 115 (191), 132 (211);  4096: 107 (142), 107 (163), 115 (183), 128 (199)
//   4 rounds instead of 8: 107 (141), 114 (163), 123 (184), 131 (198);  16, with 2048 angles: 117 (145), 110 (166), 114 (191), 130 (211)
RotationTiles tiles_of(const RotationArgs& p, int64_t heads, int64_t blocks) {
  const int64_t groups = kRotationThreads >> p.lanes_log, tokens = (int64_t)p.sequences * p.length, angles = p.a.rotary / 2;
  const int64_t fit = std::min<int64_t>(kRotationTokens, angles ? kRotationAngles / angles : kRotationTokens);
  const int64_t some = std::max<int64_t>(1, std::min(fit, groups / heads)), unit = groups / std::gcd(groups, heads);
  int64_t most = std::min(fit, std::max(some, 8 * groups / heads));
  if (unit <= most) most = most / unit * unit;
  const int64_t rounds = std::max<int64_t>(1, ceil_div(tokens, most * blocks));
  int64_t per = std::min(most, std::max(some, ceil_div(tokens, rounds * blocks)));
  if (unit <= per) per = ceil_div(per, unit) * unit;
  RotationTiles t;
  t.per = (int32_t)per;
  t.tiles = (int32_t)ceil_div(p.length, per);
  t.all = p.sequences * t.tiles;
  return t;
}

RotationArgs plan(const arrow_rotation_t* a, bool backward) {
  RotationArgs p{};
  p.a = *a;
  p.sequences = a->batch;
  p.length = a->tokens;
  if (a->tokens == 1 && a->batch > 1) {               // (tokens that are sequences' only ones)
    for (auto* s : {&p.a.q, &p.a.k, &p.a.q_out, &p.a.k_out, &p.a.dq, &p.a.dk}) s->token = s->sequence;
    p.sequences = 1;
    p.length = a->batch;
  } else if (follow(a, a->q) && follow(a, a->k) && follow(a, a->q_out) && follow(a, a->k_out) && (!backward || (follow(a, a->dq) && follow(a, a->dk)))) {
    p.sequences = std::min(a->batch, 1);
    p.length = a->batch * a->tokens;
  }
  while ((16 << p.lanes_log) < a->dim) ++p.lanes_log;
  p.whole = (16 << p.lanes_log) == a->dim;
  p.share = 1.f / (float)a->dim;
  if (!backward) {
    p.tiles[0] = tiles_of(p, a->q_heads + a->kv_heads, 1024);
    p.blocks = std::min(p.tiles[0].all, 1 << 23);    // (a launch has less than 2^32 threads)
    return p;
  }
  // Queries and keys have workgroups by their heads.
  const int32_t q = std::min(kRotationBlocks - 1, std::max(1, (int32_t)(kRotationBlocks * (int64_t)a->q_heads / (a->q_heads + a->kv_heads))));
  p.tiles[0] = tiles_of(p, a->q_heads, q);
  p.tiles[1] = tiles_of(p, a->kv_heads, kRotationBlocks - q);
  p.q_blocks = std::min(p.tiles[0].all, q);
  p.blocks = p.q_blocks + std::min(p.tiles[1].all, kRotationBlocks - q);
  return p;
}

}  // namespace

extern "C" {

int arrow_rotation_forward(const arrow_rotation_t* a, const void* q, const void* k, const void* wq, const void* wk, void* q_out, void* k_out, void* stream) {
  if (int rc = check(a)) return rc;
  if ((int64_t)a->batch * a->tokens == 0) return ARROW_OK;
  if (int rc = check_weights(a, "weights", wq, wk)) return rc;
  if (int rc = check_heads(a, "q", q, a->q, a->q_heads, false)) return rc;
  if (int rc = check_heads(a, "k", k, a->k, a->kv_heads, false)) return rc;
  if (int rc = check_heads(a, "q_out", q_out, a->q_out, a->q_heads, true)) return rc;
  if (int rc = check_heads(a, "k_out", k_out, a->k_out, a->kv_heads, true)) return rc;
  if (q_out == k || k_out == q || q_out == k_out) return refuse(ARROW_EINVAL, "q_out is k or k_out, or k_out is q");
  if ((q_out == q && !same(a->q, a->q_out)) || (k_out == k && !same(a->k, a->k_out))) return refuse(ARROW_EINVAL, "in place, but with other steps");
  const Part all[] = {{"q", rows_of(a, q, a->q, a->q_heads), false, -1}, {"k", rows_of(a, k, a->k, a->kv_heads), false, -1},
                      {"q_out", rows_of(a, q_out, a->q_out, a->q_heads), true, 0}, {"k_out", rows_of(a, k_out, a->k_out, a->kv_heads), true, 1},
                      {"a weight", weights_of(a, wq), false, -1}, {"a weight", weights_of(a, wk), false, -1}, {"positions", positions_of(a), false, -1}, {"turns", turns_of(a), false, -1}};
  if (int rc = check_apart(all)) return rc;
  RotationArgs p = plan(a, false);
  p.q = q; p.k = k; p.wq = wq; p.wk = wk;
  p.yq = q_out; p.yk = k_out;
  p.q_to = p.a.q_out; p.k_to = p.a.k_out;
  return launched("rotation forward", launch_rotation(p, false, stream));
}

size_t arrow_rotation_workspace_bytes(const arrow_rotation_t* a) {
  if (check(a)) return 0;
  return align_up((size_t)plan(a, true).blocks * a->dim * 4);
}

int arrow_rotation_backward(const arrow_rotation_t* a, const void* d_q_out, const void* d_k_out, const void* q, const void* k, const void* wq,
                            const void* wk, void* dq, void* dk, void* dwq, void* dwk, void* ws, size_t ws_bytes, void* stream) {
  if (int rc = check(a)) return rc;
  if (int rc = check_weights(a, "weights", wq, wk)) return rc;
  if (int rc = check_weights(a, "gradients of weights", dwq, dwk)) return rc;
  if (dwq && !apart(weights_of(a, dwq), weights_of(a, dwk))) return refuse(ARROW_EINVAL, "dwq and dwk are the same, or overlap");
  RotationArgs p = plan(a, true);
  const bool some = (int64_t)a->batch * a->tokens > 0;
  if (some) {
    const struct { const char* name; const void* at; const arrow_strides_t& s; int32_t heads; bool written; } all[] = {
        {"d_q_out", d_q_out, a->q_out, a->q_heads, false}, {"d_k_out", d_k_out, a->k_out, a->kv_heads, false}, {"q", q, a->q, a->q_heads, false},
        {"k", k, a->k, a->kv_heads, false}, {"dq", dq, a->dq, a->q_heads, true}, {"dk", dk, a->dk, a->kv_heads, true}};
    for (auto& m : all)
      if (int rc = check_heads(a, m.name, m.at, m.s, m.heads, m.written)) return rc;
    if (dq == dk || dq == k || dk == q || dq == d_k_out || dk == d_q_out || dq == q || dk == k)
      return refuse(ARROW_EINVAL, "dq or dk is q, k, the other's gradient, or the other");
    if ((dq == d_q_out && !same(a->dq, a->q_out)) || (dk == d_k_out && !same(a->dk, a->k_out))) return refuse(ARROW_EINVAL, "in place, but with other steps");
    const Part parts[] = {{"d_q_out", rows_of(a, d_q_out, a->q_out, a->q_heads), false, -1}, {"d_k_out", rows_of(a, d_k_out, a->k_out, a->kv_heads), false, -1},
                          {"q", rows_of(a, q, a->q, a->q_heads), false, -1}, {"k", rows_of(a, k, a->k, a->kv_heads), false, -1},
                          {"dq", rows_of(a, dq, a->dq, a->q_heads), true, 0}, {"dk", rows_of(a, dk, a->dk, a->kv_heads), true, 1},
                          {"a weight", weights_of(a, wq), false, -1}, {"a weight", weights_of(a, wk), false, -1}, {"positions", positions_of(a), false, -1},
                          {"turns", turns_of(a), false, -1}, {"dwq", weights_of(a, dwq), true, -1}, {"dwk", weights_of(a, dwk), true, -1},
                          {"the workspace", {dwq ? ws : nullptr, (int64_t)arrow_rotation_workspace_bytes(a)}, true, -1}};
    if (int rc = check_apart(parts)) return rc;
  }
  if (dwq)
    if (int rc = check_workspace(ws, ws_bytes, arrow_rotation_workspace_bytes(a))) return rc;
  if (!some && !dwq) return ARROW_OK;
  p.q = q; p.k = k; p.wq = wq; p.wk = wk; p.gq = d_q_out; p.gk = d_k_out;
  p.yq = dq; p.yk = dk;
  p.q_to = p.a.dq; p.k_to = p.a.dk;
  p.dwq = dwq; p.dwk = dwk;
  p.parts = (float*)ws;
  return launched("rotation backward", launch_rotation(p, true, stream));
}

}  // extern "C"
