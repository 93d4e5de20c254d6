// C boundary of the attention entries (include/arrow_attention.h): checks of the arguments, the plan of a call, its launches.
#include <hip/hip_runtime_api.h>

#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>

#include "arrow.h"
#include "attention_internal.h"

namespace {

using namespace arrow;

int refuse(int code, const char* fmt, ...) {
  char text[256];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(text, sizeof text, fmt, ap);
  va_end(ap);
  return fail_text(code, text);
}

int launched(const char* what, int rc) {
  return rc == 0 ? ARROW_OK : refuse(ARROW_EHIP, "%s: %s", what, hipGetErrorString((hipError_t)rc));
}

constexpr int64_t kMostStep = 1 << 24;      // elements from token to token: 64 of them stay within a descriptor's 32 bits
constexpr int32_t kMostTokens = 1 << 26;    // of a sequence

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// An operand of `len` tokens (0: nothing of it is touched, and it may be null).
int check_operand(const char* name, const void* at, const arrow_strides_t& s, int64_t len, int32_t heads, int32_t batch, bool ragged, int32_t dim,
                  bool written) {
  if (len == 0) return ARROW_OK;
  if (!at) return refuse(ARROW_EINVAL, "%s is NULL", name);
  if ((uintptr_t)at % 16) return refuse(ARROW_EINVAL, "%s is not 16-byte aligned", name);
  if (s.sequence % 8 || s.token % 8 || s.head % 8)
    return refuse(ARROW_EINVAL, "%s: steps of %lld, %lld, %lld elements are not multiples of 8", name, (long long)s.sequence, (long long)s.token,
                  (long long)s.head);
  if (s.token < 0 || s.token > kMostStep || s.head < 0 || (!ragged && s.sequence < 0))
    return refuse(ARROW_EINVAL, "%s: a step between tokens lies within 0 .. %lld, the others are not negative", name, (long long)kMostStep);
  if (written && ((len > 1 && s.token < dim) || (heads > 1 && s.head < dim) || (!ragged && batch > 1 && s.sequence < dim)))
    return refuse(ARROW_EINVAL, "%s is written, and its rows overlap", name);
  return ARROW_OK;
}

int check_heads(int32_t dtype, int32_t batch, int32_t q_heads, int32_t kv_heads, int32_t dim, int32_t window, int32_t sinks, float scale) {
  if (dtype != ARROW_BF16 && dtype != ARROW_F16) return refuse(ARROW_EINVAL, "dtype %d: attention takes ARROW_BF16 and ARROW_F16", dtype);
  if (batch < 0) return refuse(ARROW_EINVAL, "batch = %d", batch);
  if (kv_heads < 1 || q_heads < 1 || q_heads % kv_heads) return refuse(ARROW_EINVAL, "q_heads = %d is no multiple of kv_heads = %d", q_heads, kv_heads);
  if (dim < 8 || dim > 128 || dim % 8) return refuse(ARROW_EINVAL, "dim = %d is none of 8, 16, ..., 128", dim);
  if (window < 0 || sinks < 0) return refuse(ARROW_EINVAL, "window = %d, sinks = %d", window, sinks);
  if (!(scale > 0.f) || !std::isfinite(scale)) return refuse(ARROW_EINVAL, "scale = %g is not positive and finite", scale);
  return ARROW_OK;
}

int check(const arrow_attention_t* a) {
  if (!a) return refuse(ARROW_EINVAL, "NULL arguments");
  if (int rc = check_heads(a->dtype, a->batch, a->q_heads, a->kv_heads, a->dim, a->window, a->sinks, a->scale)) return rc;
  if (a->q_len < 0 || a->k_len < 0 || a->q_len > kMostTokens || a->k_len > kMostTokens)
    return refuse(ARROW_EINVAL, "q_len = %d, k_len = %d: 0 .. %d", a->q_len, a->k_len, kMostTokens);
  if (!a->q_offsets != !a->k_offsets) return refuse(ARROW_EINVAL, "offsets of queries and keys: both or neither");
  if (a->q_offsets && (a->q_tokens < 0 || a->k_tokens < 0)) return refuse(ARROW_EINVAL, "q_tokens or k_tokens is negative");
  return ARROW_OK;
}

int64_t tokens_of(const arrow_attention_t* a, bool keys) {
  if (a->batch == 0) return 0;
  const int64_t len = keys ? a->k_len : a->q_len;
  return a->q_offsets ? std::min(len, keys ? a->k_tokens : a->q_tokens) : len;
}

Operand operand(const void* at, const arrow_strides_t& s) { return {at, s.sequence, s.token, s.head}; }

AttentionArgs plan(const arrow_attention_t* a) {
  AttentionArgs p{};
  p.q_offsets = a->q_offsets; p.k_offsets = a->k_offsets;
  p.q_tokens = a->q_tokens; p.k_tokens = a->k_tokens;
  p.batch = a->batch; p.q_heads = a->q_heads; p.kv_heads = a->kv_heads; p.group = a->q_heads / a->kv_heads;
  p.dim = a->dim; p.q_len = a->q_len; p.k_len = a->k_len; p.scale = a->scale;
  p.window = a->window < a->k_len ? a->window : 0;   // one as long as any sequence hides nothing
  p.sinks = p.window ? std::min(a->sinks, a->k_len) : 0;
  // Gradients of keys: a workgroup has the queries that see a tile of keys, in steps of 64 queries of a head.
  const int64_t tiles = ceil_div(a->k_len, kKeyTile), all = ceil_div(a->q_len, kQueryStep) * p.group;
  const int64_t usual = p.window ? std::min(all, (ceil_div((int64_t)p.window + kKeyTile, kQueryStep) + 1) * p.group) : all;
  // Workgroups of 32 keys, whose wavefronts take the steps in turn, are faster than ones of 128 where there are few of those and each has
  // few steps (gradients in us, of 128 -> of 32 keys, heads of 64 and of 128):
  //   32 workgroups of 8 steps 28 -> 24, 47 -> 36;  64 of 7 steps 36 -> 31, 58 -> 48;  64 of 32 steps 40 -> 42, 69 -> 69
  //   128 of 7 steps 38 -> 45, 63 -> 68;  16 of 32 steps, cut into parts, 33 -> 38, 55 -> 57
  // They are not cut into parts, and keys that all queries see have more steps than the others (4 sinks, window of 256):
  //   16 steps 33 -> 28, 45 -> 38;  32 steps 34 -> 41, 46 -> 55;  64 steps 35 -> 66, 51 -> 93
  p.tile_parts = p.sink_parts = 1;
  p.few_keys = tiles * a->kv_heads * a->batch <= 64 && usual > 1 && usual <= 16 && (p.sinks == 0 || all <= 24);
  if (p.few_keys) return p;
  p.sink_tiles = (int32_t)std::min(tiles, ceil_div(p.sinks, kKeyTile));
  // A tile is cut into parts where that fills the chip better: the time goes by the rounds of workgroups that it holds at once, and a
  // part costs about as much as kPartSteps steps more, for its sums on their way through memory.
  constexpr int64_t kSlots = 512, kPartSteps = 10;
  const int64_t items = std::max<int64_t>(1, (tiles - p.sink_tiles) * a->kv_heads * a->batch);
  int64_t best = INT64_MAX;
  for (int32_t n = 1; n <= 16 && (n == 1 || usual / n >= 4); ++n) {
    const int64_t time = ceil_div(items * n, kSlots) * (ceil_div(usual, n) + (n > 1 ? kPartSteps : 0));
    if (time < best) { best = time; p.tile_parts = n; }
  }
  // Keys that every later query sees have far more queries than the others.  Their parts are small and come last, to fill what others leave.
  p.sink_parts = p.sink_tiles ? (int32_t)std::max<int64_t>(p.tile_parts, std::min<int64_t>(64, ceil_div(all, std::max<int64_t>(8, usual / 4)))) : 1;
  return p;
}

// Sums of parts in the workspace: a pair of them (dk, dv) for each part of a tile that is cut.
int64_t pairs_of(const AttentionArgs& p) {
  const int64_t tiles = ceil_div(p.k_len, kKeyTile);
  const int64_t a = p.sink_parts > 1 ? (int64_t)p.sink_tiles * p.sink_parts : 0, b = p.tile_parts > 1 ? (tiles - p.sink_tiles) * p.tile_parts : 0;
  return (a + b) * p.kv_heads * p.batch;
}

size_t align_up(size_t x) { return (x + 255) / 256 * 256; }

size_t rows_bytes(const arrow_attention_t* a) {
  const int64_t rows = a->q_offsets ? a->q_tokens * a->q_heads : (int64_t)a->batch * a->q_heads * a->q_len;
  return align_up((size_t)rows * 4);
}

// Notes of every 32 queries (groups_at of attention_grad.hip).
size_t notes_bytes(const arrow_attention_t* a) {
  if (a->dtype != ARROW_F16) return 0;
  const int64_t groups = a->q_offsets ? (a->q_tokens / 32 + a->batch) * a->q_heads : (int64_t)a->batch * a->q_heads * ceil_div(a->q_len, 32);
  return align_up((size_t)groups * 4);
}

int check_cache(const arrow_cache_t* c, const void* k_pool, const void* v_pool) {
  if (!c) return refuse(ARROW_EINVAL, "NULL cache");
  if (int rc = check_heads(c->dtype, c->batch, c->q_heads, c->kv_heads, c->dim, c->window, c->sinks, c->scale)) return rc;
  if (c->page < 1 || (c->page & (c->page - 1)) || c->page > (1 << 20)) return refuse(ARROW_EINVAL, "page = %d is no power of two up to 2^20", c->page);
  if (c->columns < 0 || (int64_t)c->columns * c->page > kMostTokens)
    return refuse(ARROW_EINVAL, "columns = %d of %d tokens each: 0 .. %d tokens", c->columns, c->page, kMostTokens);
  if (c->pages < 0 || c->pages > 0x7fffffff || c->max_len < 0)
    return refuse(ARROW_EINVAL, "pages = %lld, max_len = %lld", (long long)c->pages, (long long)c->max_len);
  if (c->batch == 0) return ARROW_OK;
  if (!c->lengths || (c->columns && !c->table)) return refuse(ARROW_EINVAL, "table or lengths is NULL");
  const struct { const char* name; const void* at; int64_t page, token, head; } pools[2] = {{"k_pool", k_pool, c->k_page, c->k_token, c->k_head},
                                                                                           {"v_pool", v_pool, c->v_page, c->v_token, c->v_head}};
  for (auto& m : pools) {
    if (c->pages && !m.at) return refuse(ARROW_EINVAL, "%s is NULL", m.name);
    if ((uintptr_t)m.at % 16) return refuse(ARROW_EINVAL, "%s is not 16-byte aligned", m.name);
    if (m.page % 8 || m.token % 8 || m.head % 8 || m.page < 0 || m.token < 0 || m.head < 0)
      return refuse(ARROW_EINVAL, "%s: steps of %lld, %lld, %lld elements are not multiples of 8", m.name, (long long)m.page, (long long)m.token,
                    (long long)m.head);
    if ((c->pages > 1 && m.page < c->dim) || (c->page > 1 && m.token < c->dim) || (c->kv_heads > 1 && m.head < c->dim))
      return refuse(ARROW_EINVAL, "%s is written, and its rows overlap", m.name);
  }
  if (k_pool && k_pool == v_pool) return refuse(ARROW_EINVAL, "k_pool and v_pool are the same");
  return ARROW_OK;
}

CacheArgs plan(const arrow_cache_t* c) {
  CacheArgs p{};
  p.c = *c;
  p.group = c->q_heads / c->kv_heads;
  while ((1 << p.page_log) < c->page) ++p.page_log;
  const int64_t room = (int64_t)c->columns * c->page;
  p.c.window = c->window < room ? c->window : 0;     // one as long as any sequence hides nothing
  p.c.sinks = p.c.window ? (int32_t)std::min<int64_t>(c->sinks, room) : 0;
  int64_t seen = std::min(c->max_len, room);
  if (p.c.window) seen = std::min(seen, (int64_t)p.c.window + p.c.sinks);
  const int64_t rows = std::max<int64_t>(1, (int64_t)c->batch * c->kv_heads * ceil_div(p.group, kHeadTile));
  // Stretches of the visible keys.  A workgroup takes some 14 ns per key where it has the chip to itself, the join 35 ns per stretch, so that the square root
  // of 0.4 `seen` of them take the least time together, and one where another launch is not worth it.  Where there are many rows, so many that the
  // chip is full: two workgroups to a compute unit where rows see equally many keys, as under a window, and otherwise, to even lengths out, four, and
  // stretches of up to 2048 keys (us):
  //   2 rows of 8000 keys: 16 stretches 15.0, 48 11.6, 64 11.4, 128 12.7, 256 18.1;  of 125 keys: 1 6.8, 2 8.4
  //   32 rows of 4000 .. 16,000: 16 38.4, 32 36.8, 64 39.4, 128 46.3;  128 of 500 .. 2000: 1 33.6, 4 22.6, 8 22.4, 16 23.5, 32 29.5
  //   256 rows, window of 4096: 1 69.4, 2 54.0, 4 63.9, 16 63.2;  128 rows 1 74.2, 2 52.0, 4 55.0, 8 58.8;  256 of 4000 .. 16,000: 4 295, 8 282, 16 280
  const int64_t full = p.c.window ? 512 / rows : std::max(1024 / rows, ceil_div(seen, 2048)), best = (int64_t)std::sqrt(0.4 * (double)seen);
  // A round of a workgroup's wavefronts is 64 keys: no more stretches than the longest ones' number of rounds needs.
  const int64_t rounds = std::max<int64_t>(1, ceil_div(seen, 64)), most = std::max<int64_t>(1, std::min<int64_t>({kMostSplits, full, best, rounds}));
  p.splits = seen <= 192 ? 1 : (int32_t)ceil_div(rounds, ceil_div(rounds, most));
  return p;
}

// Parts of rows in the workspace: their sums, maxima and totals.
size_t forward_bytes(const AttentionArgs& p) {
  const int64_t splits = attention_forward_splits(p);
  return splits > 1 ? align_up((size_t)p.batch * p.q_heads * p.q_len * splits * (p.dim + 2) * 4) : 0;
}

int forward(const arrow_attention_t* a, const void* q, const void* k, const void* v, void* o, float* lse, bool cut, void* ws, size_t ws_bytes, void* stream) {
  if (int rc = check(a)) return rc;
  const bool ragged = a->q_offsets != nullptr;
  const int64_t nq = tokens_of(a, false), nk = tokens_of(a, true);
  if (nq == 0) return ARROW_OK;
  if (int rc = check_operand("q", q, a->q, nq, a->q_heads, a->batch, ragged, a->dim, false)) return rc;
  if (int rc = check_operand("k", k, a->k, nk, a->kv_heads, a->batch, ragged, a->dim, false)) return rc;
  if (int rc = check_operand("v", v, a->v, nk, a->kv_heads, a->batch, ragged, a->dim, false)) return rc;
  if (int rc = check_operand("o", o, a->o, nq, a->q_heads, a->batch, ragged, a->dim, true)) return rc;
  if (o == q || o == k || o == v) return refuse(ARROW_EINVAL, "o is one of the inputs");
  if ((uintptr_t)lse % 4) return refuse(ARROW_EINVAL, "lse is not 4-byte aligned");
  AttentionArgs p = plan(a);
  p.q = operand(q, a->q); p.k = operand(k, a->k); p.v = operand(v, a->v); p.o = operand(o, a->o);
  p.lse = lse;
  p.splits = 1;
  if (cut) {
    const size_t need = forward_bytes(p);
    if (need && (!ws || (uintptr_t)ws % 256)) return refuse(ARROW_EINVAL, "workspace is NULL or not 256-byte aligned");
    if (ws_bytes < need) return refuse(ARROW_ETOOSMALL, "workspace of %zu bytes, %zu are needed", ws_bytes, need);
    p.splits = attention_forward_splits(p);
    p.parts = (float*)ws;
  }
  return launched("attention forward", launch_attention_forward(p, a->dtype, stream));
}

}  // namespace

extern "C" {

int arrow_attention_forward(const arrow_attention_t* a, const void* q, const void* k, const void* v, void* o, float* lse, void* stream) {
  return forward(a, q, k, v, o, lse, false, nullptr, 0, stream);
}

size_t arrow_attention_forward_split_bytes(const arrow_attention_t* a) {
  if (check(a) || tokens_of(a, false) == 0) return 0;
  return forward_bytes(plan(a));
}

int arrow_attention_forward_split(const arrow_attention_t* a, const void* q, const void* k, const void* v, void* o, float* lse, void* ws, size_t ws_bytes,
                                  void* stream) {
  return forward(a, q, k, v, o, lse, true, ws, ws_bytes, stream);
}

size_t arrow_attention_workspace_bytes(const arrow_attention_t* a) {
  if (check(a)) return 0;
  return 2 * rows_bytes(a) + notes_bytes(a) + align_up((size_t)pairs_of(plan(a)) * 2 * kKeyTile * a->dim * 4);
}

int arrow_attention_backward(const arrow_attention_t* a, const void* q, const void* k, const void* v, const void* o, const float* lse,
                             const void* d_o, void* dq, void* dk, void* dv, void* ws, size_t ws_bytes, void* stream) {
  if (int rc = check(a)) return rc;
  const bool ragged = a->q_offsets != nullptr;
  const int64_t nq = tokens_of(a, false), nk = tokens_of(a, true);
  const struct { const char* name; const void* at; const arrow_strides_t& s; int64_t n; int32_t heads; bool written; } all[] = {
      {"q", q, a->q, nq, a->q_heads, false}, {"k", k, a->k, nk, a->kv_heads, false}, {"v", v, a->v, nk, a->kv_heads, false},
      {"o", o, a->o, nq, a->q_heads, false}, {"d_o", d_o, a->d_o, nq, a->q_heads, false}, {"dq", dq, a->dq, nq, a->q_heads, true},
      {"dk", dk, a->dk, nk, a->kv_heads, true}, {"dv", dv, a->dv, nk, a->kv_heads, true}};
  for (auto& m : all)
    if (int rc = check_operand(m.name, m.at, m.s, m.n, m.heads, a->batch, ragged, a->dim, m.written)) return rc;
  if (nq == 0 && nk == 0) return ARROW_OK;
  for (auto& out : all)
    for (auto& other : all)
      if (out.written && &out != &other && out.n && other.n && out.at == other.at) return refuse(ARROW_EINVAL, "%s and %s are the same", out.name, other.name);
  if (nq && (!lse || (uintptr_t)lse % 4)) return refuse(ARROW_EINVAL, "lse is NULL or not 4-byte aligned");
  const size_t need = arrow_attention_workspace_bytes(a);
  if (need && (!ws || (uintptr_t)ws % 256)) return refuse(ARROW_EINVAL, "workspace is NULL or not 256-byte aligned");
  if (ws_bytes < need) return refuse(ARROW_ETOOSMALL, "workspace of %zu bytes, %zu are needed", ws_bytes, need);
  AttentionArgs p = plan(a);
  p.q = operand(q, a->q); p.k = operand(k, a->k); p.v = operand(v, a->v); p.o = operand(o, a->o); p.d_o = operand(d_o, a->d_o);
  p.dq = operand(dq, a->dq); p.dk = operand(dk, a->dk); p.dv = operand(dv, a->dv);
  p.lse_in = lse;
  p.off = (float*)ws;
  p.delta = (float*)((char*)ws + rows_bytes(a));
  p.most = (float*)((char*)ws + 2 * rows_bytes(a));
  p.parts = (float*)((char*)ws + 2 * rows_bytes(a) + notes_bytes(a));
  return launched("attention backward", launch_attention_backward(p, a->dtype, stream));
}

int arrow_cache_append(const arrow_cache_t* c, int32_t tokens, const void* k, const void* v, arrow_strides_t ks, arrow_strides_t vs,
                       void* k_pool, void* v_pool, void* stream) {
  if (int rc = check_cache(c, k_pool, v_pool)) return rc;
  if (tokens < 0 || tokens > kMostTokens) return refuse(ARROW_EINVAL, "tokens = %d", tokens);
  if (c->batch == 0 || tokens == 0 || c->pages == 0 || c->columns == 0) return ARROW_OK;
  if (int rc = check_operand("k", k, ks, tokens, c->kv_heads, c->batch, false, c->dim, false)) return rc;
  if (int rc = check_operand("v", v, vs, tokens, c->kv_heads, c->batch, false, c->dim, false)) return rc;
  CacheArgs p = plan(c);
  p.k = operand(k, ks); p.v = operand(v, vs);
  p.k_pool = k_pool; p.v_pool = v_pool;
  p.tokens = tokens;
  return launched("cache append", launch_cache_append(p, stream));
}

size_t arrow_attention_decode_workspace_bytes(const arrow_cache_t* c) {
  if (!c || c->batch < 1 || c->kv_heads < 1 || c->q_heads < 1 || c->q_heads % c->kv_heads || c->dim < 1 || c->page < 1 || c->page > (1 << 20)) return 0;
  const CacheArgs p = plan(c);
  return p.splits == 1 ? 0 : align_up((size_t)p.splits * c->batch * c->q_heads * (c->dim + 2) * 4);
}

int arrow_attention_decode(const arrow_cache_t* c, const void* q, arrow_strides_t qs, const void* k, const void* v, arrow_strides_t ks,
                           arrow_strides_t vs, void* k_pool, void* v_pool, void* o, arrow_strides_t os, void* ws, size_t ws_bytes, void* stream) {
  if (int rc = check_cache(c, k_pool, v_pool)) return rc;
  if (c->batch == 0) return ARROW_OK;
  if (!k != !v) return refuse(ARROW_EINVAL, "k and v of the new token: both or neither");
  qs.token = ks.token = vs.token = os.token = 0;
  if (int rc = check_operand("q", q, qs, 1, c->q_heads, c->batch, false, c->dim, false)) return rc;
  if (int rc = check_operand("o", o, os, 1, c->q_heads, c->batch, false, c->dim, true)) return rc;
  if (k)
    if (int rc = check_operand("k", k, ks, 1, c->kv_heads, c->batch, false, c->dim, false)) return rc;
  if (v)
    if (int rc = check_operand("v", v, vs, 1, c->kv_heads, c->batch, false, c->dim, false)) return rc;
  if (o == q || o == k || o == v || o == k_pool || o == v_pool) return refuse(ARROW_EINVAL, "o is one of the inputs");
  const size_t need = arrow_attention_decode_workspace_bytes(c);
  if (need && (!ws || (uintptr_t)ws % 256)) return refuse(ARROW_EINVAL, "workspace is NULL or not 256-byte aligned");
  if (ws_bytes < need) return refuse(ARROW_ETOOSMALL, "workspace of %zu bytes, %zu are needed", ws_bytes, need);
  CacheArgs p = plan(c);
  p.q = operand(q, qs); p.k = operand(k, ks); p.v = operand(v, vs); p.o = operand(o, os);
  p.k_pool = k_pool; p.v_pool = v_pool;
  p.parts = (float*)ws;
  return launched("attention decode", launch_attention_decode(p, stream));
}

}  // extern "C"
