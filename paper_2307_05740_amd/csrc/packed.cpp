// C boundary of the entries of include/arrow_packed.h: checks of the arguments, the plan of a call.
#include <algorithm>
#include <cmath>

#include "checks.h"
#include "packed_internal.h"

namespace {

using namespace arrow;

constexpr int32_t kMostTokens = 1 << 26;    // of a sequence

constexpr int64_t kMostStep = (int64_t)1 << 56;

Rows pool_of(const arrow_packed_t* c, const void* pool) {
  return {c->pages ? pool : nullptr, (int64_t)c->page * (c->dim + c->dim / 16), {c->pages, c->page_step}, {c->kv_heads, c->head_step}};
}

int check_pool(const arrow_packed_t* c, const void* pool) {
  if (!c) return refuse(ARROW_EINVAL, "NULL arguments");
  if (c->dtype != ARROW_BF16 && c->dtype != ARROW_F16) return refuse(ARROW_EINVAL, "dtype %d: a cache in 4 bits takes ARROW_BF16 and ARROW_F16", c->dtype);
  if (c->kv_heads < 1 || c->kv_heads > 65536) return refuse(ARROW_EINVAL, "kv_heads = %d: 1 .. 65536", c->kv_heads);
  if (c->dim != 32 && c->dim != 64 && c->dim != 128) return refuse(ARROW_EINVAL, "dim = %d is none of 32, 64, 128", c->dim);
  if (c->page < 16 || (c->page & (c->page - 1)) || c->page > (1 << 20)) return refuse(ARROW_EINVAL, "page = %d is no power of two from 16 to 2^20", c->page);
  if (c->pages < 0 || c->pages > 0x7fffffff) return refuse(ARROW_EINVAL, "pages = %lld", (long long)c->pages);
  if (c->pages == 0) return ARROW_OK;
  if (int rc = check_pointer("pool", pool, 16)) return rc;
  const int64_t block = (int64_t)c->page * (c->dim + c->dim / 16);
  if (c->page_step % 16 || c->head_step % 16 || c->page_step < 0 || c->head_step < 0 || c->page_step > kMostStep || c->head_step > kMostStep || !pool_of(c, pool).distinct())
    return refuse(ARROW_EINVAL, "pool: blocks %lld and %lld bytes apart, multiples of 16 from %lld expected that do not overlap", (long long)c->page_step,
                  (long long)c->head_step, (long long)block);
  return ARROW_OK;
}

Rows rows_of(const arrow_packed_t* c, const void* at, int64_t row, int64_t head, int64_t rows, int32_t heads) { return {at, c->dim * 2, {rows, row * 2}, {heads, head * 2}}; }

int check_rows(const arrow_packed_t* c, const char* name, const void* at, int64_t row, int64_t head, int64_t rows, int32_t heads, bool written) {
  if (int rc = check_pointer(name, at, 16)) return rc;
  if (row % 8 || head % 8 || row < 0 || head < 0 || row > kMostStep || head > kMostStep)
    return refuse(ARROW_EINVAL, "%s: steps of %lld and %lld elements are not multiples of 8", name, (long long)row, (long long)head);
  if (written && !rows_of(c, at, row, head, rows, heads).distinct()) return refuse(ARROW_EINVAL, "%s is written, and its rows overlap", name);
  return ARROW_OK;
}

int check_places(const arrow_packed_t* c, int64_t tokens, const int64_t* slots) {
  if (tokens < 0 || tokens > 0x7fffffff) return refuse(ARROW_EINVAL, "tokens = %lld: 0 .. 2^31 - 1", (long long)tokens);
  if (tokens == 0) return ARROW_OK;
  (void)c;
  return check_pointer("slots", slots, 8);
}

PackedArgs plan(const arrow_packed_t* c) {
  PackedArgs p{};
  p.c = *c;
  while ((1 << p.page_log) < c->page) ++p.page_log;
  return p;
}

int check_decode(const arrow_packed_t* c) {
  if (c->batch < 0) return refuse(ARROW_EINVAL, "batch = %d", c->batch);
  if (c->q_heads < 1 || c->q_heads % c->kv_heads) return refuse(ARROW_EINVAL, "q_heads = %d is no multiple of kv_heads = %d", c->q_heads, c->kv_heads);
  if ((int64_t)c->batch * c->q_heads > kMostBlocks) return refuse(ARROW_EINVAL, "batch = %d with q_heads = %d: 2^24 - 1 rows at most", c->batch, c->q_heads);
  if (c->window < 0 || c->sinks < 0) return refuse(ARROW_EINVAL, "window = %d, sinks = %d", c->window, c->sinks);
  if (!(c->scale > 0.f) || !std::isfinite(c->scale)) return refuse(ARROW_EINVAL, "scale = %g is not positive and finite", c->scale);
  if (c->columns < 0 || (int64_t)c->columns * c->page > kMostTokens)
    return refuse(ARROW_EINVAL, "columns = %d of %d tokens each: 0 .. %d tokens", c->columns, c->page, kMostTokens);
  if (c->max_len < 0) return refuse(ARROW_EINVAL, "max_len = %lld", (long long)c->max_len);
  if (c->batch == 0) return ARROW_OK;
  if (!c->lengths || (c->columns && !c->table)) return refuse(ARROW_EINVAL, "table or lengths is NULL");
  if ((uintptr_t)c->lengths % 4 || (uintptr_t)c->table % 4) return refuse(ARROW_EINVAL, "table or lengths is not 4-byte aligned");
  return ARROW_OK;
}

PackedArgs plan_decode(const arrow_packed_t* c) {
  PackedArgs p = plan(c);
  p.group = c->q_heads / c->kv_heads;
  const int64_t room = (int64_t)c->columns * c->page;
  p.c.window = c->window < room ? c->window : 0;     // one as long as any sequence hides nothing
  p.c.sinks = p.c.window ? (int32_t)std::min<int64_t>(c->sinks, room) : 0;
  if (c->pages == 0) p.c.columns = 0;
  int64_t seen = std::min(c->max_len, room);
  if (p.c.window) seen = std::min(seen, (int64_t)p.c.window + p.c.sinks);
  const int64_t rows = std::max<int64_t>(1, (int64_t)c->batch * c->kv_heads * ceil_div(p.group, kHeadTile));
  // Stretches of the visible keys, each a workgroup of four wavefronts; more than one take another launch, for their join.
  const bool equal = p.c.window != 0;               // (sequences that are longer than it see equally many keys; of those that are not, lengths are not known here)
  p.waves = 4;
  p.splits = 1;
  if (seen <= 512) return p;                        // (2 to 256 rows of up to 400 keys: 6.7 to 8.8 us, in two stretches 9.7 to 11.4)
  // One stretch, of eight wavefronts where these and not workgroups are what fills the chip; us, one stretch of four wavefronts, of eight, and the best of several of four:
  //   heads of 64, 128 rows of up to 1000 keys 9.0 8.5 9.8, of 2000 14 12.0 11.5; 256 of 2000 14 12.0 15, of 4000 26 19 21; 512 of 4000 34 29 32, of 8000 59 48 45; 1024 of 1000 17 21 26
  //   heads of 128, 2 rows of 1000 10.0 9.6 8.4; 160 of 1500 - 12.3 13.6, of 5000 - 28.2 23.9; 256 of 4000 31 24 26; 1024 of 8000 142 140 147
  //   under a window of 4096, 256 rows, heads of 64 28 20.7 24.6, of 128 34 26.4 30.1
  const bool eight = seen <= 1024 ? rows < 512 && (rows >= 64 || c->dim <= 64) : equal ? rows >= 192 && rows <= 768 : rows >= 160 && rows <= 768 && seen <= (rows < 192 ? 2000 : 6000);
  if (eight) {
    p.waves = 8;
    return p;
  }
  if (rows >= 512 && (equal || seen <= (rows > 768 ? 12000 : 6000))) return p;
  // Several: as many as give two workgroups to a compute unit; where lengths differ, of about 1000 keys each, and 2000 beyond eight, or where there are many rows, 2500, and 6000
  // beyond four; at most the square root of a tenth of `seen`, which is what their join is worth for few rows; no more than there are rounds of 128 keys.
  //   128 rows of up to 16,000 keys, heads of 64, 4 stretches 34.5, 8 26.0; of 128, 41.7, 33.2; 256 of 8000, heads of 64, 2 36, 4 30, 8 30; 512 of 16,000, 3 99, 4 92, 8 95, of 30,000 5 165, 15 171
  //   8 rows of 60,000, heads of 128, 16 33.1, 32 21.9, 64 20.1, 128 23.4;  2 of 1000, 4 8.4, 8 8.0, 16 7.8, 64 9.2
  const int64_t even = equal ? 1 : rows > 768 ? ceil_div(seen, 4000) : rows >= 384 ? std::max(std::min<int64_t>(4, ceil_div(seen, 2500)), ceil_div(seen, 6000))
                                                                                    : std::max(std::min<int64_t>(8, seen / 1000), ceil_div(seen, 2000));
  const int64_t rounds = ceil_div(seen, 128), best = (int64_t)std::sqrt(0.1 * (double)seen);
  const int64_t most = std::max<int64_t>(1, std::min<int64_t>({kMostSplits, std::max(512 / rows, even), best, rounds, kMostBlocks / rows}));
  p.splits = (int32_t)ceil_div(rounds, ceil_div(rounds, most));
  return p;
}

Operand operand(const void* at, const arrow_strides_t& s) { return {at, s.sequence, s.token, s.head}; }

}  // namespace

extern "C" {

int arrow_packed_append(const arrow_packed_t* c, int64_t tokens, const void* k, const void* v, arrow_strides_t ks, arrow_strides_t vs, const int64_t* slots,
                        void* pool, void* stream) {
  if (int rc = check_pool(c, pool)) return rc;
  if (int rc = check_places(c, tokens, slots)) return rc;
  if (tokens == 0) return ARROW_OK;
  if (int rc = check_rows(c, "k", k, ks.token, ks.head, tokens, c->kv_heads, false)) return rc;
  if (int rc = check_rows(c, "v", v, vs.token, vs.head, tokens, c->kv_heads, false)) return rc;
  if (pool && (k == pool || v == pool)) return refuse(ARROW_EINVAL, "k or v is the pool");
  if (c->pages == 0) return ARROW_OK;
  const Part all[] = {{"the pool", pool_of(c, pool), true, -1}, {"k", rows_of(c, k, ks.token, ks.head, tokens, c->kv_heads), false, -1},
                      {"v", rows_of(c, v, vs.token, vs.head, tokens, c->kv_heads), false, -1}, {"slots", {slots, tokens * 8}, false, -1}};
  if (int rc = check_apart(all)) return rc;
  PackedArgs p = plan(c);
  p.k = operand(k, ks); p.v = operand(v, vs);
  p.pool = pool; p.slots = slots; p.tokens = tokens;
  return launched("packed append", launch_packed_append(p, stream));
}

int arrow_packed_read(const arrow_packed_t* c, int64_t tokens, const int64_t* slots, const void* pool, void* k, void* v, arrow_strides_t ks, arrow_strides_t vs,
                      void* stream) {
  if (int rc = check_pool(c, pool)) return rc;
  if (int rc = check_places(c, tokens, slots)) return rc;
  if (tokens == 0) return ARROW_OK;
  if (int rc = check_rows(c, "k", k, ks.token, ks.head, tokens, c->kv_heads, true)) return rc;
  if (int rc = check_rows(c, "v", v, vs.token, vs.head, tokens, c->kv_heads, true)) return rc;
  if (k == v || (pool && (k == pool || v == pool))) return refuse(ARROW_EINVAL, "k or v is the other or the pool");
  const Part all[] = {{"the pool", pool_of(c, pool), false, -1}, {"k", rows_of(c, k, ks.token, ks.head, tokens, c->kv_heads), true, -1},
                      {"v", rows_of(c, v, vs.token, vs.head, tokens, c->kv_heads), true, -1}, {"slots", {slots, tokens * 8}, false, -1}};
  if (int rc = check_apart(all)) return rc;
  PackedArgs p = plan(c);
  p.k = operand(k, ks); p.v = operand(v, vs);
  p.pool = const_cast<void*>(pool); p.slots = slots; p.tokens = tokens;
  return launched("packed read", launch_packed_read(p, stream));
}

size_t arrow_packed_decode_workspace_bytes(const arrow_packed_t* c) {
  if (!c || c->batch < 1 || c->kv_heads < 1 || c->q_heads < 1 || c->q_heads % c->kv_heads || c->dim < 1 || c->dim > 128 || c->page < 1 || c->page > (1 << 20)) return 0;
  const PackedArgs p = plan_decode(c);
  return p.splits == 1 ? 0 : align_up((size_t)p.splits * c->batch * c->q_heads * (c->dim + 2) * 4);
}

int arrow_packed_decode(const arrow_packed_t* c, const void* q, arrow_strides_t qs, const void* k, const void* v, arrow_strides_t ks, arrow_strides_t vs, void* pool,
                        void* o, arrow_strides_t os, void* ws, size_t ws_bytes, void* stream) {
  if (int rc = check_pool(c, pool)) return rc;
  if (int rc = check_decode(c)) return rc;
  if (c->batch == 0) return ARROW_OK;
  if (!k != !v) return refuse(ARROW_EINVAL, "k and v of the new token: both or neither");
  if (int rc = check_rows(c, "q", q, qs.sequence, qs.head, c->batch, c->q_heads, false)) return rc;
  if (int rc = check_rows(c, "o", o, os.sequence, os.head, c->batch, c->q_heads, true)) return rc;
  if (k) {
    if (int rc = check_rows(c, "k", k, ks.sequence, ks.head, c->batch, c->kv_heads, false)) return rc;
    if (int rc = check_rows(c, "v", v, vs.sequence, vs.head, c->batch, c->kv_heads, false)) return rc;
  }
  if (o == q || o == k || o == v || (pool && o == pool)) return refuse(ARROW_EINVAL, "o is one of the inputs");
  PackedArgs p = plan_decode(c);
  const size_t need = arrow_packed_decode_workspace_bytes(c);
  if (int rc = check_workspace(ws, ws_bytes, need)) return rc;
  const Part all[] = {{"o", rows_of(c, o, os.sequence, os.head, c->batch, c->q_heads), true, -1}, {"the pool", pool_of(c, pool), k != nullptr, -1},
                      {"the workspace", {need ? ws : nullptr, (int64_t)need}, true, -1}, {"q", rows_of(c, q, qs.sequence, qs.head, c->batch, c->q_heads), false, -1},
                      {"k", rows_of(c, k, ks.sequence, ks.head, c->batch, c->kv_heads), false, -1}, {"v", rows_of(c, v, vs.sequence, vs.head, c->batch, c->kv_heads), false, -1},
                      {"table", {c->table, (int64_t)c->batch * c->columns * 4}, false, -1}, {"lengths", {c->lengths, (int64_t)c->batch * 4}, false, -1}};
  if (int rc = check_apart(all)) return rc;
  p.q = operand(q, qs); p.o = operand(o, os);
  p.k = operand(k, ks); p.v = operand(v, vs);
  p.k.token = ks.sequence; p.v.token = vs.sequence;      // (a token of each sequence)
  p.pool = pool;
  p.tokens = c->batch;
  p.parts = (float*)ws;
  if (k && c->pages)
    if (int rc = launched("packed append", launch_packed_append(p, stream))) return rc;
  return launched("packed decode", launch_packed_decode(p, stream));
}

}  // extern "C"
