// C boundary of the entry of include/arrow_pages.h: checks of the arguments, the plan of a step.
#include <algorithm>

#include "checks.h"
#include "pages_internal.h"

namespace {

using namespace arrow;

int check(const arrow_pages_t* a) {
  if (!a) return refuse(ARROW_EINVAL, "NULL arguments");
  if (a->batch < 0 || a->batch > (1 << 24)) return refuse(ARROW_EINVAL, "batch = %d: 0 .. 2^24", a->batch);
  if (a->page < 1 || (a->page & (a->page - 1)) || a->page > (1 << 20)) return refuse(ARROW_EINVAL, "page = %d is no power of two up to 2^20", a->page);
  if (a->columns < 0 || (int64_t)a->columns * a->page > (1 << 26))
    return refuse(ARROW_EINVAL, "columns = %d of %d tokens each: 0 .. 2^26 tokens", a->columns, a->page);
  if ((int64_t)a->batch * a->columns > 0x7fffffff) return refuse(ARROW_EINVAL, "a table of %d x %d entries: 2^31 - 1 at most", a->batch, a->columns);
  if (a->window < 0 || a->sinks < 0) return refuse(ARROW_EINVAL, "window = %d, sinks = %d", a->window, a->sinks);
  if (a->pages < 0 || a->pages > (1 << 30)) return refuse(ARROW_EINVAL, "pages = %lld: 0 .. 2^30", (long long)a->pages);
  if (a->offsets ? a->rows < 0 || a->rows > 0x7fffffff : a->tokens < 0 || (int64_t)a->tokens * a->batch > 0x7fffffff)
    return refuse(ARROW_EINVAL, "tokens = %d, rows = %lld: 0 .. 2^31 - 1 of all sequences", a->tokens, (long long)a->rows);
  return ARROW_OK;
}

PagesArgs plan(const arrow_pages_t* a) {
  PagesArgs p{};
  p.a = *a;
  while ((1 << p.page_log) < a->page) ++p.page_log;
  p.rows = a->offsets ? a->rows : (int64_t)a->batch * a->tokens;
  const int64_t entries = (int64_t)a->batch * a->columns;
  p.one = a->batch <= kPagesBatch && p.rows <= kPagesRows && entries <= (p.rows ? kPagesEntries : kPagesBack);
  p.two = !p.one && a->batch <= kPagesBatch && entries <= kPagesFew;
  p.chunk = p.two ? std::max(1, a->columns) : 1024;
  p.chunks = (int32_t)std::max<int64_t>(1, ceil_div(a->columns, p.chunk));
  return p;
}

size_t each_bytes(const arrow_pages_t* a) { return align_up((size_t)a->batch * plan(a).chunks * 4); }

}  // namespace

extern "C" {

size_t arrow_pages_workspace_bytes(const arrow_pages_t* a) { return check(a) || plan(a).one ? 0 : 4 * each_bytes(a) + 256; }

int arrow_pages_step(const arrow_pages_t* a, const int32_t* lengths, int32_t* held, int32_t* table, int32_t* list, int64_t* slots, void* ws, size_t ws_bytes,
                     void* stream) {
  if (int rc = check(a)) return rc;
  PagesArgs p = plan(a);
  const struct { const char* name; const void* at; int64_t n; int size; bool written; } all[] = {
      {"lengths", lengths, a->batch, 4, false}, {"offsets", a->offsets, a->offsets ? (int64_t)a->batch + 1 : 0, 4, false}, {"held", held, a->batch, 4, true},
      {"table", table, (int64_t)a->batch * a->columns, 4, true}, {"list", list, 1 + a->pages, 4, true}, {"slots", slots, p.rows, 8, true}};
  for (auto& m : all) {
    if (m.n == 0) continue;
    if (int rc = check_pointer(m.name, m.at, m.size)) return rc;
    for (auto& other : all)
      if (m.written && &m != &other && overlap(m.at, m.n * m.size, other.at, other.n * other.size)) return refuse(ARROW_EINVAL, "%s and %s overlap", m.name, other.name);
  }
  if (int rc = check_workspace(ws, ws_bytes, arrow_pages_workspace_bytes(a))) return rc;
  if (a->batch == 0 && p.rows == 0) return ARROW_OK;
  p.lengths = lengths; p.held = held; p.table = table; p.list = list; p.slots = slots;
  if (!p.one) {
    p.before = (int32_t*)ws;
    p.given = (int32_t*)((char*)ws + each_bytes(a));
    p.taken = (int32_t*)((char*)ws + 2 * each_bytes(a));
    p.first = (int32_t*)((char*)ws + 3 * each_bytes(a));
    p.sizes = (int32_t*)((char*)ws + 4 * each_bytes(a));
  }
  return launched("pages step", launch_pages_step(p, stream));
}

}  // extern "C"
