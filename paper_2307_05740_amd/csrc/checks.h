// What the C entries of the operators on sequences have in common: refusals with a text, checks of addresses.
// Everything has internal linkage; include inside a .cpp file only.
#pragma once

#include <hip/hip_runtime_api.h>

#include <algorithm>
#include <cstdarg>
#include <cstdint>
#include <cstdio>

#include "arrow.h"
#include "arrow_attention.h"

namespace arrow {

// Sets the calling thread's arrow_last_error() text and returns `code` (abi.cpp).
int fail_text(int code, const char* text);

namespace {

[[maybe_unused]] int refuse(int code, const char* fmt, ...) {
  char text[256];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(text, sizeof text, fmt, ap);
  va_end(ap);
  return fail_text(code, text);
}

[[maybe_unused]] int launched(const char* what, int rc) {
  return rc == 0 ? ARROW_OK : refuse(ARROW_EHIP, "%s: %s", what, hipGetErrorString((hipError_t)rc));
}

[[maybe_unused]] int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
[[maybe_unused]] size_t align_up(size_t x) { return (x + 255) / 256 * 256; }
[[maybe_unused]] int size_of(int32_t dtype) { return dtype == ARROW_F32 ? 4 : 2; }
[[maybe_unused]] bool is_dtype(int32_t dtype) { return dtype == ARROW_F32 || dtype == ARROW_BF16 || dtype == ARROW_F16; }

[[maybe_unused]] int check_pointer(const char* name, const void* at, int align) {
  if (!at) return refuse(ARROW_EINVAL, "%s is NULL", name);
  if ((uintptr_t)at % align) return refuse(ARROW_EINVAL, "%s is not %d-byte aligned", name, align);
  return ARROW_OK;
}

[[maybe_unused]] int check_workspace(const void* ws, size_t have, size_t need) {
  if (need && (!ws || (uintptr_t)ws % 256)) return refuse(ARROW_EINVAL, "workspace is NULL or not 256-byte aligned");
  if (have < need) return refuse(ARROW_ETOOSMALL, "workspace of %zu bytes, %zu are needed", have, need);
  return ARROW_OK;
}

[[maybe_unused]] bool overlap(const void* a, int64_t na, const void* b, int64_t nb) {
  const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
  return na > 0 && nb > 0 && x < y + (uintptr_t)nb && y < x + (uintptr_t)na;
}

// Rows of `row` bytes at every sum of some steps (in bytes, not negative), each taken 0 .. count - 1 times.
struct Rows {
  static constexpr int64_t kMost = (int64_t)1 << 60;         // (larger reaches are cut: they are only compared)
  struct Step { int64_t count, bytes; };
  uintptr_t at;
  int64_t row, reach;                        // reach: bytes from the first to the last one
  int n = 0;
  bool repeat = false;                       // a step of nothing
  Step steps[3];
  Rows(const void* p, int64_t bytes) : at((uintptr_t)p), row(std::min(bytes, kMost)), reach(row) {}
  Rows(const void* p, int64_t bytes, Step a, Step b, Step c = {1, 0}) : Rows(p, bytes) {
    add(a);
    add(b);
    add(c);
  }
  void add(const Step& s) {
    if (s.count <= 1) return;
    if (s.bytes <= 0) { repeat = true; return; }
    reach += across(s);
    steps[n++] = s;
  }
  static int64_t across(const Step& s) {
    int64_t x;
    return __builtin_mul_overflow(s.count - 1, s.bytes, &x) ? kMost : std::min(x, kMost);
  }
  // the same with the longest step first
  Rows sorted() const {
    Rows r = *this;
    std::sort(r.steps, r.steps + n, [](const Step& a, const Step& b) { return a.bytes > b.bytes; });
    return r;
  }
  // (sorted:) bytes from the first to the last one of the steps from the i-th on
  int64_t extent(int i) const {
    int64_t all = row;
    for (; i < n; ++i) all += across(steps[i]);
    return all;
  }
  int64_t count(int i, int64_t step) const { return i < n && steps[i].bytes == step ? steps[i].count : 1; }
  // whether no two rows have a byte in common, where each step is as long as what the shorter ones reach over (others are taken to have)
  bool distinct() const {
    if (repeat) return false;
    const auto nested = [](const Rows& r) {
      int64_t inner = r.row;
      for (int i = r.n - 1; i >= 0; --i) {
        if (r.steps[i].bytes < inner) return false;
        inner += across(r.steps[i]);
      }
      return true;
    };
    return nested(*this) || nested(sorted());            // (mostly they come in that order)
  }
};

// Whether no row of `a` (both are sorted), of its steps from the i-th on, has a byte in common with one of `b`, from the j-th on, which begin `off` bytes behind them.  Exact where what is shorter than the
// longest step does not reach beyond it in either, as in views of one tensor; others that reach into each other are taken to overlap.
[[maybe_unused]] bool apart(const Rows& a, int i, const Rows& b, int j, int64_t off) {
  if (off >= a.extent(i) || off <= -b.extent(j)) return true;
  const int64_t step = std::max(i < a.n ? a.steps[i].bytes : 0, j < b.n ? b.steps[j].bytes : 0);
  if (step == 0) return false;
  const int64_t na = a.count(i, step), nb = b.count(j, step);
  if (i < a.n && a.steps[i].bytes == step) ++i;
  if (j < b.n && b.steps[j].bytes == step) ++j;
  const int64_t ea = a.extent(i), eb = b.extent(j);
  if (ea > step || eb > step) return false;
  // of the distances off + t step between what is left of the two, those that are near enough
  const int64_t rest = off % step, whole = off / step;      // (t + whole is -2 .. 2 then)
  for (int64_t t = -2; t <= 2; ++t) {
    const int64_t by = rest + t * step;
    if (by >= ea || by <= -eb || t - whole < 1 - na || t - whole > nb - 1) continue;
    if (!apart(a, i, b, j, by)) return false;
  }
  return true;
}
[[maybe_unused]] bool apart(const Rows& a, const Rows& b) {
  if (!a.at || !b.at || a.row <= 0 || b.row <= 0) return true;
  const int64_t off = (int64_t)(b.at - a.at);
  return off >= a.reach || off <= -b.reach || apart(a.sorted(), 0, b.sorted(), 0, off);
}

// Operands of a call; `in_place`: of the one that it may lie on with the same steps (-1: none).
struct Part {
  const char* name;
  Rows rows;
  bool written;
  int in_place;
};
template <size_t N>
[[maybe_unused]] int check_apart(const Part (&all)[N]) {
  for (size_t i = 0; i < N; ++i) {
    const Part& m = all[i];
    if (!m.written) continue;
    for (size_t j = 0; j < N; ++j) {
      const Part& o = all[j];
      if (o.rows.at >= m.rows.at + (uintptr_t)m.rows.reach || m.rows.at >= o.rows.at + (uintptr_t)o.rows.reach) continue;    // (nearly always)
      if (i == j || (m.in_place == (int)j && m.rows.at == o.rows.at)) continue;
      if (!apart(m.rows, o.rows)) return refuse(ARROW_EINVAL, "%s is written, and overlaps %s", m.name, o.name);
    }
  }
  return ARROW_OK;
}

}  // namespace
}  // namespace arrow
