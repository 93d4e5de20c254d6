// What the C entries of the operators on sequences have in common: refusals with a text, checks of addresses.
// Everything has internal linkage; include inside a .cpp file only.
#pragma once

#include <hip/hip_runtime_api.h>

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

}  // namespace
}  // namespace arrow
