// C boundary of the embedding entries (include/arrow_embedding.h): checks of the arguments, the plan of a gradient.
#include <hip/hip_runtime_api.h>

#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>

#include "arrow.h"
#include "embedding_internal.h"

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

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
int size_of(int32_t dtype) { return dtype == ARROW_F32 ? 4 : 2; }

int check(const arrow_embedding_t* e, bool grad) {
  if (!e) return refuse(ARROW_EINVAL, "NULL arguments");
  if (e->dtype != ARROW_F32 && e->dtype != ARROW_BF16 && e->dtype != ARROW_F16) return refuse(ARROW_EINVAL, "dtype %d", e->dtype);
  if (grad && e->grad_dtype != e->dtype && e->grad_dtype != ARROW_F32) return refuse(ARROW_EINVAL, "grad_dtype %d is neither dtype nor ARROW_F32", e->grad_dtype);
  if (e->id_bytes != 4 && e->id_bytes != 8) return refuse(ARROW_EINVAL, "id_bytes = %d is neither 4 nor 8", e->id_bytes);
  if (e->columns < 1 || e->columns > (1 << 24)) return refuse(ARROW_EINVAL, "columns = %d: 1 .. 2^24", e->columns);
  if (e->rows < 1 || e->rows > 0x7ffffffe) return refuse(ARROW_EINVAL, "rows = %lld: 1 .. 2^31 - 2", (long long)e->rows);
  if (e->tokens < 0 || e->tokens > (grad ? 1 << 30 : 0x7fffffff)) return refuse(ARROW_EINVAL, "tokens = %lld", (long long)e->tokens);
  if (e->w_stride < e->columns || e->y_stride < e->columns)
    return refuse(ARROW_EINVAL, "rows %lld and %lld elements apart, of %d columns", (long long)e->w_stride, (long long)e->y_stride, e->columns);
  if (!std::isfinite(e->scale)) return refuse(ARROW_EINVAL, "scale = %g", e->scale);
  return ARROW_OK;
}

int check_pointer(const char* name, const void* at, int align) {
  if (!at) return refuse(ARROW_EINVAL, "%s is NULL", name);
  if ((uintptr_t)at % align) return refuse(ARROW_EINVAL, "%s is not %d-byte aligned", name, align);
  return ARROW_OK;
}

bool overlap(const void* a, int64_t na, const void* b, int64_t nb) {
  const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
  return na > 0 && nb > 0 && x < y + (uintptr_t)nb && y < x + (uintptr_t)na;
}

int64_t extent(int64_t rows, int64_t stride, int32_t columns, int size) { return rows ? ((rows - 1) * stride + columns) * size : 0; }

}  // namespace

namespace arrow {

EmbeddingPlan plan_embedding(const arrow_embedding_t& e) {
  EmbeddingPlan p{};
  p.direct = e.tokens <= kDirectTokens && (e.rows <= kDirectTable || e.columns * size_of(e.dtype) >= 256);
  int bits = 1;
  while ((int64_t)1 << bits <= e.rows) ++bits;                 // ids 0 .. rows, the last one for those outside the table
  p.few = e.tokens <= kFewTokens;
  const int most = p.few ? kWideDigitBits : kDigitBits;
  p.passes = (bits + most - 1) / most;
  p.bits = (bits + p.passes - 1) / p.passes;
  p.block_tokens = std::max<int64_t>(kSortTokens, ceil_div(ceil_div(e.tokens, 1024), 64) * 64);
  p.blocks = ceil_div(e.tokens, p.block_tokens);
  const int64_t eights = std::max<int64_t>(1, ceil_div(e.tokens, 512 * kChunkTokens));
  p.chunk = kChunkTokens * std::max(std::min<int64_t>(4, eights), ceil_div(e.tokens, 16384 * kChunkTokens));
  p.chunks = ceil_div(e.tokens, p.chunk);
  p.padded = ceil_div(e.columns, 8) * 8;
  size_t at = 0;
  auto room = [&](int64_t n) { const size_t was = at; at += ((size_t)n * 4 + 255) / 256 * 256; return was; };
  for (int i = 0; i < 2; ++i) { p.keys[i] = room(e.tokens); p.tokens[i] = room(e.tokens); }
  p.counts = p.few ? at : room(((int64_t)1 << p.bits) * p.blocks);
  p.begin = room(e.rows + 1);
  p.end = room(e.rows);
  p.parts = room(2 * p.chunks * p.padded);
  p.bytes = at;
  return p;
}

}  // namespace arrow

extern "C" {

int arrow_embedding_forward(const arrow_embedding_t* e, const void* W, const void* ids, void* Y, void* stream) {
  if (int rc = check(e, false)) return rc;
  if (e->tokens == 0) return ARROW_OK;
  const int size = size_of(e->dtype);
  if (int rc = check_pointer("W", W, size)) return rc;
  if (int rc = check_pointer("ids", ids, e->id_bytes)) return rc;
  if (int rc = check_pointer("Y", Y, size)) return rc;
  const int64_t y_bytes = extent(e->tokens, e->y_stride, e->columns, size);
  if (overlap(Y, y_bytes, W, extent(e->rows, e->w_stride, e->columns, size)) || overlap(Y, y_bytes, ids, e->tokens * e->id_bytes))
    return refuse(ARROW_EINVAL, "Y overlaps an input");
  return launched("embedding forward", launch_embedding_forward(*e, W, ids, Y, stream));
}

size_t arrow_embedding_workspace_bytes(const arrow_embedding_t* e) { return check(e, true) ? 0 : plan_embedding(*e).bytes; }

int arrow_embedding_backward(const arrow_embedding_t* e, const void* dY, const void* ids, void* dW, void* ws, size_t ws_bytes, void* stream) {
  if (int rc = check(e, true)) return rc;
  const int size = size_of(e->dtype);
  if (int rc = check_pointer("dW", dW, size_of(e->grad_dtype))) return rc;
  const int64_t w_bytes = extent(e->rows, e->w_stride, e->columns, size_of(e->grad_dtype));
  const EmbeddingPlan p = plan_embedding(*e);
  if (p.bytes && (!ws || (uintptr_t)ws % 256)) return refuse(ARROW_EINVAL, "workspace is NULL or not 256-byte aligned");
  if (ws_bytes < p.bytes) return refuse(ARROW_ETOOSMALL, "workspace of %zu bytes, %zu are needed", ws_bytes, p.bytes);
  if (overlap(dW, w_bytes, ws, (int64_t)p.bytes)) return refuse(ARROW_EINVAL, "dW overlaps the workspace");
  if (e->tokens) {
    if (int rc = check_pointer("dY", dY, size)) return rc;
    if (int rc = check_pointer("ids", ids, e->id_bytes)) return rc;
    if (overlap(dW, w_bytes, dY, extent(e->tokens, e->y_stride, e->columns, size)) || overlap(dW, w_bytes, ids, e->tokens * e->id_bytes))
      return refuse(ARROW_EINVAL, "dW overlaps an input");
  }
  return launched("embedding backward", launch_embedding_backward(*e, p, dY, ids, dW, ws, stream));
}

}  // extern "C"
