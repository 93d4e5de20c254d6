// Sums and maxima over neighbouring lanes, without LDS: what a lane gets from another comes as an operand's modifier, or by a swap of rows or halves.
// Everything has internal linkage; include inside a .hip file only.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace arrow {
namespace {

template <int kControl>
__device__ __forceinline__ float moved(float x) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), kControl, 0xf, 0xf, true));
}
__device__ __forceinline__ float swapped_rows(float x, float& y) {
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  y = __uint_as_float(r[1]);
  return __uint_as_float(r[0]);
}
__device__ __forceinline__ float swapped_halves(float x, float& y) {
  auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  y = __uint_as_float(r[1]);
  return __uint_as_float(r[0]);
}

// f over the groups of 2^log lanes that a lane is in, the same in all of them; f is commutative.
template <typename F>
__device__ __forceinline__ float over_lanes(float x, int log, F&& f) {
  if (log > 0) x = f(x, moved<0xb1>(x));       // lane ^ 1
  if (log > 1) x = f(x, moved<0x4e>(x));       // lane ^ 2
  if (log > 2) x = f(x, moved<0x141>(x));      // 7 - lane, of eight
  if (log > 3) x = f(x, moved<0x140>(x));      // 15 - lane, of sixteen
  float y;
  if (log > 4) { x = swapped_rows(x, y); x = f(x, y); }
  if (log > 5) { x = swapped_halves(x, y); x = f(x, y); }
  return x;
}
[[maybe_unused]] __device__ __forceinline__ float sum_of_lanes(float x, int log) {
  return over_lanes(x, log, [](float a, float b) { return a + b; });
}

}  // namespace
}  // namespace arrow
