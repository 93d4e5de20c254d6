// Norms of heads with the rotation by position, and their gradients (include/arrow_rotation.h).
//
// What bounds it is memory: every element is read once and written once (backward: two read, one written).  A lane has 16 elements of a head: the
// two pieces of 8 that are each other's partners, so that a pair is rotated within a lane; 2^n lanes have a head and add up its squares.  A workgroup
// takes some tokens with all their heads, whose angles it computes once, into LDS.
#include <hip/hip_runtime.h>

#include <cstdint>

#include "attention_common.h"
#include "lanes.h"
#include "rotation_internal.h"

namespace arrow {
namespace {

constexpr int kThreads = kRotationThreads;

struct Eight { float x[8]; };

template <typename T>
__device__ __forceinline__ Eight load8(const T* at) {
  Eight r;
  if constexpr (sizeof(T) == 4) {
    const f32x4 a = *(const f32x4*)at, b = *(const f32x4*)(at + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) { r.x[i] = a[i]; r.x[4 + i] = b[i]; }
  } else {
    const x8<T> a = *(const x8<T>*)at;
#pragma unroll
    for (int i = 0; i < 8; ++i) r.x[i] = (float)a[i];
  }
  return r;
}

template <typename T>
__device__ __forceinline__ void store8(T* at, const Eight& v) {
  if constexpr (sizeof(T) == 4) {
    *(f32x4*)at = f32x4{v.x[0], v.x[1], v.x[2], v.x[3]};
    *(f32x4*)(at + 4) = f32x4{v.x[4], v.x[5], v.x[6], v.x[7]};
  } else {
    *(x8<T>*)at = round8<T>(v.x[0], v.x[1], v.x[2], v.x[3], v.x[4], v.x[5], v.x[6], v.x[7]);
  }
}

__device__ __forceinline__ Eight zeros() { return {{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}}; }

// The turn of a pair at a position, as cosine and sine.  The product in 64 bits is off by 2^-53 of itself, at a position of 2^31 by 2^-22 of a turn.
__device__ __forceinline__ float2 turned(double turns, int64_t position) {
  const double t = turns * (double)position;
  float2 r;
  sincospif((float)(2.0 * (t - rint(t))), &r.y, &r.x);
  return r;
}

// The pairs of the lane's two pieces, rotated by (cos, sin), or back.
template <bool kBack>
__device__ __forceinline__ void rotate(Eight& a, Eight& b, const float2* cs, bool interleaved) {
  float2 t[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const f32x4 two = *(const f32x4*)(cs + 2 * i);
    t[2 * i] = {two[0], kBack ? -two[1] : two[1]};
    t[2 * i + 1] = {two[2], kBack ? -two[3] : two[3]};
  }
  if (interleaved) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      Eight& p = i < 4 ? a : b;
      const int d = 2 * (i & 3);
      const float x = p.x[d], y = p.x[d + 1];
      p.x[d] = x * t[i].x - y * t[i].y;
      p.x[d + 1] = y * t[i].x + x * t[i].y;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float x = a.x[i], y = b.x[i];
      a.x[i] = x * t[i].x - y * t[i].y;
      b.x[i] = y * t[i].x + x * t[i].y;
    }
  }
}

// What a lane does at any head: where its two pieces lie, and its pairs' turns.
struct Lane {
  int first, second;        // elements, -1: a piece that is not there
  bool turns;
  int pair;                 // the first of its eight
  __device__ __forceinline__ Lane(const arrow_rotation_t& a, int u) {
    const int pieces = a.dim / 8, rotated = a.rotary / 8;
    turns = u < rotated / 2;
    pair = 8 * u;
    int x, y;
    if (turns) {
      x = a.interleaved ? 2 * u : u;
      y = a.interleaved ? 2 * u + 1 : u + rotated / 2;
    } else {
      x = rotated + 2 * (u - rotated / 2);
      y = x + 1;
    }
    first = x < pieces ? 8 * x : -1;
    second = y < pieces ? 8 * y : -1;
  }
};

template <typename T, typename W, bool kBack>
__global__ __launch_bounds__(kThreads) void rotation_kernel(RotationArgs p) {
  __shared__ __align__(16) float2 angles[kRotationTokens * 128];
  __shared__ __align__(16) float weights[2 * 256];
  __shared__ __align__(16) float sums[kBack ? kThreads * 16 : 1];
  const arrow_rotation_t& a = p.a;
  const int tid = threadIdx.x, lanes = 1 << p.lanes_log, groups = kThreads >> p.lanes_log, group = tid >> p.lanes_log, half = a.rotary / 2;
  const Lane lane(a, tid & (lanes - 1));
  for (int i = tid; i < 2 * a.dim; i += kThreads) {
    const int d = i < a.dim ? i : i - a.dim;
    const W* w = (const W*)(i < a.dim ? p.wq : p.wk);
    weights[i] = w ? (float)w[d] : 1.f;
  }
  Eight sum[2][2] = {{zeros(), zeros()}, {zeros(), zeros()}};

  for (int64_t token0 = (int64_t)blockIdx.x * p.per; token0 < p.rows; token0 += (int64_t)gridDim.x * p.per) {
    const int tokens = (int)min((int64_t)p.per, p.rows - token0);
    __syncthreads();                                  // (the angles of the tokens before are done with)
    for (int i = tid; i < tokens * half; i += kThreads) {
      const int t = i / half, pair = i - t * half;
      const int64_t row = token0 + t;
      const int64_t position = !a.positions ? row % a.tokens : a.position_bytes == 4 ? ((const int32_t*)a.positions)[row] : ((const int64_t*)a.positions)[row];
      angles[t * half + pair] = turned(a.turns[pair], position + a.shift);
    }
    __syncthreads();
#pragma unroll
    for (int which = 0; which < 2; ++which) {         // queries, then keys
      const int heads = which ? a.kv_heads : a.q_heads;
      const arrow_strides_t& from = which ? a.k : a.q;
      const arrow_strides_t& to = which ? p.k_to : p.q_to;
      const arrow_strides_t& grad = which ? a.k_out : a.q_out;
      const float* w = weights + which * a.dim;
      for (int i = group; i < tokens * heads; i += groups) {
        const int t = i / heads, head = i - t * heads;
        const int64_t row = token0 + t, b = row / a.tokens, at = row - b * a.tokens;
        const T* x = (const T*)(which ? p.k : p.q) + b * from.sequence + at * from.token + head * from.head;
        T* y = (T*)(which ? p.yk : p.yq) + b * to.sequence + at * to.token + head * to.head;
        Eight xa = zeros(), xb = zeros(), wa = zeros(), wb = zeros(), ga = zeros(), gb = zeros();
        if (lane.first >= 0) { xa = load8(x + lane.first); wa = load8(w + lane.first); }
        if (lane.second >= 0) { xb = load8(x + lane.second); wb = load8(w + lane.second); }
        if constexpr (kBack) {
          const T* g = (const T*)(which ? p.gk : p.gq) + b * grad.sequence + at * grad.token + head * grad.head;
          if (lane.first >= 0) ga = load8(g + lane.first);
          if (lane.second >= 0) gb = load8(g + lane.second);
        }
        float square = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) square = fmaf(xa.x[j], xa.x[j], fmaf(xb.x[j], xb.x[j], square));
        const float r = 1.f / sqrtf(sum_of_lanes(square, p.lanes_log) / (float)a.dim + a.eps);
        const float2* cs = angles + t * half + lane.pair;
        if constexpr (!kBack) {
#pragma unroll
          for (int j = 0; j < 8; ++j) { xa.x[j] *= r * wa.x[j]; xb.x[j] *= r * wb.x[j]; }
          if (lane.turns) rotate<false>(xa, xb, cs, a.interleaved);
        } else {
          if (lane.turns) rotate<true>(ga, gb, cs, a.interleaved);
          float mean = 0.f;
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            xa.x[j] *= r; xb.x[j] *= r;               // n
            const float da = ga.x[j] * xa.x[j], db = gb.x[j] * xb.x[j];
            sum[which][0].x[j] += da;
            sum[which][1].x[j] += db;
            mean = fmaf(wa.x[j], da, fmaf(wb.x[j], db, mean));
          }
          mean = sum_of_lanes(mean, p.lanes_log) / (float)a.dim;
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            xa.x[j] = r * (wa.x[j] * ga.x[j] - xa.x[j] * mean);
            xb.x[j] = r * (wb.x[j] * gb.x[j] - xb.x[j] * mean);
          }
        }
        if (lane.first >= 0) store8(y + lane.first, xa);
        if (lane.second >= 0) store8(y + lane.second, xb);
      }
    }
  }

  if constexpr (kBack) {
    if (!p.dwq) return;
    // the groups' sums of an element, one after the other
    for (int which = 0; which < 2; ++which) {
      __syncthreads();
      float* mine = sums + group * lanes * 16;
      if (lane.first >= 0) store8(mine + lane.first, sum[which][0]);
      if (lane.second >= 0) store8(mine + lane.second, sum[which][1]);
      __syncthreads();
      for (int d = tid; d < a.dim; d += kThreads) {
        float all = 0.f;
        for (int i = 0; i < groups; ++i) all += sums[i * lanes * 16 + d];
        p.parts[((int64_t)blockIdx.x * 2 + which) * a.dim + d] = all;
      }
    }
  }
}

// The workgroups' sums of the weights' gradients, 16 elements to a workgroup.
template <typename W>
__global__ __launch_bounds__(kThreads) void rotation_join_kernel(RotationArgs p) {
  __shared__ float sums[kThreads];
  const int c = blockIdx.x * 16 + (threadIdx.x & 15), part = threadIdx.x >> 4, columns = 2 * p.a.dim;
  float all = 0.f;
#pragma unroll 4
  for (int i = part; i < p.blocks; i += kThreads / 16) all += p.parts[(int64_t)i * columns + c];
  sums[threadIdx.x] = all;
  __syncthreads();
  if (threadIdx.x >= 16) return;
  for (int i = 1; i < kThreads / 16; ++i) all += sums[i * 16 + threadIdx.x];
  W* to = (W*)(c < p.a.dim ? p.dwq : p.dwk);
  to[c < p.a.dim ? c : c - p.a.dim] = (W)all;
}

template <typename T, typename W>
int launch(const RotationArgs& p, bool backward, void* stream) {
  hipStream_t s = (hipStream_t)stream;
  if (p.blocks) {
    if (backward) rotation_kernel<T, W, true><<<dim3((unsigned)p.blocks), dim3(kThreads), 0, s>>>(p);
    else rotation_kernel<T, W, false><<<dim3((unsigned)p.blocks), dim3(kThreads), 0, s>>>(p);
  }
  if (backward && p.dwq) rotation_join_kernel<W><<<dim3((unsigned)(2 * p.a.dim / 16)), dim3(kThreads), 0, s>>>(p);
  return (int)hipGetLastError();
}

}  // namespace

int launch_rotation(const RotationArgs& p, bool backward, void* stream) {
  const bool wide = p.a.weight_dtype == ARROW_F32;
  if (p.a.dtype == ARROW_F32) return launch<float, float>(p, backward, stream);
  if (p.a.dtype == ARROW_BF16) return wide ? launch<__bf16, float>(p, backward, stream) : launch<__bf16, __bf16>(p, backward, stream);
  return wide ? launch<_Float16, float>(p, backward, stream) : launch<_Float16, _Float16>(p, backward, stream);
}

}  // namespace arrow
