// Norms of heads with the rotation by position, and their gradients (include/arrow_rotation.h).
//
// What bounds it is memory: every element is read once and written once (backward: two read, one written).  A lane has 16 elements of a head: the
// two pieces of 8 that are each other's partners, so that a pair is rotated within a lane; 2^n lanes have a head and add up its squares.  A workgroup
// takes some tokens with all their heads, whose angles it computes once, into LDS: with 40 heads of 128 they are a fortieth of the work, but with three of 256 a third
// (tiles_of in rotation.cpp has the times).
//
// Measured with 4 x 4096 tokens of 32/8 heads of 128 in bfloat16: forward 64 us, 5.2 TB/s of what it has to move (a 1 GiB copy: 5.1), vector instructions issue in 44 % of the cycles;
// gradients 110 us, 4.6 TB/s, 43 %, and 5 us for the join of the weights' gradients (in float32 131 and 207 together); a few tokens 5.2 us, which is a launch.
#include <hip/hip_runtime.h>

#include <cstdint>

#include "attention_common.h"
#include "lanes.h"
#include "rotation_internal.h"

namespace arrow {
namespace {

constexpr int kThreads = kRotationThreads;

struct Eight { float x[8]; };

// Eight elements as they lie in memory.
template <typename T> struct Raw { x8<T> v; };
template <> struct Raw<float> { f32x4 v[2]; };

template <typename T>
__device__ __forceinline__ Raw<T> raw8(const T* at) {
  if constexpr (sizeof(T) == 4) return {{*(const f32x4*)at, *(const f32x4*)(at + 4)}};
  else return {*(const x8<T>*)at};
}
// Zeros where the piece is not there.
template <typename T>
__device__ __forceinline__ Raw<T> only(const Raw<T>& r, bool in) {
  union { Raw<T> r; uint32_t u[sizeof(Raw<T>) / 4]; } x;
  x.r = r;
#pragma unroll
  for (auto& u : x.u) u = in ? u : 0;
  return x.r;
}
template <typename T>
__device__ __forceinline__ Eight wide(const Raw<T>& r) {
  Eight e;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if constexpr (sizeof(T) == 4) e.x[i] = r.v[i / 4][i % 4];
    else e.x[i] = (float)r.v[i];
  }
  return e;
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

// The same, and what was made of it before is not kept in registers.
template <typename T>
__device__ __forceinline__ Raw<T> again(const Raw<T>& r) {
  if constexpr (sizeof(T) == 4) {
    return {{here(r.v[0]), here(r.v[1])}};
  } else {
    union { x8<T> v; u32x4 u; } x;
    x.v = r.v;
    x.u = here(x.u);
    return {x.v};
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
template <bool kBack, bool kInterleaved>
__device__ __forceinline__ void rotate(Eight& a, Eight& b, const float2* cs) {
#pragma unroll
  for (int i = 0; i < 8; i += 2) {
    const f32x4 two = *(const f32x4*)(cs + i);
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const float c = two[2 * k], s = kBack ? -two[2 * k + 1] : two[2 * k + 1];
      if constexpr (kInterleaved) {
        Eight& p = i < 4 ? a : b;
        const int d = 2 * ((i + k) & 3);
        const float x = p.x[d], y = p.x[d + 1];
        p.x[d] = x * c - y * s;
        p.x[d + 1] = y * c + x * s;
      } else {
        const float x = a.x[i + k], y = b.x[i + k];
        a.x[i + k] = x * c - y * s;
        b.x[i + k] = y * c + x * s;
      }
    }
  }
}

// What a lane does at any head: where its two pieces lie, and its pairs' turns.
struct Lane {
  int first, second;        // elements
  bool has_first, has_second;
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
    has_first = x < pieces;
    has_second = y < pieces;
    first = has_first ? 8 * x : 0;           // (a piece that is not there is read as the first one)
    second = has_second ? 8 * y : 0;
  }
};

// Some tokens of one sequence.
struct Tokens {
  uint32_t b, at;           // the sequence, and the first of them in it
  int count;
  __device__ __forceinline__ Tokens(const RotationArgs& p, const RotationTiles& tiles, uint32_t tile) {
    b = tile / (uint32_t)tiles.tiles;
    at = (tile - b * tiles.tiles) * tiles.per;
    count = min(tiles.per, p.length - (int)at);
  }
};

// Their heads, of queries or keys (kKeys): 2^n lanes each, the next one's elements on their way while one is worked on, the first ones' from the start.
template <typename T, bool kBack, bool kKeys, bool kInterleaved>
struct Heads {
  struct Pieces { Raw<T> xa, xb, ga, gb; };
  const RotationArgs& p;
  const Lane& lane;
  const arrow_strides_t &from, &to, &grad;
  const T *x, *g;
  T* y;
  int heads, n, i, t, head;           // head i of n: of token t
  Pieces next;

  __device__ __forceinline__ Heads(const RotationArgs& args, const Lane& l, const Tokens& of)
      : p(args), lane(l), from(kKeys ? args.a.k : args.a.q), to(kKeys ? args.k_to : args.q_to), grad(kKeys ? args.a.k_out : args.a.q_out) {
    heads = kKeys ? p.a.kv_heads : p.a.q_heads;
    n = of.count * heads;
    x = (const T*)(kKeys ? p.k : p.q) + of.b * from.sequence + of.at * from.token;
    g = kBack ? (const T*)(kKeys ? p.gk : p.gq) + of.b * grad.sequence + of.at * grad.token : nullptr;
    y = (T*)(kKeys ? p.yk : p.yq) + of.b * to.sequence + of.at * to.token;
    i = threadIdx.x >> p.lanes_log;
    const int j = min(i, n - 1);
    t = (uint32_t)j / (uint32_t)heads;
    head = j - t * heads;
    load();
  }
  __device__ __forceinline__ void load() {
    const T* at = x + t * from.token + head * from.head;
    next.xa = raw8(at + lane.first);
    next.xb = raw8(at + lane.second);
    if constexpr (kBack) {
      at = g + t * grad.token + head * grad.head;
      next.ga = raw8(at + lane.first);
      next.gb = raw8(at + lane.second);
    }
  }
  __device__ __forceinline__ void run(const float2* angles, const float* w, Eight* sum);
};

template <typename T, bool kBack, bool kKeys, bool kInterleaved>
__device__ __forceinline__ void Heads<T, kBack, kKeys, kInterleaved>::run(const float2* angles, const float* w, Eight* sum) {
  if (i >= n) return;
  const arrow_rotation_t& a = p.a;
  const int half = a.rotary / 2, step = kThreads >> p.lanes_log, step_t = step / heads, step_head = step - step_t * heads;
  while (true) {
    Pieces now = next;
    const int now_t = t, now_head = head;
    i += step;
    const bool more = i < n;
    head += step_head;
    t += step_t;
    if (head >= heads) { head -= heads; ++t; }
    if (!more) { t = now_t; head = now_head; }
    load();
    if (!p.whole) {
      now.xa = only(now.xa, lane.has_first);
      now.xb = only(now.xb, lane.has_second);
      if constexpr (kBack) {
        now.ga = only(now.ga, lane.has_first);
        now.gb = only(now.gb, lane.has_second);
      }
    }
    Eight xa = wide<T>(now.xa), xb = wide<T>(now.xb);
    float square = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) square = fmaf(xa.x[j], xa.x[j], fmaf(xb.x[j], xb.x[j], square));
    const float r = rsqrtf(fmaf(sum_of_lanes(square, p.lanes_log), p.share, a.eps));
    const float2* cs = angles + now_t * half + lane.pair;
    if constexpr (!kBack) {
#pragma unroll
      for (int j = 0; j < 8; ++j) { xa.x[j] *= r * w[lane.first + j]; xb.x[j] *= r * w[lane.second + j]; }
      if (lane.turns) rotate<false, kInterleaved>(xa, xb, cs);
    } else {
      Eight ga = wide<T>(now.ga), gb = wide<T>(now.gb);
      if (lane.turns) rotate<true, kInterleaved>(ga, gb, cs);
      __builtin_amdgcn_sched_barrier(0);          // (the weights are not loaded before the angles are done with)
      xa = wide<T>(again(now.xa));
      xb = wide<T>(again(now.xb));
      float mean = 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        xa.x[j] *= r; xb.x[j] *= r;               // n
        sum[0].x[j] = fmaf(ga.x[j], xa.x[j], sum[0].x[j]);
        sum[1].x[j] = fmaf(gb.x[j], xb.x[j], sum[1].x[j]);
        ga.x[j] *= w[lane.first + j];
        gb.x[j] *= w[lane.second + j];
        mean = fmaf(ga.x[j], xa.x[j], fmaf(gb.x[j], xb.x[j], mean));
      }
      mean = sum_of_lanes(mean, p.lanes_log) * p.share;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        xa.x[j] = r * (ga.x[j] - xa.x[j] * mean);
        xb.x[j] = r * (gb.x[j] - xb.x[j] * mean);
      }
    }
    T* at = y + now_t * to.token + now_head * to.head;
    if (lane.has_first) store8(at + lane.first, xa);
    if (lane.has_second) store8(at + lane.second, xb);
    if (!more) return;
  }
}

// Their angles, `half` each.
__device__ __forceinline__ void find_angles(const RotationArgs& p, const Tokens& of, float2* angles) {
  const arrow_rotation_t& a = p.a;
  const int half = a.rotary / 2;
  for (int i = threadIdx.x; i < of.count * half; i += kThreads) {
    const uint32_t t = (uint32_t)i / (uint32_t)half, pair = i - t * half, row = of.b * p.length + of.at + t;
    const int64_t position = !a.positions ? row % (uint32_t)a.tokens : a.position_bytes == 4 ? ((const int32_t*)a.positions)[row] : ((const int64_t*)a.positions)[row];
    angles[i] = turned(a.turns[pair], position + a.shift);
  }
}

template <typename W>
__device__ __forceinline__ void find_weights(const RotationArgs& p, bool keys, float* weights) {
  const W* w = (const W*)(keys ? p.wk : p.wq);
  for (int d = threadIdx.x; d < p.a.dim; d += kThreads) weights[d] = w ? (float)w[d] : 1.f;
}

template <typename T, typename W, bool kInterleaved>
__global__ __launch_bounds__(kThreads) void rotation_kernel(RotationArgs p) {
  __shared__ __align__(16) float2 angles[kRotationAngles];
  __shared__ __align__(16) float weights[2][256];
  const Lane lane(p.a, threadIdx.x & ((1 << p.lanes_log) - 1));
  for (uint32_t tile = blockIdx.x; tile < (uint32_t)p.tiles[0].all; tile += gridDim.x) {
    const Tokens of(p, p.tiles[0], tile);
    Heads<T, false, false, kInterleaved> queries(p, lane, of);
    Heads<T, false, true, kInterleaved> keys(p, lane, of);
    if (tile == blockIdx.x) {
      find_weights<W>(p, false, weights[0]);
      find_weights<W>(p, true, weights[1]);
    } else {
      __syncthreads();                                // (the angles of the tokens before are done with)
    }
    find_angles(p, of, angles);
    __syncthreads();
    queries.run(angles, weights[0], nullptr);
    keys.run(angles, weights[1], nullptr);
  }
}

// Gradients: a workgroup has queries or keys, so that it holds the sums of one weight's gradient only, in 16 registers; both would be 32, and spill.  Workgroups stay on the chip
// and go round, four to a compute unit, so that there are 1024 such sums to join (1280 workgroups, five to one: 194 us for 4 x 4096 tokens, 188 with 1024; with registers
// held to five, 164 bytes of a lane spill and the kernel takes 236 us, not 124).
template <typename T, typename W, bool kKeys, bool kInterleaved>
__device__ __forceinline__ void rotate_back(const RotationArgs& p, uint32_t block, uint32_t blocks, float2* angles, float* weights, float* sums) {
  const int lanes = 1 << p.lanes_log, groups = kThreads >> p.lanes_log;
  const Lane lane(p.a, threadIdx.x & (lanes - 1));
  find_weights<W>(p, kKeys, weights);
  Eight sum[2] = {zeros(), zeros()};
  for (uint32_t tile = block; tile < (uint32_t)p.tiles[kKeys].all; tile += blocks) {
    const Tokens of(p, p.tiles[kKeys], tile);
    Heads<T, true, kKeys, kInterleaved> heads(p, lane, of);
    __syncthreads();                                  // (the angles of the tokens before are done with)
    find_angles(p, of, angles);
    __syncthreads();
    heads.run(angles, weights, sum);
  }
  if (!p.dwq) return;
  // the groups' sums of an element, one after the other
  __syncthreads();
  float* mine = sums + (threadIdx.x >> p.lanes_log) * lanes * 16;
  if (lane.has_first) store8(mine + lane.first, sum[0]);
  if (lane.has_second) store8(mine + lane.second, sum[1]);
  __syncthreads();
  for (int d = threadIdx.x; d < p.a.dim; d += kThreads) {
    float all = 0.f;
    for (int i = 0; i < groups; ++i) all += sums[i * lanes * 16 + d];
    p.parts[(int64_t)blockIdx.x * p.a.dim + d] = all;
  }
}

template <typename T, typename W, bool kInterleaved>
__global__ __launch_bounds__(kThreads, sizeof(T) == 4 ? 3 : 4) void rotation_grad_kernel(RotationArgs p) {
  static_assert(sizeof(float2) * kRotationAngles >= sizeof(float) * kThreads * 16, "the sums have the angles' place");
  __shared__ __align__(16) float2 angles[kRotationAngles];
  __shared__ __align__(16) float weights[256];
  float* sums = (float*)angles;
  const uint32_t block = blockIdx.x, q_blocks = p.q_blocks;
  if (block < q_blocks) rotate_back<T, W, false, kInterleaved>(p, block, q_blocks, angles, weights, sums);
  else rotate_back<T, W, true, kInterleaved>(p, block - q_blocks, gridDim.x - q_blocks, angles, weights, sums);
}

// The workgroups' sums of the weights' gradients, 16 elements to a workgroup: one launch more, 5 us, for sums that come in the same order every time.
template <typename W>
__global__ __launch_bounds__(kThreads) void rotation_join_kernel(RotationArgs p) {
  __shared__ float sums[kThreads];
  const bool keys = blockIdx.y;
  const int c = blockIdx.x * 16 + (threadIdx.x & 15), part = threadIdx.x >> 4;
  const int first = keys ? p.q_blocks : 0, end = keys ? p.blocks : p.q_blocks;
  float all = 0.f;
  if (c < p.a.dim) {
#pragma unroll 8
    for (int i = first + part; i < end; i += kThreads / 16) all += p.parts[(int64_t)i * p.a.dim + c];
  }
  sums[threadIdx.x] = all;
  __syncthreads();
  if (threadIdx.x >= 16 || c >= p.a.dim) return;
  for (int i = 1; i < kThreads / 16; ++i) all += sums[i * 16 + threadIdx.x];
  ((W*)(keys ? p.dwk : p.dwq))[c] = (W)all;
}

template <typename T, typename W, bool kInterleaved>
int launch(const RotationArgs& p, bool backward, hipStream_t s) {
  if (p.blocks) {
    if (backward) rotation_grad_kernel<T, W, kInterleaved><<<dim3((unsigned)p.blocks), dim3(kThreads), 0, s>>>(p);
    else rotation_kernel<T, W, kInterleaved><<<dim3((unsigned)p.blocks), dim3(kThreads), 0, s>>>(p);
  }
  if (backward && p.dwq) rotation_join_kernel<W><<<dim3((unsigned)((p.a.dim + 15) / 16), 2), dim3(kThreads), 0, s>>>(p);
  return (int)hipGetLastError();
}
template <typename T, typename W>
int launch(const RotationArgs& p, bool backward, void* stream) {
  return p.a.interleaved ? launch<T, W, true>(p, backward, (hipStream_t)stream) : launch<T, W, false>(p, backward, (hipStream_t)stream);
}

}  // namespace

int launch_rotation(const RotationArgs& p, bool backward, void* stream) {
  const bool wide = p.a.weight_dtype == ARROW_F32;
  if (p.a.dtype == ARROW_F32) return launch<float, float>(p, backward, stream);
  if (p.a.dtype == ARROW_BF16) return wide ? launch<__bf16, float>(p, backward, stream) : launch<__bf16, __bf16>(p, backward, stream);
  return wide ? launch<_Float16, float>(p, backward, stream) : launch<_Float16, _Float16>(p, backward, stream);
}

}  // namespace arrow
