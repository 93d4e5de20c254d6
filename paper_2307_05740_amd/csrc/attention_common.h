// Helpers shared by the attention kernels: 16-bit types and their matrix instructions, tiles of rows in LDS.
// Everything has internal linkage; include inside a .hip file only.
//
// Matrix instructions.  D = A B + C over 32 x 32 with 16 inner steps; lane l holds row (A) or column (B) l % 32 at inner
// steps 8 (l / 32) + 0..7, and of C and D column l % 32, rows 8 (i / 4) + 4 (l / 32) + i % 4 for i = 0..15.  A product whose inner steps
// run over the rows of an earlier result takes that result as its B operand without any exchange between lanes: the inner steps may come
// in any order as long as A has the same one, so lane half h = l / 32 simply holds rows 4 h + 0..3 and 8 + 4 h + 0..3 of each 16.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "attention_internal.h"

namespace arrow {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

template <typename T> struct Wide;
template <> struct Wide<__bf16> {
  typedef __bf16 x8 __attribute__((ext_vector_type(8)));
  typedef __bf16 x4 __attribute__((ext_vector_type(4)));
  typedef __bf16 x2 __attribute__((ext_vector_type(2)));
};
template <> struct Wide<_Float16> {
  typedef _Float16 x8 __attribute__((ext_vector_type(8)));
  typedef _Float16 x4 __attribute__((ext_vector_type(4)));
  typedef _Float16 x2 __attribute__((ext_vector_type(2)));
};
template <typename T> using x8 = typename Wide<T>::x8;
template <typename T> using x4 = typename Wide<T>::x4;
template <typename T> using x2 = typename Wide<T>::x2;

__device__ __forceinline__ f32x16 mma32(x8<__bf16> a, x8<__bf16> b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x16 mma32(x8<_Float16> a, x8<_Float16> b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 mma16(x8<__bf16> a, x8<__bf16> b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 mma16(x8<_Float16> a, x8<_Float16> b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
__device__ __forceinline__ float minus_infinity() { return -__builtin_inff(); }

// max / sum of a value and that of the lane 32 further on, in both.
__device__ __forceinline__ float max_halves(float x) {
  auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float add_halves(float x) {
  auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Eight values rounded to T, to nearest even.
template <typename T>
__device__ __forceinline__ x8<T> round8(float a, float b, float c, float d, float e, float f, float g, float h) {
  x8<T> r;
  r[0] = (T)a; r[1] = (T)b; r[2] = (T)c; r[3] = (T)d; r[4] = (T)e; r[5] = (T)f; r[6] = (T)g; r[7] = (T)h;
  return r;
}

// Sum of eight values and of c, in 32 bits.
__device__ __forceinline__ float add8(x8<__bf16> x, float c) {
  const x2<__bf16> one = {(__bf16)1.f, (__bf16)1.f};
#pragma unroll
  for (int i = 0; i < 8; i += 2) c = __builtin_amdgcn_fdot2_f32_bf16(x2<__bf16>{x[i], x[i + 1]}, one, c, false);
  return c;
}
__device__ __forceinline__ float add8(x8<_Float16> x, float c) {
  const x2<_Float16> one = {(_Float16)1.f, (_Float16)1.f};
#pragma unroll
  for (int i = 0; i < 8; i += 2) c = __builtin_amdgcn_fdot2(x2<_Float16>{x[i], x[i + 1]}, one, c, false);
  return c;
}

__device__ __forceinline__ int wave_id() { return __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)); }

// A tile of rows of D 16-bit elements in LDS, in pieces of 16 bytes.  Piece c of row r lies at place c ^ turn(r) of the row, so
// that both ways of reading it touch every bank once: 16 rows' pieces of one number (`rows`, an operand whose inner steps run
// along the rows), and four rows' runs of 64 bytes (`columns`, one whose inner steps run across them, transposed on the way).
template <int D>
struct Tile {
  static constexpr int kPieces = D / 8;
  static constexpr int kRowBytes = 2 * D;
  static constexpr int kRowsOfKiB = 1024 / kRowBytes;
  __device__ static int turn(int r) {
    return D == 128 ? ((r & 3) << 2) | ((r >> 2) & 3) : (((r >> 1) & 1) << 2) | ((r >> 2) & 3);
  }
};

// Columns of the tiles in which heads of up to C = 64, 96 or 128 columns lie.  Products leave out those from C on (training over 1531 tokens, heads
// of 96: 155 us with all 128, 141 without the last ones).
constexpr int columns_of_tile(int C) { return C <= 64 ? 64 : 128; }

typedef __attribute__((address_space(3))) void lds_void;
typedef __attribute__((address_space(3))) unsigned char lds_byte;

template <typename T>
__device__ __forceinline__ x8<T> lds_read8(uint32_t at) { return *(const __attribute__((address_space(3))) x8<T>*)(uintptr_t)at; }
__device__ __forceinline__ f32x4 lds_read4(uint32_t at) { return *(const __attribute__((address_space(3))) f32x4*)(uintptr_t)at; }
// (`restrict` tells these reads apart from the loads to LDS that are on their way to other tiles, for which they would wait otherwise;
// so does that a kernel has all its LDS in one array)
__device__ __forceinline__ i16x4 lds_transposed(const lds_byte* __restrict p) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4*)p);
}
__device__ __forceinline__ uint32_t lds_address(const lds_byte* p) { return (uint32_t)(uintptr_t)p; }

// This lane's places in the tile at an address whose low byte is 0.  Those of other inner steps and columns differ by an exclusive
// or of a constant, which costs an instruction each and no registers from tile to tile.
template <int D>
struct TileReads {
  uint32_t rows, columns;
  __device__ __forceinline__ explicit TileReads(int l) {
    const int g = l >> 4, i = l & 15, row = 4 * (g >> 1) + (i >> 2), piece = 2 * (g & 1) + ((i & 3) >> 1);
    rows = (l & 31) * Tile<D>::kRowBytes + (((l >> 5) ^ Tile<D>::turn(l & 31)) << 4);
    columns = row * Tile<D>::kRowBytes + ((piece ^ Tile<D>::turn(row)) << 4) + ((i & 1) << 3);
  }
};
// The same value, computed where it stands: what is derived from it is not kept in registers from one round of a loop to the next.
template <typename X>
__device__ __forceinline__ X here(X x) {
  asm volatile("" : "+v"(x));
  return x;
}
// A or B of a tile's rows (32 from a multiple of 32 on, `skip` bytes into the tile) and its columns 16 s .. 16 s + 15: lane l has row l % 32,
// columns 16 s + 8 (l / 32) + 0..7.  at: the tile's address + TileReads::rows.
template <typename T>
__device__ __forceinline__ x8<T> read_rows(uint32_t at, int s, int skip) { return lds_read8<T>((at ^ (s << 5)) + skip); }
// A of the transposed tile: its rows are the tile's columns 32 m .. 32 m + 31, its inner steps 16 rows of the tile (from a multiple of 16 on, `skip` bytes into
// it) in the order of an earlier result's.  at: the tile's address + TileReads::columns.
template <typename T, int D>
__device__ __forceinline__ x8<T> read_columns(uint32_t at, int m, int skip) {
  union { i16x4 half[2]; x8<T> all; } r;
  r.half[0] = lds_transposed((const lds_byte*)(uintptr_t)((at ^ (m << 6)) + skip));
  r.half[1] = lds_transposed((const lds_byte*)(uintptr_t)((at ^ (m << 6 | 32)) + skip + 8 * Tile<D>::kRowBytes));
  return r.all;
}

// Elements apart: the finite ones, and of the others 1 for infinity, 128 for minus infinity and 129 for NaN: the sum of up to 127 of these says which there are.
template <typename T> struct Apart { x8<T> finite, other; };
template <typename T>
__device__ __forceinline__ Apart<T> apart(x8<T> x) {
  typedef uint16_t u16x8 __attribute__((ext_vector_type(8)));
  constexpr uint16_t infinity = std::is_same<T, __bf16>::value ? 0x7f80 : 0x7c00;
  union { x8<T> all; u16x8 bits; } u;
  u.all = x;
  Apart<T> r;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint16_t size = u.bits[i] & 0x7fff;
    const bool odd = size >= infinity, minus = u.bits[i] >> 15;
    r.finite[i] = odd ? (T)0.f : x[i];
    r.other[i] = !odd ? (T)0.f : size > infinity ? (T)129.f : minus ? (T)128.f : (T)1.f;
  }
  return r;
}

// Nothing that follows begins before these sums are there.
__device__ __forceinline__ void one_by_one(f32x16& x) {
  x = here(x);
  __builtin_amdgcn_sched_barrier(0);
}

// acc += X^T W, where X is 16 kSteps rows of a tile and 32 of its columns, 32 m on, of which elements that are not finite are taken out.
// (Little is on its way at a time: these are not to take more registers than the products that they stand beside.)
template <typename T, int D, int kSteps>
__device__ __forceinline__ void add_finite(f32x16& acc, uint32_t at, int m, const x8<T>* w) {
#pragma unroll
  for (int u = 0; u < kSteps; ++u) {
    acc = mma32(apart<T>(read_columns<T, D>(at, m, 16 * u * Tile<D>::kRowBytes)).finite, w[u], acc);
    one_by_one(acc);
  }
}

// What was taken out: an element counts where seen(u, i) says so of the lane's column and the row that element i of operand u has, as itself whatever its weight (kSigned:
// weights are not negative) or as NaN, and does not elsewhere.  A product with the weights would make it NaN everywhere.
template <typename T, int D, int kSteps, bool kSigned, typename F>
__device__ __forceinline__ void add_others(f32x16& acc, uint32_t at, int m, F&& seen) {
  f32x16 others = (f32x16)(0.f);
#pragma unroll
  for (int u = 0; u < kSteps; ++u) {
    x8<T> one;
#pragma unroll
    for (int i = 0; i < 8; ++i) one[i] = seen(u, i) ? (T)1.f : (T)0.f;
    others = mma32(apart<T>(read_columns<T, D>(at, m, 16 * u * Tile<D>::kRowBytes)).other, one, others);
    one_by_one(others);
  }
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int n = (int)others[i];
    if (kSigned) acc[i] += (n & 127 ? __builtin_inff() : 0.f) - (n >> 7 ? __builtin_inff() : 0.f);
    else acc[i] = n ? __builtin_nanf("") : acc[i];
  }
  one_by_one(acc);
}

// Whether any of the workgroup's four wavefronts says so.  flags: four words in LDS that nothing else uses, and are written once.
__device__ __forceinline__ bool any_wave(bool x, lds_byte* flags) {
  typedef __attribute__((address_space(3))) uint32_t lds_word;
  lds_word* at = (lds_word*)flags;
  const bool mine = __any(x);
  if ((threadIdx.x & 63) == 0) at[wave_id()] = mine;
  __syncthreads();
  return __builtin_amdgcn_readfirstlane((int)(at[0] | at[1] | at[2] | at[3])) != 0;
}

// Copies ROWS rows of an operand into a Tile, straight to LDS, WAVES wavefronts together.  Rows that are not there and columns from `dim` on
// become 0: the buffer descriptor ends with the last row.
template <int D, int ROWS, int WAVES>
struct Loader {
  static constexpr int kStepRows = WAVES * Tile<D>::kRowsOfKiB, kSteps = ROWS / kStepRows;
  static_assert(kSteps * kStepRows == ROWS, "whole steps");
  // what step i changes of a row's turn
  __device__ static constexpr int turn_of(int i) { return (D == 128 ? i * WAVES : 2 * i * WAVES) & 3; }
  uint32_t offset;                                               // of this lane's row
  int piece, dim;
  uint32_t stride_bytes, tile_bytes;                             // (of a tile whose rows are all there; 127 of the longest steps are below 2^32)
  __device__ __forceinline__ Loader(int wave, int lane, int64_t stride, int dim_) {
    const int row = wave * Tile<D>::kRowsOfKiB + lane / Tile<D>::kPieces;
    piece = (lane % Tile<D>::kPieces) ^ Tile<D>::turn(row);
    stride_bytes = (uint32_t)(stride * 2);
    dim = dim_;
    tile_bytes = (ROWS - 1) * stride_bytes + 2 * dim;
    offset = row * stride_bytes;
  }
  // base: the tile's first row (the same in all lanes); rows: those that are there, any number
  __device__ __forceinline__ void load(const void* base, int rows, lds_byte* tile, int wave) const {
    const uint32_t bytes = rows >= ROWS ? tile_bytes : rows > 0 ? (rows - 1) * stride_bytes + 2 * dim : 0;
    auto rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, (int)bytes, 0x00020000);
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      const int p = piece ^ turn_of(i);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (lds_void*)(tile + (i * WAVES + wave) * 1024), 16,
                                               8 * p < dim ? offset + i * kStepRows * stride_bytes + 16 * p : 0xfffffff0u, 0, 0, 0);
    }
  }
};

// Tokens of one sequence: where they start in its operands, and how many there are.
struct Span { int64_t first; int count; };
__device__ __forceinline__ Span span_of(const int32_t* offsets, int b, int64_t tokens, int len) {
  if (!offsets) return {0, len};
  int64_t first = offsets[b], end = offsets[b + 1];
  first = first < 0 ? 0 : first > tokens ? tokens : first;
  end = end < first ? first : end > tokens ? tokens : end;
  const int64_t n = end - first;
  // (b is the same in all lanes, and so are these, in scalar registers)
  return {(int64_t)__builtin_amdgcn_readfirstlane((int)first), __builtin_amdgcn_readfirstlane((int)(n < len ? n : len))};
}
__device__ __forceinline__ const char* rows_of(const Operand& m, bool ragged, int b, int64_t first, int64_t head) {
  return (const char*)m.at + 2 * (head * m.head + (ragged ? first * m.token : b * m.sequence));
}

// Which tiles of K keys the queries at positions low .. high see: the first `sinks` ones, then those of the window.
struct SeenTiles {
  int lead, rest, total;
  __device__ __forceinline__ int at(int t) const { return t < lead ? t : t - lead + rest; }
};
template <int K>
__device__ __forceinline__ SeenTiles seen_tiles(int low, int high, int window, int sinks) {
  SeenTiles s{0, 0, 0};
  if (high < 0) return s;
  const int last = high / K;
  const int64_t begin = (int64_t)low - window + 1;
  s.rest = window && begin > 0 ? (int)(begin / K) : 0;
  s.lead = window ? min((int)(((int64_t)sinks + K - 1) / K), s.rest) : 0;
  s.total = s.lead + last - s.rest + 1;
  return s;
}

// 32 rows (columns 32 m on of the operand) of a transposed result and 32 columns (the operand's rows, this lane's at `to`), rounded and stored.  A lane
// has columns 32 m + 16 u + 4 half + 0..3 and + 8..11; with the other half's it gets eight in a row.
template <typename T>
__device__ __forceinline__ void store_block(const f32x16& acc, int m, T* to, int half, int dim) {
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    union { x8<T> all; uint32_t w[4]; } r, x;
    r.all = round8<T>(acc[8 * u], acc[8 * u + 1], acc[8 * u + 2], acc[8 * u + 3], acc[8 * u + 4], acc[8 * u + 5], acc[8 * u + 6], acc[8 * u + 7]);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      auto y = __builtin_amdgcn_permlane32_swap(r.w[i], r.w[2 + i], false, false);
      x.w[i] = y[0];
      x.w[2 + i] = y[1];
    }
    const int d = 32 * m + 16 * u + 8 * half;
    if (d < dim) *(x8<T>*)(to + d) = x.all;
  }
}
template <typename T, int D>
__device__ __forceinline__ void store_columns(const f32x16* acc, T* to, int half, int dim) {
#pragma unroll
  for (int m = 0; m < D / 32; ++m) store_block<T>(acc[m], m, to, half, dim);
}

// Where the sums of a part of a key tile lie in the workspace, counted in pairs (dk, dv): only tiles in several parts have places.
__device__ __forceinline__ int64_t part_place(const AttentionArgs& a, int tiles, int64_t unit, int tile, int part) {
  const int lead = a.sink_parts > 1 ? a.sink_tiles * a.sink_parts : 0;
  const int per_unit = lead + (a.tile_parts > 1 ? (tiles - a.sink_tiles) * a.tile_parts : 0);
  return unit * per_unit + (tile < a.sink_tiles ? tile * a.sink_parts : lead + (tile - a.sink_tiles) * a.tile_parts) + part;
}

// The order of a block's instructions: kAhead LDS reads first, then kPer of them for each of kProducts matrix instructions, and the same for a second
// kind of products, so that a product's operands are on their way while earlier ones run.  (By itself the compiler reads one operand
// at a time and waits for it.)
template <int kAhead, int kProducts, int kPer, int kProducts2 = 0, int kPer2 = 0>
__device__ __forceinline__ void reads_ahead() {
  constexpr int kReads = kProducts * kPer + kProducts2 * kPer2;
  __builtin_amdgcn_sched_group_barrier(0x100, kAhead, 0);
#pragma unroll
  for (int i = 0; i < kProducts + kProducts2; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    const int done = kAhead + (i < kProducts ? i * kPer : kProducts * kPer + (i - kProducts) * kPer2);
    if (done < kReads) {
      if (i < kProducts) __builtin_amdgcn_sched_group_barrier(0x100, kPer, 0);
      else __builtin_amdgcn_sched_group_barrier(0x100, kPer2, 0);
    }
  }
}

__device__ __forceinline__ void wait_for_tiles() {
  // (the builtins of loads to LDS count as vector memory)
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup");
}

// The same for tiles that only this wavefront loads and reads.
__device__ __forceinline__ void wait_for_own_tiles() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

}  // namespace
}  // namespace arrow
