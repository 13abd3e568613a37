// Shared definitions of attention and of the quantised cache: matrix fragments of the three element types, where rows,
// sequences and cache slots lie.
//
// Fragments.  A 16 x 16 product of 32 contraction elements takes 8 elements a lane: lane 16 g + n holds row (or column) n,
// elements 8 g .. 8 g + 7; its result has column n, rows 4 g .. 4 g + 3 in lane 16 g + n.  The contraction's order is free as
// long as both operands agree, so two results of 16 tokens each, side by side in their lanes, are an operand of 32
// tokens for the next product without moving between lanes: element j of lane group g is token 4 g + j (j < 4) or
// 16 + 4 g + j - 4.  Scores are therefore computed with the tokens as rows, and outputs with the head's elements as rows.
// binary32 takes eight products of 4 elements for the same lanes.
#pragma once

#include "squant_lin.h"

namespace squant {
namespace att {

using lin::Brain;
using lin::brain8;
using lin::exp2_fast;
using lin::float4v;
using lin::Half;
using lin::half2v;
using lin::half8;
using lin::kLn2;
using lin::kLog2E;
using lin::load_any;
using lin::magnitude;
using lin::power_of_two;
using lin::store_any;
using lin::uint2v;
using lin::uint4v;

constexpr int kThreads = 256;
constexpr int kGroup = 32;  // elements of a head that share a scale in the cache

typedef float float8 __attribute__((ext_vector_type(8)));
typedef _Float16 half4 __attribute__((ext_vector_type(4)));
typedef __bf16 brain4 __attribute__((ext_vector_type(4)));

struct Single {
  typedef float8 frag;
  static __device__ __forceinline__ float4v mma(frag a, frag b, float4v c) {
#pragma unroll
    for (int j = 0; j < 8; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[j], b[j], c, 0, 0, 0);
    return c;
  }
};
template <class T> struct MatrixOf;
template <> struct MatrixOf<_Float16> { typedef Half type; };
template <> struct MatrixOf<__bf16> { typedef Brain type; };
template <> struct MatrixOf<float> { typedef Single type; };

// Elements of [rows][heads][head_dim], strides in elements.
struct Strided {
  char* p;
  int64_t row, head;
};
template <class T> __device__ __forceinline__ T* element(const Strided& s, int64_t row, int head) {
  return reinterpret_cast<T*>(s.p) + row * s.row + head * s.head;
}

__device__ __forceinline__ uint64_t lanes_where(bool c) { return __builtin_amdgcn_ballot_w64(c); }

// The largest i in [0, n) with f(i) <= x, for f that does not fall; -1 if there is none.  By all lanes of a wave: 64 values a step.
template <class F> __device__ __forceinline__ int last_not_above(F f, int n, int64_t x) {
  const int lane = (int)(threadIdx.x & 63u);
  int first = 0, found = -1;
  while (n > 0) {
    const int step = (n + 63) / 64;
    const int i = lane * step;
    const int count = __popcll(lanes_where(i < n && f(first + (i < n ? i : 0)) <= x));
    if (count == 0) break;
    const int at = (count - 1) * step;
    found = first + at;
    n = min(step - 1, n - at - 1);
    first = found + 1;
  }
  return __builtin_amdgcn_readfirstlane(found);
}

// Rows of packed sequences.  Sequence `count` stands for the rows behind the last one.
struct Packed {
  const int32_t* starts;  // null: one sequence of all rows, or (one_each) a row for each
  int32_t count;
  int32_t rows;
  bool one_each;
  __device__ __forceinline__ int start(int i) const {
    if (!starts) return one_each ? min(i, rows) : i ? rows : 0;
    return min(max(starts[i], 0), rows);
  }
  __device__ __forceinline__ int length(int i) const {
    return max((i < count ? start(i + 1) : rows) - start(i), 0);
  }
  // The sequence of a row; `count` behind the last, -1 before the first.
  __device__ __forceinline__ int sequence_of(int64_t row) const {
    if (!starts) return one_each ? (int)(row < count ? row : count) : 0;
    return last_not_above([&](int i) { return (int64_t)start(i); }, count + 1, row);
  }
};

// Sequences are cut into tiles of `tile` units, `per_row` units a row.  The host knows only how many rows there are, so
// sequence i is given the tiles from start(i) * per_row / tile + i on: at least as many as it needs, whatever the starts.
__host__ __device__ __forceinline__ int64_t tiles_bound(int64_t rows, int per_row, int tile, int sequences) {
  return rows * per_row / tile + sequences + 1;
}
struct Tile {
  int sequence;  // -1: this tile is no one's
  int start, length;  // its sequence's rows
  int first;     // its first unit within the sequence
  int index, tiles;
};
__device__ __forceinline__ Tile find_tile(const Packed& p, int64_t id, int per_row, int tile) {
  Tile t;
  auto place = [&](int start, int i) { return (int64_t)start * per_row / tile + i; };
  if (p.starts && p.count < 63) {
    // a lane for each sequence: what is found of it is in another lane's registers already
    const int lane = (int)(threadIdx.x & 63u), mine = p.start(min(lane, p.count));
    const int found = __popcll(lanes_where(lane <= p.count && place(mine, lane) <= id)) - 1;
    t.sequence = __builtin_amdgcn_readfirstlane(found);
    if (t.sequence < 0) return t;
    t.start = __builtin_amdgcn_readlane(mine, t.sequence);
    t.length = max((t.sequence < p.count ? __builtin_amdgcn_readlane(mine, t.sequence + 1) : p.rows) - t.start, 0);
  } else {
    t.sequence = last_not_above([&](int i) { return place(p.start(i), i); }, p.count + 1, id);
    if (t.sequence < 0) return t;
    t.start = p.start(t.sequence);
    t.length = p.length(t.sequence);
  }
  const int64_t units = (int64_t)t.length * per_row, at = id - place(t.start, t.sequence);
  t.tiles = (int)((units + tile - 1) / tile);
  t.index = (int)at;
  t.first = (int)(at * tile);
  if (at < 0 || at * tile >= units) t.sequence = -1;  // below 0: starts that fall
  return t;
}

// A value over the four lanes that hold a column of a result (16 apart).  Swapping a register's rows of lanes with its own copy's puts
// a lane's value and its neighbour's side by side.
template <class OP> __device__ __forceinline__ float over_groups(float v, OP op) {
  const uint32_t u = __float_as_uint(v);
  const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  const uint32_t w = __float_as_uint(op(__uint_as_float(a[0]), __uint_as_float(a[1])));
  const auto b = __builtin_amdgcn_permlane32_swap(w, w, false, false);
  return op(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float over_groups_max(float v) {
  return over_groups(v, [](float x, float y) { return fmaxf(x, y); });
}
__device__ __forceinline__ float over_groups_sum(float v) {
  return over_groups(v, [](float x, float y) { return x + y; });
}

template <class T> struct Eight { T t[8]; };
template <class T> __device__ __forceinline__ void load8(const T* p, float (&v)[8]) {
  const Eight<T> e = load_any<Eight<T>>(p);
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = (float)e.t[i];
}

// Weights are 2^(score * factor - largest) in one operation, whose product keeps all of its bits; the largest's were rounded.  From
// scores of 2^20 on that difference is no longer small against 1 (at 2^25 a weight leaves binary16, at 2^31 binary32): such a
// wave takes the largest off first, so that its own weight is exact.
__device__ __forceinline__ bool far_scores(float largest) {
  const float m = fabsf(largest);
  return lanes_where(m > 0x1p20f && m < __builtin_inff()) != 0;
}

template <bool B> struct Constant { static constexpr bool value = B; };

constexpr float kInfinity = __builtin_inff();

}  // namespace att
}  // namespace squant
