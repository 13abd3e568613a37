// The quantised cache: where a token lies, and the kernels that write tokens to it and read them back.
//
// Both are bound by memory.  A lane takes 8 elements (a 16-byte load or store of a 16-bit type; 4 or 8 bytes of codes), four
// lanes the 32 that share a scale, so the largest magnitude takes two moves within a quad and no LDS.
#pragma once

#include "squant_att.h"

namespace squant {
namespace att {

struct Cache {
  uint8_t* codes[2];    // keys, values
  uint16_t* scales[2];
  int32_t pages, page_size, heads, dim;
  // t / page_size for 0 <= t < 2^31 as the high word of t * magic, shifted
  uint32_t magic;
  int32_t shift;        // -1: pages of one token
  const int32_t* table;
  int32_t table_width;
  const int32_t* lengths;

  __device__ __forceinline__ int32_t page_of(int32_t t) const {
    return shift < 0 ? t : (int32_t)(__umulhi((uint32_t)t, magic) >> shift);
  }
  __device__ __forceinline__ int32_t table_at(int sequence, int32_t page) const {
    return (uint32_t)page < (uint32_t)table_width ? table[(int64_t)sequence * table_width + page] : -1;
  }
  // The row [page][head][slot] of head 0, or -1 for a token whose page is none; the rows of other heads lie page_size apart.
  __device__ __forceinline__ int32_t row_of(int32_t t, int32_t page, int32_t id) const {
    return (uint32_t)id < (uint32_t)pages ? id * heads * page_size + (t - page * page_size) : -1;
  }
};

struct CacheRowsArgs {
  Cache cache;
  Packed rows;
  Strided x[2];          // keys, values
  int32_t pieces;        // 8 elements each, of a row's keys and values
  uint32_t piece_magic;  // i / pieces for the indices of a workgroup
  int32_t dim_pieces, rows_each;
};

constexpr int kMostRows = 64;  // of a workgroup

// Slots of a workgroup's rows: the cache row of head 0, -1: no page, -2: not a token of any sequence.
__device__ __forceinline__ void find_slots(const CacheRowsArgs& a, int64_t first, int32_t (&slots)[kMostRows]) {
  const int wave = (int)threadIdx.x / 64, lane = (int)threadIdx.x % 64;
  for (int r = wave; r < a.rows_each; r += kThreads / 64) {
    const int64_t row = first + r;
    int32_t slot = -2;
    if (row < a.rows.rows) {
      const int s = a.rows.sequence_of(row);
      if (s >= 0 && s < a.rows.count) {
        const int32_t t = a.cache.lengths[s] - (int32_t)(a.rows.start(s) + a.rows.length(s) - row);
        if (t >= 0) {
          const int32_t page = a.cache.page_of(t);
          slot = a.cache.row_of(t, page, a.cache.table_at(s, page));
        }
      }
    }
    if (lane == 0) slots[r] = slot;
  }
  __syncthreads();
}

template <class T> __device__ __forceinline__ void load8(const T* p, float (&v)[8]) {
  struct Eight { T t[8]; };
  const Eight e = load_any<Eight>(p);
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = (float)e.t[i];
}
template <class T> __device__ __forceinline__ void store8(T* p, const float (&v)[8]) {
  struct Eight { T t[8]; };
  Eight e;
#pragma unroll
  for (int i = 0; i < 8; ++i) e.t[i] = (T)v[i];
  store_any(p, e);
}

__device__ __forceinline__ uint16_t bfloat16_bits(float v) { return __builtin_bit_cast(uint16_t, (__bf16)v); }
__device__ __forceinline__ float from_bfloat16(uint32_t bits) { return __uint_as_float(bits << 16); }

// Codes of 8 elements.  scale has 8 significant bits, so (code + 1/2) * scale are binary32 numbers, and no other quotient of
// binary32 numbers rounds to a code and a half: the nearest integer of the rounded quotient is that of the real one.
template <int FMT>
__device__ __forceinline__ void encode(const float (&v)[8], float scale, uint32_t (&o)[FMT == SQUANT_OUT_INT4 ? 1 : 2]) {
  constexpr float top = FMT == SQUANT_OUT_INT4 ? 7.0f : 127.0f;
  int c[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float q = fminf(fmaxf(__builtin_rintf(v[i] / scale), -top), top);
    c[i] = scale > 0.0f ? (int)q : 0;
  }
  if constexpr (FMT == SQUANT_OUT_INT4) {
    o[0] = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) o[0] |= ((uint32_t)c[i] & 15u) << (4 * i);
  } else {
#pragma unroll
    for (int d = 0; d < 2; ++d) {
      o[d] = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) o[d] |= ((uint32_t)c[4 * d + i] & 255u) << (8 * i);
    }
  }
}

template <int FMT>
__device__ __forceinline__ void decode(const uint32_t (&o)[FMT == SQUANT_OUT_INT4 ? 1 : 2], float scale, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int c = FMT == SQUANT_OUT_INT4 ? (int)(o[0] << (28 - 4 * i)) >> 28 : (int)(int8_t)(o[(i >> 2) * (FMT != SQUANT_OUT_INT4)] >> (8 * (i & 3)));
    v[i] = (float)c * scale;
  }
}

template <class T, int FMT> __global__ __launch_bounds__(kThreads) void cache_write(CacheRowsArgs a) {
  constexpr int W = FMT == SQUANT_OUT_INT4 ? 1 : 2;
  constexpr float top = FMT == SQUANT_OUT_INT4 ? 7.0f : 127.0f;
  __shared__ int32_t slots[kMostRows];
  const int64_t first = (int64_t)blockIdx.x * a.rows_each;
  find_slots(a, first, slots);
  const int items = a.rows_each * a.pieces;  // pieces is a multiple of 4: the lanes of a quad share a group
  for (int at = (int)threadIdx.x; at < items; at += kThreads) {
    const int r = (int)__umulhi((uint32_t)at, a.piece_magic), piece = at - r * a.pieces;
    const int32_t slot = slots[r];
    if (slot < 0) continue;
    const int half = a.pieces / 2, tensor = piece >= half, p = piece - tensor * half;
    const int head = p / a.dim_pieces, d = p - head * a.dim_pieces;
    float v[8];
    load8(element<T>(a.x[tensor], first + r, head) + d * 8, v);
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, magnitude(v[i]));
    m = max(m, (uint32_t)__shfl_xor((int)m, 1));
    m = max(m, (uint32_t)__shfl_xor((int)m, 2));
    const uint16_t bits = m < 0x7f800000u ? bfloat16_bits(__uint_as_float(m) / top) : (uint16_t)0x7fc0;
    uint32_t o[W];
    encode<FMT>(v, from_bfloat16(bits), o);
    const int64_t row = (int64_t)slot + (int64_t)head * a.cache.page_size;
    struct Words { uint32_t w[W]; } words;
#pragma unroll
    for (int i = 0; i < W; ++i) words.w[i] = o[i];
    *reinterpret_cast<Words*>(a.cache.codes[tensor] + row * (a.cache.dim / 8 * 4 * W) + d * 4 * W) = words;
    if ((d & 3) == 0) a.cache.scales[tensor][row * (a.cache.dim / kGroup) + d / 4] = bits;
  }
}

template <class T, int FMT> __global__ __launch_bounds__(kThreads) void cache_read(CacheRowsArgs a) {
  constexpr int W = FMT == SQUANT_OUT_INT4 ? 1 : 2;
  __shared__ int32_t slots[kMostRows];
  const int64_t first = (int64_t)blockIdx.x * a.rows_each;
  find_slots(a, first, slots);
  const int items = a.rows_each * a.pieces;
  for (int at = (int)threadIdx.x; at < items; at += kThreads) {
    const int r = (int)__umulhi((uint32_t)at, a.piece_magic), piece = at - r * a.pieces;
    if (first + r >= a.rows.rows) continue;
    const int32_t slot = slots[r];
    const int half = a.pieces / 2, tensor = piece >= half, p = piece - tensor * half;
    const int head = p / a.dim_pieces, d = p - head * a.dim_pieces;
    const int64_t row = (int64_t)max(slot, 0) + (int64_t)head * a.cache.page_size;
    struct Words { uint32_t w[W]; };
    const Words words = *reinterpret_cast<const Words*>(a.cache.codes[tensor] + row * (a.cache.dim / 8 * 4 * W) + d * 4 * W);
    uint32_t o[W];
#pragma unroll
    for (int i = 0; i < W; ++i) o[i] = words.w[i];
    const float scale = from_bfloat16(a.cache.scales[tensor][row * (a.cache.dim / kGroup) + d / 4]);
    float v[8];
    decode<FMT>(o, slot == -1 ? __builtin_nanf("") : scale, v);
    if (slot == -2) {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = 0.0f;
    }
    store8(element<T>(a.x[tensor], first + r, head) + d * 8, v);
  }
}

typedef void (*cache_rows_t)(CacheRowsArgs);
cache_rows_t cache_write_kernel(int type, int format);
cache_rows_t cache_read_kernel(int type, int format);

}  // namespace att
}  // namespace squant
