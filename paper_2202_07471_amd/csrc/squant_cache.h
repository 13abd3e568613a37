// The quantised cache: where a token lies, and the kernels that write tokens to it and read them back.
//
// Both are bound by memory.  A lane takes 8 elements at a time (a 16-byte load or store of a 16-bit type; 4 or 8 bytes of codes), four
// lanes the 32 that share a scale, so the largest magnitude takes two moves within a quad and no LDS.  A workgroup takes up
// to 64 rows, whose slots it finds at once, a thread each; a thread has the loads of four pieces on their way.
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
  uint32_t piece_magic;  // i / pieces for the indices of a workgroup, as a high word
  int32_t dim_pieces;    // of a head
  uint32_t dim_magic;
  int32_t rows_each;     // of a workgroup
};

constexpr int kMostRows = 64;
constexpr int kKnownStarts = kThreads;  // that fit the LDS

// Slots of a workgroup's rows: the cache row of head 0, -1: no page, -2: not a token of any sequence.
__device__ __forceinline__ void find_slots(const CacheRowsArgs& a, int64_t first, int32_t (&slots)[kMostRows], int32_t (&starts)[kKnownStarts]) {
  const Packed& p = a.rows;
  const bool known = p.count < kKnownStarts;
  if (p.starts && known) {
    starts[threadIdx.x] = p.start(min((int)threadIdx.x, p.count));
    __syncthreads();
  }
  const int64_t row = first + (int)threadIdx.x;
  if ((int)threadIdx.x < a.rows_each) {
    int32_t slot = -2;
    if (row < p.rows) {
      // the last sequence that begins at the row or before
      int s = (int)min(row, (int64_t)p.count);
      if (p.starts) {
        auto start = [&](int i) { return known ? starts[i] : p.start(i); };
        int below = -1, above = p.count + 1;  // start(below) <= row < start(above)
        while (above - below > 1) {
          const int middle = (above + below) / 2;
          if (start(middle) <= row) below = middle;
          else above = middle;
        }
        s = below;
      }
      if (s >= 0 && s < p.count) {
        const int64_t t = (int64_t)a.cache.lengths[s] - (p.one_each ? 1 : p.start(s + 1) - row);
        if (t >= 0) {
          const int32_t page = a.cache.page_of((int32_t)t);
          slot = a.cache.row_of((int32_t)t, page, a.cache.table_at(s, page));
        }
      }
    }
    slots[threadIdx.x] = slot;
  }
  __syncthreads();
}

// Piece `at` of a workgroup's rows.
struct Piece {
  int row, tensor, head, d;  // d: in pieces
  __device__ __forceinline__ Piece(const CacheRowsArgs& a, int at) {
    row = (int)__umulhi((uint32_t)at, a.piece_magic);
    const int piece = at - row * a.pieces, half = a.pieces / 2;
    tensor = piece >= half;
    const int p = piece - tensor * half;
    head = (int)__umulhi((uint32_t)p, a.dim_magic);
    d = p - head * a.dim_pieces;
  }
};
constexpr int kAtOnce = 4;  // pieces of a thread on their way

// Past the caches: what is read back is more than they hold, and kept there it goes to memory in pieces (66815 tokens of 8 heads of 128 in 4 bits
// to bfloat16 106 us, 66 like this).
typedef uint32_t stream4v __attribute__((ext_vector_type(4), aligned(2)));
template <class T> __device__ __forceinline__ void stream8(T* p, const float (&v)[8]) {
  Eight<T> e;
#pragma unroll
  for (int i = 0; i < 8; ++i) e.t[i] = (T)v[i];
  struct Pieces { stream4v w[sizeof(T) / 2]; };
  const Pieces pieces = __builtin_bit_cast(Pieces, e);
#pragma unroll
  for (int i = 0; i < (int)sizeof(T) / 2; ++i) __builtin_nontemporal_store(pieces.w[i], reinterpret_cast<stream4v*>(p) + i);
}

__device__ __forceinline__ uint16_t bfloat16_bits(float v) { return __builtin_bit_cast(uint16_t, (__bf16)v); }
__device__ __forceinline__ float from_bfloat16(uint32_t bits) { return __uint_as_float(bits << 16); }

// Codes of 8 elements.  scale has 8 significant bits, so (code + 1/2) * scale are binary32 numbers with at most 16 significant bits, and a
// quotient that is no code and a half is at least 2^-24 (1 + 2^-8) of it away: the nearest integer of the quotient rounded to binary32 is
// that of the real one.  That holds for the quotient by the reciprocal and one correction as well (2^-46 of it off before its
// rounding), which is a third of a division's instructions; scales at the ends of binary32's range are divided by.
template <int FMT>
__device__ __forceinline__ void encode(const float (&v)[8], float scale, uint32_t (&o)[FMT == SQUANT_OUT_INT4 ? 1 : 2]) {
  constexpr float top = FMT == SQUANT_OUT_INT4 ? 7.0f : 127.0f;
  float q[8];
  if (scale > 0x1p-90f && scale < 0x1p90f) {
    const float r = 1.0f / scale;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float guess = v[i] * r;
      q[i] = __builtin_fmaf(__builtin_fmaf(-guess, scale, v[i]), r, guess);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) q[i] = scale > 0.0f ? v[i] / scale : 0.0f;
  }
  // an integer of a byte, added to 1.5 * 2^23, is the low byte of the sum; the addition rounds to it, ties to even
  uint32_t c[8], bytes[2];
#pragma unroll
  for (int i = 0; i < 8; ++i) c[i] = __float_as_uint(__builtin_amdgcn_fmed3f(q[i], -top, top) + 12582912.0f);
#pragma unroll
  for (int d = 0; d < 2; ++d)
    bytes[d] = scale > 0.0f ? lin::pick(c[4 * d + 1], c[4 * d], 0x0c0c0400u) | lin::pick(c[4 * d + 3], c[4 * d + 2], 0x04000c0cu) : 0u;
  if constexpr (FMT == SQUANT_OUT_INT4) {
#pragma unroll
    for (int d = 0; d < 2; ++d) {
      bytes[d] &= 0x0f0f0f0fu;
      bytes[d] |= bytes[d] >> 4;
    }
    o[0] = lin::pick(bytes[1], bytes[0], 0x06040200u);
  } else {
    o[0] = bytes[0], o[1] = bytes[1];
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
  __shared__ int32_t slots[kMostRows], starts[kKnownStarts];
  const int64_t first = (int64_t)blockIdx.x * a.rows_each;
  find_slots(a, first, slots, starts);
  const int items = a.rows_each * a.pieces;  // pieces is a multiple of 4: the lanes of a quad share a group
  for (int at = (int)threadIdx.x; at < items; at += kAtOnce * kThreads) {
    float v[kAtOnce][8];
    int32_t slot[kAtOnce];
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      const int here = at + i * kThreads;
      const Piece p(a, min(here, items - 1));
      slot[i] = here < items ? slots[p.row] : -1;
#pragma unroll
      for (int e = 0; e < 8; ++e) v[i][e] = 0.0f;
      if (slot[i] >= 0) load8(element<T>(a.x[p.tensor], first + p.row, p.head) + p.d * 8, v[i]);
    }
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      const Piece p(a, min(at + i * kThreads, items - 1));
      uint32_t m = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) m = max(m, magnitude(v[i][e]));
      m = max(m, (uint32_t)__shfl_xor((int)m, 1));
      m = max(m, (uint32_t)__shfl_xor((int)m, 2));
      const uint16_t bits = m < 0x7f800000u ? bfloat16_bits(__uint_as_float(m) / top) : (uint16_t)0x7fc0;
      uint32_t o[W];
      encode<FMT>(v[i], from_bfloat16(bits), o);
      if (slot[i] < 0) continue;
      const int64_t row = (int64_t)slot[i] + (int64_t)p.head * a.cache.page_size;
      struct Words { uint32_t w[W]; } words;
#pragma unroll
      for (int k = 0; k < W; ++k) words.w[k] = o[k];
      *reinterpret_cast<Words*>(a.cache.codes[p.tensor] + row * (a.cache.dim / 8 * 4 * W) + p.d * 4 * W) = words;
      if ((p.d & 3) == 0) a.cache.scales[p.tensor][row * (a.cache.dim / kGroup) + p.d / 4] = bits;
    }
  }
}

template <class T, int FMT> __global__ __launch_bounds__(kThreads) void cache_read(CacheRowsArgs a) {
  constexpr int W = FMT == SQUANT_OUT_INT4 ? 1 : 2;
  __shared__ int32_t slots[kMostRows], starts[kKnownStarts];
  const int64_t first = (int64_t)blockIdx.x * a.rows_each;
  find_slots(a, first, slots, starts);
  const int items = (int)min((int64_t)a.rows_each, a.rows.rows - first) * a.pieces;
  for (int at = (int)threadIdx.x; at < items; at += kAtOnce * kThreads) {
    struct Words { uint32_t w[W]; } words[kAtOnce];
    uint16_t scale[kAtOnce];
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      const Piece p(a, min(at + i * kThreads, items - 1));
      const int64_t row = (int64_t)max(slots[p.row], 0) + (int64_t)p.head * a.cache.page_size;
      words[i] = *reinterpret_cast<const Words*>(a.cache.codes[p.tensor] + row * (a.cache.dim / 8 * 4 * W) + p.d * 4 * W);
      scale[i] = a.cache.scales[p.tensor][row * (a.cache.dim / kGroup) + p.d / 4];
    }
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      if (at + i * kThreads >= items) break;
      const Piece p(a, at + i * kThreads);
      const int32_t slot = slots[p.row];
      uint32_t o[W];
#pragma unroll
      for (int k = 0; k < W; ++k) o[k] = slot == -2 ? 0 : words[i].w[k];
      float v[8];
      decode<FMT>(o, slot == -1 ? __builtin_nanf("") : slot == -2 ? 0.0f : from_bfloat16(scale[i]), v);
      stream8(element<T>(a.x[p.tensor], first + p.row, p.head) + p.d * 8, v);
    }
  }
}

typedef void (*cache_rows_t)(CacheRowsArgs);
cache_rows_t cache_write_kernel(int type, int format);
cache_rows_t cache_read_kernel(int type, int format);

}  // namespace att
}  // namespace squant
