// Attention of one or a few new tokens of each sequence over the quantised cache.
//
//   out[r] = sum_t p[r, t] V[t],  p = softmax_t(scale * Q[r] . K[t]),  K and V = codes * scales.
//
// A workgroup takes 16 or 32 rows (new tokens times the query heads of a key head) and a stretch of the sequence, its four
// waves 32 tokens each in turn; a wave reads codes and scales from memory straight into the lanes that multiply them, a block of
// tokens ahead.  Codes become binary16 numbers code * scale * 2^e with an exponent for the wave (running: a block with a
// larger scale lowers it, and the output's sums with it).  For 4 bits that is exact, 3 bits of a code and 8 of a scale being 11, for scales
// down to about 2^-24 of the largest that the wave has met; below, an element loses bits (`wide` says what of them).
// For 8 bits it would round to 11 bits (2^-12 of an element): binary16 and binary32 calls take the remainder as a second plane
// (11 drafted tokens' binary16 outputs 5.5e-4 off without it, 2.1e-4 with), bfloat16 ones do without.  Queries are
// binary16 with an exponent for each row: two planes for binary32, whose lower one does not meet the remainders (2^-24 of a product).  Softmax
// weights are rounded to 11 bits times 2^14 (binary32: two planes).  Sums are binary32.
//
// Layout of a block: lane 16 g + n.
//   keys    lane holds token n (and 16 + n), the g-th quarter of its codes: NG fragments of 8 codes.
//   scores  column n = row of the queries, tokens 4 g .. 4 g + 3 (and 16 + those): after exp they are the operand
//           of the second product as they are.
//   values  lane holds the same 8 tokens' codes of elements 2 NG n .. 2 NG n + 2 NG - 1, transposed in registers.
#pragma once

#include "squant_cache.h"

namespace squant {
namespace att {

struct CacheAttentionArgs {
  Cache cache;
  Packed rows;
  Strided q, out;
  int32_t heads, group;  // query heads, and of a key head
  int32_t splits;
  int32_t chunk;         // tokens of a split, a multiple of 128
  float scale;           // times log2(e)
  float* partial;        // [splits][rows][heads][dim]
  float2* stats;         // [splits][rows][heads]: largest score (base 2), sum of weights
};

constexpr int kTokens = 32;                 // of a wave's block
constexpr int kWaves = kThreads / 64;
constexpr float kWeightUnit = 14.0f;        // weights are held times 2^14

// A type's `a` and `b` as the two halves.
__device__ __forceinline__ half2v pair(_Float16 a, _Float16 b) { return half2v{a, b}; }

template <int FMT, int NG> struct Layout {
  static constexpr int kBits = FMT == SQUANT_OUT_INT4 ? 4 : 8;
  static constexpr int kRow = NG * kGroup * kBits / 8;   // bytes
  static constexpr int kKeyWords = kRow / 16;            // a lane's quarter
  static constexpr int kValueBytes = kRow / 16;          // a lane's sixteenth
  static constexpr int kValueWords = (kValueBytes + 3) / 4;
  // Scale groups that a lane's quarter of a key, or its sixteenth of a value, lies in; NG of 3 and 6 have it in two at most.
  static constexpr int kKeyScales = NG % 4 == 0 ? NG / 4 : NG <= 2 ? 1 : 2;
  static constexpr int kValueScales = NG == 3 || NG == 6 ? 2 : 1;
};

// Bits that make a 4-bit two's complement code in the low, or the high, half of a byte the binary16 number 1024 + code + 8, or
// 1024 + 16 (code + 8): (u & mask) ^ magic.  One instruction, which takes one constant from a scalar register; these are in vector registers.
struct Magic {
  uint32_t low, high;
  __device__ __forceinline__ Magic() {
    asm("v_mov_b32 %0, 0x64086408" : "=v"(low));
    asm("v_mov_b32 %0, 0x64806480" : "=v"(high));
  }
};

// 8 codes as binary16 integers (times 16 where `slot_unit` says so); element order as `slot_element` has it.
template <int FMT> __device__ __forceinline__ void key_codes(const uint32_t* w, const Magic& magic, half2v (&o)[4]) {
  if constexpr (FMT == SQUANT_OUT_INT4) {
    const uint32_t u = w[0], v = u >> 8;
    const half2v low = pair((_Float16)1032.0f, (_Float16)1032.0f), high = pair((_Float16)1152.0f, (_Float16)1152.0f);
    o[0] = lin::as_half2((u & 0x000f000fu) ^ magic.low) - low;
    o[1] = lin::as_half2((u & 0x00f000f0u) ^ magic.high) - high;
    o[2] = lin::as_half2((v & 0x000f000fu) ^ magic.low) - low;
    o[3] = lin::as_half2((v & 0x00f000f0u) ^ magic.high) - high;
  } else {
    const half2v bias = pair((_Float16)1152.0f, (_Float16)1152.0f);
#pragma unroll
    for (int d = 0; d < 2; ++d) {
      const uint32_t u = w[d] ^ 0x80808080u;
      o[2 * d] = lin::as_half2(lin::pick(0x64646464u, u, 0x04010400u)) - bias;
      o[2 * d + 1] = lin::as_half2(lin::pick(0x64646464u, u, 0x04030402u)) - bias;
    }
  }
}
// The element (of 8) in slot s of a key's fragment, and the power of two its code is held times.
template <int FMT> __device__ __forceinline__ constexpr int slot_element(int s) {
  return FMT == SQUANT_OUT_INT4 ? (s >> 1) + 4 * (s & 1) : s;
}
template <int FMT> __device__ __forceinline__ constexpr float slot_unit(int s) {
  return FMT == SQUANT_OUT_INT4 && (s & 2) ? 0.0625f : 1.0f;
}

// Codes of tokens 2 m and 2 m + 1 for one element: byte `p` (low or high half of it) of a and b.  Codes of high halves are times 16.
template <int FMT> __device__ __forceinline__ half2v value_codes(uint32_t a, uint32_t b, const Magic& magic, int p, int high) {
  const uint32_t u = lin::pick(b, a, 0x0c040c00u + 0x00010001u * (uint32_t)p);
  if constexpr (FMT == SQUANT_OUT_INT4)
    return high ? lin::as_half2((u & 0x00f000f0u) ^ magic.high) - pair((_Float16)1152.0f, (_Float16)1152.0f)
                : lin::as_half2((u & 0x000f000fu) ^ magic.low) - pair((_Float16)1032.0f, (_Float16)1032.0f);
  return lin::as_half2(u ^ magic.high) - pair((_Float16)1152.0f, (_Float16)1152.0f);
}

__device__ __forceinline__ uint32_t over_lanes_max(uint32_t v) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) v = max(v, (uint32_t)__shfl_xor((int)v, o));
  return v;
}

// Scales times 2^e stay below 512 (times 8 or 16 of a code, in binary16).  The exponent that brings the largest finite one to
// [2^7, 2^8).
__device__ __forceinline__ int scale_exponent(uint32_t top) {
  if (top == 0) return 126;
  return min(7 - ((int)(top >> 23) - 127), 126);
}
__device__ __forceinline__ uint32_t finite_bits(float v) {
  const uint32_t m = magnitude(v);
  return m < 0x7f800000u ? m : 0u;
}
// bfloat16 bits of 512 / 2^e: scales from there on are too large for e, or no numbers.
__device__ __forceinline__ uint32_t too_large(int e) { return min((uint32_t)(9 - e + 127) << 7, 0x7f80u); }

// Waves a SIMD that registers are kept for.  Three are what most take; asked for more, heads of 128 spill (96 sequences 171 us, 211), and so do
// 32 rows at three (eleven sequences' drafts 36 us, 61).  At two, heads of 256 over 8 bits keep 22 to 43 registers in memory, binary32 calls
// 101 to 126 (9 to 33 of others with 32 rows or heads of 192).
constexpr int cache_occupancy(int ng, int rt) { return ng <= 2 && rt == 1 ? 3 : 2; }

// One row by a wave, token by token: for tiles whose rows cannot share exponents, which are seldom.  Scores and sums are binary64: with powers of two
// of their own, the other rows' do not leave binary32 either.  A lane for each token, then for each element.
template <class T, int FMT, int NG>
__device__ __forceinline__ void row_alone(const CacheAttentionArgs& a, int seq, int row, int qhead, int head, int split, int begin, int upto, bool beyond) {
  constexpr int W = FMT == SQUANT_OUT_INT4 ? 1 : 2, D = NG * kGroup, E = (D + 63) / 64;
  const Cache& c = a.cache;
  const int lane = (int)threadIdx.x & 63;
  const T* q = element<T>(a.q, row, qhead);
  // the token's row of the cache, -1: its page is none
  auto where = [&](int t) -> int64_t {
    const int page = c.page_of(t);
    const int32_t r = c.row_of(t, page, c.table_at(seq, page));
    return r < 0 ? -1 : (int64_t)r + (int64_t)head * c.page_size;
  };
  auto scale_of = [&](int tensor, int64_t r, int group) {
    const uint16_t bits = r < 0 ? (uint16_t)0x7fc0 : c.scales[tensor][r * NG + group];
    return (bits & 0x7fffu) < 0x7f80u ? from_bfloat16(bits) : __builtin_nanf("");
  };
  auto score = [&](int t) {
    const int64_t r = where(t);
    double s = 0.0;
#pragma unroll 1
    for (int i = 0; i < 4 * NG; ++i) {
      uint32_t words[W];
#pragma unroll
      for (int w = 0; w < W; ++w) words[w] = *reinterpret_cast<const uint32_t*>(c.codes[0] + max(r, (int64_t)0) * (D / 8 * 4 * W) + (i * W + w) * 4);
      float x[8], y[8];
      load8(q + 8 * i, x);
      decode<FMT>(words, scale_of(0, r, i >> 2), y);
#pragma unroll
      for (int e = 0; e < 8; ++e) s = __builtin_fma((double)x[e], (double)y[e], s);
    }
    return s;
  };
  double top = -(double)kInfinity;
#pragma unroll 1
  for (int t = begin + lane; t < upto; t += 64) top = fmax(top, score(t));
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) top = fmax(top, __shfl_xor(top, o));
  const double none = top == -(double)kInfinity ? 0.0 : top, scale = fmaxf(a.scale, 0x1p-149f);
  double total = beyond ? (double)__builtin_nanf("") : 0.0, sum[E] = {};
#pragma unroll 1
  for (int t0 = begin; t0 < upto; t0 += 64) {
    const float w = t0 + lane < upto ? exp2_fast((float)((score(t0 + lane) - none) * scale)) : 0.0f;
    total += w;
    const int count = min(64, upto - t0);
#pragma unroll 1
    for (int i = 0; i < count; ++i) {
      const int64_t r = where(t0 + i);
      const float one = __shfl(w, i);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int d = lane + 64 * e;
        if (d >= D) continue;
        const uint8_t byte = c.codes[1][max(r, (int64_t)0) * (D / 2 * W) + (FMT == SQUANT_OUT_INT4 ? d / 2 : d)];
        const int code = FMT == SQUANT_OUT_INT4 ? (int)((uint32_t)byte << (28 - 4 * (d & 1))) >> 28 : (int)(int8_t)byte;
        sum[e] = __builtin_fma((double)one, (double)code * (double)scale_of(1, r, d / kGroup), sum[e]);
      }
    }
  }
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) total += __shfl_xor(total, o);
  const int64_t at = ((int64_t)split * a.rows.rows + row) * a.heads + qhead;
  if (a.splits > 1 && lane == 0) a.stats[at] = make_float2((float)(top * scale), (float)total);
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const int d = lane + 64 * e;
    if (d >= D) continue;
    if (a.splits > 1) a.partial[at * D + d] = (float)sum[e];
    else element<T>(a.out, row, qhead)[d] = (T)(float)(total == 0.0 ? 0.0 : sum[e] / total);
  }
}

// All rows of a tile, dealt to the workgroup's waves.  Arguments are read anew, from a pointer that the compiler does not know: kept until here
// they would take registers from the loop before.
template <class T, int FMT, int NG>
__device__ __forceinline__ void rows_alone(int seq, int row0, int first, int count, int said, int rows_each) {
  typedef const __attribute__((address_space(4))) CacheAttentionArgs* args_t;
  args_t p = (args_t)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(p));
  const CacheAttentionArgs& a = *(const CacheAttentionArgs*)p;
  const int head = (int)blockIdx.x % a.cache.heads, split = (int)blockIdx.y;
  const int64_t capacity = (int64_t)a.cache.table_width * a.cache.page_size;
  const int begin = split * a.chunk, end = min((int)min((int64_t)said, capacity), begin + a.chunk);
#pragma unroll 1
  for (int r = first + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6); r < min(first + rows_each, count * a.group); r += kWaves) {
    const int token = r / a.group, upto = said - count + token + 1;
    row_alone<T, FMT, NG>(a, seq, row0 + token, head * a.group + r - token * a.group, head, split, begin, min(max(upto, 0), end), upto > capacity);
  }
}

// HALVES: pages of a multiple of 16 tokens, of which each half of a block has consecutive rows: their addresses are a number for the
// wave plus one of the lane that stays.
//
// One body for all blocks, with branches of the wave around what only some need: a call of a short sequence spends its time
// on fetching instructions for the first time (with a body of its own for blocks that hide tokens and two blocks a turn
// one token of 8192 took 12 us in this kernel, whether it multiplied or only read).  The next block's keys are on their way from
// a block's beginning on, its values from the end of the products, into the registers that have become free there.
//
// What bounds it: 96 sequences of 1024 to 16384 tokens, 32 heads of 128 on 8, 4 bits: 167 us, 3.4 TB/s of codes and scales; reading them
// without the products takes 125, and vector instructions (1.7 a code: place, centre, scale) issue for about half of the time.
// One token of 8192: 12 us, of which reading alone takes nearly all: a chain of lengths, table, codes, and two joins.
template <class T, int FMT, int NG, int RT, bool HALVES>
__global__ __launch_bounds__(kThreads, cache_occupancy(NG, RT)) void cache_attention(CacheAttentionArgs a) {
  typedef Layout<FMT, NG> L;
  constexpr int PL = sizeof(T) == 4 ? 2 : 1;                                 // planes of queries and weights
  constexpr bool LOW = FMT == SQUANT_OUT_INT8 && !__is_same(T, __bf16);      // the remainder of an element as well
  constexpr int D = NG * kGroup, F = D / 16, TR = 16 * RT, kStep = kWaves * kTokens;
  extern __shared__ float lds[];
  const Cache& c = a.cache;
  const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int n = lane & 15, g = lane >> 4;
  const int head = (int)blockIdx.x % c.heads;
  const int split = (int)blockIdx.y;

  // whose rows these are; of few sequences, lengths are on their way meanwhile
  Tile tile;
  const int tile_id = (int)(blockIdx.x / (uint32_t)c.heads);
  const bool few = a.rows.count <= 64;
  const int lane_length = few && a.rows.count ? c.lengths[min(lane, a.rows.count - 1)] : 0;
  if (a.rows.one_each) {
    const int each = (a.group + TR - 1) / TR;
    tile.sequence = tile_id / each;
    tile.first = (tile_id - tile.sequence * each) * TR;
    tile.start = tile.sequence, tile.length = 1;
    if (tile.sequence >= a.rows.count) return;
  } else {
    tile = find_tile(a.rows, tile_id, a.group, TR);
  }
  if (tile.sequence < 0) return;
  const int seq = tile.sequence, row0 = tile.start, count = tile.length;
  const int64_t capacity = (int64_t)c.table_width * c.page_size;
  int said = 0;
  if (seq < a.rows.count) said = max(few ? __builtin_amdgcn_readlane(lane_length, seq) : c.lengths[seq], 0);
  const int length = (int)min((int64_t)said, capacity);
  const int begin = split * a.chunk, end = min(length, begin + a.chunk);
  if (a.splits > 1 && (begin >= max(length, 1) || seq == a.rows.count)) return;  // the join knows

  // this lane's columns of the scores: rows of the queries
  int row[RT], qhead[RT], seen[RT];
  bool live[RT], beyond[RT];  // beyond: it sees tokens past the table, and is NaN
  int least_seen = 0x7fffffff;
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int r = tile.first + 16 * rt + n;
    const int token = r / a.group;
    live[rt] = r < count * a.group;
    row[rt] = row0 + (live[rt] ? token : 0);
    qhead[rt] = head * a.group + (live[rt] ? r - token * a.group : 0);
    const int upto = live[rt] ? said - count + token + 1 : 0;
    beyond[rt] = upto > capacity;
    seen[rt] = min(max(upto, 0), end);
    if (live[rt]) least_seen = min(least_seen, seen[rt]);
  }
  // rows of a tile see no less than its first
  least_seen = min(__builtin_amdgcn_readfirstlane(least_seen), end);

  // where a block's tokens are: on its way before the queries
  const uint32_t head_row = (uint32_t)head * (uint32_t)c.page_size;
  auto page_ids = [&](int t0, int32_t (&id)[2]) {
    id[0] = id[1] = -1;
    if (seq >= a.rows.count) return;  // rows behind the last sequence have no row of the table
    if constexpr (HALVES) {
#pragma unroll
      for (int h = 0; h < 2; ++h) id[h] = __builtin_amdgcn_readfirstlane(c.table_at(seq, c.page_of(t0 + 16 * h)));
    } else {
      id[0] = id[1] = c.table_at(seq, c.page_of(t0 + (lane & 31)));
    }
  };
  int t0 = begin + wave * kTokens;
  int32_t ids[2];
  page_ids(t0, ids);

  half8 q[RT][PL][NG];
  int q_e[RT];  // queries are held times 2^q_e
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    float x[NG][8];
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < NG; ++i) {
      load8(element<T>(a.q, row[rt], qhead[rt]) + (g * NG + i) * 8, x[i]);
#pragma unroll
      for (int s = 0; s < 8; ++s) top = max(top, finite_bits(x[i][s]));
    }
    top = max(top, (uint32_t)__shfl_xor((int)top, 16));
    top = max(top, (uint32_t)__shfl_xor((int)top, 32));
    const int e = lin::row_exponent(top);
    const float up = power_of_two(e);
    q_e[rt] = e;
#pragma unroll
    for (int i = 0; i < NG; ++i)
#pragma unroll
      for (int s = 0; s < 8; ++s) {
        const float v = x[i][slot_element<FMT>(s)] * up * slot_unit<FMT>(s);
        const _Float16 hi = (_Float16)v;
        q[rt][0][i][s] = hi;
        if constexpr (PL == 2) q[rt][1][i][s] = magnitude(v) < 0x7f800000u ? (_Float16)(v - (float)hi) : (_Float16)0.0f;
      }
  }

  // Where a block's tokens lie, those past the sequence's end wherever the table says.  `bad`: tokens whose page is none.
  struct Where {
    int64_t first[2];  // HALVES: rows of the halves' first tokens
    int32_t row;       // else: the row of token t0 + lane % 32
    uint32_t bad;
  };
  auto find = [&](Where& w, int t0, const int32_t (&id)[2]) {
    w.bad = 0;
    if constexpr (HALVES) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int t = t0 + 16 * h;
        const int32_t r = c.row_of(t, c.page_of(t), id[h]);
        if (r < 0) w.bad |= 0xffffu << (16 * h);
        w.first[h] = r < 0 ? 0 : (int64_t)(r + head_row);  // rows 0 to 15 are there
      }
    } else {
      const int t = t0 + (lane & 31);
      const int32_t r = c.row_of(t, c.page_of(t), id[0]);
      w.bad = (uint32_t)lanes_where(r < 0);
      w.row = r < 0 ? 0 : (int32_t)(r + head_row);
    }
  };
  // bases for the wave and offsets of the lane
  struct Place {
    const uint8_t* codes;
    const uint16_t* scales;
    uint32_t byte, scale;
  };
  auto place = [&](const Where& w, int tensor, int h, int token) {
    if constexpr (HALVES) {
      return Place{c.codes[tensor] + w.first[h] * L::kRow, c.scales[tensor] + w.first[h] * NG, (uint32_t)(token * L::kRow), (uint32_t)(token * NG)};
    } else {
      const int64_t r = __shfl(w.row, 16 * h + token);
      return Place{c.codes[tensor] + r * L::kRow, c.scales[tensor] + r * NG, 0, 0};
    }
  };
  uint32_t key[2][L::kKeyWords], value[8][L::kValueWords];
  uint16_t key_scale[2][L::kKeyScales], value_scale[8][L::kValueScales];
  // key token 16 tt + n, value token 4 g + j (j < 4), 16 + 4 g + j - 4
  uint32_t next_key[2][L::kKeyWords];
  uint16_t next_key_scale[2][L::kKeyScales];
  auto load_keys = [&](const Where& w, uint32_t (&key)[2][L::kKeyWords], uint16_t (&key_scale)[2][L::kKeyScales]) {
#pragma unroll
    for (int tt = 0; tt < 2; ++tt) {
      struct Words { uint32_t w[L::kKeyWords]; };
      const Place at = place(w, 0, tt, n);
      const Words v = load_any<Words>(at.codes + (uint32_t)(at.byte + (uint32_t)(g * (L::kRow / 4))));
#pragma unroll
      for (int i = 0; i < L::kKeyWords; ++i) key[tt][i] = v.w[i];
#pragma unroll
      for (int k = 0; k < L::kKeyScales; ++k) key_scale[tt][k] = at.scales[(uint32_t)(at.scale + (uint32_t)min(((g * NG) >> 2) + k, NG - 1))];
    }
  };
  auto load_values = [&](const Where& w) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const Place at = place(w, 1, j >> 2, 4 * g + (j & 3));
      const uint8_t* p = at.codes + (uint32_t)(at.byte + (uint32_t)(n * L::kValueBytes));
      if constexpr (L::kValueBytes % 4 == 0) {
        struct Words { uint32_t w[L::kValueWords]; };
        const Words v = *reinterpret_cast<const Words*>(p);
#pragma unroll
        for (int i = 0; i < L::kValueWords; ++i) value[j][i] = v.w[i];
      } else if constexpr (L::kValueBytes == 6) {
        struct Halves { uint16_t w[3]; };
        const Halves v = *reinterpret_cast<const Halves*>(p);
        value[j][0] = v.w[0] | (uint32_t)v.w[1] << 16;
        value[j][1] = v.w[2];
      } else if constexpr (L::kValueBytes == 2) {
        value[j][0] = *reinterpret_cast<const uint16_t*>(p);
      } else if constexpr (L::kValueBytes == 3) {
        value[j][0] = p[0] | (uint32_t)p[1] << 8 | (uint32_t)p[2] << 16;
      } else {
        static_assert(L::kValueBytes == 1, "");
        value[j][0] = p[0];
      }
#pragma unroll
      for (int k = 0; k < L::kValueScales; ++k) value_scale[j][k] = at.scales[(uint32_t)(at.scale + (uint32_t)min(((2 * NG * n) >> 5) + k, NG - 1))];
    }
  };

  float4v o[F][RT];
#pragma unroll
  for (int f = 0; f < F; ++f)
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) o[f][rt] = float4v{0, 0, 0, 0};
  float largest[RT], sum[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) largest[rt] = -kInfinity, sum[rt] = beyond[rt] ? __builtin_nanf("") : 0.0f;
  int key_e = 126, value_e = 126;
  const Magic magic;
  // Tokens share exponents, and large scales cost small ones their bits.  What a row gets must not depend on tokens that it does not see:
  // `wide` where some row sees a token that another does not, with a scale more than 2^7 times all of those before (of this
  // block, or met by the wave).  An element is otherwise off by at most 9 * 2^-25 (a code's product and its scale, both rounded next to 0)
  // where the largest that the row sees is at least 7 * 2^0: 2^-24 of it.
  bool wide = false;

  Where at, next;
  if (t0 < end) {
    find(at, t0, ids);
    load_keys(at, key, key_scale);
    load_values(at);
    page_ids(t0 + kStep, ids);
  }
#pragma unroll 1
  for (; t0 < end; t0 += kStep) {
    const bool more = t0 + kStep < end;
    if (more) {
      find(next, t0 + kStep, ids);
      load_keys(next, next_key, next_key_scale);
      page_ids(t0 + 2 * kStep, ids);
    }

    const bool some_hidden = t0 + kTokens > least_seen;  // of the block's tokens, for some row
    uint32_t nan_tokens = at.bad;                         // rows that see one of them are NaN
    // Whether the block's largest scale, `most`, is too large for e and for the tokens that are before those which only some rows see.  e stands for
    // scales below 2^(8 - e): an exponent of 134 - e; 126 before there are any.
    auto spread = [&](int e, uint32_t most, auto each) {
      const int cut = max(least_seen, t0 + (e == 126 ? 1 : 0)), top = (int)(most >> 23) - 7;
      if (cut >= min(end, t0 + kTokens) || top <= 134 - e) return false;
      uint32_t before = 0;
      each([&](int t, uint32_t scale) { before = max(before, t < cut ? scale & 0x7fffu : 0u); });
      return lanes_where((int)(before >> 7) >= top) == 0;
    };

    uint32_t top = 0;
#pragma unroll
    for (int tt = 0; tt < 2; ++tt)
#pragma unroll
      for (int k = 0; k < L::kKeyScales; ++k) {
        if (some_hidden && t0 + 16 * tt + n >= end) key_scale[tt][k] = 0;
        top = max(top, (uint32_t)key_scale[tt][k] & 0x7fffu);
      }
    if (lanes_where(top >= too_large(key_e))) {
      uint32_t m = 0;
#pragma unroll
      for (int tt = 0; tt < 2; ++tt) {
        bool none = false;
#pragma unroll
        for (int k = 0; k < L::kKeyScales; ++k) {
          none |= (key_scale[tt][k] & 0x7fffu) >= 0x7f80u;
          m = max(m, finite_bits(from_bfloat16(key_scale[tt][k])));
        }
        // four lanes, 16 apart, share a token.  An infinite scale's products may all be minus infinity: a weight of 0, unless marked
        const uint64_t odd = lanes_where(none), pairs = odd | odd >> 32;
        nan_tokens |= (uint32_t)((pairs | pairs >> 16) & 0xffffu) << (16 * tt);
      }
      const uint32_t most = (uint32_t)__builtin_amdgcn_readfirstlane((int)over_lanes_max(m));
      if (__builtin_expect(some_hidden, false))
        wide |= spread(key_e, most, [&](auto take) {
#pragma unroll
          for (int tt = 0; tt < 2; ++tt)
#pragma unroll
            for (int k = 0; k < L::kKeyScales; ++k) take(t0 + 16 * tt + n, key_scale[tt][k]);
        });
      key_e = min(key_e, scale_exponent(most));
    }
    float4v s[2][RT];
#pragma unroll
    for (int tt = 0; tt < 2; ++tt) {
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) s[tt][rt] = float4v{0, 0, 0, 0};
      _Float16 scale[L::kKeyScales];
#pragma unroll
      for (int k = 0; k < L::kKeyScales; ++k) scale[k] = (_Float16)(from_bfloat16(key_scale[tt][k]) * power_of_two(key_e));
#pragma unroll
      for (int i = 0; i < NG; ++i) {
        _Float16 w = scale[0];
        if constexpr (NG % 4 == 0) w = scale[i >> 2];
        else if constexpr (L::kKeyScales == 2) w = ((g * NG + i) >> 2) > ((g * NG) >> 2) ? scale[1] : scale[0];
        half2v codes[4];
        key_codes<FMT>(key[tt] + i * (L::kBits / 4), magic, codes);
        half8 hi, lo = {};
#pragma unroll
        for (int d = 0; d < 4; ++d) {
          const half2v v = codes[d] * pair(w, w);
          hi[2 * d] = v[0], hi[2 * d + 1] = v[1];
          if constexpr (LOW) {
            const half2v rest = __builtin_elementwise_fma(codes[d], pair(w, w), -v);
            lo[2 * d] = rest[0], lo[2 * d + 1] = rest[1];
          }
        }
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
          s[tt][rt] = Half::mma(hi, q[rt][0][i], s[tt][rt]);
          if constexpr (PL == 2) s[tt][rt] = Half::mma(hi, q[rt][1][i], s[tt][rt]);
          if constexpr (LOW) s[tt][rt] = Half::mma(lo, q[rt][0][i], s[tt][rt]);
        }
      }
    }
    // the values' scales: 0 for tokens past the end, whatever is there, and for those that make rows NaN
    top = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
      for (int k = 0; k < L::kValueScales; ++k) {
        const int token = 4 * g + (j & 3) + 16 * (j >> 2);
        if (some_hidden && t0 + token >= end) value_scale[j][k] = 0;
        top = max(top, (uint32_t)value_scale[j][k] & 0x7fffu);
      }
    if (nan_tokens || lanes_where(top >= too_large(value_e))) {
      uint32_t m = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int token = 4 * g + (j & 3) + 16 * (j >> 2);
        bool none = nan_tokens >> token & 1;
#pragma unroll
        for (int k = 0; k < L::kValueScales; ++k) none |= (value_scale[j][k] & 0x7fffu) >= 0x7f80u;
        const uint64_t odd = lanes_where(none);  // sixteen lanes of a group share a token
#pragma unroll
        for (int g2 = 0; g2 < 4; ++g2)
          if (odd >> (16 * g2) & 0xffffu) nan_tokens |= 1u << (4 * g2 + (j & 3) + 16 * (j >> 2));
      }
#pragma unroll
      for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int k = 0; k < L::kValueScales; ++k) {
          if (nan_tokens >> (4 * g + (j & 3) + 16 * (j >> 2)) & 1) value_scale[j][k] = 0;
          m = max(m, finite_bits(from_bfloat16(value_scale[j][k])));
        }
      const uint32_t most = (uint32_t)__builtin_amdgcn_readfirstlane((int)over_lanes_max(m));
      if (__builtin_expect(some_hidden, false))
        wide |= spread(value_e, most, [&](auto take) {
#pragma unroll
          for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int k = 0; k < L::kValueScales; ++k) take(t0 + 4 * g + (j & 3) + 16 * (j >> 2), value_scale[j][k]);
        });
      const int e = min(value_e, scale_exponent(most));
#pragma unroll
      for (int f = 0; f < F; ++f)
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
          for (int i = 0; i < 4; ++i) o[f][rt][i] = ldexpf(o[f][rt][i], e - value_e);
      value_e = e;
    }
    if (some_hidden || nan_tokens) {
#pragma unroll
      for (int rt = 0; rt < RT; ++rt)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int token = 4 * g + (j & 3) + 16 * (j >> 2);
          if (nan_tokens >> token & 1) s[j >> 2][rt][j & 3] = __builtin_nanf("");
          if (t0 + token >= seen[rt]) s[j >> 2][rt][j & 3] = -kInfinity;
        }
    }

    // softmax weights of the block, times 2^14; what they add up to stays with the lane until the end
    half8 p[RT][PL];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      // Both powers at once: where keys are zeros so far and queries small, or scale is 0, they leave binary32.  Never 0 itself, nor
      // infinite: a hidden score's minus infinity stays one, and a score of 0 too; others times 2^-149 are nothing.
      float f = __builtin_amdgcn_fmed3f(ldexpf(a.scale, -(q_e[rt] + key_e)), 0x1p-149f, 0x1.fffffep127f);
      float m = -kInfinity;
#pragma unroll
      for (int j = 0; j < 8; ++j) m = fmaxf(m, s[j >> 2][rt][j & 3]);
      m = over_groups_max(m) * f;
      if (lanes_where(m > largest[rt])) {
        const float most = fmaxf(m, largest[rt]);
        const float shrink = most == -kInfinity ? 1.0f : exp2_fast(largest[rt] - most);
        sum[rt] *= shrink;
#pragma unroll
        for (int f2 = 0; f2 < F; ++f2)
#pragma unroll
          for (int i = 0; i < 4; ++i) o[f2][rt][i] *= shrink;
        largest[rt] = most;
      }
      float base = largest[rt] == -kInfinity ? 0.0f : kWeightUnit - largest[rt];
      if (__builtin_expect(far_scores(largest[rt]), false)) {
        const float from = largest[rt] == -kInfinity ? 0.0f : largest[rt];
#pragma unroll
        for (int j = 0; j < 8; ++j) s[j >> 2][rt][j & 3] = s[j >> 2][rt][j & 3] * f - from;
        f = 1.0f, base = kWeightUnit;
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float w = exp2_fast(__builtin_fmaf(s[j >> 2][rt][j & 3], f, base));
        sum[rt] += w;
        const _Float16 hi = (_Float16)w;
        p[rt][0][j] = hi;
        if constexpr (PL == 2) p[rt][1][j] = (_Float16)(w - (float)hi);
      }
    }

    half2v scale2[4][L::kValueScales];
#pragma unroll
    for (int m = 0; m < 4; ++m)
#pragma unroll
      for (int k = 0; k < L::kValueScales; ++k)
        scale2[m][k] = pair((_Float16)(from_bfloat16(value_scale[2 * m][k]) * power_of_two(value_e)),
                            (_Float16)(from_bfloat16(value_scale[2 * m + 1][k]) * power_of_two(value_e)));
#pragma unroll
    for (int f = 0; f < F; ++f) {
      const int byte = FMT == SQUANT_OUT_INT4 ? f / 2 : f;
      half8 hi, lo = {};
#pragma unroll
      for (int m = 0; m < 4; ++m) {
        half2v w = scale2[m][0];
        if constexpr (L::kValueScales == 2) w = ((2 * NG * n + f) >> 5) > ((2 * NG * n) >> 5) ? scale2[m][1] : scale2[m][0];
        const half2v codes = value_codes<FMT>(value[2 * m][byte / 4], value[2 * m + 1][byte / 4], magic, byte % 4, f & 1);
        const half2v v = codes * w;
        hi[2 * m] = v[0], hi[2 * m + 1] = v[1];
        if constexpr (LOW) {
          const half2v rest = __builtin_elementwise_fma(codes, w, -v);
          lo[2 * m] = rest[0], lo[2 * m + 1] = rest[1];
        }
      }
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        o[f][rt] = Half::mma(hi, p[rt][0], o[f][rt]);
        if constexpr (PL == 2) o[f][rt] = Half::mma(hi, p[rt][1], o[f][rt]);
        if constexpr (LOW) o[f][rt] = Half::mma(lo, p[rt][0], o[f][rt]);
      }
    }
    if (more) {
      load_values(next);
      at = next;
#pragma unroll
      for (int tt = 0; tt < 2; ++tt) {
#pragma unroll
        for (int i = 0; i < L::kKeyWords; ++i) key[tt][i] = next_key[tt][i];
#pragma unroll
        for (int k = 0; k < L::kKeyScales; ++k) key_scale[tt][k] = next_key_scale[tt][k];
      }
    }
  }

  // the waves' sums become one
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) sum[rt] = over_groups_sum(sum[rt]);
  float* stats = lds;                      // [wave][2][TR]
  float* wides = lds + kWaves * 2 * TR;    // [wave]
  float* pile = wides + kWaves;            // [2][F][RT][64] of four
  if (lane == 0) wides[wave] = wide ? 1.0f : 0.0f;
  if (g == 0) {
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      stats[(wave * 2 + 0) * TR + 16 * rt + n] = largest[rt];
      stats[(wave * 2 + 1) * TR + 16 * rt + n] = sum[rt];
    }
  }
  __syncthreads();
  const float4v any = *reinterpret_cast<const float4v*>(wides);
  if (__builtin_expect(__builtin_amdgcn_readfirstlane(any[0] + any[1] + any[2] + any[3] != 0.0f), false)) {
    rows_alone<T, FMT, NG>(seq, row0, tile.first, count, said, TR);
    return;
  }
  float total[RT], most[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    float m = -kInfinity, l = 0.0f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) m = fmaxf(m, stats[w * 2 * TR + 16 * rt + n]);
    const float base = m == -kInfinity ? 0.0f : m;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) l += stats[(w * 2 + 1) * TR + 16 * rt + n] * exp2_fast(stats[w * 2 * TR + 16 * rt + n] - base);
    // without the weights' unit from here on: with it, values from 2^113 on left binary32
    total[rt] = l * 0x1p-14f, most[rt] = m;
    const float mine = exp2_fast(largest[rt] - base);
#pragma unroll
    for (int f = 0; f < F; ++f)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        // odd elements of 4-bit codes are held times 16
        o[f][rt][i] = ldexpf(o[f][rt][i] * mine, -value_e - (int)kWeightUnit - (FMT == SQUANT_OUT_INT4 && (f & 1) ? 4 : 0));
  }
  float4v* piles = reinterpret_cast<float4v*>(pile);
#pragma unroll
  for (int half = 2; half >= 1; half >>= 1) {
    if (wave >= half && wave < 2 * half) {
#pragma unroll
      for (int f = 0; f < F; ++f)
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) piles[(((wave - half) * F + f) * RT + rt) * 64 + lane] = o[f][rt];
    }
    __syncthreads();
    if (wave < half) {
#pragma unroll
      for (int f = 0; f < F; ++f)
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) o[f][rt] += piles[((wave * F + f) * RT + rt) * 64 + lane];
    }
    __syncthreads();
  }
  if (wave != 0) return;
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    if (!live[rt]) continue;
    const int64_t at = ((int64_t)split * a.rows.rows + row[rt]) * a.heads + qhead[rt];
    const float inverse = a.splits > 1 ? 1.0f : total[rt] == 0.0f ? 0.0f : 1.0f / total[rt];
    if (a.splits > 1 && g == 0) a.stats[at] = make_float2(most[rt], total[rt]);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int d = 2 * NG * (4 * g + i);
#pragma unroll
      for (int f = 0; f < F; f += 2) {
        const float v0 = o[f][rt][i] * inverse, v1 = o[f + 1][rt][i] * inverse;
        if (a.splits > 1) {
          *reinterpret_cast<float2*>(a.partial + at * D + d + f) = make_float2(v0, v1);
        } else {
          struct Two { T v[2]; };
          store_any(element<T>(a.out, row[rt], qhead[rt]) + d + f, Two{{(T)v0, (T)v1}});
        }
      }
    }
  }
}

// The splits of each row and head become its output: a wave for each, lanes in groups of dim / 4 that take a split each, four
// splits of a group on their way at once.
template <class T> __global__ __launch_bounds__(kThreads) void join_splits(CacheAttentionArgs a) {
  const int lane = (int)threadIdx.x & 63;
  const int64_t at = (int64_t)blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int64_t all = (int64_t)a.rows.rows * a.heads;
  if (at >= all) return;
  const int row = (int)(at / a.heads), head = (int)(at - (int64_t)row * a.heads), dim = a.cache.dim;
  const int s = a.rows.sequence_of(row);
  int parts = 0;
  if (s >= 0 && s < a.rows.count) {
    const int64_t length = min((int64_t)max(a.cache.lengths[s], 0), (int64_t)a.cache.table_width * a.cache.page_size);
    parts = (int)((length + a.chunk - 1) / a.chunk);
  }
  // 64, 32 (dim 96: 24), 16 or 8 lanes hold a row of four elements each
  const int lanes = dim / 4, groups = dim == 192 ? 1 : 64 / lanes, group = lane / lanes, d = (lane - group * lanes) * 4;
  const bool mine = group < groups;
  float m = -kInfinity;
  for (int i = lane; i < parts; i += 64) m = fmaxf(m, a.stats[i * all + at].x);
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) m = fmaxf(m, __shfl_xor(m, o));
  const float base = m == -kInfinity ? 0.0f : m;
  float total = 0.0f;
  float4v v = {0, 0, 0, 0};
  for (int i = group; i < parts; i += 4 * groups) {
    float2 st[4];
    float4v p[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int64_t j = min(i + k * groups, parts - 1);
      st[k] = a.stats[j * all + at];
      p[k] = *reinterpret_cast<const float4v*>(a.partial + (j * all + at) * dim + d);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float w = mine && i + k * groups < parts ? exp2_fast(st[k].x - base) : 0.0f;
      if (w == 0.0f && i + k * groups >= parts) continue;
      total += st[k].y * w;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = __builtin_fmaf(p[k][e], w, v[e]);
    }
  }
  // the groups' sums, in their order
  float sum = 0.0f;
  float4v out = {0, 0, 0, 0};
  for (int g = 0; g < groups; ++g) {
    const int from = g * lanes + d / 4;
    sum += __shfl(total, from);
#pragma unroll
    for (int e = 0; e < 4; ++e) out[e] += __shfl(v[e], from);
  }
  if (group != 0) return;
  const float inverse = sum == 0.0f ? 0.0f : 1.0f / sum;
  struct Four { T v[4]; } o;
#pragma unroll
  for (int e = 0; e < 4; ++e) o.v[e] = (T)(out[e] * inverse);
  store_any(element<T>(a.out, row, head) + d, o);
}

// LDS of a workgroup: the waves' statistics, and half of their sums.
inline size_t cache_attention_lds(int ng, int rt) { return (size_t)kWaves * 2 * 16 * rt * 4 + kWaves * 4 + (size_t)2 * (ng * 2) * rt * 64 * 16; }

typedef void (*cache_attention_t)(CacheAttentionArgs);
template <class T, int FMT, bool HALVES> cache_attention_t cache_attention_of(int ng, int rt) {
  if constexpr (HALVES) {
    if (rt == 2) switch (ng) {
      case 1: return cache_attention<T, FMT, 1, 2, HALVES>;
      case 2: return cache_attention<T, FMT, 2, 2, HALVES>;
      case 3: return cache_attention<T, FMT, 3, 2, HALVES>;
      case 4: return cache_attention<T, FMT, 4, 2, HALVES>;
    }
  }
  switch (ng) {
    case 1: return cache_attention<T, FMT, 1, 1, HALVES>;
    case 2: return cache_attention<T, FMT, 2, 1, HALVES>;
    case 3: return cache_attention<T, FMT, 3, 1, HALVES>;
    case 4: return cache_attention<T, FMT, 4, 1, HALVES>;
    case 6: return cache_attention<T, FMT, 6, 1, HALVES>;
    case 8: return cache_attention<T, FMT, 8, 1, HALVES>;
    default: return nullptr;
  }
}
template <class T, int FMT> cache_attention_t cache_attention_of(int ng, int rt, bool halves) {
  return halves ? cache_attention_of<T, FMT, true>(ng, rt) : cache_attention_of<T, FMT, false>(ng, rt);
}
cache_attention_t cache_attention_int4_bf16(int ng, int rt, bool halves);
cache_attention_t cache_attention_int4_f16(int ng, int rt, bool halves);
cache_attention_t cache_attention_int4_f32(int ng, int rt, bool halves);
cache_attention_t cache_attention_int8_bf16(int ng, int rt, bool halves);
cache_attention_t cache_attention_int8_f16(int ng, int rt, bool halves);
cache_attention_t cache_attention_int8_f32(int ng, int rt, bool halves);
cache_attention_t join_splits_kernel(int type);

}  // namespace att
}  // namespace squant
