// Attention of one or a few new tokens of each sequence over the quantised cache.
//
//   out[r] = sum_t p[r, t] V[t],  p = softmax_t(scale * Q[r] . K[t]),  K and V = codes * scales.
//
// A workgroup takes 16 or 32 rows (new tokens times the query heads of a key head) and a stretch of the sequence, its four
// waves 32 tokens each in turn; a wave reads codes and scales from memory straight into the lanes that multiply them, a block of
// tokens ahead.  Codes become binary16 numbers code * scale * 2^e with an exponent for the wave (running: a block with a
// larger scale lowers it, and the output's sums with it), which for 4 bits is exact: 3 bits of a code and 8 of a scale are 11.
// For 8 bits it would round to 11 bits (2^-12 of an element): binary16 and binary32 calls take the remainder as a second plane
// (11 drafted tokens' binary16 outputs 5.5e-4 off without it, 2.1e-4 with), bfloat16 ones do without.  Queries are
// binary16 with an exponent for each row: exact for 16-bit types, two planes for binary32.  Softmax weights
// are rounded to 11 bits times 2^14 (binary32: two planes).  Sums are binary32.
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
  int type;
  int32_t heads, group;  // query heads, and of a key head
  int32_t tiles;         // of rows
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

// A block of tokens on its way or at work.  `bad`: those whose page is none.
template <int FMT, int NG> struct Block {
  typedef Layout<FMT, NG> L;
  uint32_t key[2][L::kKeyWords];
  uint32_t value[8][L::kValueWords];
  uint16_t key_scale[2][L::kKeyScales];
  uint16_t value_scale[8][L::kValueScales];
  uint32_t bad;
};

// 8 codes as binary16 integers (times 16 where `sixteen` says so); element order as `slot_element` has it.
template <int FMT> __device__ __forceinline__ void key_codes(const uint32_t* w, half2v (&o)[4]) {
  if constexpr (FMT == SQUANT_OUT_INT4) {
    const uint32_t u = w[0] ^ 0x88888888u, v = u >> 8;
    const half2v low = pair((_Float16)1032.0f, (_Float16)1032.0f), high = pair((_Float16)1152.0f, (_Float16)1152.0f);
    o[0] = lin::as_half2((u & 0x000f000fu) | 0x64006400u) - low;
    o[1] = lin::as_half2((u & 0x00f000f0u) | 0x64006400u) - high;
    o[2] = lin::as_half2((v & 0x000f000fu) | 0x64006400u) - low;
    o[3] = lin::as_half2((v & 0x00f000f0u) | 0x64006400u) - high;
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

// Codes of tokens 2 m and 2 m + 1 for one element: byte `p` (low or high half of it) of a and b, which hold codes plus 8 or
// 128.  Codes of high halves are times 16.
template <int FMT> __device__ __forceinline__ half2v value_codes(uint32_t a, uint32_t b, int p, int high) {
  const uint32_t u = lin::pick(b, a, 0x0c040c00u + 0x00010001u * (uint32_t)p);
  if constexpr (FMT == SQUANT_OUT_INT4) {
    const half2v bias = high ? pair((_Float16)1152.0f, (_Float16)1152.0f) : pair((_Float16)1032.0f, (_Float16)1032.0f);
    return lin::as_half2((u & (high ? 0x00f000f0u : 0x000f000fu)) | 0x64006400u) - bias;
  }
  return lin::as_half2(u | 0x64006400u) - pair((_Float16)1152.0f, (_Float16)1152.0f);
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

// Waves a SIMD that the registers are kept for.  The wave waits for memory: three hide it better than two with more loads on their way.
constexpr int cache_occupancy(int ng, int rt) { return ng <= 2 ? 4 : ng <= 4 && rt == 1 ? 3 : 2; }

// PL: planes of queries and weights; LOW: the remainder of an 8-bit element as well.  HALVES: pages of a multiple of 16 tokens, of
// which each half of a block has consecutive rows: their addresses are a number for the wave plus one of the lane that stays.
template <int FMT, int NG, int PL, bool LOW, int RT, bool HALVES>
__global__ __launch_bounds__(kThreads, cache_occupancy(NG, RT)) void cache_attention(CacheAttentionArgs a) {
  typedef Layout<FMT, NG> L;
  typedef Block<FMT, NG> B;
  constexpr int D = NG * kGroup, F = D / 16, TR = 16 * RT;
  extern __shared__ float lds[];
  const Cache& c = a.cache;
  const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int n = lane & 15, g = lane >> 4;
  const int head = (int)blockIdx.x % c.heads;
  const int split = (int)blockIdx.y;

  // whose rows these are
  Tile tile;
  const int64_t tile_id = blockIdx.x / (uint32_t)c.heads;
  if (a.rows.one_each) {
    const int each = (a.group + TR - 1) / TR;
    tile.sequence = (int)(tile_id / each);
    tile.first = (int)(tile_id - (int64_t)tile.sequence * each) * TR;
    if (tile.sequence >= a.rows.count) return;
  } else {
    tile = find_tile(a.rows, tile_id, a.group, TR);
  }
  if (tile.sequence < 0) return;
  const int seq = tile.sequence, row0 = a.rows.start(seq), count = a.rows.length(seq);
  int64_t capacity = (int64_t)c.table_width * c.page_size;
  const int said = seq < a.rows.count ? max(c.lengths[seq], 0) : 0;
  const int length = (int)min((int64_t)said, capacity);
  const int begin = split * a.chunk, end = min(length, begin + a.chunk);
  if (a.splits > 1 && begin >= max(length, 1)) return;  // the join knows
  if (a.splits > 1 && seq == a.rows.count) return;

  // this lane's columns of the scores: rows of the queries
  int row[RT], qhead[RT], seen[RT];
  bool live[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int r = tile.first + 16 * rt + n;
    const int token = r / a.group;
    live[rt] = r < count * a.group;
    row[rt] = row0 + (live[rt] ? token : 0);
    qhead[rt] = head * a.group + (r - token * a.group);
    seen[rt] = live[rt] ? min(max(said - count + token + 1, 0), length) : 0;
    if (!live[rt]) qhead[rt] = head * a.group;
  }
  const float poison = said > length ? __builtin_nanf("") : 1.0f;

  half8 q[RT][PL][NG];
  float factor[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    float x[NG][8];
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < NG; ++i) {
      const int d = (g * NG + i) * 8;
      if (a.type == SQUANT_W_F32) load8(element<float>(a.q, row[rt], qhead[rt]) + d, x[i]);
      else if (a.type == SQUANT_W_F16) load8(element<_Float16>(a.q, row[rt], qhead[rt]) + d, x[i]);
      else load8(element<__bf16>(a.q, row[rt], qhead[rt]) + d, x[i]);
#pragma unroll
      for (int s = 0; s < 8; ++s) top = max(top, finite_bits(x[i][s]));
    }
    top = max(top, (uint32_t)__shfl_xor((int)top, 16));
    top = max(top, (uint32_t)__shfl_xor((int)top, 32));
    const int e = lin::row_exponent(top);
    const float up = power_of_two(e);
    factor[rt] = a.scale * power_of_two(-e) * poison;
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

  // where tokens lie: pages of the block's halves, or of token t0 + lane % 32
  const uint32_t head_row = (uint32_t)head * (uint32_t)c.page_size;
  const int last = max(length - 1, 0);
  auto page_ids = [&](int t0, int32_t (&id)[2]) {
    if constexpr (HALVES) {
#pragma unroll
      for (int h = 0; h < 2; ++h) id[h] = __builtin_amdgcn_readfirstlane(c.table_at(seq, c.page_of(min(t0 + 16 * h, last))));
    } else {
      id[0] = id[1] = c.table_at(seq, c.page_of(min(t0 + (lane & 31), last)));
    }
  };
  auto load_value = [&](uint32_t (&o)[L::kValueWords], const uint8_t* p) {
    __builtin_memset(o, 0, sizeof(o));
    if constexpr (L::kValueBytes % 4 == 0) {
      struct Words { uint32_t w[L::kValueWords]; };
      const Words w = *reinterpret_cast<const Words*>(p);
#pragma unroll
      for (int i = 0; i < L::kValueWords; ++i) o[i] = w.w[i];
    } else if constexpr (L::kValueBytes == 6) {
      struct Halves { uint16_t w[3]; };
      const Halves w = *reinterpret_cast<const Halves*>(p);
      o[0] = w.w[0] | (uint32_t)w.w[1] << 16;
      o[1] = w.w[2];
    } else if constexpr (L::kValueBytes == 2) {
      o[0] = *reinterpret_cast<const uint16_t*>(p);
    } else if constexpr (L::kValueBytes == 3) {
      o[0] = p[0] | (uint32_t)p[1] << 8 | (uint32_t)p[2] << 16;
    } else {
      static_assert(L::kValueBytes == 1, "");
      o[0] = p[0];
    }
  };
  // codes and scales of key token 16 tt + n and of value token 4 g + j (j < 4), 16 + 4 g + j - 4, by their rows
  auto load_rows = [&](B& b, auto row_of) {
#pragma unroll
    for (int tt = 0; tt < 2; ++tt) {
      struct Words { uint32_t w[L::kKeyWords]; };
      const auto at = row_of(tt, n, g * (L::kRow / 4));
      const Words w = load_any<Words>(c.codes[0] + at.bytes);
#pragma unroll
      for (int i = 0; i < L::kKeyWords; ++i) b.key[tt][i] = w.w[i];
#pragma unroll
      for (int k = 0; k < L::kKeyScales; ++k) b.key_scale[tt][k] = c.scales[0][at.scales + min(((g * NG) >> 2) + k, NG - 1)];
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const auto at = row_of(j >> 2, 4 * g + (j & 3), n * L::kValueBytes);
      load_value(b.value[j], c.codes[1] + at.bytes);
#pragma unroll
      for (int k = 0; k < L::kValueScales; ++k) b.value_scale[j][k] = c.scales[1][at.scales + min(((2 * NG * n) >> 5) + k, NG - 1)];
    }
  };
  struct Place { int64_t bytes, scales; };
  auto load_block = [&](B& b, int t0, const int32_t (&id)[2]) {
    if constexpr (HALVES) {
      int64_t first[2];
      b.bad = 0;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int t = min(t0 + 16 * h, last);
        const int32_t r = c.row_of(t / 16 * 16, c.page_of(t), id[h]);
        if (r < 0) b.bad |= 0xffffu << (16 * h);
        first[h] = r < 0 ? 0 : (int64_t)(r + head_row);  // rows 0 to 15 are there
      }
      load_rows(b, [&](int h, int token, int byte) {
        return Place{first[h] * L::kRow + (uint32_t)(token * L::kRow + byte), first[h] * NG + (uint32_t)(token * NG)};
      });
    } else {
      const int t = min(t0 + (lane & 31), last);
      const int32_t r = c.row_of(t, c.page_of(t), id[0]);
      b.bad = (uint32_t)lanes_where(r < 0);
      const int32_t mine = r < 0 ? 0 : (int32_t)(r + head_row);
      load_rows(b, [&](int h, int token, int byte) {
        const int64_t row = __shfl(mine, 16 * h + token);
        return Place{row * L::kRow + byte, row * NG};
      });
    }
  };

  float4v o[F][RT];
#pragma unroll
  for (int f = 0; f < F; ++f)
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) o[f][rt] = float4v{0, 0, 0, 0};
  float largest[RT], sum[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) largest[rt] = -kInfinity, sum[rt] = 0.0f;
  int key_e = 126, value_e = 126;
  int least_seen = 0x7fffffff;
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) least_seen = min(least_seen, live[rt] ? seen[rt] : 0x7fffffff);
#pragma unroll
  for (int w = 1; w < 16; w <<= 1) least_seen = min(least_seen, __shfl_xor(least_seen, w));
  least_seen = __builtin_amdgcn_readfirstlane(least_seen);

  constexpr int kStep = kWaves * kTokens;
  auto work = [&](B& cur, int t0, auto hidden) {
    constexpr bool kHidden = decltype(hidden)::value;
    // a token whose page is none makes its rows NaN; tokens past the end count nothing, whatever is there
    float key_scale[2][L::kKeyScales], value_scale[8][L::kValueScales];
    float top = 0.0f;
#pragma unroll
    for (int tt = 0; tt < 2; ++tt)
#pragma unroll
      for (int k = 0; k < L::kKeyScales; ++k) {
        float s = from_bfloat16(cur.key_scale[tt][k]);
        if constexpr (kHidden) s = t0 + 16 * tt + n >= end ? 0.0f : cur.bad >> (16 * tt + n) & 1 ? __builtin_nanf("") : s;
        key_scale[tt][k] = s;
        top = fmaxf(top, fabsf(s));
      }
    if (lanes_where(top * power_of_two(key_e) >= 512.0f)) {
      uint32_t m = 0;
#pragma unroll
      for (int tt = 0; tt < 2; ++tt)
#pragma unroll
        for (int k = 0; k < L::kKeyScales; ++k) m = max(m, finite_bits(key_scale[tt][k]));
      key_e = min(key_e, __builtin_amdgcn_readfirstlane(scale_exponent(over_lanes_max(m))));
    }

    float4v s[2][RT];
#pragma unroll
    for (int tt = 0; tt < 2; ++tt) {
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) s[tt][rt] = float4v{0, 0, 0, 0};
      _Float16 scale[L::kKeyScales];
#pragma unroll
      for (int k = 0; k < L::kKeyScales; ++k) scale[k] = (_Float16)(key_scale[tt][k] * power_of_two(key_e));
#pragma unroll
      for (int i = 0; i < NG; ++i) {
        _Float16 w = scale[0];
        if constexpr (NG % 4 == 0) w = scale[i >> 2];
        else if constexpr (L::kKeyScales == 2) w = ((g * NG + i) >> 2) > ((g * NG) >> 2) ? scale[1] : scale[0];
        half2v codes[4];
        key_codes<FMT>(cur.key[tt] + i * (L::kBits / 4), codes);
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

    // softmax weights of the block, times 2^14; what they add up to stays with the lane until the end
    half8 p[RT][PL];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      const float f = factor[rt] * power_of_two(-key_e);
      float x[8];
      float m = -kInfinity;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        x[j] = s[j >> 2][rt][j & 3] * f;
        if constexpr (kHidden) x[j] = t0 + 16 * (j >> 2) + 4 * g + (j & 3) < min(seen[rt], end) ? x[j] : -kInfinity;
        m = fmaxf(m, x[j]);
      }
      m = over_groups_max(m);
      if (lanes_where(m > largest[rt])) {
        const float more = fmaxf(m, largest[rt]);
        const float shrink = more == -kInfinity ? 1.0f : exp2_fast(largest[rt] - more);
        sum[rt] *= shrink;
#pragma unroll
        for (int f2 = 0; f2 < F; ++f2)
#pragma unroll
          for (int i = 0; i < 4; ++i) o[f2][rt][i] *= shrink;
        largest[rt] = more;
      }
      const float base = largest[rt] == -kInfinity ? 0.0f : largest[rt] - kWeightUnit;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float w = exp2_fast(x[j] - base);
        sum[rt] += w;
        const _Float16 hi = (_Float16)w;
        p[rt][0][j] = hi;
        if constexpr (PL == 2) p[rt][1][j] = (_Float16)(w - (float)hi);
      }
    }

    top = 0.0f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int at = 4 * g + (j & 3) + 16 * (j >> 2);
#pragma unroll
      for (int k = 0; k < L::kValueScales; ++k) {
        float v = from_bfloat16(cur.value_scale[j][k]);
        if constexpr (kHidden) v = t0 + at >= end ? 0.0f : cur.bad >> at & 1 ? __builtin_nanf("") : v;
        value_scale[j][k] = v;
        top = fmaxf(top, fabsf(v));
      }
    }
    if (lanes_where(top * power_of_two(value_e) >= 512.0f)) {
      uint32_t m = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int k = 0; k < L::kValueScales; ++k) m = max(m, finite_bits(value_scale[j][k]));
      const int e = min(value_e, __builtin_amdgcn_readfirstlane(scale_exponent(over_lanes_max(m))));
#pragma unroll
      for (int f = 0; f < F; ++f)
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
          for (int i = 0; i < 4; ++i) o[f][rt][i] = ldexpf(o[f][rt][i], e - value_e);
      value_e = e;
    }
    half2v scale2[4][L::kValueScales];
#pragma unroll
    for (int m = 0; m < 4; ++m)
#pragma unroll
      for (int k = 0; k < L::kValueScales; ++k)
        scale2[m][k] = pair((_Float16)(value_scale[2 * m][k] * power_of_two(value_e)),
                            (_Float16)(value_scale[2 * m + 1][k] * power_of_two(value_e)));
    // a scale of NaN or infinity at a token that some row does not see: that row's weight of 0 would not keep it out
    bool odd = false;
    if constexpr (kHidden) {
      bool any = false;
#pragma unroll
      for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int k = 0; k < L::kValueScales; ++k) any |= !(fabsf(value_scale[j][k]) < kInfinity);
      odd = lanes_where(any) != 0;
    }
    // codes plus 8 or 128
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
      for (int i = 0; i < L::kValueWords; ++i) cur.value[j][i] ^= FMT == SQUANT_OUT_INT4 ? 0x88888888u : 0x80808080u;
    auto element_operand = [&](int f, half8& hi, half8& lo) {
      const int byte = FMT == SQUANT_OUT_INT4 ? f / 2 : f;
#pragma unroll
      for (int m = 0; m < 4; ++m) {
        half2v w = scale2[m][0];
        if constexpr (L::kValueScales == 2) w = ((2 * NG * n + f) >> 5) > ((2 * NG * n) >> 5) ? scale2[m][1] : scale2[m][0];
        const half2v codes = value_codes<FMT>(cur.value[2 * m][byte / 4], cur.value[2 * m + 1][byte / 4], byte % 4, f & 1);
        const half2v v = codes * w;
        hi[2 * m] = v[0], hi[2 * m + 1] = v[1];
        if constexpr (LOW) {
          const half2v rest = __builtin_elementwise_fma(codes, w, -v);
          lo[2 * m] = rest[0], lo[2 * m + 1] = rest[1];
        }
      }
    };
    auto add = [&](const half8& h, const half8& l, float4v acc, int rt) {
      acc = Half::mma(h, p[rt][0], acc);
      if constexpr (PL == 2) acc = Half::mma(h, p[rt][1], acc);
      if constexpr (LOW) acc = Half::mma(l, p[rt][0], acc);
      return acc;
    };
    if (!odd) {
#pragma unroll
      for (int f = 0; f < F; ++f) {
        half8 hi, lo = {};
        element_operand(f, hi, lo);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) o[f][rt] = add(hi, lo, o[f][rt], rt);
      }
    } else {
      // token by token, rows that do not see it left out
#pragma unroll 1
      for (int t = 0; t < kTokens; ++t)
#pragma unroll
        for (int f = 0; f < F; ++f) {
          half8 hi, lo = {};
          element_operand(f, hi, lo);
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (4 * g + (j & 3) + 16 * (j >> 2) != t) hi[j] = lo[j] = (_Float16)0.0f;
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) {
            const float4v alone = add(hi, lo, float4v{0, 0, 0, 0}, rt);
            if (t0 + t < min(seen[rt], end)) o[f][rt] += alone;
          }
        }
    }
  };
  // Blocks of which all rows see all tokens, the next one on its way; then the others, one by one.
  B cur;
  int t0 = begin + wave * kTokens;
  const int seen_by_all = min(end, least_seen);
  if (t0 + kTokens <= seen_by_all) {
    int32_t ids[2];
    page_ids(t0, ids);
    load_block(cur, t0, ids);
    page_ids(t0 + kStep, ids);
#pragma unroll 1
    while (!cur.bad) {
      B next;
      const bool more = t0 + kStep + kTokens <= seen_by_all;
      if (more) {
        load_block(next, t0 + kStep, ids);
        page_ids(t0 + 2 * kStep, ids);
      }
      work(cur, t0, Constant<false>{});
      t0 += kStep;
      if (!more) break;
      cur = next;
    }
  }
#pragma unroll 1
  for (; t0 < end; t0 += kStep) {
    int32_t ids[2];
    page_ids(t0, ids);
    load_block(cur, t0, ids);
    work(cur, t0, Constant<true>{});
  }

  // the waves' sums become one
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) sum[rt] = over_groups_sum(sum[rt]);
  float* stats = lds;                      // [wave][2][TR]
  float* pile = lds + kWaves * 2 * TR;     // [2][F][RT][64] of four
  if (g == 0) {
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      stats[(wave * 2 + 0) * TR + 16 * rt + n] = largest[rt];
      stats[(wave * 2 + 1) * TR + 16 * rt + n] = sum[rt];
    }
  }
  __syncthreads();
  float total[RT], most[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    float m = -kInfinity, l = 0.0f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) m = fmaxf(m, stats[w * 2 * TR + 16 * rt + n]);
    const float base = m == -kInfinity ? 0.0f : m;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) l += stats[(w * 2 + 1) * TR + 16 * rt + n] * exp2_fast(stats[w * 2 * TR + 16 * rt + n] - base);
    total[rt] = l, most[rt] = m;
    const float mine = exp2_fast(largest[rt] - base);
#pragma unroll
    for (int f = 0; f < F; ++f)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        // odd elements of 4-bit codes are held times 16
        o[f][rt][i] = ldexpf(o[f][rt][i] * mine, -value_e - (FMT == SQUANT_OUT_INT4 && (f & 1) ? 4 : 0));
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
        } else if (a.type == SQUANT_W_F32) {
          struct Two { float v[2]; };
          store_any(element<float>(a.out, row[rt], qhead[rt]) + d + f, Two{{v0, v1}});
        } else if (a.type == SQUANT_W_F16) {
          struct Two { _Float16 v[2]; };
          store_any(element<_Float16>(a.out, row[rt], qhead[rt]) + d + f, Two{{(_Float16)v0, (_Float16)v1}});
        } else {
          struct Two { __bf16 v[2]; };
          store_any(element<__bf16>(a.out, row[rt], qhead[rt]) + d + f, Two{{(__bf16)v0, (__bf16)v1}});
        }
      }
    }
  }
}

// The splits of each row and head become its output: a wave for each.
template <int FORMATS> __global__ __launch_bounds__(kThreads) void join_splits(CacheAttentionArgs a) {
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
  float m = -kInfinity;
  for (int i = lane; i < parts; i += 64) m = fmaxf(m, a.stats[i * all + at].x);
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) m = fmaxf(m, __shfl_xor(m, o));
  const float base = m == -kInfinity ? 0.0f : m;
  float total = 0.0f, v[4] = {0, 0, 0, 0};
  for (int i = 0; i < parts; ++i) {
    const float2 st = a.stats[i * all + at];
    const float w = exp2_fast(st.x - base);
    total += st.y * w;
    const float* p = a.partial + (i * all + at) * dim;
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (k * 64 + lane < dim) v[k] = __builtin_fmaf(p[k * 64 + lane], w, v[k]);
  }
  const float inverse = total == 0.0f ? 0.0f : 1.0f / total;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int d = k * 64 + lane;
    if (d >= dim) continue;
    const float x = v[k] * inverse;
    if (a.type == SQUANT_W_F32) element<float>(a.out, row, head)[d] = x;
    else if (a.type == SQUANT_W_F16) element<_Float16>(a.out, row, head)[d] = (_Float16)x;
    else element<__bf16>(a.out, row, head)[d] = (__bf16)x;
  }
}

// LDS of a workgroup: the waves' statistics, and half of their sums.
inline size_t cache_attention_lds(int ng, int rt) { return (size_t)kWaves * 2 * 16 * rt * 4 + (size_t)2 * (ng * 2) * rt * 64 * 16; }

typedef void (*cache_attention_t)(CacheAttentionArgs);
template <int FMT, int PL, bool LOW, bool HALVES> cache_attention_t cache_attention_of(int ng, int rt) {
  if constexpr (HALVES) {
    if (rt == 2) switch (ng) {
      case 1: return cache_attention<FMT, 1, PL, LOW, 2, HALVES>;
      case 2: return cache_attention<FMT, 2, PL, LOW, 2, HALVES>;
      case 3: return cache_attention<FMT, 3, PL, LOW, 2, HALVES>;
      case 4: return cache_attention<FMT, 4, PL, LOW, 2, HALVES>;
    }
  }
  switch (ng) {
    case 1: return cache_attention<FMT, 1, PL, LOW, 1, HALVES>;
    case 2: return cache_attention<FMT, 2, PL, LOW, 1, HALVES>;
    case 3: return cache_attention<FMT, 3, PL, LOW, 1, HALVES>;
    case 4: return cache_attention<FMT, 4, PL, LOW, 1, HALVES>;
    case 6: return cache_attention<FMT, 6, PL, LOW, 1, HALVES>;
    case 8: return cache_attention<FMT, 8, PL, LOW, 1, HALVES>;
    default: return nullptr;
  }
}
template <int FMT, int PL, bool LOW> cache_attention_t cache_attention_of(int ng, int rt, bool halves) {
  return halves ? cache_attention_of<FMT, PL, LOW, true>(ng, rt) : cache_attention_of<FMT, PL, LOW, false>(ng, rt);
}
// By format, and by type: bfloat16 (8 bits only), 16 bits, binary32.
cache_attention_t cache_attention_int4(int ng, int rt, bool halves);
cache_attention_t cache_attention_int4_f32(int ng, int rt, bool halves);
cache_attention_t cache_attention_int8_bf16(int ng, int rt, bool halves);
cache_attention_t cache_attention_int8_f16(int ng, int rt, bool halves);
cache_attention_t cache_attention_int8_f32(int ng, int rt, bool halves);
cache_attention_t join_splits_kernel();

}  // namespace att
}  // namespace squant
