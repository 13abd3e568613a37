// Shared definitions of the operators that multiply by codes: arguments, the conversion of codes to
// matrix-unit operands, activations, and what happens to a finished piece of a product.
//
// Every product is rows x codes: out[m, c] = sum_i a[m, i] w[i, c], with w[i, c] = code(c, i) for the layer
// itself (the contraction runs along a code row) and code(i, c) for its gradient (it runs across them).
// Codes are integers of at most 8 bits, exact in binary16 and in bfloat16, so the matrix units multiply
// exactly and add in binary32; the scale of an output channel is applied once, to the finished sum (layer)
// or to the row operand (gradient).  Row operands:
//   bfloat16, binary16  as they are;
//   binary32            two binary16 planes, hi + lo = x * 2^e with one e a row (its largest finite element
//                       lands in [2^14, 2^15)): 22 bits of an element, or 2^-40 of the row's largest where
//                       that is more.  bfloat16 would take three planes for the same.  A pass of its own lays them
//                       out; few rows are split in registers, with an exponent of what a wave has seen of a row;
//   gradients           one plane like this for 16-bit outputs (at most 2^-11 of an element: an eighth of what a
//                       bfloat16 gradient would be off by, for a binary16 one as much as its output's rounding,
//                       1.4 times that in all; two planes would take twice the products), two for binary32.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "squant.h"

namespace squant {
namespace lin {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef __bf16 brain8 __attribute__((ext_vector_type(8)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef uint32_t uint4v __attribute__((ext_vector_type(4)));
typedef uint32_t uint2v __attribute__((ext_vector_type(2)));

constexpr int kLanes = 64;
constexpr int kBlock = 64;   // contraction elements a step of the main loops takes
constexpr int kTile = 64;    // columns of a wave, and the columns that share a scale of the kept pre-activation
constexpr int kWide = 256;   // columns of a workgroup of `product`

enum Kind { kLinear = 0, kPartial = 1, kStats = 2, kProb = 3, kGrad = 4, kGradLoss = 5 };

// What a finished piece of a product needs; one structure for every kind, so that a kernel's main loop
// is compiled once.
struct Finish {
  int kind;
  int act;
  int keep;
  int out_type;             // squant_wtype_t of `out` where the kernel does not fix it
  float unit;               // the product's codes are held as multiples of this: 1, 2^-4, 2^-9
  int64_t rows;
  int32_t cols;             // of the output
  const float* row_factor;  // 2^-e of each row, or null
  const float* scales;
  const void* bias;
  const void* residual;
  int64_t ldr;
  void* out;
  int64_t ldo;
  void* kept;               // int8 [rows][cols] or out's type
  float* kept_scales;       // [rows][ceil(cols / 64)]
  float4v* partial;         // kPartial: [slice][row fragment][column fragment][lane]
  // cross entropy
  const int64_t* labels;
  int64_t ignore;
  float2* stats;            // [rows][chunks]: largest logit and sum of exponentials, base 2
  float* label_logit;       // [rows], base 2
  const float* lse;
  const float* dloss;
  const float* prob_unit;   // [1]: 2^E that brings p * scale into binary16's range
  _Float16* prob;           // [rows][planes][ld_prob]
  int64_t ld_prob;          // elements between rows
  int64_t prob_plane;       // elements between planes
  float* label_prob;        // [rows]
  float* other_sums;        // [tiles of columns][rows]: sums of the probabilities beside the label's
  int32_t other_tiles;
  int32_t first_col;        // vocabulary entry of column 0 of the piece
  int32_t vocabulary;
  const uint8_t* codes;     // kGradLoss: the label's row
  int64_t code_row;
  int32_t format;
};

struct ProductArgs {
  const void* a;       // row operand [rows][planes][blocks * 64], zero beyond the contraction's length
  int64_t lda;         // elements between rows
  int64_t plane;       // elements between planes
  const uint8_t* w;    // codes; for a piece of the vocabulary, its first row.  `product`: rows of whole 16-byte words, for a
                       // layer of whole steps
  int64_t w_row;       // bytes of a code row
  int32_t w_rows;      // code rows
  int32_t w_cols;      // codes of a row
  const uint8_t* w_end;
  int32_t blocks;      // ceil(contraction / 64)
  int32_t slices;      // the contraction is cut into this many
  int32_t tiles_m, tiles_n;
  int accumulate;      // kPartial, kProb: the sums are added to those in `partial`, `other_sums`
  Finish f;
};

typedef void (*product_t)(ProductArgs);

// ---------------------------------------------------------------------------
// loads at any alignment
// ---------------------------------------------------------------------------

template <class V>
__device__ __forceinline__ V load_any(const void* p) {
  V v;
  __builtin_memcpy(&v, p, sizeof(V));
  return v;
}
template <class V>
__device__ __forceinline__ void store_any(void* p, V v) {
  __builtin_memcpy(p, &v, sizeof(V));
}

// ---------------------------------------------------------------------------
// codes to operands
// ---------------------------------------------------------------------------

__device__ __forceinline__ uint32_t pick(uint32_t hi, uint32_t lo, uint32_t sel) {
  return __builtin_amdgcn_perm(hi, lo, sel);
}

__device__ __forceinline__ half2v as_half2(uint32_t u) { return __builtin_bit_cast(half2v, u); }

// u in the low byte of each half is the binary16 subnormal u * 2^-24: one fused multiply-add makes it
// (u - zero) * 2^-9, exactly.
__device__ __forceinline__ half2v centred(uint32_t u, float zero) {
  const half2v up = {(_Float16)32768.0f, (_Float16)32768.0f};
  const _Float16 z = (_Float16)(-zero / 512.0f);
  return __builtin_elementwise_fma(as_half2(u), up, half2v{z, z});
}

struct Half {
  typedef half8 frag;
  static __device__ __forceinline__ float4v mma(frag w, frag x, float4v c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(w, x, c, 0, 0, 0);
  }
};
struct Brain {
  typedef brain8 frag;
  static __device__ __forceinline__ float4v mma(frag w, frag x, float4v c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, x, c, 0, 0, 0);
  }
};

template <int FMT> struct Codes;
template <> struct Codes<SQUANT_OUT_INT8> {
  typedef uint4v row16;                       // 16 codes of a row
  static constexpr int kRow16 = 16;           // its bytes
  typedef uint32_t col4;                      // 4 codes of a row, one for each of 4 columns
  static __device__ __forceinline__ int64_t offset(int64_t i) { return i; }
  static __device__ __forceinline__ int value(const uint8_t* row, int64_t i) { return (int8_t)row[i]; }
};
template <> struct Codes<SQUANT_OUT_INT4> {
  typedef uint2v row16;
  static constexpr int kRow16 = 8;
  typedef uint16_t col4;
  static __device__ __forceinline__ int64_t offset(int64_t i) { return i >> 1; }
  static __device__ __forceinline__ int value(const uint8_t* row, int64_t i) {
    return (int)((uint32_t)row[i >> 1] << ((i & 1) ? 24 : 28)) >> 28;
  }
};

// The multiple that a converted code is held as; the finished sum is multiplied by its inverse.
template <class F, int FMT> struct CodeUnit;
template <> struct CodeUnit<Half, SQUANT_OUT_INT8> { static constexpr float inverse = 1.0f; };
template <> struct CodeUnit<Brain, SQUANT_OUT_INT8> { static constexpr float inverse = 1.0f; };
template <> struct CodeUnit<Half, SQUANT_OUT_INT4> { static constexpr float inverse = 512.0f; };
template <> struct CodeUnit<Brain, SQUANT_OUT_INT4> { static constexpr float inverse = 16.0f; };
constexpr float kColumnUnitInverse = 512.0f;  // of convert_columns

// Codes 8h .. 8h+7 of 16 consecutive ones.  About 1 instruction a code for binary16, 1.5 otherwise.
template <class F, int FMT>
__device__ __forceinline__ typename F::frag convert(const typename Codes<FMT>::row16& r, int h) {
  uint32_t o[4];
  if constexpr (FMT == SQUANT_OUT_INT8 && __is_same(F, Half)) {
#pragma unroll
    for (int d = 0; d < 2; ++d) {
      const uint32_t u = r[2 * h + d] ^ 0x80808080u;  // code + 128, then 1024 + that by its bits
      const half2v bias = {(_Float16)1152.0f, (_Float16)1152.0f};
      o[2 * d] = __builtin_bit_cast(uint32_t, as_half2(pick(0x64646464u, u, 0x04010400u)) - bias);
      o[2 * d + 1] = __builtin_bit_cast(uint32_t, as_half2(pick(0x64646464u, u, 0x04030402u)) - bias);
    }
  } else if constexpr (FMT == SQUANT_OUT_INT8) {
#pragma unroll
    for (int d = 0; d < 4; ++d) {  // an integer of 8 bits is exact in the upper half of its binary32
      const uint32_t u = r[2 * h + (d >> 1)];
      const int s = (d & 1) * 16;
      const float a = (float)(int8_t)(u >> s), b = (float)(int8_t)(u >> (s + 8));
      o[d] = pick(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
    }
  } else if constexpr (__is_same(F, Half)) {
    const uint32_t u = r[h] ^ 0x88888888u;  // code + 8
    const uint32_t even = u & 0x0f0f0f0fu, odd = (u >> 4) & 0x0f0f0f0fu;
#pragma unroll
    for (int d = 0; d < 4; ++d)
      o[d] = __builtin_bit_cast(uint32_t, centred(pick(odd, even, 0x0c040c00u + 0x00010001u * (uint32_t)d), 8.0f));
  } else {
#pragma unroll
    for (int d = 0; d < 4; ++d) {  // the instruction makes code / 16 of four bits
      const float a = __builtin_amdgcn_cvt_off_f32_i4((int)(r[h] >> (8 * d)));
      const float b = __builtin_amdgcn_cvt_off_f32_i4((int)(r[h] >> (8 * d + 4)));
      o[d] = pick(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
    }
  }
  const uint4v v = {o[0], o[1], o[2], o[3]};
  return __builtin_bit_cast(typename F::frag, v);
}

// Column j of 8 code rows of 4 columns each, as multiples of 2^-9.
template <int FMT>
__device__ __forceinline__ half8 convert_columns(const typename Codes<FMT>::col4* r, int j) {
  uint32_t o[4];
#pragma unroll
  for (int d = 0; d < 4; ++d) {
    if constexpr (FMT == SQUANT_OUT_INT8) {
      const uint32_t a = r[2 * d] ^ 0x80808080u, b = r[2 * d + 1] ^ 0x80808080u;
      o[d] = __builtin_bit_cast(uint32_t, centred(pick(b, a, 0x0c040c00u + 0x00010001u * (uint32_t)j), 128.0f));
    } else {
      const uint32_t u = ((uint32_t)r[2 * d] | (uint32_t)r[2 * d + 1] << 16) ^ 0x88888888u;
      o[d] = __builtin_bit_cast(uint32_t, centred((u >> (4 * j)) & 0x000f000fu, 8.0f));
    }
  }
  const uint4v v = {o[0], o[1], o[2], o[3]};
  return __builtin_bit_cast(half8, v);
}

// sizeof(V) bytes from each p[i] on, where `end` ends the buffer.  Past a row's end they are the next row's, which
// the callers multiply by zero or do not store; past the buffer's end nothing is read, and the value's upper bytes
// are zeros.  `bytes` is the whole buffer's size: one below sizeof(V) is read byte by byte.
template <class V> struct Shifted { typedef V type; };
template <> struct Shifted<uint4v> { typedef __uint128_t type; };
template <> struct Shifted<uint2v> { typedef uint64_t type; };
template <class V, int N>
__device__ __forceinline__ void load_before(V (&o)[N], const uint8_t* const (&p)[N], const uint8_t* end, int64_t bytes) {
  typedef typename Shifted<V>::type U;
  constexpr int n = (int)sizeof(V);
  U u[N];
  if (bytes < n) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      u[i] = 0;
#pragma unroll 1
      for (int b = 0; b < n; ++b)
        if (p[i] + b < end) u[i] |= (U)p[i][b] << (8 * b);
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) u[i] = load_any<U>(p[i] + n > end ? end - n : p[i]);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int64_t past = p[i] + n - end;
      u[i] = past >= n ? (U)0 : past > 0 ? (U)(u[i] >> (8 * (int)past)) : u[i];
    }
  }
#pragma unroll
  for (int i = 0; i < N; ++i) o[i] = __builtin_bit_cast(V, u[i]);
}

// ---------------------------------------------------------------------------
// types, activations
// ---------------------------------------------------------------------------

template <class T> __device__ __forceinline__ float widen(T v) { return (float)v; }
template <class T> __device__ __forceinline__ T narrow(float v) { return (T)v; }

constexpr float kLog2E = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// erfc(x) exp(x^2) for x >= 0: a polynomial in t = 1 / (1 + x / 2), least squares of the relative error (weights
// moved towards equal ripples).  FINE: x in [0, 10], where erfc leaves binary32's range, to 3e-8 in exact arithmetic
// and 2.9e-7 in binary32.  Otherwise, for 16-bit results: x in [0, 5], to 6.4e-6, a thirtieth of half a binary16
// step, with 4 multiply-adds less.
template <bool FINE>
__device__ __forceinline__ float erfcx_poly(float x) {
  const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.5f, x, 1.0f));
  if constexpr (FINE) {
    float r = -5.505337939e-02f;
    r = __builtin_fmaf(r, t, 2.639137506e-01f);
    r = __builtin_fmaf(r, t, -4.415010214e-01f);
    r = __builtin_fmaf(r, t, 2.212197632e-01f);
    r = __builtin_fmaf(r, t, 1.705580018e-02f);
    r = __builtin_fmaf(r, t, 1.812604517e-01f);
    r = __builtin_fmaf(r, t, 2.497902513e-01f);
    r = __builtin_fmaf(r, t, 2.810990512e-01f);
    r = __builtin_fmaf(r, t, 2.822213173e-01f);
    return __builtin_fmaf(r, t, -6.008548098e-06f);
  }
  float r = -2.049253434e-01f;
  r = __builtin_fmaf(r, t, 5.639148951e-01f);
  r = __builtin_fmaf(r, t, 1.532078534e-02f);
  r = __builtin_fmaf(r, t, 3.542144001e-01f);
  r = __builtin_fmaf(r, t, 2.707676291e-01f);
  return __builtin_fmaf(r, t, 7.012577262e-04f);
}

// exp(-z^2 / 2).  FINE: the square's rounding error would be magnified by the exponent, so it is carried along.
template <bool FINE>
__device__ __forceinline__ float exp_half_square(float z) {
  const float c = -0.5f * kLog2E;
  const float a = z * z, e = a * c;
  if constexpr (!FINE) return exp2_fast(e);
  const float lost = __builtin_fmaf(z, z, -a);
  const float tail = __builtin_fmaf(a, c, -e) + (lost * c + a * -9.6299e-9f);
  return e < -160.0f ? 0.0f : exp2_fast(e) * (1.0f + kLn2 * tail);
}

// The normal distribution's Phi(z), and exp(-z^2 / 2) beside it.
template <bool FINE>
__device__ __forceinline__ float normal_cdf(float z, float& density) {
  density = exp_half_square<FINE>(z);
  const float tail = 0.5f * erfcx_poly<FINE>(fabsf(z) * 0.70710678118654752f) * density;
  return z < 0.0f ? tail : 1.0f - tail;
}

__device__ __forceinline__ float sigmoid(float z) {
  return __builtin_amdgcn_rcpf(1.0f + exp2_fast(-kLog2E * z));
}

// N values at a time, so that the choice of activation is made once for them, and four at a time in registers.
// T: the type of the result.
__device__ __forceinline__ void after_four(int i) {
  if ((i & 3) == 3) __builtin_amdgcn_sched_barrier(0);
}
template <class T, int N>
__device__ __forceinline__ void activate(float (&z)[N], int act) {
  constexpr bool fine = sizeof(T) == 4;
  if (act == SQUANT_ACT_RELU) {
#pragma unroll
    for (int i = 0; i < N; ++i) z[i] = z[i] < 0.0f ? 0.0f : z[i];  // a NaN stays
  } else if (act == SQUANT_ACT_GELU) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float density;
      z[i] *= normal_cdf<fine>(z[i], density);
      after_four(i);
    }
  } else if (act == SQUANT_ACT_SILU) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      z[i] *= sigmoid(z[i]);
      after_four(i);
    }
  }
}

// v *= act'(z)
template <class T, int N>
__device__ __forceinline__ void apply_slope(float (&v)[N], const float (&z)[N], int act) {
  constexpr bool fine = sizeof(T) == 4;
  if (act == SQUANT_ACT_RELU) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] *= z[i] > 0.0f ? 1.0f : z[i] <= 0.0f ? 0.0f : z[i];
  } else if (act == SQUANT_ACT_GELU) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float density;
      const float cdf = normal_cdf<fine>(z[i], density);
      const float d = 0.3989422804014327f * density;
      v[i] *= d > 0.0f ? __builtin_fmaf(z[i], d, cdf) : cdf + 0.0f * d;  // z may be infinite where the density is 0
    }
  } else if (act == SQUANT_ACT_SILU) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      // 1 - p = e p without its cancellation; where p or e has left the range of numbers the slope is p
      const float e = exp2_fast(-kLog2E * z[i]), p = __builtin_amdgcn_rcpf(1.0f + e);
      v[i] *= p > 0.0f && e > 0.0f ? p * __builtin_fmaf(z[i], e * p, 1.0f) : p;
    }
  }
}

// Largest magnitude by the bits: a NaN is larger than any number and stays.
__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// A value over the 4 lanes (16 apart) that hold the 64 columns of a row.
__device__ __forceinline__ uint32_t group_max(uint32_t v) {
  v = max(v, (uint32_t)__shfl_xor((int)v, 16));
  return max(v, (uint32_t)__shfl_xor((int)v, 32));
}

// The power of two that brings a row's largest finite magnitude into [2^14, 2^15), as an exponent.  It stops
// at 126 (2^-126 and its inverse are normal numbers).
__device__ __forceinline__ int row_exponent(uint32_t top) {
  if (top == 0) return 0;
  const int e = (int)(top >> 23) - 127;  // a subnormal counts as 2^-127
  return min(14 - e, 126);
}
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// ---------------------------------------------------------------------------
// finished pieces
// ---------------------------------------------------------------------------

// NC elements in whole.  16-bit ones of rows of odd lengths begin between 32-bit words, where a wide access costs
// several times an aligned one: they go as the words that hold them, shifted by an element, and by themselves at the
// ends (777 x 2559 outputs with residual and kept pre-activation 36.4 us, now 32.7 us).
template <class T, int NC> struct Pack { T v[NC]; };
template <class T> __device__ __forceinline__ bool between_words(const T* p) {
  return sizeof(T) == 2 && (reinterpret_cast<uintptr_t>(p) & 2u) != 0;
}
template <int NC, class T>
__device__ __forceinline__ Pack<T, NC> load_pack(const T* p) {
  if constexpr (sizeof(T) == 2 && NC >= 4) {
    const bool between = between_words(p);
    if (__any(between)) {
      struct Words { uint32_t w[NC / 2]; };
      const char* from = (const char*)p - (between ? 2 : 0);
      Words a;
      __builtin_memcpy(&a, __builtin_assume_aligned(from, 4), sizeof(a));
      const uint32_t after = between ? *(const uint32_t*)(from + 2 * NC) : 0;
#pragma unroll
      for (int i = 0; i < NC / 2; ++i) a.w[i] = __builtin_amdgcn_alignbyte(i + 1 < NC / 2 ? a.w[i + 1 < NC / 2 ? i + 1 : 0] : after, a.w[i], between ? 2 : 0);
      return __builtin_bit_cast(Pack<T, NC>, a);
    }
  }
  return load_any<Pack<T, NC>>(p);
}
template <int NC, class T>
__device__ __forceinline__ void store_pack(T* p, const Pack<T, NC>& k) {
  if constexpr (sizeof(T) == 2 && NC >= 4) {
    const bool between = between_words(p);
    if (__any(between)) {
      struct Words { uint32_t w[NC / 2]; };
      struct Inner { uint32_t w[NC / 2 - 1]; };
      const Words a = __builtin_bit_cast(Words, k);
      Inner o;
#pragma unroll
      for (int i = 0; i + 1 < NC / 2; ++i) o.w[i] = __builtin_amdgcn_alignbyte(a.w[i + 1], a.w[i], between ? 2 : 0);
      __builtin_memcpy(__builtin_assume_aligned((char*)p + (between ? 2 : 0), 4), &o, sizeof(o));
      if (between) {
        p[0] = k.v[0];
        p[NC - 1] = k.v[NC - 1];
      } else {
        *(uint32_t*)(p + NC - 2) = a.w[NC / 2 - 1];
      }
      return;
    }
  }
  store_any(p, k);
}

template <int NC, class T>
__device__ __forceinline__ void load_cols(float (&o)[NC], const T* p, int valid) {
  if (valid >= NC) {
    const Pack<T, NC> k = load_pack<NC, T>(p);
#pragma unroll
    for (int i = 0; i < NC; ++i) o[i] = widen(k.v[i]);
  } else {
#pragma unroll
    for (int i = 0; i < NC; ++i) o[i] = 0.0f;
    if (valid > 0) {
      T v[NC];  // every load on its way before the first is waited for
#pragma unroll
      for (int i = 0; i < NC; ++i) v[i] = p[i < valid ? i : 0];
#pragma unroll
      for (int i = 0; i < NC; ++i) o[i] = i < valid ? widen(v[i]) : 0.0f;
    }
  }
}

template <int NC, class T>
__device__ __forceinline__ void store_cols(T* p, const float (&o)[NC], int valid) {
  if (valid >= NC) {
    Pack<T, NC> k;
#pragma unroll
    for (int i = 0; i < NC; ++i) k.v[i] = narrow<T>(o[i]);
    store_pack<NC, T>(p, k);
  } else {
#pragma unroll
    for (int i = 0; i < NC; ++i)
      if (i < valid) p[i] = narrow<T>(o[i]);
  }
}

// What a lane's columns share over the rows: loaded once.
template <int NC> struct Columns {
  float scale[NC], bias[NC];
};
template <int NC, class T>
__device__ __forceinline__ void load_columns(Columns<NC>& k, const Finish& f, int32_t col) {
  const int valid = min(max(f.cols - col, 0), NC);
  load_cols<NC, float>(k.scale, f.scales + col, valid);
#pragma unroll
  for (int i = 0; i < NC; ++i) k.bias[i] = 0.0f;
  if (f.kind == kLinear && f.bias) load_cols<NC, T>(k.bias, (const T*)f.bias + col, valid);
}

// What a row's outputs share.  `product` fetches it once into the LDS: loaded for each fragment of rows it is a trip to
// memory in each (loss and gradient of 2048 rows over 32768 entries 799 us with, 785 us without).
struct RowValues {
  float factor;  // of a row held in planes
  int32_t label;  // kStats, kProb: the label's column, or -1
  float lse;      // kProb: base 2
};
__device__ __forceinline__ RowValues row_values(const Finish& f, int64_t row) {
  RowValues r = {1.0f, -1, 0.0f};
  if (row >= f.rows) return r;
  if (f.row_factor) r.factor = f.row_factor[row];
  if (f.kind == kStats || f.kind == kProb) {
    const int64_t at = f.labels[row] - f.first_col;
    r.label = at >= 0 && at < f.cols ? (int32_t)at : -1;
  }
  if (f.kind == kProb) r.lse = f.lse[row] * kLog2E;
  return r;
}

// A lane's NC consecutive columns of one row, `v` the bare sums.  With NC = 16 the lanes l, l^16, l^32, l^48
// hold the row's 64 columns of one tile (every lane of the wave calls).  T: the output's type.
template <int NC, class T>
__device__ __forceinline__ void finish_layer(const Finish& f, const Columns<NC>& k, int64_t row, int32_t col, float (&v)[NC],
                                             const RowValues& shared) {
  const bool live = row < f.rows;
  const int valid = live ? min(max(f.cols - col, 0), NC) : 0;
  const float factor = f.unit * shared.factor;
  float s[NC];
  const bool add = f.kind == kLinear && f.residual;
  if (add) load_cols<NC, T>(s, (const T*)f.residual + row * f.ldr + col, valid);
  // the scale first: a large row's factor alone may overflow
#pragma unroll
  for (int i = 0; i < NC; ++i) v[i] = v[i] * k.scale[i] * factor;
  if (f.kind == kLinear) {
#pragma unroll
    for (int i = 0; i < NC; ++i) v[i] += k.bias[i];
    if constexpr (NC == 16) {
      if (f.keep == SQUANT_KEEP_FULL) store_cols<NC, T>((T*)f.kept + row * f.cols + col, v, valid);
      if (f.keep == SQUANT_KEEP_INT8) {
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < NC; ++i) top = max(top, i < valid ? magnitude(v[i]) : 0u);
        top = group_max(top);
        const float t = __uint_as_float(top);
        // next to zero 127 / t leaves binary32's range: the group is taken 2^60 times as large
        const float up = t < 0x1p-60f ? 0x1p60f : 1.0f, per = top ? 127.0f / (t * up) : 0.0f;
        if (live && col < f.cols && (col & (kTile - 1)) == 0)
          f.kept_scales[row * ((f.cols + kTile - 1) / kTile) + col / kTile] = top ? t / 127.0f : 1.0f;
        uint32_t q[4];
#pragma unroll
        for (int d = 0; d < 4; ++d) {
          q[d] = 0;
#pragma unroll
          for (int b = 0; b < 4; ++b) {
            const float c = fminf(fmaxf(rintf(v[4 * d + b] * up * per), -127.0f), 127.0f);
            q[d] |= ((uint32_t)(int)c & 255u) << (8 * b);
          }
        }
        int8_t* out = (int8_t*)f.kept + row * f.cols + col;
        if (valid >= NC) {
          store_any(out, uint4v{q[0], q[1], q[2], q[3]});
        } else {
#pragma unroll
          for (int i = 0; i < NC; ++i)
            if (i < valid) out[i] = (int8_t)(q[i >> 2] >> (8 * (i & 3)));
        }
      }
    }
    activate<T, NC>(v, f.act);
    if (add) {
#pragma unroll
      for (int i = 0; i < NC; ++i) v[i] += s[i];
    }
    store_cols<NC, T>((T*)f.out + row * f.ldo + col, v, valid);
    return;
  }
  if constexpr (NC == 16) {
    if (f.kind == kStats) {
      // base 2: the label's logit, and the chunk's largest logit and sum of exponentials
      float top = -__builtin_inff();
#pragma unroll
      for (int i = 0; i < NC; ++i) {
        v[i] = i < valid ? v[i] * kLog2E : -__builtin_inff();
        top = fmaxf(top, v[i]);
      }
      if (live) {
        const int32_t at = shared.label - col;
        if (at >= 0 && at < valid) {
#pragma unroll
          for (int i = 0; i < NC; ++i)
            if (at == i) f.label_logit[row] = v[i];
        }
      }
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      float sum = 0.0f;
      const float from = top == -__builtin_inff() ? 0.0f : top;  // a chunk without a finite logit adds nothing
#pragma unroll
      for (int i = 0; i < NC; ++i) sum += i < valid ? exp2_fast(v[i] - from) : 0.0f;
      sum += __shfl_xor(sum, 16);
      sum += __shfl_xor(sum, 32);
      if (live && col < f.cols && (col & (kTile - 1)) == 0)
        f.stats[row * ((f.cols + kTile - 1) / kTile) + col / kTile] = make_float2(top, sum);
    }
  }
}

// The gradient's row operand from 16 logits of a row, on the same lanes: p * scale * 2^E in PL planes, zero at the label and
// from the piece's end to its next multiple of 64 columns.  Returns the sum of the tile's probabilities beside the label's.
template <int PL>
__device__ __forceinline__ float finish_prob(const Finish& f, const Columns<16>& k, int64_t row, int32_t col, float (&v)[16],
                                             const RowValues& shared, float prob_unit) {
  const bool live = row < f.rows;
  const int valid = live ? min(max(f.cols - col, 0), 16) : 0;
  const float factor = f.unit * shared.factor;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    v[i] = v[i] * k.scale[i] * factor;
    v[i] = i < valid ? exp2_fast(__builtin_fmaf(v[i], kLog2E, -shared.lse)) : 0.0f;
  }
  const int32_t at = shared.label - col;
  if (__any(at >= 0 && at < valid)) {
    if (at >= 0 && at < valid) {
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (at == i) f.label_prob[row] = v[i];
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = at == i ? 0.0f : v[i];
  }
  float others = 0.0f;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    others += v[i];
    v[i] *= k.scale[i] * prob_unit;
  }
  if (live && col < (f.cols + kTile - 1) / kTile * kTile) {
    _Float16* p = f.prob + row * f.ld_prob + col;
    store_cols<16, _Float16>(p, v, 16);
    if (PL == 2) {
#pragma unroll
      for (int i = 0; i < 16; ++i) v[i] -= (float)(_Float16)v[i];
      store_cols<16, _Float16>(p + f.prob_plane, v, 16);
    }
  }
  others += __shfl_xor(others, 16);
  return others + __shfl_xor(others, 32);
}

// kProb: a row's sum of one tile of columns.  Pieces of the vocabulary add to the same sums.
__device__ __forceinline__ void store_others(const Finish& f, int64_t row, int32_t tile, float sum, bool accumulate) {
  if (row >= f.rows) return;
  float* p = f.other_sums + tile * f.rows + row;
  *p = accumulate ? *p + sum : sum;
}

// The same for the gradients: columns are the layer's inputs.
//
// Of the loss: dh = g * (sum over v != y of p_v w_v - (1 - p_y) w_y).  Where p_y > 1/2, 1 - p_y is the other probabilities' sum: as
// a difference it would be off by the rounding of p_y, many times the gradient of a row whose label is likely.
// `row_factor`: 2^-e of the row, or 1 - p_y (kGradLoss).
template <class T>
__device__ __forceinline__ void finish_grad_as(const Finish& f, int64_t row, int32_t col, float (&v)[16], float row_factor) {
  const int valid = row < f.rows ? min(max(f.cols - col, 0), 16) : 0;
  if (valid == 0) return;
  if (f.kind == kGrad) {
    const float factor = f.unit * row_factor;
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] *= factor;
  } else {
    const int64_t label = f.labels[row];
    if (label == f.ignore) {
#pragma unroll
      for (int i = 0; i < 16; ++i) v[i] = 0.0f;
    } else if (label < 0 || label >= f.vocabulary) {
#pragma unroll
      for (int i = 0; i < 16; ++i) v[i] = __builtin_nanf("");
    } else {
      const float factor = f.unit / *f.prob_unit, g = f.dloss[row], s = row_factor * f.scales[label];
      const uint8_t* codes = f.codes + label * f.code_row;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        float c = 0.0f;
        if (i < valid)
          c = (float)(f.format == SQUANT_OUT_INT8 ? Codes<SQUANT_OUT_INT8>::value(codes, col + i)
                                                  : Codes<SQUANT_OUT_INT4>::value(codes, col + i));
        v[i] = g * (v[i] * factor - s * c);
      }
    }
  }
  store_cols<16, T>((T*)f.out + row * f.ldo + col, v, valid);
}

__device__ __forceinline__ void finish_grad(const Finish& f, int64_t row, int32_t col, float (&v)[16], float row_factor) {
  if (f.out_type == SQUANT_W_F32) finish_grad_as<float>(f, row, col, v, row_factor);
  else if (f.out_type == SQUANT_W_F16) finish_grad_as<_Float16>(f, row, col, v, row_factor);
  else finish_grad_as<__bf16>(f, row, col, v, row_factor);
}

// The type of a layer's output by its row operand.
template <class F, int PL> struct OutOf { typedef float type; };
template <> struct OutOf<Half, 1> { typedef _Float16 type; };
template <> struct OutOf<Brain, 1> { typedef __bf16 type; };

// Where the 4 values of column fragment `c` of a lane group of 4 lanes go among its 16 columns: the layer's
// fragments hold 4 consecutive columns, the gradient's every fourth.
template <bool GRAD>
__device__ __forceinline__ constexpr int column_of(int c, int i) { return GRAD ? 4 * i + c : 4 * c + i; }

}  // namespace lin
}  // namespace squant
