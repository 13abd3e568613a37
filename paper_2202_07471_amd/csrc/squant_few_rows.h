// The product of at most 64 rows (binary32: 32) with codes: bound by the codes' bytes, or by a few trips to memory where they are
// few.
//
// A workgroup owns 16 * NF columns and its waves share the contraction, a unit of 16 bytes of each code row at a time
// in turn, so that neighbouring waves read neighbouring bytes.  Codes go straight to registers; rows come from the
// caches, where the other workgroups' reads leave them.  Every load of up to kAhead units is on its way before the
// first is multiplied: a wave of a 4096-wide layer waits for memory once.  The waves' sums meet in the LDS.
//
// Loads off a 32-bit boundary cost two to three times an aligned one (8 rows by 16384 x 2049 int8 codes 21.3 us, now 13.5
// us), so code rows that do not begin at whole words (WORDS false) are read as the words that hold them, one more than
// there are words of codes, and shifted into place by their address's low two bits.  No word is read that holds no byte
// of the buffer: the row has more codes after these, or the shift is not 0.
#pragma once

#include "squant_lin.h"

namespace squant {
namespace lin {

// Waves of a workgroup: 16 where its columns are few and the waves' registers and sums fit.
constexpr int few_waves(int mf, int nf) { return nf == 4 || mf * nf > 4 ? 8 : 16; }
constexpr size_t few_lds(int mf, int nf) { return (size_t)few_waves(mf, nf) * mf * (nf * kLanes * 16 + 16 * 4); }

// Rows up to which `few_rows` is taken.  Every workgroup splits its binary32 rows anew: past 32 of them a pass of
// its own costs less.
constexpr int few_rows_limit(int planes) { return planes == 1 ? 64 : 32; }

// 8 binary32 numbers as hi + lo of binary16, times `up`.
struct Planes { half8 v[2]; };
__device__ __forceinline__ Planes split8(const uint4v (&x)[2], float up) {
  Planes o;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float f = __uint_as_float(x[i >> 2][i & 3]) * up;
    o.v[0][i] = (_Float16)f;
    o.v[1][i] = magnitude(f) < 0x7f800000u ? (_Float16)(f - (float)o.v[0][i]) : (_Float16)0.0f;  // an infinity has no remainder
  }
  return o;
}

// 8 elements of a row from element k on, zeros from element `cols` on.
__device__ __forceinline__ uint4v load_row8(const char* row, int64_t k, int64_t cols) {
  if (k + 8 <= cols) return load_any<uint4v>(row + 2 * k);
  uint4v o = {0, 0, 0, 0};
  if (k >= cols) return o;
  uint32_t v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = load_any<uint16_t>(row + 2 * (k + i < cols ? k + i : k));
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (k + i < cols) o[i >> 1] |= v[i] << (16 * (i & 1));
  return o;
}

// T: the type of the rows and of the output; binary32 with F = Half.
template <class F, class T, int FMT, int MF, int NF, bool WORDS>
__global__ void __launch_bounds__(few_waves(MF, NF) * kLanes, sizeof(T) == 2 && MF * NF <= 8 ? 4 : 2) few_rows(ProductArgs a) {
  constexpr int kWaves = few_waves(MF, NF);
  constexpr int kHalves = FMT == SQUANT_OUT_INT4 ? 4 : 2;  // groups of 8 codes in 16 bytes
  constexpr int kUnit = 32 * kHalves;                      // contraction elements of a unit
  constexpr bool kSplit = sizeof(T) == 4;                  // rows are split into planes
  constexpr int PL = kSplit ? 2 : 1;                         // 16-byte loads of 8 elements
  constexpr int kRowFrags = PL * kHalves * MF;             // of a unit
  constexpr bool kRowsAhead = kRowFrags <= 8;              // its rows are loaded with its codes
  constexpr int kAheadMost = 16 / (NF + (kRowsAhead ? kRowFrags : 0));  // by 64 registers
  constexpr int kAhead = kAheadMost >= 4 && kRowsAhead ? 4 : kAheadMost >= 2 ? 2 : 1;
  typedef typename Codes<FMT>::row16 codes16;
  extern __shared__ __align__(16) unsigned char smem[];
  const int lane = threadIdx.x & (kLanes - 1);
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kLanes);  // known to be uniform
  const int sub = lane & 15, quad = lane >> 4;
  const int32_t col0 = (int32_t)blockIdx.x * (16 * NF);
  const int32_t row0 = (int32_t)blockIdx.y * (16 * MF);

  const int64_t w_bytes = (int64_t)a.w_rows * a.w_row;
  const uint8_t* w[NF];
  uint32_t shift[NF];  // to the words that hold the row's codes
#pragma unroll
  for (int c = 0; c < NF; ++c) {
    const int32_t n = NF == 4 ? col0 + (sub >> 2) * 16 + c * 4 + (sub & 3) : col0 + c * 16 + sub;
    w[c] = a.w + (int64_t)min(n, a.w_rows - 1) * a.w_row + quad * 16;
    shift[c] = WORDS ? 0 : (uint32_t)(reinterpret_cast<uintptr_t>(w[c]) & 3u);
  }
  const char* x[MF];
#pragma unroll
  for (int m = 0; m < MF; ++m) x[m] = (const char*)a.a + min((int64_t)(row0 + m * 16 + sub), a.f.rows - 1) * a.lda * (int)sizeof(T);

  float4v acc[MF][NF];
#pragma unroll
  for (int m = 0; m < MF; ++m)
#pragma unroll
    for (int c = 0; c < NF; ++c) acc[m][c] = float4v{0.0f, 0.0f, 0.0f, 0.0f};

  struct Operands {
    uint4v codes[NF];
    uint32_t after[WORDS ? 1 : NF];
    uint4v rows[kRowsAhead ? PL : 1][kRowsAhead ? kHalves : 1][kRowsAhead ? MF : 1];
  };
  auto element = [&](int u, int h) { return (int64_t)u * kUnit + quad * (kUnit / 4) + h * 8; };
  // Row elements of a unit; `ends`: it may reach past the row's end.
  auto row_frag = [&](int u, int p, int h, int m, bool ends) {
    const int64_t k = element(u, h);
    if constexpr (kSplit) {
      const float* f = (const float*)x[m] + k + 4 * p;
      if (!ends) return load_any<uint4v>(f);
      uint4v o = {0, 0, 0, 0};
      if (k + 4 * p >= a.w_cols) return o;
#pragma unroll
      for (int i = 0; i < 4; ++i) o[i] = load_any<uint32_t>(f + (k + 4 * p + i < a.w_cols ? i : 0));
#pragma unroll
      for (int i = 0; i < 4; ++i) o[i] = k + 4 * p + i < a.w_cols ? o[i] : 0;
      return o;
    } else {
      if (ends) return load_row8(x[m], k, a.w_cols);
      return load_any<uint4v>(x[m] + 2 * k);
    }
  };
  auto load_unit = [&](int u, Operands& o, bool ends) {
    if (ends) {
      const uint8_t* at[NF];
#pragma unroll
      for (int c = 0; c < NF; ++c) at[c] = w[c] + (int64_t)u * 64;
      load_before(o.codes, at, a.w_end, w_bytes);
    } else {
#pragma unroll
      for (int c = 0; c < NF; ++c) {
        o.codes[c] = load_any<uint4v>(w[c] - shift[c] + (int64_t)u * 64);
        if constexpr (!WORDS) o.after[c] = load_any<uint32_t>(w[c] - shift[c] + (int64_t)u * 64 + 16);
      }
    }
    if constexpr (kRowsAhead) {
#pragma unroll
      for (int p = 0; p < PL; ++p)
#pragma unroll
        for (int h = 0; h < kHalves; ++h)
#pragma unroll
          for (int m = 0; m < MF; ++m) o.rows[p][h][m] = row_frag(u, p, h, m, ends);
    }
  };
  // binary32: what a lane adds up belongs to one row, so that the row's exponent is a number of the lane's.  It
  // follows the largest element seen; the sums so far are brought to it.
  int exponent[kSplit ? MF : 1];
#pragma unroll
  for (int m = 0; m < (kSplit ? MF : 1); ++m) exponent[m] = 126;
  auto raise = [&](const uint4v (&rows)[PL], int m) {
    uint32_t top = 0;
#pragma unroll
    for (int p = 0; p < PL; ++p)
#pragma unroll
      for (int i = 0; i < 4; ++i) top = max(top, rows[p][i] & 0x7fffffffu);
    top = group_max(min(top, 0x7f7fffffu));  // an infinity or a NaN: as the largest number
    const int e = min(exponent[m], row_exponent(top));
    if (!__any(top != 0 && e < exponent[m])) return;
    const int drop = top != 0 ? max(e - exponent[m], -126) : 0;
    exponent[m] = top != 0 ? e : exponent[m];
#pragma unroll
    for (int c = 0; c < NF; ++c) acc[m][c] *= power_of_two(drop);
  };
  auto multiply = [&](int u, const Operands& o, bool ends) {
#pragma unroll
    for (int h = 0; h < kHalves; ++h) {
      if constexpr (!kRowsAhead) __builtin_amdgcn_sched_barrier(0);  // one half's rows at a time in registers
      typename F::frag wf[NF];
#pragma unroll
      for (int c = 0; c < NF; ++c) {
        uint4v q = o.codes[c];
        if (!WORDS && !ends) {
#pragma unroll
          for (int i = h * 4 / kHalves; i < (h + 1) * 4 / kHalves; ++i)
            q[i] = __builtin_amdgcn_alignbyte(i < 3 ? o.codes[c][i < 3 ? i + 1 : 3] : o.after[c], o.codes[c][i], shift[c]);
        }
        codes16 r;
        if constexpr (FMT == SQUANT_OUT_INT4) r = h < 2 ? codes16{q[0], q[1]} : codes16{q[2], q[3]};
        else r = q;
        wf[c] = convert<F, FMT>(r, h & 1);
      }
#pragma unroll
      for (int m = 0; m < MF; ++m) {
        uint4v rows[PL];
#pragma unroll
        for (int p = 0; p < PL; ++p) {
          if constexpr (kRowsAhead) rows[p] = o.rows[p][h][m];
          else rows[p] = row_frag(u, p, h, m, ends);
        }
        if constexpr (kSplit) {
          raise(rows, m);
          const Planes x = split8(rows, power_of_two(exponent[m]));
#pragma unroll
          for (int p = 1; p >= 0; --p)
#pragma unroll
            for (int c = 0; c < NF; ++c) acc[m][c] = F::mma(wf[c], x.v[p], acc[m][c]);
        } else {
#pragma unroll
          for (int c = 0; c < NF; ++c) acc[m][c] = F::mma(wf[c], __builtin_bit_cast(typename F::frag, rows[0]), acc[m][c]);
        }
      }
    }
  };

  const int whole = a.w_cols / kUnit, units = (a.w_cols + kUnit - 1) / kUnit;
  int u = wave;
#pragma unroll 1
  for (; u + (kAhead - 1) * kWaves < whole; u += kAhead * kWaves) {
    Operands o[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) load_unit(u + i * kWaves, o[i], false);
#pragma unroll
    for (int i = 0; i < kAhead; ++i) multiply(u + i * kWaves, o[i], false);
  }
  if constexpr (kAhead > 1) {
#pragma unroll 1
    for (; u < whole; u += kWaves) {
      Operands o;
      load_unit(u, o, false);
      multiply(u, o, false);
    }
  }
  if (u < units) {  // the one unit that ends within
    Operands o;
    load_unit(u, o, true);
    multiply(u, o, true);
  }

  float4v* sums = reinterpret_cast<float4v*>(smem);
  int* exponents = reinterpret_cast<int*>(smem + (size_t)kWaves * MF * NF * kLanes * 16);  // [wave][m][row], binary32
#pragma unroll
  for (int m = 0; m < MF; ++m) {
#pragma unroll
    for (int c = 0; c < NF; ++c) sums[((wave * MF + m) * NF + c) * kLanes + lane] = acc[m][c];
    if (kSplit && lane < 16) exponents[(wave * MF + m) * 16 + lane] = exponent[kSplit ? m : 0];
  }
  __syncthreads();
  auto least = [&](int m) {
    int e = exponents[m * 16 + sub];
#pragma unroll 4
    for (int o = 1; o < kWaves; ++o) e = min(e, exponents[(o * MF + m) * 16 + sub]);
    return e;
  };
  auto total = [&](int m, int c, int e) {
    float4v t = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
    for (int o = 0; o < kWaves; ++o) {
      const float4v s = sums[((o * MF + m) * NF + c) * kLanes + lane];
      if constexpr (kSplit) t += s * power_of_two(max(e - exponents[(o * MF + m) * 16 + sub], -126));
      else t += s;
    }
    return t;
  };
  if constexpr (NF == 4) {
    if (wave >= MF) return;
    Columns<16> columns;
    load_columns<16, T>(columns, a.f, col0 + quad * 16);
    const int e = kSplit ? least(wave) : 0;
    float v[16];
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const float4v t = total(wave, c, e);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[4 * c + i] = t[i];
    }
    RowValues shared = row_values(a.f, row0 + wave * 16 + sub);
    shared.factor = power_of_two(-e);
    const int64_t row = row0 + wave * 16 + sub;
    if (a.f.kind == kProb) {
      const float others = finish_prob<PL>(a.f, columns, row, col0 + quad * 16, v, shared, *a.f.prob_unit);
      if (quad == 0) store_others(a.f, row, blockIdx.x, others, a.accumulate);
    } else {
      finish_layer<16, T>(a.f, columns, row, col0 + quad * 16, v, shared);
    }
  } else {
    if (wave >= MF * NF) return;
    const int m = wave / NF, c = wave % NF;
    const int32_t col = col0 + c * 16 + quad * 4;
    Columns<4> columns;
    load_columns<4, T>(columns, a.f, col);
    const int e = kSplit ? least(m) : 0;
    const float4v t = total(m, c, e);
    float v[4] = {t[0], t[1], t[2], t[3]};
    finish_layer<4, T>(a.f, columns, row0 + m * 16 + sub, col, v, RowValues{power_of_two(-e), -1, 0.0f});
  }
}

template <class F, class T, int FMT, int NF, bool WORDS>
product_t few_rows_of(int mf) {
  if (mf == 1) return few_rows<F, T, FMT, 1, NF, WORDS>;
  if constexpr (sizeof(T) == 2)
    if (mf == 4) return few_rows<F, T, FMT, 4, NF, WORDS>;
  return few_rows<F, T, FMT, 2, NF, WORDS>;
}
template <class F, class T, int FMT>
product_t few_of(int mf, int nf, bool words) {
  if (nf == 4) return words ? few_rows_of<F, T, FMT, 4, true>(mf) : few_rows_of<F, T, FMT, 4, false>(mf);
  if (nf == 2) return words ? few_rows_of<F, T, FMT, 2, true>(mf) : few_rows_of<F, T, FMT, 2, false>(mf);
  return words ? few_rows_of<F, T, FMT, 1, true>(mf) : few_rows_of<F, T, FMT, 1, false>(mf);
}

}  // namespace lin
}  // namespace squant
