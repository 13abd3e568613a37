// The product of at most 64 rows with codes: bound by the codes' bytes, or by a few trips to memory where they are
// few.
//
// A workgroup owns 16 * NF columns and its waves share the contraction, a unit of 16 bytes of each code row at a time
// in turn, so that neighbouring waves read neighbouring bytes.  Codes go straight to registers; rows come from the
// caches, where the other workgroups' reads leave them.  Every load of up to kAhead units is on its way before the
// first is multiplied: a wave of a 4096-wide layer waits for memory once.  The waves' sums meet in the LDS.
#pragma once

#include "squant_lin.h"

namespace squant {
namespace lin {

// Waves of a workgroup: 16 where its columns are few and the waves' registers and sums fit.
constexpr int few_waves(int mf, int nf) { return nf == 4 || mf * nf > 4 ? 8 : 16; }
constexpr size_t few_lds(int mf, int nf) { return (size_t)few_waves(mf, nf) * mf * nf * kLanes * 16; }

// 8 elements of a row from element k on, zeros from element `cols` on.
__device__ __forceinline__ uint4v load_row8(const char* row, int64_t k, int64_t cols) {
  if (k + 8 <= cols) return load_any<uint4v>(row + 2 * k);
  uint4v o = {0, 0, 0, 0};
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (k + i < cols) o[i >> 1] |= (uint32_t)load_any<uint16_t>(row + 2 * (k + i)) << (16 * (i & 1));
  return o;
}

template <class F, int PL, int FMT, int MF, int NF, bool WORDS>
__global__ void __launch_bounds__(few_waves(MF, NF) * kLanes) few_rows(ProductArgs a) {
  constexpr int kWaves = few_waves(MF, NF);
  constexpr int kHalves = FMT == SQUANT_OUT_INT4 ? 4 : 2;  // groups of 8 codes in 16 bytes
  constexpr int kUnit = 32 * kHalves;                      // contraction elements of a unit
  constexpr int kRowFrags = PL * kHalves * MF;             // of a unit
  constexpr bool kRowsAhead = kRowFrags <= 8;              // its rows are loaded with its codes
  constexpr int kAheadMost = 16 / (NF + (kRowsAhead ? kRowFrags : 0));  // by 64 registers
  constexpr int kAhead = kAheadMost >= 4 ? 4 : kAheadMost >= 2 ? 2 : 1;
  typedef typename Codes<FMT>::row16 codes16;
  typedef typename OutOf<F, PL>::type T;
  extern __shared__ __align__(16) unsigned char smem[];
  const int lane = threadIdx.x & (kLanes - 1), wave = threadIdx.x / kLanes;
  const int sub = lane & 15, quad = lane >> 4;
  const int32_t col0 = (int32_t)blockIdx.x * (16 * NF);

  const int64_t w_bytes = (int64_t)a.w_rows * a.w_row;
  const uint8_t* w[NF];
  uint32_t shift[NF];  // see RowCodes
#pragma unroll
  for (int c = 0; c < NF; ++c) {
    const int32_t n = NF == 4 ? col0 + (sub >> 2) * 16 + c * 4 + (sub & 3) : col0 + c * 16 + sub;
    w[c] = a.w + (int64_t)min(n, a.w_rows - 1) * a.w_row + quad * 16;
    shift[c] = WORDS ? 0 : (uint32_t)(reinterpret_cast<uintptr_t>(w[c]) & 3u);
  }
  const char* x[MF];
#pragma unroll
  for (int m = 0; m < MF; ++m) x[m] = (const char*)a.a + min((int64_t)(m * 16 + sub), a.f.rows - 1) * a.lda * 2;

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
    if (ends) return load_row8(x[m] + 2 * p * a.plane, element(u, h), a.w_cols);
    return load_any<uint4v>(x[m] + 2 * (p * a.plane + element(u, h)));
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
      for (int p = 0; p < PL; ++p)
#pragma unroll
        for (int m = 0; m < MF; ++m) {
          uint4v rows;
          if constexpr (kRowsAhead) rows = o.rows[p][h][m];
          else rows = row_frag(u, p, h, m, ends);
#pragma unroll
          for (int c = 0; c < NF; ++c) acc[m][c] = F::mma(wf[c], __builtin_bit_cast(typename F::frag, rows), acc[m][c]);
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
#pragma unroll
  for (int m = 0; m < MF; ++m)
#pragma unroll
    for (int c = 0; c < NF; ++c) sums[((wave * MF + m) * NF + c) * kLanes + lane] = acc[m][c];
  __syncthreads();
  auto total = [&](int m, int c) {
    float4v t = sums[(m * NF + c) * kLanes + lane];
#pragma unroll 4
    for (int o = 1; o < kWaves; ++o) t += sums[((o * MF + m) * NF + c) * kLanes + lane];
    return t;
  };
  if constexpr (NF == 4) {
    if (wave >= MF) return;
    Columns<16> columns;
    load_columns<16, T>(columns, a.f, col0 + quad * 16);
    float v[16];
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const float4v t = total(wave, c);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[4 * c + i] = t[i];
    }
    finish_layer<16, T>(a.f, columns, wave * 16 + sub, col0 + quad * 16, v, PL);
  } else {
    if (wave >= MF * NF) return;
    const int m = wave / NF, c = wave % NF;
    const int32_t col = col0 + c * 16 + quad * 4;
    Columns<4> columns;
    load_columns<4, T>(columns, a.f, col);
    const float4v t = total(m, c);
    float v[4] = {t[0], t[1], t[2], t[3]};
    finish_layer<4, T>(a.f, columns, m * 16 + sub, col, v, PL);
  }
}

template <class F, int PL, int FMT, int NF, bool WORDS>
product_t few_rows_of(int mf) {
  if (mf == 1) return few_rows<F, PL, FMT, 1, NF, WORDS>;
  if (mf == 2) return few_rows<F, PL, FMT, 2, NF, WORDS>;
  return few_rows<F, PL, FMT, 4, NF, WORDS>;
}
template <class F, int PL, int FMT>
product_t few_of(int mf, int nf, bool words) {
  if (nf == 4) return words ? few_rows_of<F, PL, FMT, 4, true>(mf) : few_rows_of<F, PL, FMT, 4, false>(mf);
  if (nf == 2) return words ? few_rows_of<F, PL, FMT, 2, true>(mf) : few_rows_of<F, PL, FMT, 2, false>(mf);
  return words ? few_rows_of<F, PL, FMT, 1, true>(mf) : few_rows_of<F, PL, FMT, 1, false>(mf);
}

}  // namespace lin
}  // namespace squant
