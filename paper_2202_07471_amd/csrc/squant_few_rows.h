// The product of at most 64 rows with codes: bound by the codes' bytes.
//
// A workgroup owns 16 * NF columns and its waves share the contraction, 64 elements in turn, so that neighbouring
// waves read neighbouring bytes of the code rows.  Codes go straight to registers; rows come from the caches, where
// the other workgroups' reads leave them.  The waves' sums meet in the LDS.  Where the columns make too few
// workgroups to fill the chip, workgroups share the contraction too and leave partial sums (NF = 4 only).
#pragma once

#include "squant_lin.h"

namespace squant {
namespace lin {

constexpr int kFewWaves = 8;

template <class F, int PL, int FMT, int MF, int NF>
__global__ void __launch_bounds__(kFewWaves * kLanes) few_rows(ProductArgs a) {
  typedef typename Codes<FMT>::row16 codes16;
  extern __shared__ __align__(16) unsigned char smem[];
  const int lane = threadIdx.x & (kLanes - 1), wave = threadIdx.x / kLanes;
  const int sub = lane & 15, quad = lane >> 4;
  const int32_t col0 = (int32_t)blockIdx.x * (16 * NF);
  const int slice = blockIdx.y;
  const int first = (int)((int64_t)a.blocks * slice / a.slices), last = (int)((int64_t)a.blocks * (slice + 1) / a.slices);

  const int64_t w_bytes = (int64_t)a.w_rows * a.w_row;
  const uint8_t* w[NF];
#pragma unroll
  for (int c = 0; c < NF; ++c) {
    const int32_t n = NF == 4 ? col0 + (sub >> 2) * 16 + c * 4 + (sub & 3) : col0 + c * 16 + sub;
    w[c] = a.w + (int64_t)min(n, a.w_rows - 1) * a.w_row;
  }
  const char* x[MF];
#pragma unroll
  for (int m = 0; m < MF; ++m)
    x[m] = (const char*)a.a + min((int64_t)(m * 16 + sub), a.f.rows - 1) * a.lda * 2 + quad * 32;

  float4v acc[MF][NF];
#pragma unroll
  for (int m = 0; m < MF; ++m)
#pragma unroll
    for (int c = 0; c < NF; ++c) acc[m][c] = float4v{0.0f, 0.0f, 0.0f, 0.0f};

  auto multiply = [&](int b, const codes16 (&r)[NF]) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      typename F::frag wf[NF];
#pragma unroll
      for (int c = 0; c < NF; ++c) wf[c] = convert<F, FMT>(r[c], h);
#pragma unroll
      for (int p = 0; p < PL; ++p)
#pragma unroll
        for (int m = 0; m < MF; ++m) {
          const typename F::frag xf =
              load_any<typename F::frag>(x[m] + p * a.plane * 2 + (int64_t)b * (kBlock * 2) + h * 16);
#pragma unroll
          for (int c = 0; c < NF; ++c) acc[m][c] = F::mma(wf[c], xf, acc[m][c]);
        }
    }
  };

  // whole blocks, kAhead of them loaded before the first is multiplied
  constexpr int kAhead = NF * MF >= 8 ? 2 : 4;
  const int whole = min(last, a.w_cols / kBlock);
  int b = first + wave;
  for (; b + (kAhead - 1) * kFewWaves < whole; b += kAhead * kFewWaves) {
    codes16 r[kAhead][NF];
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
#pragma unroll
      for (int c = 0; c < NF; ++c)
        r[u][c] = load_any<codes16>(w[c] + Codes<FMT>::offset((int64_t)(b + u * kFewWaves) * kBlock + quad * 16));
#pragma unroll
    for (int u = 0; u < kAhead; ++u) multiply(b + u * kFewWaves, r[u]);
  }
  for (; b < last; b += kFewWaves) {
    codes16 r[NF];
    const uint8_t* at[NF];
#pragma unroll
    for (int c = 0; c < NF; ++c) at[c] = w[c] + Codes<FMT>::offset((int64_t)b * kBlock + quad * 16);
    load_before(r, at, a.w_end, w_bytes);
    multiply(b, r);
  }

  float4v* sums = reinterpret_cast<float4v*>(smem);
#pragma unroll
  for (int m = 0; m < MF; ++m)
#pragma unroll
    for (int c = 0; c < NF; ++c) sums[((wave * MF + m) * NF + c) * kLanes + lane] = acc[m][c];
  __syncthreads();
  for (int m = wave; m < MF; m += kFewWaves) {
    float v[4 * NF];
#pragma unroll
    for (int c = 0; c < NF; ++c) {
      float4v t = sums[(m * NF + c) * kLanes + lane];
#pragma unroll
      for (int o = 1; o < kFewWaves; ++o) t += sums[((o * MF + m) * NF + c) * kLanes + lane];
      if (a.f.kind == kPartial) {
        const int64_t row_frag = ((int64_t)slice + a.slice0) * a.tiles_m + m;
        a.f.partial[(row_frag * (a.tiles_n * NF) + blockIdx.x * NF + c) * kLanes + lane] = t;
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) v[4 * c + i] = t[i];
    }
    if (a.f.kind == kPartial) continue;
    const int64_t row = m * 16 + sub;
    typedef typename OutOf<F, PL>::type T;
    if constexpr (NF == 4) {
      finish_layer<16, T>(a.f, row, col0 + quad * 16, v, PL);
    } else {
#pragma unroll
      for (int c = 0; c < NF; ++c) {
        float t[4] = {v[4 * c], v[4 * c + 1], v[4 * c + 2], v[4 * c + 3]};
        finish_layer<4, T>(a.f, row, col0 + c * 16 + quad * 4, t, PL);
      }
    }
  }
}

template <class F, int PL, int FMT, int NF>
product_t few_rows_of(int mf) {
  if (mf == 1) return few_rows<F, PL, FMT, 1, NF>;
  if (mf == 2) return few_rows<F, PL, FMT, 2, NF>;
  return few_rows<F, PL, FMT, 4, NF>;
}

}  // namespace lin
}  // namespace squant
