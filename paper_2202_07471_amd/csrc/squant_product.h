// The product of many rows with codes, for a layer and for the logits of the loss's gradient (the contraction runs along a
// code row) and for gradients (it runs across the code rows).
//
// A workgroup makes MT x 256 outputs with waves of (MT / 2) x 64 (64 x 64 where MT is 64: halves of it that convert
// the same codes twice took 41 us where it takes 29, 1024 x 4096 x 2048).  Rows and codes go to the LDS without passing
// through registers, 64 contraction elements at a time; the 16-byte chunks of what lies there in one row are exchanged so
// that lanes that read at once use more banks.  Waves read the codes of their 64 columns and make them operands in
// registers.  Codes that do not lie in whole steps at multiples of 16 bytes are laid out so before (lay_codes): read as
// they were they cost twice the time (777 x 2049 x 2559 45 us, 777 x 2048 x 2560 23 us).  Codes are the matrix
// instruction's first operand, rows its second, so that a lane ends with 16 consecutive columns of one row.
//
// Bound by no unit alone: of 280 K cycles of 4096 x 4096 x 4096 (bfloat16, int8 codes, 256 rows; 133 us under the counters, at 2.1 GHz) the
// matrix units are busy 131 K, vector instructions issue in 96 K, the LDS reads in 84 K, 41 K of them bank conflicts, and waves wait
// for 35 % of their 247 K.  A step of 64 of a 256 x 256 tile takes 1.62 us on all compute units, 1.33 PFLOP/s; a round's start and end
// overlap with nothing (4096 x 4096 x 4096 113 us, 10 of them; 4096 x 4096 x 8192 with gelu and residual 254 us, 23 in each of two rounds).
#pragma once

#include "squant_lin.h"

namespace squant {
namespace lin {

template <int MT> struct Shape {
  static constexpr int kWavesM = MT == 64 ? 1 : 2;
  static constexpr int kWaveRows = MT / kWavesM;
  // Groups of waves that take every other step of the contraction, each with row buffers of its own; their sums meet
  // in the LDS at the end.  A tile of 64 rows has work for 4 waves, one a SIMD, that wait for each other's latencies.
  static constexpr int kGroups = MT == 64 ? 2 : 1;
  static constexpr int kWaves = kWavesM * (kWide / kTile);  // of a group
  static constexpr int kThreads = kGroups * kWaves * kLanes;
  static constexpr int kFrags = kWaveRows / 16;
  static constexpr int kOwn = kFrags / kGroups;  // fragments of rows that a wave finishes
};

constexpr int kLdsBytes = 160 * 1024;
// LDS of one step: the rows' planes, then the codes.
constexpr int step_codes(int format) { return format == SQUANT_OUT_INT4 ? kWide * kBlock / 2 : kWide * kBlock; }
constexpr int step_bytes(int mt, int planes, int format) { return mt * kBlock * 2 * planes + step_codes(format); }
constexpr int row_groups(int mt) { return mt == 64 ? Shape<64>::kGroups : 1; }
// Steps in flight or at work: a step of 256 rows takes longer than memory's latency, one of 64 rows a quarter.
constexpr int product_depth(int mt, int planes, int format) {
  const int wanted = mt == 64 ? 4 : mt == 128 ? 3 : 2;
  const int each = step_bytes(mt, planes, format) * row_groups(mt);
  return wanted * each <= kLdsBytes ? wanted : kLdsBytes / each;
}
constexpr int product_lds(int mt, int planes, int format) {
  return product_depth(mt, planes, format) * step_bytes(mt, planes, format) * row_groups(mt);
}

// 16 bytes a lane from memory to LDS bytes [lds, lds + 1024), in lane order.
__device__ __forceinline__ void to_lds(const void* p, void* lds) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)p,
                                   (__attribute__((address_space(3))) void*)lds, 16, 0, 0);
}

// What a product is for.  The loss gradient's logits have kernels of their own: with their epilogue beside the layer's the
// latter spills registers (256 rows: 6 registers, 15 with the sums of the probabilities; 4096 x 4096 x 8192 with gelu and
// residual 258 us, 268 us).
enum Role { kLayer, kProbabilities, kGradient };

// A wave's codes of one step: 16 of each of its lanes' 4 columns (layer), or 4 columns of 16 rows (gradient).
template <int FMT, bool GRAD> struct Raw { typename Codes<FMT>::row16 v[4]; };
template <int FMT> struct Raw<FMT, true> { typename Codes<FMT>::col4 v[16]; };

template <class F, int PL, int FMT, int MT, Role ROLE>
__global__ void __launch_bounds__(Shape<MT>::kThreads, 2) product(ProductArgs a) {
  typedef Shape<MT> S;
  constexpr bool GRAD = ROLE == kGradient;
  constexpr bool kInt8 = FMT == SQUANT_OUT_INT8;
  constexpr int D = product_depth(MT, PL, FMT);
  constexpr int kPlaneBytes = MT * kBlock * 2;
  constexpr int kBufBytes = step_bytes(MT, PL, FMT);
  extern __shared__ __align__(1024) unsigned char smem[];
  const int lane = threadIdx.x & (kLanes - 1);
  const int wave_of_all = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kLanes);  // known to be uniform
  const int group = wave_of_all / S::kWaves, wave = wave_of_all % S::kWaves;
  unsigned char* buffers = smem + group * (kBufBytes * D);
  const int wave_m = wave % S::kWavesM, wave_n = wave / S::kWavesM;

  // Each XCD takes a run of consecutive tiles; within it, bands of 8 tiles of rows run along the columns, so that
  // what an XCD's cache holds of rows and of codes is used by several workgroups.
  const int tiles = a.tiles_m * a.tiles_n;
  int tile = blockIdx.x;
  {
    const int per = tiles / 8, rest = tiles % 8, x = tile % 8;
    tile = x * per + min(x, rest) + tile / 8;
  }
  const int band = tile / (8 * a.tiles_n);
  const int band_rows = min(8, a.tiles_m - band * 8);
  const int in_band = tile - band * 8 * a.tiles_n;
  const int tile_m = band * 8 + in_band % band_rows, tile_n = in_band / band_rows;
  const int slice = blockIdx.y;
  const int first = (int)((int64_t)a.blocks * slice / a.slices), last = (int)((int64_t)a.blocks * (slice + 1) / a.slices);

  const int64_t row0 = (int64_t)tile_m * MT;
  const int32_t col0 = tile_n * kWide + wave_n * kTile;
  const int sub = lane & 15, quad = lane >> 4;

  // row operand: 8 rows an instruction; a row past the end is the last one again
  constexpr int kLoads = MT / 8 / S::kWaves;
  uint32_t src[kLoads];  // bytes from the tile's first row: kMaxSide keeps them in 32 bits
  const char* rows = (const char*)a.a + row0 * a.lda * 2;
  const int last_row = (int)min((int64_t)MT, a.f.rows - row0) - 1;
#pragma unroll
  for (int i = 0; i < kLoads; ++i) {
    const int r = (wave * kLoads + i) * 8 + (lane >> 3);
    src[i] = (uint32_t)min(r, last_row) * (uint32_t)(a.lda * 2) + (((lane & 7) ^ ((r >> 1) & 7)) << 4);
  }
  auto load_rows = [&](int b, int buf) {
#pragma unroll
    for (int p = 0; p < PL; ++p)
#pragma unroll
      for (int i = 0; i < kLoads; ++i)
        to_lds(rows + (p * a.plane * 2 + (int64_t)b * (kBlock * 2)) + src[i],
               buffers + buf * kBufBytes + p * kPlaneBytes + (wave * kLoads + i) * 1024);
  };

  // Codes: 64 of each column in turn (layer), columns in the order in which a lane group reads them as operands, or 256
  // columns of each row in turn (gradient).  A column or row past the end is the last one again: the columns are not
  // stored, the rows' operands are zero.
  constexpr int kCodeLoads = step_codes(FMT) / 1024 / S::kWaves;
  constexpr int kCodeRow = (GRAD ? kWide : kBlock) / (kInt8 ? 1 : 2);  // bytes of a column or row of a step
  const int32_t tile_col = tile_n * kWide;
  const uint8_t* codes = a.w + (GRAD ? 0 : (int64_t)tile_col * a.w_row);
  uint32_t csrc[kCodeLoads];
  int crow[GRAD ? kCodeLoads : 1];
#pragma unroll
  for (int i = 0; i < kCodeLoads; ++i) {
    const int place = ((wave * kCodeLoads + i) * 1024 + lane * 16) / kCodeRow, chunk = lane & (kCodeRow / 16 - 1);
    if constexpr (GRAD) {
      crow[i] = place;
      const int32_t at = (int32_t)Codes<FMT>::offset(tile_col) + (chunk ^ (place >> 4) * (kCodeRow / 64)) * 16;
      csrc[i] = (uint32_t)min(at, (int32_t)a.w_row - 16);
    } else {
      const int sub16 = place & 15;
      const int32_t col = (place >> 6) * 64 + (sub16 >> 2) * 16 + ((place >> 4) & 3) * 4 + (sub16 & 3);
      csrc[i] = (uint32_t)min(col, a.w_rows - 1 - tile_col) * (uint32_t)a.w_row + (uint32_t)(chunk ^ (sub16 >> (kInt8 ? 2 : 3))) * 16;
    }
  }
  auto load_codes = [&](int b, int buf) {
    const uint8_t* p = codes + (GRAD ? (int64_t)b * kBlock * a.w_row : Codes<FMT>::offset((int64_t)b * kBlock));
    const int last_code_row = a.w_rows - 1 - b * kBlock;
#pragma unroll
    for (int i = 0; i < kCodeLoads; ++i) {
      uint32_t at = csrc[i];
      if constexpr (GRAD) at += (uint32_t)min(crow[i], last_code_row) * (uint32_t)a.w_row;
      to_lds(p + at, buffers + buf * kBufBytes + PL * kPlaneBytes + (wave * kCodeLoads + i) * 1024);
    }
  };
  auto read_codes = [&](int buf, Raw<FMT, GRAD>& o) {
    const unsigned char* p = buffers + buf * kBufBytes + PL * kPlaneBytes;
    if constexpr (GRAD) {
      typedef typename Codes<FMT>::col4 col4;
      p += quad * 16 * kCodeRow + ((wave_n ^ quad) * 16 + sub) * (int)sizeof(col4);
#pragma unroll
      for (int i = 0; i < 16; ++i) o.v[i] = *(const col4*)(p + i * kCodeRow);
    } else {
      p += (wave_n * 64 + sub) * kCodeRow + (kInt8 ? (quad ^ (sub >> 2)) * 16 : ((quad >> 1) ^ (sub >> 3)) * 16 + (quad & 1) * 8);
#pragma unroll
      for (int c = 0; c < 4; ++c) o.v[c] = *(const typename Codes<FMT>::row16*)(p + c * 16 * kCodeRow);
    }
  };

  float4v acc[S::kFrags][4];
#pragma unroll
  for (int m = 0; m < S::kFrags; ++m)
#pragma unroll
    for (int c = 0; c < 4; ++c) acc[m][c] = float4v{0.0f, 0.0f, 0.0f, 0.0f};

  auto operand = [&](const Raw<FMT, GRAD>& r, int h, int c) {
    if constexpr (GRAD) return convert_columns<FMT>(r.v + 8 * h, c);
    else return convert<F, FMT>(r.v[c], h);
  };
  auto row_frag = [&](int buf, int p, int h, int m) {
    return *(const typename F::frag*)(buffers + buf * kBufBytes + p * kPlaneBytes + m * 2048 + wave_m * S::kWaveRows * 128 +
                                      sub * 128 + (((quad * 2 + h) ^ (sub >> 1)) << 4));
  };
  // A half step is 16 fragments of products a fragment of rows; the next fragment of rows is read, and the next
  // half's codes are converted, between them.
  auto multiply = [&](int buf) {
    constexpr int kHalf = PL * S::kFrags, kSteps = 2 * kHalf;
    Raw<FMT, GRAD> r;
    read_codes(buf, r);
    typename F::frag w[2][4], x[2];
#pragma unroll
    for (int c = 0; c < 4; ++c) w[0][c] = operand(r, 0, c);
    x[0] = row_frag(buf, 0, 0, 0);
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      const int h = s / kHalf, in = s % kHalf, m = in % S::kFrags;
      if (s + 1 < kSteps) {
        const int n = s + 1, nin = n % kHalf;
        x[n & 1] = row_frag(buf, nin / S::kFrags, n / kHalf, nin % S::kFrags);
      }
      if (h == 0) {
        // the next half's operands, dealt to this half's fragments of rows
#pragma unroll
        for (int c = in * 4 / kHalf; c < (in + 1) * 4 / kHalf; ++c) w[1][c] = operand(r, 1, c);
      }
      __builtin_amdgcn_sched_barrier(0x6);  // what is not arithmetic stays in its fragment
#pragma unroll
      for (int c = 0; c < 4; ++c) acc[m][c] = F::mma(w[h][c], x[s & 1], acc[m][c]);
      __builtin_amdgcn_sched_barrier(0x6);
    }
  };
  // A step's loads are issued D - 1 steps before it, without branches around them, so that what is on its way can be
  // counted: past the last step the last block is loaded again, and not multiplied.  The barrier also says that the
  // buffer to be loaded next is read out.
  constexpr int kOthers = (kLoads * PL + kCodeLoads) * (D - 2);  // may be on their way when a step begins
  static_assert(D >= 2 && kOthers < 64, "the wait counter has six bits");
  // No load moves over this: the count of one step's is told from the next one's.
  auto in_order = []() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  };
  if (first < last) {  // a short last piece of the vocabulary may leave a slice without a step
#pragma unroll
    for (int i = 0; i < D - 1; ++i) {
      const int b = min(first + i * S::kGroups + group, last - 1);
      load_rows(b, i);
      load_codes(b, i);
      in_order();
    }
#pragma unroll 1
    for (int b0 = first; b0 < last; b0 += D * S::kGroups) {
#pragma unroll
      for (int i = 0; i < D; ++i) {
        // not __syncthreads(), which would wait for every load
        in_order();
        __builtin_amdgcn_s_waitcnt((kOthers & 15) | (kOthers >> 4) << 14 | 0x070);
        __builtin_amdgcn_s_barrier();
        in_order();
        const int b = b0 + i * S::kGroups + group, ahead = min(b + (D - 1) * S::kGroups, last - 1);
        load_rows(ahead, (i + D - 1) % D);
        load_codes(ahead, (i + D - 1) % D);
        if (b < last) multiply(i);
      }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
  }
  if constexpr (S::kGroups == 2) {
    // each group hands half of its fragments to the other and keeps the sums of the other half
    float4v* given = reinterpret_cast<float4v*>(smem) + wave * (S::kOwn * 4 * kLanes) + lane;
    constexpr int kGiven = S::kWaves * S::kOwn * 4 * kLanes;  // of a group
#pragma unroll
    for (int m = 0; m < S::kOwn; ++m)
#pragma unroll
      for (int c = 0; c < 4; ++c) given[group * kGiven + (m * 4 + c) * kLanes] = acc[group == 0 ? m + S::kOwn : m][c];
    __syncthreads();
#pragma unroll
    for (int m = 0; m < S::kOwn; ++m)
#pragma unroll
      for (int c = 0; c < 4; ++c) acc[m][c] = acc[group == 0 ? m : m + S::kOwn][c] + given[(1 - group) * kGiven + (m * 4 + c) * kLanes];
  }
  const int first_frag = wave_m * S::kFrags + group * S::kOwn;  // of those that this wave finishes, in the tile

  if (ROLE != kProbabilities && a.f.kind == kPartial) {
    const int64_t frags_n = (int64_t)a.tiles_n * (kWide / 16);
#pragma unroll
    for (int m = 0; m < S::kOwn; ++m) {
      const int64_t row_frag = (int64_t)slice * a.tiles_m * (MT / 16) + tile_m * (MT / 16) + first_frag + m;
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        float4v* p = a.f.partial + (row_frag * frags_n + (col0 / 16 + c)) * kLanes + lane;
        if (a.accumulate) acc[m][c] += *p;
        *p = acc[m][c];
      }
    }
    return;
  }
  // One copy of the epilogue's code: the fragment is picked by uniform branches, so that every register is
  // named (unrolled eight times it is larger than the instruction cache, indexed it sends the sums to scratch memory).
  typedef typename OutOf<F, PL>::type T;
  // What columns and rows share waits in the LDS, where it costs no registers beside the sums and no trip to memory
  // for each fragment.
  float* shared_columns = reinterpret_cast<float*>(smem);              // [2][kWide]
  float* shared_sums = shared_columns + 2 * kWide;                      // [kWide / kTile][MT], kProb
  RowValues* shared_rows = reinterpret_cast<RowValues*>(shared_sums + kWide / kTile * MT);  // [MT]
  __syncthreads();
  if (threadIdx.x < kWide) {
    if constexpr (!GRAD) {
      Columns<1> one;
      load_columns<1, T>(one, a.f, tile_n * kWide + (int)threadIdx.x);
      shared_columns[threadIdx.x] = one.scale[0];
      shared_columns[kWide + threadIdx.x] = one.bias[0];
    }
    if (threadIdx.x < MT) shared_rows[threadIdx.x] = row_values(a.f, row0 + threadIdx.x);
  }
  const float prob_unit = ROLE == kProbabilities ? *a.f.prob_unit : 1.0f;
  const int32_t out_col = col0 + quad * 16;
  __syncthreads();
#pragma unroll 1
  for (int m = 0; m < S::kOwn; ++m) {
    float4v t[4];
#pragma unroll
    for (int j = 0; j < S::kOwn; ++j)
      if (m == j) {
#pragma unroll
        for (int c = 0; c < 4; ++c) t[c] = acc[j][c];
      }
    float v[16];
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i) v[column_of<GRAD>(c, i)] = t[c][i];
    const int in_tile = (first_frag + m) * 16 + sub;
    const int64_t row = row0 + in_tile;
    if constexpr (GRAD) {
      finish_grad(a.f, row, out_col, v, shared_rows[in_tile].factor);
    } else {
      Columns<16> columns;
      asm volatile("" ::: "memory");  // read again for each fragment
#pragma unroll
      for (int i = 0; i < 16; ++i) columns.scale[i] = shared_columns[wave_n * kTile + quad * 16 + i];
#pragma unroll
      for (int i = 0; i < 16; ++i) columns.bias[i] = shared_columns[kWide + wave_n * kTile + quad * 16 + i];
      if constexpr (ROLE == kProbabilities) {
        const float sum = finish_prob<PL>(a.f, columns, row, out_col, v, shared_rows[in_tile], prob_unit);
        if (quad == 0) shared_sums[wave_n * MT + in_tile] = sum;
      } else {
        finish_layer<16, T>(a.f, columns, row, out_col, v, shared_rows[in_tile]);
      }
    }
  }
  if constexpr (ROLE == kProbabilities) {
    __syncthreads();
    if (threadIdx.x >= MT) return;
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < kWide / kTile; ++i) sum += shared_sums[i * MT + threadIdx.x];
    store_others(a.f, row0 + threadIdx.x, tile_n, sum, a.accumulate);
  }
}

template <class F, int PL, int FMT, Role ROLE>
product_t product_of(int mt) {
  if (mt == 256) return product<F, PL, FMT, 256, ROLE>;
  if (mt == 128) return product<F, PL, FMT, 128, ROLE>;
  return product<F, PL, FMT, 64, ROLE>;
}

}  // namespace lin
}  // namespace squant
