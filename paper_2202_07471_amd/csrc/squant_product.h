// The product of many rows with codes, for a layer (GRAD = false: the contraction runs along a code row) and
// for its gradient (GRAD = true: across the code rows).
//
// A workgroup makes MT x 256 outputs with waves of (MT / 2) x 64 (64 x 64 where MT is 64: halves
// of it that convert the same codes twice took 41 us where it takes 29, 1024 x 4096 x 2048).  The row operand goes to
// the LDS without passing through registers, 64 contraction elements at a time in two buffers; rows of 128 bytes
// with their 16-byte chunks exchanged by the row's low three bits, so that 8 lanes that read the same chunk of
// 8 rows use all banks.  Codes go from memory to the registers of the waves that own their columns and are made
// operands there: they are half or a quarter of the operand's bytes, each wave reads each of its codes once, and
// no LDS traffic is spent on them.  Codes are the matrix instruction's first operand, rows its second, so that a
// lane ends with 16 consecutive columns of one row.
#pragma once

#include "squant_lin.h"

namespace squant {
namespace lin {

template <int MT> struct Shape {
  static constexpr int kWavesM = MT == 64 ? 1 : 2;
  static constexpr int kWaveRows = MT / kWavesM;
  static constexpr int kWaves = kWavesM * (kWide / kTile);
  static constexpr int kThreads = kWaves * kLanes;
  static constexpr int kFrags = kWaveRows / 16;
  // Steps in flight or at work: a step of 256 rows takes longer than memory's latency, one of 64 rows a quarter.
  static constexpr int kDepth = MT == 256 ? 2 : MT == 128 ? 3 : 4;
};

// 16 bytes a lane from memory to LDS bytes [lds, lds + 1024), in lane order.
__device__ __forceinline__ void to_lds(const void* p, void* lds) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)p,
                                   (__attribute__((address_space(3))) void*)lds, 16, 0, 0);
}

// The codes of one step, as loaded.
template <int FMT, bool GRAD, bool WORDS> struct Raw;
template <int FMT, bool WORDS> struct Raw<FMT, false, WORDS> { RowCodes<FMT, WORDS> v[4]; };
template <int FMT, bool WORDS> struct Raw<FMT, true, WORDS> { typename Codes<FMT>::col4 v[16]; };

// WORDS: code rows begin at whole 32-bit words (see RowCodes; a gradient takes them as they are).
template <class F, int PL, int FMT, int MT, bool GRAD, bool WORDS>
__global__ void __launch_bounds__(Shape<MT>::kThreads, 2) product(ProductArgs a) {
  typedef Shape<MT> S;
  constexpr int kPlaneBytes = MT * kBlock * 2;
  constexpr int kBufBytes = kPlaneBytes * PL;
  extern __shared__ __align__(1024) unsigned char smem[];
  const int lane = threadIdx.x & (kLanes - 1);
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kLanes);  // known to be uniform
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
    src[i] = (uint32_t)min(r, last_row) * (uint32_t)(a.lda * 2) + (((lane & 7) ^ (r & 7)) << 4);
  }
  auto load_rows = [&](int b, int buf) {
#pragma unroll
    for (int p = 0; p < PL; ++p)
#pragma unroll
      for (int i = 0; i < kLoads; ++i)
        to_lds(rows + (p * a.plane * 2 + (int64_t)b * (kBlock * 2)) + src[i],
               smem + buf * kBufBytes + p * kPlaneBytes + (wave * kLoads + i) * 1024);
  };

  // Codes.  For a layer each lane reads 16 codes of 4 rows; for a gradient 4 columns of 16 rows, lanes whose columns
  // do not exist those of the row's last bytes.  `inside`: blocks that no read leaves the buffer for.
  const int64_t w_bytes = (int64_t)a.w_rows * a.w_row;
  uint32_t wsrc[GRAD ? 1 : 4];
  const uint8_t* w_base = a.w;
  int inside;
  if constexpr (GRAD) {
    constexpr int n = (int)sizeof(typename Codes<FMT>::col4);
    // a row's last load may pass its end by less than n bytes
    const bool even = a.w_row % n == 0;
    const uint32_t at = (uint32_t)min(Codes<FMT>::offset(col0 + 4 * sub), a.w_row - (even ? n : 1));
    wsrc[0] = (uint32_t)quad * 16 * (uint32_t)a.w_row + at;
    inside = (int)max((w_bytes - (even ? 0 : n - 1)) / (kBlock * a.w_row), (int64_t)0);
  } else {
    w_base += (int64_t)min(col0, a.w_rows - 1) * a.w_row;
#pragma unroll
    for (int c = 0; c < 4; ++c)
      wsrc[c] = (uint32_t)max(min(col0 + (sub >> 2) * 16 + c * 4 + (sub & 3), a.w_rows - 1) - min(col0, a.w_rows - 1), 0) *
                (uint32_t)a.w_row + (uint32_t)Codes<FMT>::offset(quad * 16);
    inside = a.w_cols / kBlock;
    if constexpr (!WORDS) {
      const uint32_t off = (uint32_t)(reinterpret_cast<uintptr_t>(w_base) & 3u);
      w_base -= off;
#pragma unroll
      for (int c = 0; c < 4; ++c) wsrc[c] += off;
    }
  }
  uint32_t shift[4] = {0, 0, 0, 0};
  if constexpr (!GRAD && !WORDS) {
#pragma unroll
    for (int c = 0; c < 4; ++c) shift[c] = wsrc[c] & 3u;
  }
  auto load_codes = [&](int b, Raw<FMT, GRAD, WORDS>& o) {
    if constexpr (GRAD) {
      const uint8_t* p = w_base + (int64_t)b * kBlock * a.w_row;
#pragma unroll
      for (int i = 0; i < 16; ++i) o.v[i] = load_any<typename Codes<FMT>::col4>(p + i * a.w_row + wsrc[0]);
    } else {
      const uint8_t* p = w_base + Codes<FMT>::offset((int64_t)b * kBlock);
#pragma unroll
      for (int c = 0; c < 4; ++c) o.v[c].load(p + (wsrc[c] - shift[c]));
    }
  };
  // the same at the buffer's end
  auto load_last_codes = [&](int b, Raw<FMT, GRAD, WORDS>& o) {
    constexpr int n = GRAD ? 16 : 4;
    const uint8_t* at[n];
#pragma unroll
    for (int i = 0; i < n; ++i)
      at[i] = GRAD ? w_base + ((int64_t)b * kBlock + i) * a.w_row + wsrc[0]
                   : w_base + Codes<FMT>::offset((int64_t)b * kBlock) + wsrc[GRAD ? 0 : i];
    if constexpr (GRAD) {
      load_before(o.v, at, a.w_end, w_bytes);
    } else {
      typename Codes<FMT>::row16 v[4];
      load_before(v, at, a.w_end, w_bytes);
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        o.v[c].set(v[c]);
        shift[c] = 0;  // nothing is read as whole words after this
      }
    }
  };

  float4v acc[S::kFrags][4];
#pragma unroll
  for (int m = 0; m < S::kFrags; ++m)
#pragma unroll
    for (int c = 0; c < 4; ++c) acc[m][c] = float4v{0.0f, 0.0f, 0.0f, 0.0f};

  auto operand = [&](const Raw<FMT, GRAD, WORDS>& r, int h, int c) {
    if constexpr (GRAD) return convert_columns<FMT>(r.v + 8 * h, c);
    else return convert<F, FMT>(r.v[c].aligned(h, shift[c]), h);
  };
  auto row_frag = [&](int buf, int p, int h, int m) {
    return *(const typename F::frag*)(smem + buf * kBufBytes + p * kPlaneBytes + m * 2048 + wave_m * S::kWaveRows * 128 +
                                      sub * 128 + (((quad * 2 + h) ^ (sub & 7)) << 4));
  };
  // A half step is 16 fragments of products a fragment of rows; the next fragment of rows is read, and the next
  // half's codes are converted, between them.
  auto multiply = [&](int buf, const Raw<FMT, GRAD, WORDS>& r) {
    constexpr int kSteps = 2 * PL * S::kFrags;
    typename F::frag w[2][4], x[2];
#pragma unroll
    for (int c = 0; c < 4; ++c) w[0][c] = operand(r, 0, c);
    x[0] = row_frag(buf, 0, 0, 0);
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      const int h = s / (PL * S::kFrags), in = s % (PL * S::kFrags), m = in % S::kFrags;
      if (s + 1 < kSteps) {
        const int n = s + 1, nin = n % (PL * S::kFrags);
        x[n & 1] = row_frag(buf, nin / S::kFrags, n / (PL * S::kFrags), nin % S::kFrags);
      }
      if (h == 0) {
        // the next half's operands, dealt to this half's fragments of rows
#pragma unroll
        for (int c = in * 4 / (PL * S::kFrags); c < (in + 1) * 4 / (PL * S::kFrags); ++c) w[1][c] = operand(r, 1, c);
      }
      __builtin_amdgcn_sched_barrier(0x6);  // what is not arithmetic stays in its fragment
#pragma unroll
      for (int c = 0; c < 4; ++c) acc[m][c] = F::mma(w[h][c], x[s & 1], acc[m][c]);
      __builtin_amdgcn_sched_barrier(0x6);
    }
  };
  // A step's loads are issued kDepth - 1 steps before it, without branches around them, so that what is on its way
  // can be counted: past the last step the last block is loaded again, and not multiplied.  (With a branch around
  // them the compiler waits for everything before it touches a step's codes.)  The barrier also says that the buffer
  // to be loaded next is read out.
  constexpr int D = S::kDepth;
  constexpr int kIssued = kLoads * PL + (GRAD ? 16 : WORDS ? 4 : 8);
  constexpr int kOthers = kIssued * (D - 2);  // may be on their way when a step begins
  static_assert(kOthers < 64, "the wait counter has six bits");
  const int steady = min(last, inside);
  // No load moves over this: the count of one step's is told from the next one's.
  auto in_order = []() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  };
  if (first < steady) {
    Raw<FMT, GRAD, WORDS> raw[D];
#pragma unroll
    for (int i = 0; i < D - 1; ++i) {
      load_rows(min(first + i, steady - 1), i);
      load_codes(min(first + i, steady - 1), raw[i]);
      in_order();
    }
#pragma unroll 1
    for (int b0 = first; b0 < steady; b0 += D) {
#pragma unroll
      for (int i = 0; i < D; ++i) {
        // not __syncthreads(), which would wait for every load
        in_order();
        __builtin_amdgcn_s_waitcnt((kOthers & 15) | (kOthers >> 4) << 14 | 0x070);
        __builtin_amdgcn_s_barrier();
        in_order();
        const int ahead = min(b0 + i + D - 1, steady - 1);
        load_rows(ahead, (i + D - 1) % D);
        load_codes(ahead, raw[(i + D - 1) % D]);
        if (b0 + i < steady) multiply(i, raw[i]);
      }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
  }
  for (int b = max(first, steady); b < last; ++b) {  // what ends within a block
    Raw<FMT, GRAD, WORDS> raw;
    load_rows(b, 0);
    load_last_codes(b, raw);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    multiply(0, raw);
    __syncthreads();
  }

  if (a.f.kind == kPartial) {
    const int64_t frags_n = (int64_t)a.tiles_n * (kWide / 16);
#pragma unroll
    for (int m = 0; m < S::kFrags; ++m) {
      const int64_t row_frag = (int64_t)slice * a.tiles_m * (MT / 16) + tile_m * (MT / 16) + wave_m * S::kFrags + m;
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
  // The columns' scales and biases wait in the LDS, where they cost no registers beside the sums.
  float* shared_columns = reinterpret_cast<float*>(smem);  // [2][kWide]
  if constexpr (!GRAD) {
    __syncthreads();
    if (threadIdx.x < kWide) {
      Columns<1> one;
      load_columns<1, T>(one, a.f, tile_n * kWide + (int)threadIdx.x);
      shared_columns[threadIdx.x] = one.scale[0];
      shared_columns[kWide + threadIdx.x] = one.bias[0];
    }
    __syncthreads();
  }
#pragma unroll 1
  for (int m = 0; m < S::kFrags; ++m) {
    float4v t[4];
#pragma unroll
    for (int j = 0; j < S::kFrags; ++j)
      if (m == j) {
#pragma unroll
        for (int c = 0; c < 4; ++c) t[c] = acc[j][c];
      }
    float v[16];
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i) v[column_of<GRAD>(c, i)] = t[c][i];
    const int64_t row = row0 + wave_m * S::kWaveRows + m * 16 + sub;
    if constexpr (GRAD) {
      finish_grad(a.f, row, col0 + quad * 16, v);
    } else {
      Columns<16> columns;
      asm volatile("" ::: "memory");  // read again for each fragment
#pragma unroll
      for (int i = 0; i < 16; ++i) columns.scale[i] = shared_columns[wave_n * kTile + quad * 16 + i];
#pragma unroll
      for (int i = 0; i < 16; ++i) columns.bias[i] = shared_columns[kWide + wave_n * kTile + quad * 16 + i];
      finish_layer<16, T>(a.f, columns, row, col0 + quad * 16, v, row_factor_of(a.f, row), PL);
    }
  }
}

template <class F, int PL, int FMT, bool GRAD, bool WORDS>
product_t product_of(int mt) {
  if (mt == 256) return product<F, PL, FMT, 256, GRAD, WORDS>;
  if (mt == 128) return product<F, PL, FMT, 128, GRAD, WORDS>;
  return product<F, PL, FMT, 64, GRAD, WORDS>;
}
template <class F, int PL, int FMT>
product_t layer_of(int mt, bool words) {
  return words ? product_of<F, PL, FMT, false, true>(mt) : product_of<F, PL, FMT, false, false>(mt);
}

}  // namespace lin
}  // namespace squant
