// What goes before and after the products with codes: row operands laid out, gradients of the activation, partial
// sums joined, the loss from its chunks.
#pragma once

#include "squant_lin.h"

namespace squant {
namespace lin {

constexpr int kRowThreads = 256;
constexpr int kRowGroup = 16;  // most rows a workgroup of gradient_rows takes

// Code rows copied to rows of whole steps at multiples of 16 bytes, zeros at their ends: by the workgroups of a launch
// past `first_block`, so that it costs no launch where there are rows to lay out as well.
struct CodesArgs {
  const uint8_t* codes;
  int64_t row;              // bytes
  uint8_t* out;
  int32_t out_row;          // bytes
  int64_t chunks;           // 16 bytes of `out` each; 0: nothing to lay out
  int64_t first_block;
};

struct RowsArgs {
  CodesArgs w;
  const void* x;            // rows, or the output's gradient
  int64_t ldx;
  int64_t rows;
  int32_t cols;
  void* out;                // [rows][planes][padded]
  int32_t padded;           // cols up to a multiple of 64
  float* row_factor;
  // gradient rows only
  const float* scales;
  const void* kept;
  const float* kept_scales;
  int act, keep;
  int rows_per_group;
  float* column_sums;       // [partials][cols], or null
};

__device__ __forceinline__ uint32_t finite_magnitude(float v) {
  const uint32_t m = magnitude(v);
  return m < 0x7f800000u ? m : 0u;
}

__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
#pragma unroll
  for (int o = 1; o < kLanes; o <<= 1) v = max(v, (uint32_t)__shfl_xor((int)v, o));
  return v;
}

// hi + lo of 8 values, written to one or two planes.
template <int PL>
__device__ __forceinline__ void store_planes(_Float16* p, int64_t plane, const float (&v)[8]) {
  half8 hi, lo;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    hi[i] = (_Float16)v[i];
    // an infinity has no remainder
    lo[i] = magnitude(v[i]) < 0x7f800000u ? (_Float16)(v[i] - (float)hi[i]) : (_Float16)0.0f;
  }
  *(half8*)p = hi;
  if (PL == 2) *(half8*)(p + plane) = lo;
}

__device__ __forceinline__ void lay_codes(const CodesArgs& w, int64_t block) {
  const int64_t at = block * kRowThreads + threadIdx.x;
  if (at >= w.chunks) return;
  const int32_t per = w.out_row / 16;
  int64_t row;
  if (w.chunks <= 0xffffffffLL) row = (uint32_t)at / (uint32_t)per;  // a third of the instructions of 64 bits
  else row = at / per;
  const int32_t c = (int32_t)(at - row * per) * 16;
  const uint8_t* p = w.codes + row * w.row + c;
  uint4v o = {0, 0, 0, 0};
  if (c + 16 <= w.row) {
    // the words that hold the bytes: the last one is read only if it holds some
    const uint32_t off = (uint32_t)(reinterpret_cast<uintptr_t>(p) & 3u);
    const uint32_t* words = reinterpret_cast<const uint32_t*>(p - off);
    uint32_t v[5];
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = words[i];
    v[4] = off ? words[4] : 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = __builtin_amdgcn_alignbyte(v[i + 1], v[i], off);
  } else {
    if (c < w.row) {
      uint32_t v[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) v[i] = p[c + i < w.row ? i : 0];
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (c + i < w.row) o[i >> 2] |= v[i] << (8 * (i & 3));
    }
  }
  *(uint4v*)(w.out + at * 16) = o;
}

// 16-bit rows copied to where they are aligned and end with zeros.  Any 16-bit type.
__global__ void __launch_bounds__(kRowThreads) pad_rows(RowsArgs a);
// binary32 rows to two planes, a workgroup a row.
__global__ void __launch_bounds__(kRowThreads) split_rows(RowsArgs a);

// Rows of dz * scale, dz = dy * act'(z), as PL binary16 planes with an exponent a row, and the column sums of dz.
// The exponent comes from the largest |dy * scale| (the slopes stay below 1.13), so that it costs no second
// evaluation of the slope: dy is read twice, the second time from the cache.  A workgroup takes a few rows; where
// they have few columns its threads share out the rows as well, and where there are few rows several workgroups
// share out their columns.
template <class T, int PL>
__global__ void __launch_bounds__(kRowThreads) gradient_rows(RowsArgs a) {
  __shared__ uint32_t tops[kRowGroup];
  if (a.w.chunks && blockIdx.x >= a.w.first_block) return lay_codes(a.w, (blockIdx.x - a.w.first_block) * gridDim.y + blockIdx.y);
  const int lane = threadIdx.x & (kLanes - 1);
  const int64_t row0 = (int64_t)blockIdx.x * a.rows_per_group;
  const int n_rows = (int)min((int64_t)a.rows_per_group, a.rows - row0);
  if (threadIdx.x < kRowGroup) tops[threadIdx.x] = 0;
  __syncthreads();
  for (int r = 0; r < n_rows; ++r) {
    const T* dy = (const T*)a.x + (row0 + r) * a.ldx;
    uint32_t top = 0;
#pragma unroll 2
    for (int32_t c = threadIdx.x * 8; c < a.cols; c += kRowThreads * 8) {
      float v[8], s[8];
      load_cols<8, T>(v, dy + c, a.cols - c);
      load_cols<8, float>(s, a.scales + c, a.cols - c);
#pragma unroll
      for (int i = 0; i < 8; ++i) top = max(top, finite_magnitude(v[i] * s[i]));
    }
    top = wave_max(top);
    if (lane == 0) atomicMax(&tops[r], top);  // in the LDS; a maximum does not depend on the order
  }
  __syncthreads();
  if (blockIdx.y == 0 && (int)threadIdx.x < n_rows) a.row_factor[row0 + threadIdx.x] = power_of_two(1 - row_exponent(tops[threadIdx.x]));
  const int vectors = a.padded / 8;
  const int shares = max(1, kRowThreads / vectors), share = shares > 1 ? (int)threadIdx.x / vectors : 0;
  if (share >= shares) return;
  const int32_t chunks = (a.cols + kTile - 1) / kTile;
  // with one share the columns are dealt to the workgroups of these rows as well
  for (int j = shares > 1 ? (int)threadIdx.x % vectors : (int)(blockIdx.y * kRowThreads + threadIdx.x); j < vectors;
       j += (int)gridDim.y * kRowThreads) {
    const int32_t c = j * 8;
    const int valid = min(max(a.cols - c, 0), 8);
    float s[8], sum[8];
    load_cols<8, float>(s, a.scales + c, valid);
#pragma unroll
    for (int i = 0; i < 8; ++i) sum[i] = 0.0f;
#pragma unroll 4
    for (int r = share; r < n_rows; r += shares) {
      const int64_t row = row0 + r;
      const float up = power_of_two(row_exponent(tops[r]) - 1);  // room for slopes beyond 1
      float v[8];
      load_cols<8, T>(v, (const T*)a.x + row * a.ldx + c, valid);
      if (a.keep == SQUANT_KEEP_FULL) {
        float z[8];
        load_cols<8, T>(z, (const T*)a.kept + row * a.cols + c, valid);
        apply_slope<T, 8>(v, z, a.act);
      } else if (a.keep == SQUANT_KEEP_INT8) {
        float z[8];
        const float unit = valid ? a.kept_scales[row * chunks + c / kTile] : 0.0f;
        load_cols<8, int8_t>(z, (const int8_t*)a.kept + row * a.cols + c, valid);
#pragma unroll
        for (int i = 0; i < 8; ++i) z[i] *= unit;
        apply_slope<T, 8>(v, z, a.act);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        v[i] = i < valid ? v[i] : 0.0f;
        sum[i] += v[i];
        v[i] = v[i] * s[i] * up;
      }
      store_planes<PL>((_Float16*)a.out + row * PL * a.padded + c, a.padded, v);
    }
    if (a.column_sums) {
      float* out = a.column_sums + ((int64_t)blockIdx.x * shares + share) * a.cols + c;
      store_cols<8, float>(out, sum, valid);
    }
  }
}

struct ColumnSumArgs {
  const float* partial;
  int64_t partials;
  int32_t cols;
  void* out;
  int out_type;
};
__global__ void __launch_bounds__(1024) column_sums(ColumnSumArgs a);

struct JoinArgs {
  const float4v* partial;
  int slices;
  int64_t row_frags, col_frags;
  Finish f;
};
// Adds the slices of a split product in their order: one wave a fragment of 16 rows and 64 columns.
template <bool GRAD, class T>
__global__ void __launch_bounds__(kRowThreads) join(JoinArgs a) {
  const int lane = threadIdx.x & (kLanes - 1);
  const int64_t at = (int64_t)blockIdx.x * (kRowThreads / kLanes) + threadIdx.x / kLanes;
  const int64_t tiles = a.col_frags / 4;
  if (at >= a.row_frags * tiles) return;
  const int64_t rf = at / tiles, tile = at % tiles;
  float4v t[4];
#pragma unroll
  for (int c = 0; c < 4; ++c) t[c] = float4v{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
  for (int s = 0; s < a.slices; ++s) {
    const float4v* p = a.partial + ((s * a.row_frags + rf) * a.col_frags + tile * 4) * kLanes + lane;
#pragma unroll
    for (int c = 0; c < 4; ++c) t[c] += p[c * kLanes];
  }
  float v[16];
#pragma unroll
  for (int c = 0; c < 4; ++c)
#pragma unroll
    for (int i = 0; i < 4; ++i) v[column_of<GRAD>(c, i)] = t[c][i];
  const int64_t row = rf * 16 + (lane & 15);
  const int32_t col = (int32_t)tile * kTile + (lane >> 4) * 16;
  const RowValues shared = row_values(a.f, row);
  if constexpr (GRAD) {
    float factor = shared.factor;
    if (a.f.kind == kGradLoss) {
      const int64_t at = min(row, a.f.rows - 1);
      const float label = a.f.label_prob[at];
      factor = 1.0f - label;
      if (__any(label > 0.5f)) {
        float others = 0.0f;
#pragma unroll 8
        for (int32_t i = lane >> 4; i < a.f.other_tiles; i += 4) others += a.f.other_sums[i * a.f.rows + at];
        others += __shfl_xor(others, 16);
        others += __shfl_xor(others, 32);
        factor = label > 0.5f ? others : factor;
      }
    }
    finish_grad(a.f, row, col, v, factor);
  } else {
    Columns<16> columns;
    load_columns<16, T>(columns, a.f, col);
    finish_layer<16, T>(a.f, columns, row, col, v, shared);
  }
}

struct LossArgs {
  const float2* stats;
  int32_t chunks;
  const float* label_logit;  // base 2
  const int64_t* labels;
  int64_t ignore;
  int32_t vocabulary;
  int64_t rows;
  float* loss;
  float* lse;
};
// A workgroup a row: the chunks' sums brought to one largest logit.
__global__ void __launch_bounds__(kRowThreads) loss_rows(LossArgs a);

// 2^E of the gradient's probabilities: the largest scale of the vocabulary comes into [2^13, 2^14).
__global__ void __launch_bounds__(1024) probability_unit(const float* scales, int32_t n, float* unit);

typedef void (*rows_kernel_t)(RowsArgs);
typedef void (*join_kernel_t)(JoinArgs);

}  // namespace lin
}  // namespace squant
