// The kernels around the products with codes.
#include "squant_lin_kernels.h"

namespace squant {
namespace lin {

__global__ void __launch_bounds__(kRowThreads) pad_rows(RowsArgs a) {
  if (a.w.chunks && blockIdx.x >= a.w.first_block) return lay_codes(a.w, blockIdx.x - a.w.first_block);
  const int64_t vectors = a.padded / 8;
  const int64_t at = (int64_t)blockIdx.x * kRowThreads + threadIdx.x;
  if (at >= a.rows * vectors) return;
  const int64_t row = at / vectors;
  const int32_t c = (int32_t)(at % vectors) * 8;
  const uint16_t* x = (const uint16_t*)a.x + row * a.ldx + c;
  uint4v o = {0, 0, 0, 0};
  if (c + 8 <= a.cols) {
    o = load_any<uint4v>(x);
  } else if (c < a.cols) {
    uint32_t v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = x[c + i < a.cols ? i : 0];
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c + i < a.cols) o[i >> 1] |= v[i] << (16 * (i & 1));
  }
  *(uint4v*)((uint16_t*)a.out + row * a.padded + c) = o;
}

__global__ void __launch_bounds__(kRowThreads) split_rows(RowsArgs a) {
  constexpr int kHeld = 4;  // vectors of 8 elements a thread keeps: rows up to 8192 are read once
  __shared__ uint32_t tops[kRowThreads / kLanes];
  if (a.w.chunks && blockIdx.x >= a.w.first_block) return lay_codes(a.w, blockIdx.x - a.w.first_block);
  const int64_t row = blockIdx.x;
  const float* x = (const float*)a.x + row * a.ldx;
  float v[kHeld][8];
  uint32_t top = 0;
  for (int32_t c0 = 0; c0 < a.padded; c0 += kHeld * kRowThreads * 8) {
#pragma unroll
    for (int j = 0; j < kHeld; ++j) {
      const int32_t c = c0 + (j * kRowThreads + (int)threadIdx.x) * 8;
      load_cols<8, float>(v[j], x + c, max(a.cols - c, 0));
    }
#pragma unroll
    for (int j = 0; j < kHeld; ++j)
#pragma unroll
      for (int i = 0; i < 8; ++i) top = max(top, finite_magnitude(v[j][i]));
  }
  top = wave_max(top);
  if ((threadIdx.x & (kLanes - 1)) == 0) tops[threadIdx.x / kLanes] = top;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kRowThreads / kLanes; ++i) top = max(top, tops[i]);
  const int e = row_exponent(top);
  const float up = power_of_two(e);
  if (threadIdx.x == 0) a.row_factor[row] = power_of_two(-e);
  _Float16* out = (_Float16*)a.out + row * 2 * a.padded;
  const bool held = a.padded <= kHeld * kRowThreads * 8;
  for (int32_t c0 = 0; c0 < a.padded; c0 += kHeld * kRowThreads * 8) {
#pragma unroll
    for (int j = 0; j < kHeld; ++j) {
      const int32_t c = c0 + (j * kRowThreads + (int)threadIdx.x) * 8;
      if (c >= a.padded) break;
      if (!held) load_cols<8, float>(v[j], x + c, max(a.cols - c, 0));
#pragma unroll
      for (int i = 0; i < 8; ++i) v[j][i] *= up;
      store_planes<2>(out + c, a.padded, v[j]);
    }
  }
}

__global__ void __launch_bounds__(1024) column_sums(ColumnSumArgs a) {
  __shared__ float part[16][kLanes];
  const int lane = threadIdx.x & (kLanes - 1), group = threadIdx.x / kLanes;
  const int32_t c = (int32_t)blockIdx.x * kLanes + lane;
  float s = 0.0f;
  if (c < a.cols) {
    int64_t p = group;
    for (; p + 7 * 16 < a.partials; p += 8 * 16) {
      float v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = a.partial[(p + i * 16) * a.cols + c];
#pragma unroll
      for (int i = 0; i < 8; ++i) s += v[i];
    }
    for (; p < a.partials; p += 16) s += a.partial[p * a.cols + c];
  }
  part[group][lane] = s;
  __syncthreads();
  if (group != 0 || c >= a.cols) return;
#pragma unroll
  for (int g = 1; g < 16; ++g) s += part[g][lane];
  if (a.out_type == SQUANT_W_F32) ((float*)a.out)[c] = s;
  else if (a.out_type == SQUANT_W_F16) ((_Float16*)a.out)[c] = (_Float16)s;
  else ((__bf16*)a.out)[c] = (__bf16)s;
}

__global__ void __launch_bounds__(kRowThreads) loss_rows(LossArgs a) {
  constexpr int kWaves = kRowThreads / kLanes;
  __shared__ float tops[kWaves], sums[kWaves];
  const int lane = threadIdx.x & (kLanes - 1), wave = threadIdx.x / kLanes;
  const int64_t row = blockIdx.x;
  const float2* s = a.stats + row * a.chunks;
  float top = -__builtin_inff();
#pragma unroll 4
  for (int32_t c = threadIdx.x; c < a.chunks; c += kRowThreads) top = fmaxf(top, s[c].x);
#pragma unroll
  for (int o = 1; o < kLanes; o <<= 1) top = fmaxf(top, __shfl_xor(top, o));
  if (lane == 0) tops[wave] = top;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kWaves; ++i) top = fmaxf(top, tops[i]);
  float sum = 0.0f;
#pragma unroll 4
  for (int32_t c = threadIdx.x; c < a.chunks; c += kRowThreads) {
    const float2 t = s[c];
    sum += t.y * exp2_fast(t.x - top);
  }
#pragma unroll
  for (int o = 1; o < kLanes; o <<= 1) sum += __shfl_xor(sum, o);
  if (lane == 0) sums[wave] = sum;
  __syncthreads();
  if (threadIdx.x != 0) return;
  sum = 0.0f;
#pragma unroll
  for (int i = 0; i < kWaves; ++i) sum += sums[i];
  const float rest = log2f(sum);
  a.lse[row] = (top + rest) * kLn2;
  const int64_t label = a.labels[row];
  if (label == a.ignore) a.loss[row] = 0.0f;
  else if (label < 0 || label >= a.vocabulary) a.loss[row] = __builtin_nanf("");
  else a.loss[row] = ((top - a.label_logit[row]) + rest) * kLn2;  // not by the log-sum-exp, whose rounding is that of a logit
}

__global__ void __launch_bounds__(1024) probability_unit(const float* scales, int32_t n, float* unit) {
  __shared__ uint32_t tops[1024 / kLanes];
  uint32_t top = 0;
  #pragma unroll 4
  for (int64_t i = (int64_t)threadIdx.x * 4; i < n; i += 4096) {
    float v[4];
    load_cols<4, float>(v, scales + i, (int)min((int64_t)4, n - i));
#pragma unroll
    for (int j = 0; j < 4; ++j) top = max(top, finite_magnitude(v[j]));
  }
  top = wave_max(top);
  if ((threadIdx.x & (kLanes - 1)) == 0) tops[threadIdx.x / kLanes] = top;
  __syncthreads();
  if (threadIdx.x != 0) return;
#pragma unroll
  for (int i = 0; i < 1024 / kLanes; ++i) top = max(top, tops[i]);
  *unit = power_of_two(row_exponent(top) - 1);
}

rows_kernel_t pad_rows_kernel() { return pad_rows; }
rows_kernel_t split_rows_kernel() { return split_rows; }
rows_kernel_t gradient_rows_kernel(int type) {
  if (type == SQUANT_W_F32) return gradient_rows<float, 2>;
  if (type == SQUANT_W_F16) return gradient_rows<_Float16, 1>;
  return gradient_rows<__bf16, 1>;
}
join_kernel_t join_kernel(bool grad, int type) {
  if (grad) return join<true, float>;
  if (type == SQUANT_W_F32) return join<false, float>;
  if (type == SQUANT_W_F16) return join<false, _Float16>;
  return join<false, __bf16>;
}
void (*column_sums_kernel())(ColumnSumArgs) { return column_sums; }
void (*loss_rows_kernel())(LossArgs) { return loss_rows; }
void (*probability_unit_kernel())(const float*, int32_t, float*) { return probability_unit; }

}  // namespace lin
}  // namespace squant
