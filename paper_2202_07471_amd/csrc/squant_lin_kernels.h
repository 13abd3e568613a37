// The kernels of the operators that multiply by codes, by translation unit.
#pragma once

#include "squant_lin_rows.h"

namespace squant {
namespace lin {

// `mt` 64, 128 or 256 rows a workgroup; `mf` fragments of 16 rows, 1, 2 or 4; `nf` of 16 columns, 1, 2 or 4;
// `words`: code rows begin at whole 32-bit words.
product_t layer_bf16(int format, int mt);
product_t layer_f16(int format, int mt);
product_t layer_f32(int format, int mt);
product_t prob_bf16(int format, int mt);
product_t prob_f16(int format, int mt);
product_t prob_f32(int format, int mt);
product_t gradient_1(int format, int mt);  // planes of the row operand
product_t gradient_2(int format, int mt);
product_t few_bf16(int format, int mf, int nf, bool words);
product_t few_f16(int format, int mf, int nf, bool words);
product_t few_f32(int format, int mf, int nf, bool words);
rows_kernel_t pad_rows_kernel();
rows_kernel_t split_rows_kernel();
rows_kernel_t gradient_rows_kernel(int type);
join_kernel_t join_kernel(bool grad, int type);
void (*column_sums_kernel())(ColumnSumArgs);
void (*loss_rows_kernel())(LossArgs);
void (*probability_unit_kernel())(const float*, int32_t, float*);

}  // namespace lin
}  // namespace squant
