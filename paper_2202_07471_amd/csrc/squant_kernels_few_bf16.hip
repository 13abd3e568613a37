// Products of few bfloat16 rows with codes.
#include "squant_few_rows.h"
#include "squant_lin_kernels.h"

namespace squant {
namespace lin {

product_t few_bf16(int format, int mf, int nf) {
  if (nf == 4)
    return format == SQUANT_OUT_INT4 ? few_rows_of<Brain, 1, SQUANT_OUT_INT4, 4>(mf)
                                     : few_rows_of<Brain, 1, SQUANT_OUT_INT8, 4>(mf);
  return format == SQUANT_OUT_INT4 ? few_rows_of<Brain, 1, SQUANT_OUT_INT4, 1>(mf)
                                   : few_rows_of<Brain, 1, SQUANT_OUT_INT8, 1>(mf);
}

}  // namespace lin
}  // namespace squant
