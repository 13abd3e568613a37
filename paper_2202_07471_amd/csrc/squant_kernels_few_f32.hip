// Products of few binary32 rows with codes.
#include "squant_few_rows.h"
#include "squant_lin_kernels.h"

namespace squant {
namespace lin {

product_t few_f32(int format, int mf, int nf, bool words) {
  return format == SQUANT_OUT_INT4 ? few_of<Half, float, SQUANT_OUT_INT4>(mf, nf, words)
                                   : few_of<Half, float, SQUANT_OUT_INT8>(mf, nf, words);
}

}  // namespace lin
}  // namespace squant
