// Gradients through codes, row operands of 1 plane.
#include "squant_lin_kernels.h"
#include "squant_product.h"

namespace squant {
namespace lin {

product_t gradient_1(int format, int mt) {
  return format == SQUANT_OUT_INT4 ? product_of<Half, 1, SQUANT_OUT_INT4, kGradient>(mt)
                                   : product_of<Half, 1, SQUANT_OUT_INT8, kGradient>(mt);
}

}  // namespace lin
}  // namespace squant
