// Products of binary32 rows with codes.
#include "squant_lin_kernels.h"
#include "squant_product.h"

namespace squant {
namespace lin {

product_t layer_f32(int format, int mt) {
  return format == SQUANT_OUT_INT4 ? product_of<Half, 2, SQUANT_OUT_INT4, kLayer>(mt)
                                   : product_of<Half, 2, SQUANT_OUT_INT8, kLayer>(mt);
}

}  // namespace lin
}  // namespace squant
