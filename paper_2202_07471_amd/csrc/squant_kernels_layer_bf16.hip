// Products of bfloat16 rows with codes.
#include "squant_lin_kernels.h"
#include "squant_product.h"

namespace squant {
namespace lin {

product_t layer_bf16(int format, int mt, bool words) {
  return format == SQUANT_OUT_INT4 ? layer_of<Brain, 1, SQUANT_OUT_INT4>(mt, words)
                                   : layer_of<Brain, 1, SQUANT_OUT_INT8>(mt, words);
}

}  // namespace lin
}  // namespace squant
