// Logits of bfloat16 rows against a vocabulary of codes, as the loss gradient's probabilities.
#include "squant_lin_kernels.h"
#include "squant_product.h"

namespace squant {
namespace lin {

product_t prob_bf16(int format, int mt) {
  return format == SQUANT_OUT_INT4 ? product_of<Brain, 1, SQUANT_OUT_INT4, kProbabilities>(mt)
                                   : product_of<Brain, 1, SQUANT_OUT_INT8, kProbabilities>(mt);
}

}  // namespace lin
}  // namespace squant
