// Gradients of attention over whole prompts, bfloat16: keys and values.
#include "squant_prompt.h"

namespace squant {
namespace att {

PromptKernel prompt_keys_bf16(int dim, bool direct, bool many) { return backward_for<__bf16, true>(dim, direct, many); }

}  // namespace att
}  // namespace squant
