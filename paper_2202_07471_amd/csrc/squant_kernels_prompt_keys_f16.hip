// Gradients of attention over whole prompts, binary16: keys and values.
#include "squant_prompt.h"

namespace squant {
namespace att {

PromptKernel prompt_keys_f16(int dim) { return backward_for<_Float16, true>(dim); }

}  // namespace att
}  // namespace squant
