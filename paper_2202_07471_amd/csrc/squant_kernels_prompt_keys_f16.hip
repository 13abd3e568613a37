// Gradients of attention over whole prompts, binary16: keys and values.
#include "squant_prompt.h"

namespace squant {
namespace att {

PromptKernel prompt_keys_f16(int dim, bool direct, bool many) { return backward_for<_Float16, true>(dim, direct, many); }

}  // namespace att
}  // namespace squant
