// Gradients of attention over whole prompts, binary32: keys and values.
#include "squant_prompt.h"

namespace squant {
namespace att {

PromptKernel prompt_keys_f32(int dim, bool direct, bool many) { return backward_for<float, true>(dim, direct, many); }

}  // namespace att
}  // namespace squant
