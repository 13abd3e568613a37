// Attention over whole prompts, bfloat16.
#include "squant_prompt.h"

namespace squant {
namespace att {

PromptKernel prompt_forward_bf16(int dim, bool direct) { return forward_for<__bf16>(dim, direct); }

}  // namespace att
}  // namespace squant
