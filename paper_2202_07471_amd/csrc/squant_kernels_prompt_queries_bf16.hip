// Gradients of attention over whole prompts, bfloat16: queries.
#include "squant_prompt.h"

namespace squant {
namespace att {

PromptKernel prompt_queries_bf16(int dim, bool direct, bool many) { return backward_for<__bf16, false>(dim, direct, many); }

}  // namespace att
}  // namespace squant
