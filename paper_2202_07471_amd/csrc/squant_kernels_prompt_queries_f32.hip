// Gradients of attention over whole prompts, binary32: queries.
#include "squant_prompt.h"

namespace squant {
namespace att {

PromptKernel prompt_queries_f32(int dim) { return backward_for<float, false>(dim); }

}  // namespace att
}  // namespace squant
