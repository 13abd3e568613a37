// Gradients of attention over whole prompts, binary32: queries.
#include "squant_prompt.h"

namespace squant {
namespace att {

PromptKernel prompt_queries_f32(int dim, bool direct, bool many) { return backward_for<float, false>(dim, direct, many); }

}  // namespace att
}  // namespace squant
