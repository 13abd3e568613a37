// Gradients of attention over whole prompts, binary16: queries.
#include "squant_prompt.h"

namespace squant {
namespace att {

PromptKernel prompt_queries_f16(int dim, bool direct, bool many) { return backward_for<_Float16, false>(dim, direct, many); }

}  // namespace att
}  // namespace squant
