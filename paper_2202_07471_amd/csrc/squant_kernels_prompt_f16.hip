// Attention over whole prompts, binary16.
#include "squant_prompt.h"

namespace squant {
namespace att {

PromptKernel prompt_forward_f16(int dim, bool direct) { return forward_for<_Float16>(dim, direct); }

}  // namespace att
}  // namespace squant
