// Attention over whole prompts, binary32.
#include "squant_prompt.h"

namespace squant {
namespace att {

PromptKernel prompt_forward_f32(int dim, bool direct) { return forward_for<float>(dim, direct); }

prompt_t prompt_join_forward_kernel(int type) {
  return type == SQUANT_W_F32 ? prompt_join_forward<float> : type == SQUANT_W_F16 ? prompt_join_forward<_Float16> : prompt_join_forward<__bf16>;
}
prompt_t prompt_join_kernel(int type, bool keys) {
  if (keys) return type == SQUANT_W_F32 ? prompt_join<float, true> : type == SQUANT_W_F16 ? prompt_join<_Float16, true> : prompt_join<__bf16, true>;
  return prompt_join<float, false>;
}

}  // namespace att
}  // namespace squant
