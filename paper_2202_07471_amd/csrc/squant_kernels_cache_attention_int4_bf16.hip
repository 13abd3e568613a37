// Attention over a cache of 4-bit codes, bfloat16; the join of pieces for all types.
#include "squant_cache_attention.h"

namespace squant {
namespace att {

cache_attention_t cache_attention_int4_bf16(int ng, int rt, bool halves) { return cache_attention_of<__bf16, SQUANT_OUT_INT4>(ng, rt, halves); }
cache_attention_t join_splits_kernel(int type) {
  return type == SQUANT_W_F32 ? join_splits<float> : type == SQUANT_W_F16 ? join_splits<_Float16> : join_splits<__bf16>;
}

}  // namespace att
}  // namespace squant
