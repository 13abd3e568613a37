// Attention over a cache of 4-bit codes, bfloat16.
#include "squant_cache_attention.h"

namespace squant {
namespace att {

cache_attention_t cache_attention_int4_bf16(int ng, int rt, bool halves) { return cache_attention_of<__bf16, SQUANT_OUT_INT4>(ng, rt, halves); }
cache_attention_t join_splits_kernel() { return join_splits<0>; }

}  // namespace att
}  // namespace squant
