// Attention over a cache of 8-bit codes, binary32 queries.
#include "squant_cache_attention.h"

namespace squant {
namespace att {

cache_attention_t cache_attention_int8_2(int ng, int rt) { return cache_attention_of<SQUANT_OUT_INT8, 2>(ng, rt); }

}  // namespace att
}  // namespace squant
