// Attention over a cache of 4-bit codes, binary16.
#include "squant_cache_attention.h"

namespace squant {
namespace att {

cache_attention_t cache_attention_int4_f16(int ng, int rt, bool halves) { return cache_attention_of<_Float16, SQUANT_OUT_INT4>(ng, rt, halves); }

}  // namespace att
}  // namespace squant
