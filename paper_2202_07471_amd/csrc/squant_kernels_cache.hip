// Tokens into the quantised cache and back.
#include "squant_cache.h"

namespace squant {
namespace att {

cache_rows_t cache_write_kernel(int type, int format) {
  if (format == SQUANT_OUT_INT4)
    return type == SQUANT_W_F32 ? cache_write<float, SQUANT_OUT_INT4> : type == SQUANT_W_F16 ? cache_write<_Float16, SQUANT_OUT_INT4> : cache_write<__bf16, SQUANT_OUT_INT4>;
  return type == SQUANT_W_F32 ? cache_write<float, SQUANT_OUT_INT8> : type == SQUANT_W_F16 ? cache_write<_Float16, SQUANT_OUT_INT8> : cache_write<__bf16, SQUANT_OUT_INT8>;
}

cache_rows_t cache_read_kernel(int type, int format) {
  if (format == SQUANT_OUT_INT4)
    return type == SQUANT_W_F32 ? cache_read<float, SQUANT_OUT_INT4> : type == SQUANT_W_F16 ? cache_read<_Float16, SQUANT_OUT_INT4> : cache_read<__bf16, SQUANT_OUT_INT4>;
  return type == SQUANT_W_F32 ? cache_read<float, SQUANT_OUT_INT8> : type == SQUANT_W_F16 ? cache_read<_Float16, SQUANT_OUT_INT8> : cache_read<__bf16, SQUANT_OUT_INT8>;
}

}  // namespace att
}  // namespace squant
