// Products of few binary16 rows with codes.
#include "squant_few_rows.h"
#include "squant_lin_kernels.h"

namespace squant {
namespace lin {

namespace {
template <int NF>
product_t by_format(int format, int mf) {
  return format == SQUANT_OUT_INT4 ? few_rows_of<Half, 1, SQUANT_OUT_INT4, NF>(mf)
                                   : few_rows_of<Half, 1, SQUANT_OUT_INT8, NF>(mf);
}
}  // namespace

product_t few_f16(int format, int mf, int nf) {
  return nf == 4 ? by_format<4>(format, mf) : nf == 2 ? by_format<2>(format, mf) : by_format<1>(format, mf);
}

}  // namespace lin
}  // namespace squant
