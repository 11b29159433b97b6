// The persistent grouped GEMM's variants that add the rows' low-rank adapters (gemm_fast.h, adapter_core.h): a file of its own because
// a variant takes seconds to compile.

#include "gemm_fast.h"

namespace ppmoe {

FastKernel fast_kernel_with_adapters(int dtype, bool gelu, bool ragged, bool b_by_rows) {
  using fast::grouped_gemm_fast_kernel;
  if (b_by_rows && (gelu || ragged)) return nullptr;
#define PPMOE_VARIANT(DT)                                                         \
  b_by_rows          ? grouped_gemm_fast_kernel<0, 0, DT, false, true, true>      \
  : gelu && ragged ? grouped_gemm_fast_kernel<1, 0, DT, true, false, true>        \
  : gelu           ? grouped_gemm_fast_kernel<1, 0, DT, false, false, true>       \
  : ragged         ? grouped_gemm_fast_kernel<0, 0, DT, true, false, true>        \
                   : grouped_gemm_fast_kernel<0, 0, DT, false, false, true>
  if (dtype == MOE_F16) return PPMOE_VARIANT(MOE_F16);
  return PPMOE_VARIANT(MOE_BF16);
#undef PPMOE_VARIANT
}

}  // namespace ppmoe
