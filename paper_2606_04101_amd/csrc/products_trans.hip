// The experts' products in bf16 on weights [K][N]: the gradient of the forward product's
// input.
#include "products_thin.hpp"

namespace uep {

hipError_t launch_product_trans(const ProductArgs &a, int32_t act, int32_t type, hipStream_t stream) {
  if (act == ULTRAEP_NO_ACT) choose_type<kMath16, true, ULTRAEP_NO_ACT>(a, type, stream);
  else if (act == ULTRAEP_SWIGLU) choose_type<kMath16, true, ULTRAEP_SWIGLU>(a, type, stream);
  else choose_type<kMath16, true, ULTRAEP_SWIGLU_GRAD>(a, type, stream);
  return hipGetLastError();
}

}  // namespace uep
