// The experts' products in bf16 on weights [N][K].
#include "products_thin.hpp"

namespace uep {

hipError_t launch_product_trans(const ProductArgs &a, int32_t act, int32_t type, hipStream_t stream);

hipError_t launch_expert_matmul_bf16(const uint16_t *x, int64_t M, const uint16_t *w, int32_t n_w,
                                     int64_t w_stride, int32_t N, int32_t K, int32_t trans,
                                     const int64_t *block_off, const int32_t *block_w,
                                     int32_t n_block, int32_t act, uint16_t *pre, void *y,
                                     int32_t type, int32_t *status, hipStream_t stream) {
  const ProductArgs a{reinterpret_cast<const int8_t *>(x), reinterpret_cast<const int8_t *>(w),
                      nullptr, nullptr, block_off, block_w, pre, y, status, M, w_stride, n_w, N, K,
                      n_block, act == ULTRAEP_SWIGLU ? N / 2 : N};
  if (trans) return launch_product_trans(a, act, type, stream);
  if (act == ULTRAEP_NO_ACT) choose_type<kMath16, false, ULTRAEP_NO_ACT>(a, type, stream);
  else if (act == ULTRAEP_SWIGLU) choose_type<kMath16, false, ULTRAEP_SWIGLU>(a, type, stream);
  else choose_type<kMath16, false, ULTRAEP_SWIGLU_GRAD>(a, type, stream);
  return hipGetLastError();
}

}  // namespace uep

// Which of product_tile's tiles a call takes, for the tests (host only): eight, whether of 8 bits
extern "C" int uep_product_tile(int64_t M, int32_t n_block, int32_t N, int32_t K, int32_t eight, int32_t trans,
                                int32_t act, int32_t type) {
  const uep::Math kind = !eight ? uep::kMath16 : type == ULTRAEP_BF16 ? uep::kMath8 : uep::kMathWide;
  return uep::product_tile(kind, trans, act, M, n_block, N, K);
}
