// C ABI of the operators around the balancing path (see include/ultraep.h):
// argument validation on the host, then stream-ordered kernel launches.  No
// allocation, no host synchronisation, no memset, no state.
#include <math.h>
#include <stdint.h>

#include "operators.hpp"

namespace {

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
bool aligned4(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

int rc(hipError_t e) { return e == hipSuccess ? ULTRAEP_OK : ULTRAEP_EDEVICE; }

bool type_ok(int32_t type) { return type == ULTRAEP_F32 || type == ULTRAEP_BF16; }

bool router_ok(const ultraep_router *r) {
  if (!r || r->E < 1 || r->E > 1024 || r->k < 1 || r->k > 64 || r->k > r->E) return false;
  if (r->score != ULTRAEP_SOFTMAX && r->score != ULTRAEP_SIGMOID) return false;
  if (r->renorm != 0 && r->renorm != 1) return false;
  if (!isfinite(r->scale) || r->seq_len < 0) return false;
  if (r->n_group == 0) return r->top_group == 0;
  if (r->n_group < 1 || r->n_group > 64 || r->E % r->n_group != 0) return false;
  const int32_t size = r->E / r->n_group;
  if (size < 2 || r->top_group < 1 || r->top_group > r->n_group) return false;
  return r->k <= r->top_group * size;
}

constexpr int64_t kMaxTokens = int64_t(1) << 23;

bool logits_ok(const void *logits, int32_t type, int64_t T, int64_t ld, const ultraep_router *r) {
  if (!type_ok(type) || T < 0 || T > kMaxTokens || !router_ok(r) || ld < r->E || ld > 1 << 20)
    return false;
  if (T > 0 && !logits) return false;
  return (reinterpret_cast<uintptr_t>(logits) & (type == ULTRAEP_BF16 ? 1u : 3u)) == 0;
}

// M rows in blocks of n_w weights
bool blocks_ok(int64_t M, int32_t n_w, const int64_t *block_off, int32_t n_block) {
  return M >= 0 && M < (int64_t(1) << 31) && n_w >= 1 && n_block >= 1 &&
         n_block <= uep::kMaxBlocks && block_off;
}
bool extent_ok(int32_t n, int32_t step) { return n >= step && n % step == 0 && n <= 1 << 20; }
// elements from one weight to the next
bool stride_ok(int64_t stride, int32_t N, int32_t K) {
  return stride >= static_cast<int64_t>(N) * K && stride % 8 == 0 && stride <= int64_t(1) << 40;
}
// gradients of n_w weights: their tiles are numbered in 31 bits
bool weights_ok(int32_t n_w, int32_t N, int32_t K) {
  return n_w >= 1 && n_w <= 1 << 20 && extent_ok(N, 8) && extent_ok(K, 8) &&
         int64_t(n_w) * ((N + 63) / 64) * ((K + 63) / 64) < int64_t(1) << 31;
}

}  // namespace

extern "C" {

size_t ultraep_route_ws_bytes(int64_t T, const ultraep_router *r) {
  if (T < 0 || T > kMaxTokens || !router_ok(r)) return 0;
  return uep::route_ws_bytes(T, *r);
}

int ultraep_route(const void *logits, int32_t type, int64_t T, int64_t ld,
                  const ultraep_router *r, const float *bias, const uint8_t *mask,
                  int32_t *topk, float *gate, int32_t *counts, float *prob_sum,
                  int32_t *tokens, void *ws, size_t ws_bytes, int32_t *status,
                  hipStream_t stream) {
  if (!logits_ok(logits, type, T, ld, r) || !status) return ULTRAEP_EINVAL;
  if (T > 0 && (!topk || !gate)) return ULTRAEP_EINVAL;
  const bool stats = counts != nullptr;
  if (stats != (prob_sum != nullptr) || stats != (tokens != nullptr)) return ULTRAEP_EINVAL;
  if (stats && (!ws || !aligned4(ws) || ws_bytes < uep::route_ws_need(T, *r)))
    return ULTRAEP_EINVAL;
  if (T == 0 && !stats) return ULTRAEP_OK;
  return rc(uep::launch_route(logits, type, T, ld, *r, bias, mask, topk, gate, counts, prob_sum,
                              tokens, ws, status, stream));
}

int ultraep_balance_loss(const int32_t *counts, const int32_t *load_tokens,
                         const float *prob_sum, const int32_t *tokens, int64_t n_seg,
                         const ultraep_router *r, float alpha, float *loss, float *coef,
                         hipStream_t stream) {
  if (!router_ok(r) || n_seg < 0 || n_seg > kMaxTokens || !isfinite(alpha) || !loss)
    return ULTRAEP_EINVAL;
  if (n_seg > 0 && (!counts || !load_tokens || !prob_sum || !tokens || !coef))
    return ULTRAEP_EINVAL;
  return rc(uep::launch_balance_loss(counts, load_tokens, prob_sum, tokens, n_seg, *r, alpha, loss,
                                     coef, stream));
}

int ultraep_route_grad(const void *logits, int32_t type, int64_t T, int64_t ld,
                       const ultraep_router *r, const uint8_t *mask, const int32_t *topk,
                       const float *dgate, const float *coef, const float *dloss,
                       void *dlogits, int32_t *status, hipStream_t stream) {
  if (!logits_ok(logits, type, T, ld, r) || !logits_ok(dlogits, type, T, ld, r) || !status)
    return ULTRAEP_EINVAL;
  if (T == 0) return ULTRAEP_OK;
  if (!topk) return ULTRAEP_EINVAL;
  return rc(uep::launch_route_grad(logits, type, T, ld, *r, mask, topk, dgate, coef, dloss, dlogits,
                                   status, stream));
}

int ultraep_combine_grad(const uint16_t *dout, const uint16_t *y, int64_t n_rows,
                         const float *gate, const int32_t *row_of_slot, int64_t T, int32_t k,
                         int32_t H, const int64_t *n_routed, uint16_t *dy, float *dgate,
                         int32_t *status, hipStream_t stream) {
  if (T < 0 || k < 1 || k > 64 || H < 8 || H % 8 != 0 || n_rows < 0 || !n_routed || !status)
    return ULTRAEP_EINVAL;
  if (T * static_cast<int64_t>(k) >= (int64_t(1) << 31) || n_rows >= (int64_t(1) << 31))
    return ULTRAEP_EINVAL;
  if (T > 0 && (!dout || !aligned16(dout) || !gate || !row_of_slot || !dgate))
    return ULTRAEP_EINVAL;
  if (n_rows > 0 && (!y || !aligned16(y) || !dy || !aligned16(dy) || dy == y))
    return ULTRAEP_EINVAL;
  if (T == 0 && n_rows == 0) return ULTRAEP_OK;
  return rc(uep::launch_combine_grad(dout, y, n_rows, gate, row_of_slot, T, k, H, n_routed, dy,
                                     dgate, status, stream));
}

int ultraep_quant_rows(const void *x, int32_t type, int64_t rows, int64_t K, int64_t ld,
                       int8_t *q, int64_t ldq, float *scale, hipStream_t stream) {
  if (!type_ok(type) || rows < 0 || rows >= (int64_t(1) << 31)) return ULTRAEP_EINVAL;
  if (K < 8 || K % 8 != 0 || ld < K || ld % 8 != 0 || ld > 1 << 20) return ULTRAEP_EINVAL;
  if (ldq < K || ldq % 16 != 0 || ldq > 1 << 20) return ULTRAEP_EINVAL;
  if (rows == 0) return ULTRAEP_OK;
  if (!x || !q || !scale || !aligned16(x) || !aligned16(q)) return ULTRAEP_EINVAL;
  return rc(uep::launch_quant_rows(x, type, rows, K, ld, q, ldq, scale, stream));
}

int ultraep_expert_matmul(const int8_t *xq, const float *x_scale, int64_t M,
                          const int8_t *wq, const float *w_scale, int32_t n_w, int32_t N,
                          int32_t K, const int64_t *block_off, const int32_t *block_w,
                          int32_t n_block, int32_t act, void *y, int32_t type,
                          int32_t *status, hipStream_t stream) {
  if (M < 0 || M >= (int64_t(1) << 31) || n_w < 1 || n_block < 1 || n_block > uep::kMaxBlocks ||
      !type_ok(type) || (act != 0 && act != 1) || !block_off || !status)
    return ULTRAEP_EINVAL;
  if (K < 16 || K % 16 != 0 || K > 1 << 16) return ULTRAEP_EINVAL;
  if (N < 8 || N % (act ? 16 : 8) != 0 || N > 1 << 20) return ULTRAEP_EINVAL;
  if (M * static_cast<int64_t>(N) >= int64_t(1) << 38) return ULTRAEP_EINVAL;
  if (!wq || !aligned16(wq) || !w_scale) return ULTRAEP_EINVAL;
  if (M == 0) return ULTRAEP_OK;
  if (!xq || !aligned16(xq) || !x_scale || !y || !aligned16(y)) return ULTRAEP_EINVAL;
  return rc(uep::launch_expert_matmul(xq, x_scale, M, wq, w_scale, n_w, N, K, block_off, block_w,
                                      n_block, act, y, type, status, stream));
}

int ultraep_expert_matmul_bf16(const uint16_t *x, int64_t M, const uint16_t *w, int32_t n_w,
                               int64_t w_stride, int32_t N, int32_t K, int32_t trans,
                               const int64_t *block_off, const int32_t *block_w,
                               int32_t n_block, int32_t act, uint16_t *pre, void *y,
                               int32_t type, int32_t *status, hipStream_t stream) {
  if (!blocks_ok(M, n_w, block_off, n_block) || !type_ok(type) || !status) return ULTRAEP_EINVAL;
  if (trans != 0 && trans != 1) return ULTRAEP_EINVAL;
  if (act != ULTRAEP_NO_ACT && act != ULTRAEP_SWIGLU && act != ULTRAEP_SWIGLU_GRAD)
    return ULTRAEP_EINVAL;
  if (!extent_ok(K, 8) || !extent_ok(N, act == ULTRAEP_SWIGLU ? 16 : 8)) return ULTRAEP_EINVAL;
  if (M * static_cast<int64_t>(N) >= int64_t(1) << 38) return ULTRAEP_EINVAL;
  if (!stride_ok(w_stride, N, K) || !w || !aligned16(w)) return ULTRAEP_EINVAL;
  if ((act == ULTRAEP_NO_ACT && pre) || !aligned16(pre)) return ULTRAEP_EINVAL;
  if (M == 0) return ULTRAEP_OK;
  if (act == ULTRAEP_SWIGLU_GRAD && !pre) return ULTRAEP_EINVAL;
  if (!x || !aligned16(x) || !y || !aligned16(y)) return ULTRAEP_EINVAL;
  // only a bf16 gradient may take its pre's place
  if (y == pre && !(act == ULTRAEP_SWIGLU_GRAD && type == ULTRAEP_BF16)) return ULTRAEP_EINVAL;
  if (y == x || y == w || (pre && (pre == x || pre == w))) return ULTRAEP_EINVAL;
  return rc(uep::launch_expert_matmul_bf16(x, M, w, n_w, w_stride, N, K, trans, block_off, block_w,
                                           n_block, act, pre, y, type, status, stream));
}

size_t ultraep_expert_weight_grad_ws_bytes(int64_t M, int32_t N, int32_t K, int32_t n_w) {
  if (M < 0 || M >= int64_t(1) << 31 || !weights_ok(n_w, N, K)) return 0;
  return uep::weight_grad_ws_bytes(M, N, K, n_w);
}

int ultraep_expert_weight_grad(const uint16_t *dy, const uint16_t *x, int64_t M, int32_t N,
                               int32_t K, const int64_t *block_off, const int32_t *block_w,
                               int32_t n_block, int32_t n_w, int64_t dw_stride,
                               int32_t accumulate, void *dw, int32_t type, void *ws,
                               size_t ws_bytes, int32_t *status, hipStream_t stream) {
  if (!blocks_ok(M, n_w, block_off, n_block) || !type_ok(type) || !status) return ULTRAEP_EINVAL;
  if ((accumulate != 0 && accumulate != 1) || !weights_ok(n_w, N, K)) return ULTRAEP_EINVAL;
  if (!stride_ok(dw_stride, N, K) || !dw || !aligned16(dw)) return ULTRAEP_EINVAL;
  if (ws && (!aligned16(ws) || ws_bytes < uep::weight_grad_ws_bytes(M, N, K, n_w)))
    return ULTRAEP_EINVAL;
  if (M > 0 && (!dy || !aligned16(dy) || !x || !aligned16(x))) return ULTRAEP_EINVAL;
  if (dw == dy || dw == x || (ws && (ws == dw || ws == dy || ws == x))) return ULTRAEP_EINVAL;
  return rc(uep::launch_expert_weight_grad(dy, x, M, N, K, block_off, block_w, n_block, n_w,
                                           dw_stride, accumulate, dw, type, ws, status, stream));
}

int ultraep_quant_blocks(const void *x, int32_t type, int64_t rows, int64_t K, int64_t ld,
                         uint8_t *q, int64_t ldq, uint8_t *scale, hipStream_t stream) {
  if (!type_ok(type) || rows < 0 || rows >= (int64_t(1) << 31)) return ULTRAEP_EINVAL;
  if (K < 8 || K % 8 != 0 || ld < K || ld % 8 != 0 || ld > 1 << 20) return ULTRAEP_EINVAL;
  if (ldq < K || ldq % 16 != 0 || ldq > 1 << 20) return ULTRAEP_EINVAL;
  if (rows == 0) return ULTRAEP_OK;
  if (!x || !q || !scale || !aligned16(x) || !aligned16(q) || !aligned4(scale) || q == x || scale == x || scale == q)
    return ULTRAEP_EINVAL;
  return rc(uep::launch_quant_blocks(x, type, rows, K, ld, q, ldq, scale, stream));
}

int ultraep_expert_matmul_fp8(const uint8_t *xq, const uint8_t *x_scale, int64_t M,
                              const uint8_t *wq, const uint8_t *w_scale, int32_t n_w, int32_t N,
                              int32_t K, const int64_t *block_off, const int32_t *block_w,
                              int32_t n_block, int32_t act, void *y, int32_t type,
                              int32_t *status, hipStream_t stream) {
  if (!blocks_ok(M, n_w, block_off, n_block) || !type_ok(type) || !status) return ULTRAEP_EINVAL;
  if (act != ULTRAEP_NO_ACT && act != ULTRAEP_SWIGLU) return ULTRAEP_EINVAL;
  if (!extent_ok(K, 16) || K > 1 << 18 || !extent_ok(N, act ? 16 : 8)) return ULTRAEP_EINVAL;
  if (M * static_cast<int64_t>(N) >= int64_t(1) << 38) return ULTRAEP_EINVAL;
  if (!wq || !aligned16(wq) || !w_scale || !aligned4(w_scale)) return ULTRAEP_EINVAL;
  if (M == 0) return ULTRAEP_OK;
  if (!xq || !aligned16(xq) || !x_scale || !aligned4(x_scale) || !y || !aligned16(y))
    return ULTRAEP_EINVAL;
  if (y == xq || y == wq || y == x_scale || y == w_scale) return ULTRAEP_EINVAL;
  return rc(uep::launch_expert_matmul_fp8(xq, x_scale, M, wq, w_scale, n_w, N, K, block_off,
                                          block_w, n_block, act, y, type, status, stream));
}

}  // extern "C"
