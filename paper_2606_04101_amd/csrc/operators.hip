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
  if (M < 0 || M >= (int64_t(1) << 31) || n_w < 1 || n_block < 1 || n_block > 2048 ||
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

}  // extern "C"
