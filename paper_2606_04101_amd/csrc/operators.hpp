// Launchers of the operators around the balancing path (router, combine's
// backward pass, 8-bit expert products) and the numeric helpers they share.
// Internal header; the C ABI in operators.hip validates arguments and calls
// these.
#pragma once

#include "common.hpp"

namespace uep {

typedef uint32_t v2u __attribute__((ext_vector_type(2)));
typedef float v4f __attribute__((ext_vector_type(4)));

// route workspace: one partial of every statistic per chunk of a sequence
struct RouteShape {
  int64_t n_seg;    // sequences
  int64_t seq;      // tokens of a sequence (the last may have fewer)
  int64_t chunk;    // tokens of a workgroup
  int64_t n_chunk;  // workgroups of a sequence
};
RouteShape route_shape(int64_t T, const ultraep_router &r);
size_t route_ws_need(int64_t T, const ultraep_router &r);   // of a call of T tokens
size_t route_ws_bytes(int64_t T, const ultraep_router &r);  // of any of up to T

hipError_t launch_route(const void *logits, int32_t type, int64_t T, int64_t ld,
                        const ultraep_router &r, const float *bias, const uint8_t *mask,
                        int32_t *topk, float *gate, int32_t *counts, float *prob_sum,
                        int32_t *tokens, void *ws, int32_t *status, hipStream_t stream);
hipError_t launch_balance_loss(const int32_t *counts, const int32_t *load_tokens,
                               const float *prob_sum, const int32_t *tokens, int64_t n_seg,
                               const ultraep_router &r, float alpha, float *loss, float *coef,
                               hipStream_t stream);
hipError_t launch_route_grad(const void *logits, int32_t type, int64_t T, int64_t ld,
                             const ultraep_router &r, const uint8_t *mask, const int32_t *topk,
                             const float *dgate, const float *coef, const float *dloss,
                             void *dlogits, int32_t *status, hipStream_t stream);
hipError_t launch_combine_grad(const uint16_t *dout, const uint16_t *y, int64_t n_rows,
                               const float *gate, const int32_t *row_of_slot, int64_t T, int32_t k,
                               int32_t H, const int64_t *n_routed, uint16_t *dy, float *dgate,
                               int32_t *status, hipStream_t stream);
hipError_t launch_quant_rows(const void *x, int32_t type, int64_t rows, int64_t K, int64_t ld,
                             int8_t *q, int64_t ldq, float *scale, hipStream_t stream);
hipError_t launch_expert_matmul(const int8_t *xq, const float *xs, int64_t M, const int8_t *wq,
                                const float *ws, int32_t n_w, int32_t N, int32_t K,
                                const int64_t *block_off, const int32_t *block_w, int32_t n_block,
                                int32_t act, void *y, int32_t type, int32_t *status,
                                hipStream_t stream);

__device__ __forceinline__ float bf16_at_low(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_at_high(uint32_t w) {
  return __uint_as_float(w & 0xFFFF0000u);
}

// fp32 -> bf16, to nearest-even; NaN -> 0x7FC0
__device__ __forceinline__ uint32_t round_bf16(float f) {
  const uint32_t u = __float_as_uint(f);
  if ((u & 0x7FFFFFFFu) > 0x7F800000u) return 0x7FC0u;
  return (u + 0x7FFFu + ((u >> 16) & 1u)) >> 16;
}

// two of them, a in the low half, by the converter (a NaN stays one)
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  typedef float v2f __attribute__((ext_vector_type(2)));
  typedef __bf16 v2b __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((v2f{a, b}), v2b));
}

__device__ __forceinline__ float readlane_f(float v, int l) {
  return __int_as_float(readlane(__float_as_int(v), l));
}

// Reductions over rows of 16 lanes (DPP mirrors) or over the 64 of a wave (the rows'
// results in order), each in one fixed order.  Every lane must be active.
template <int kCtrl>
__device__ __forceinline__ int dpp_i(int v) {
  // (each control used reads a lane of the row for every lane)
  return __builtin_amdgcn_mov_dpp(v, kCtrl, 0xF, 0xF, true);
}
template <int kCtrl>
__device__ __forceinline__ float dpp_f(float v) {
  return __int_as_float(dpp_i<kCtrl>(__float_as_int(v)));
}
template <int kLanes>
__device__ __forceinline__ float lanes_sum(float v) {
  // (rounded before the first sum: fused into it, a product would be the exact one in one
  // lane and the rounded one in its neighbour, and their sums two numbers)
  asm("" : "+v"(v));
  v += dpp_f<0xB1>(v);   // quad_perm 1,0,3,2
  v += dpp_f<0x4E>(v);   // quad_perm 2,3,0,1
  v += dpp_f<0x141>(v);  // row_half_mirror
  v += dpp_f<0x140>(v);  // row_mirror
  if (kLanes == 16) return v;
  return (readlane_f(v, 0) + readlane_f(v, 16)) + (readlane_f(v, 32) + readlane_f(v, 48));
}
// the larger, as one instruction (no NaN among them)
__device__ __forceinline__ float larger(float a, float b) {
  return __builtin_amdgcn_fmed3f(a, b, __builtin_inff());
}
template <int kLanes>
__device__ __forceinline__ float lanes_max(float v) {
  v = larger(v, dpp_f<0xB1>(v));
  v = larger(v, dpp_f<0x4E>(v));
  v = larger(v, dpp_f<0x141>(v));
  v = larger(v, dpp_f<0x140>(v));
  if (kLanes == 16) return v;
  return larger(larger(readlane_f(v, 0), readlane_f(v, 16)),
                larger(readlane_f(v, 32), readlane_f(v, 48)));
}
template <int kLanes>
__device__ __forceinline__ int lanes_max(int v) {
  return kLanes == 16 ? row_max(v) : wave_max(v);
}
__device__ __forceinline__ float wave_sum_f(float v) { return lanes_sum<kWave>(v); }

// exp by the hardware's exp2, 1 ulp.  The product with log2(e) is rounded before it, so a
// result between 2^-126 and infinity is (|x| + 2) 2^-24 off at most, relatively; below it is 0.
__device__ __forceinline__ float fast_exp(float x) {
  return __builtin_amdgcn_exp2f(x * 1.44269504088896341f);
}
// The same for x <= 0, -inf among them, within 2 ulp: what t = x log2(e) misses is
// x - t ln 2 to first order, with ln 2 in two parts (Cody and Waite).  In the router's scores
// it costs 1 to 4 % of a call with statistics (16384 tokens of 256 16.8 us, with fast_exp
// 16.5; 65536 47 and 45) and keeps a score of logit -30 at 10 x 2^-24 instead of 40.
__device__ __forceinline__ float exp_neg(float x) {
  x = larger(x, -128.f);  // (0 from there on, and no -inf below)
  const float t = x * 1.44269504088896341f, e = __builtin_amdgcn_exp2f(t);
  const float missed = fmaf(-t, -0x1.05c610p-29f, fmaf(-t, 0x1.62e430p-1f, x));
  return fmaf(e, missed, e);
}
// 1 / x to 1 ulp, for x of ordinary size
__device__ __forceinline__ float fast_rcp(float x) { return __builtin_amdgcn_rcpf(x); }

// s = 1 / (1 + exp(-z)) and 1 - s, each without overflow or cancellation for any z
struct Sigmoid {
  float s, rest;
};
__device__ __forceinline__ Sigmoid sigmoid_both(float z) {
  const float e = exp_neg(-fabsf(z)), r = fast_rcp(1.f + e), q = e * r;
  return z >= 0.f ? Sigmoid{r, q} : Sigmoid{q, r};
}
__device__ __forceinline__ float sigmoid(float z) { return sigmoid_both(z).s; }
// s over exp(c), c <= 0: of weight where sigmoid(z) itself vanishes
__device__ __forceinline__ float sigmoid_over(float z, float c) {
  return exp_neg(fminf(z, 0.f) - c) * fast_rcp(1.f + exp_neg(-fabsf(z)));
}

}  // namespace uep
