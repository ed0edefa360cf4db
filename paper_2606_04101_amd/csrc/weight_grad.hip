// The gradient of the experts' weights: for each weight the sum, over its blocks' rows, of
// the outer products of the two sides' rows.
#include "operators.hpp"

namespace uep {

struct GradArgs {
  const uint16_t *dy, *x;
  const int64_t *block_off;
  const int32_t *block_w;
  void *dw;
  int32_t *status;
  int64_t M, dw_stride;
  int32_t n_w, N, K, n_block, accumulate, bf16;
};

constexpr int kTile = 64, kStepM = 16;

// 64 x 64 elements of one weight's gradient, 4 x 4 a thread, on the vector units.
__global__ void __launch_bounds__(256) k_weight_grad(GradArgs a, int32_t tn, int32_t tk) {
  __shared__ float s_y[kStepM][kTile], s_x[kStepM][kTile];
  const int tid = threadIdx.x;
  bool sound = true;  // no block is out of order, out of [0, M] or without a weight
  for (int g = tid; g < a.n_block; g += 256) {
    const int64_t lo = a.block_off[g], hi = a.block_off[g + 1];
    const int w = a.block_w ? a.block_w[g] : g;
    sound &= lo >= 0 && hi >= lo && hi <= a.M && (hi == lo || (w >= 0 && w < a.n_w));
  }
  if (!__syncthreads_and(sound)) {
    if (tid == 0) report(a.status, ULTRAEP_EDATA);
    return;
  }
  const int tr = tid / 16, tc = tid % 16;
  for (int64_t item = blockIdx.x; item < static_cast<int64_t>(a.n_w) * tn * tk; item += gridDim.x) {
    const int w = static_cast<int>(item / (tn * tk)), n0 = static_cast<int>(item / tk % tn) * kTile;
    const int k0 = static_cast<int>(item % tk) * kTile;
    float v[4][4] = {};
    for (int g = 0; g < a.n_block; ++g) {
      if ((a.block_w ? a.block_w[g] : g) != w) continue;
      const int64_t lo = a.block_off[g], hi = a.block_off[g + 1];
      for (int64_t m0 = lo; m0 < hi; m0 += kStepM) {
        for (int i = tid; i < kStepM * kTile; i += 256) {
          const int64_t m = m0 + i / kTile;
          const int n = n0 + i % kTile, k = k0 + i % kTile;
          s_y[i / kTile][i % kTile] = m < hi && n < a.N ? bf16_at_low(a.dy[m * a.N + n]) : 0.f;
          s_x[i / kTile][i % kTile] = m < hi && k < a.K ? bf16_at_low(a.x[m * a.K + k]) : 0.f;
        }
        __syncthreads();
        for (int m = 0; m < kStepM; ++m)
          for (int i = 0; i < 4; ++i)
            for (int j = 0; j < 4; ++j)
              v[i][j] = fmaf(s_y[m][tr + i * 16], s_x[m][tc + j * 16], v[i][j]);
        __syncthreads();
      }
    }
    for (int i = 0; i < 4; ++i)
      for (int j = 0; j < 4; ++j) {
        const int n = n0 + tr + i * 16, k = k0 + tc + j * 16;
        if (n >= a.N || k >= a.K) continue;
        const int64_t at = w * a.dw_stride + static_cast<int64_t>(n) * a.K + k;
        if (a.bf16) {
          uint16_t *p = static_cast<uint16_t *>(a.dw) + at;
          *p = round_bf16(a.accumulate ? bf16_at_low(*p) + v[i][j] : v[i][j]);
        } else {
          float *p = static_cast<float *>(a.dw) + at;
          *p = a.accumulate ? *p + v[i][j] : v[i][j];
        }
      }
  }
}

size_t weight_grad_ws_bytes(int64_t, int32_t, int32_t, int32_t) { return 16; }

hipError_t launch_expert_weight_grad(const uint16_t *dy, const uint16_t *x, int64_t M, int32_t N,
                                     int32_t K, const int64_t *block_off, const int32_t *block_w,
                                     int32_t n_block, int32_t n_w, int64_t dw_stride,
                                     int32_t accumulate, void *dw, int32_t type, void *,
                                     int32_t *status, hipStream_t stream) {
  const GradArgs a{dy, x, block_off, block_w, dw, status, M, dw_stride, n_w, N, K, n_block,
                   accumulate, type == ULTRAEP_BF16};
  const int32_t tn = (N + kTile - 1) / kTile, tk = (K + kTile - 1) / kTile;
  const int64_t items = static_cast<int64_t>(n_w) * tn * tk;
  const dim3 grid(static_cast<unsigned>(items < 1 << 16 ? items : 1 << 16));
  hipLaunchKernelGGL(k_weight_grad, grid, dim3(256), 0, stream, a, tn, tk);
  return hipGetLastError();
}

}  // namespace uep
