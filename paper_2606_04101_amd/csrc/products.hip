// The experts' products in floating point: bf16 (forward, or on transposed weights for
// the gradient of the input) and 8-bit with a scale for each 128 elements.
#include "operators.hpp"
#include "tiles.hpp"

namespace uep {

struct ProductArgs {
  const uint8_t *x, *w;    // elements
  const uint8_t *xs, *ws;  // scales (8-bit)
  const int64_t *block_off;
  const int32_t *block_w;
  uint16_t *pre;
  void *y;
  int32_t *status;
  int64_t M, w_stride;  // (elements)
  int32_t n_w, N, K, n_block, trans, act, bf16;
};

__device__ __forceinline__ float e4m3(uint8_t v) {
  return __builtin_amdgcn_cvt_f32_fp8(static_cast<int>(v), 0);
}
__device__ __forceinline__ float power(uint8_t b) {  // 2^(b - 127)
  return b == 255 ? __builtin_nanf("") : ldexpf(1.f, static_cast<int>(b) - 127);
}

constexpr int kTile = 64, kStepK = 16;

// 64 rows x 64 channels, 4 x 4 a thread, on the vector units.
template <bool kFp8>
__global__ void __launch_bounds__(256) k_product(ProductArgs a, int32_t n_col) {
  __shared__ float s_x[kStepK][kTile + 1], s_w[kStepK][kTile + 1];
  __shared__ int s_run[32];
  const int tid = threadIdx.x;
  RowTiles<kTile> tiles;
  tiles.count(a, s_run, __builtin_amdgcn_readfirstlane(tid / kWave), 4);
  const int n_item = tiles.total * n_col;
  const bool glu = a.act == ULTRAEP_SWIGLU;
  const int half = a.N / 2, n_out = glu ? half : a.N, out = glu ? kTile / 2 : kTile;
  const int pitch = scale_pitch(a.K);
  const int tr = tid / 16, tc = tid % 16;
  for (int item = blockIdx.x; item < n_item; item += gridDim.x) {
    const RowTile tile = tiles.find(a, item / n_col);
    const int n0 = item % n_col * out;
    // the tile's channel j: with SwiGLU 32 gates, then their partners
    auto channel = [&](int j) { return n0 + j % out + j / out * half; };
    auto in_range = [&](int j) { return n0 + j % out < n_out; };
    float v[4][4] = {};
    for (int k0 = 0; k0 < a.K; k0 += kStepK) {
      for (int i = tid; i < kTile * kStepK; i += 256) {
        const int r = i / kStepK, k = k0 + i % kStepK;
        float f = 0.f;
        if (r < tile.rows && k < a.K) {
          const int64_t row = tile.row + r, at = row * a.K + k;
          f = kFp8 ? e4m3(a.x[at]) * power(a.xs[row * pitch + k / kScaleBlock])
                   : bf16_at_low(reinterpret_cast<const uint16_t *>(a.x)[at]);
        }
        s_x[i % kStepK][r] = f;
      }
      for (int i = tid; i < kTile * kStepK; i += 256) {
        const int j = a.trans ? i % kTile : i / kStepK, kk = a.trans ? i / kTile : i % kStepK;
        const int k = k0 + kk;
        float f = 0.f;
        if (in_range(j) && k < a.K) {
          const int64_t n = channel(j), base = tile.w * a.w_stride;
          const int64_t at = base + (a.trans ? static_cast<int64_t>(k) * a.N + n : n * a.K + k);
          f = kFp8 ? e4m3(a.w[at]) *
                         power(a.ws[(static_cast<int64_t>(tile.w) * a.N + n) * pitch + k / kScaleBlock])
                   : bf16_at_low(reinterpret_cast<const uint16_t *>(a.w)[at]);
        }
        s_w[kk][j] = f;
      }
      __syncthreads();
      for (int k = 0; k < kStepK; ++k)
        for (int i = 0; i < 4; ++i)
          for (int j = 0; j < 4; ++j)
            v[i][j] = fmaf(s_x[k][tr + i * 16], s_w[k][tc + j * 16], v[i][j]);
      __syncthreads();
    }
    auto store = [&](int64_t at, float f) {
      if (a.bf16) static_cast<uint16_t *>(a.y)[at] = round_bf16(f);
      else static_cast<float *>(a.y)[at] = f;
    };
    for (int i = 0; i < 4; ++i) {
      const int64_t row = tile.row + tr + i * 16;
      if (tr + i * 16 >= tile.rows) continue;
      for (int j = 0; j < 4; ++j) {
        const int c = tc + j * 16, n = channel(c);
        if (!in_range(c)) continue;
        if (glu) {
          if (a.pre) a.pre[row * a.N + n] = round_bf16(v[i][j]);
          if (j < 2) store(row * half + n, v[i][j] * sigmoid(v[i][j]) * v[i][j < 2 ? j + 2 : j]);
        } else if (a.act == ULTRAEP_SWIGLU_GRAD) {
          const int64_t at = row * 2 * a.N + n;
          const float g = bf16_at_low(a.pre[at]), u = bf16_at_low(a.pre[at + a.N]);
          const Sigmoid s = sigmoid_both(g);
          store(at, v[i][j] * u * s.s * (1.f + g * s.rest));
          store(at + a.N, v[i][j] * g * s.s);
        } else {
          store(row * a.N + n, v[i][j]);
        }
      }
    }
  }
}

template <bool kFp8>
static hipError_t start_product(const ProductArgs &a, hipStream_t stream) {
  const bool glu = a.act == ULTRAEP_SWIGLU;
  const int out = glu ? kTile / 2 : kTile, n_out = glu ? a.N / 2 : a.N;
  const int32_t n_col = (n_out + out - 1) / out;
  const int64_t items = (a.M / kTile + (a.M < a.n_block ? a.M : a.n_block)) * n_col;
  const dim3 grid(static_cast<unsigned>(items < 1 << 16 ? items : 1 << 16));
  hipLaunchKernelGGL((k_product<kFp8>), grid, dim3(256), 0, stream, a, n_col);
  return hipGetLastError();
}

hipError_t launch_expert_matmul_bf16(const uint16_t *x, int64_t M, const uint16_t *w, int32_t n_w,
                                     int64_t w_stride, int32_t N, int32_t K, int32_t trans,
                                     const int64_t *block_off, const int32_t *block_w,
                                     int32_t n_block, int32_t act, uint16_t *pre, void *y,
                                     int32_t type, int32_t *status, hipStream_t stream) {
  const ProductArgs a{reinterpret_cast<const uint8_t *>(x), reinterpret_cast<const uint8_t *>(w),
                      nullptr, nullptr, block_off, block_w, pre, y, status, M, w_stride,
                      n_w, N, K, n_block, trans, act, type == ULTRAEP_BF16};
  return start_product<false>(a, stream);
}

hipError_t launch_expert_matmul_fp8(const uint8_t *xq, const uint8_t *xs, int64_t M,
                                    const uint8_t *wq, const uint8_t *ws, int32_t n_w, int32_t N,
                                    int32_t K, const int64_t *block_off, const int32_t *block_w,
                                    int32_t n_block, int32_t act, void *y, int32_t type,
                                    int32_t *status, hipStream_t stream) {
  const ProductArgs a{xq, wq, xs, ws, block_off, block_w, nullptr, y, status, M,
                      static_cast<int64_t>(N) * K, n_w, N, K, n_block, 0, act,
                      type == ULTRAEP_BF16};
  return start_product<true>(a, stream);
}

// ---------------------------------------------------------------- quantisation

// One wave a block of 128 elements, two a lane.
template <bool kBf16>
__global__ void __launch_bounds__(256)
k_quant_blocks(const char *x, int64_t rows, int32_t K, int64_t ld, uint8_t *q, int64_t ldq,
               uint8_t *scale) {
  const int lane = lane_id(), pitch = scale_pitch(K);
  const int n = static_cast<int>((ldq + kScaleBlock - 1) / kScaleBlock);
  const int64_t nw = static_cast<int64_t>(gridDim.x) * 4;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * 4 + threadIdx.x / kWave; i < rows * n; i += nw) {
    const int64_t r = i / n;
    const int b = static_cast<int>(i % n), k = b * kScaleBlock + lane * 2;
    float f[2] = {0.f, 0.f};
    for (int j = 0; j < 2; ++j)
      if (k + j < K)
        f[j] = kBf16 ? bf16_at_low(reinterpret_cast<const uint16_t *>(x)[r * ld + k + j])
                     : reinterpret_cast<const float *>(x)[r * ld + k + j];
    const int most = wave_max(max(__float_as_int(f[0]) & 0x7FFFFFFF, __float_as_int(f[1]) & 0x7FFFFFFF));
    uint8_t byte = 255, o[2] = {0x7F, 0x7F};
    if (most < 0x7F800000) {
      // 448 = 1.75 * 2^8: e = exponent - 8, one more where the mantissa is above 1.75
      const int e = max((most >> 23) - 127 - 8 + ((most & 0x7FFFFF) > 0x600000), -127);
      byte = static_cast<uint8_t>(e + 127);
      const int two = __builtin_amdgcn_cvt_pk_fp8_f32(ldexpf(f[0], -e), ldexpf(f[1], -e), 0, false);
      o[0] = static_cast<uint8_t>(two);
      o[1] = static_cast<uint8_t>(two >> 8);
    }
    for (int j = 0; j < 2; ++j)
      if (k + j < ldq) q[r * ldq + k + j] = k + j < K ? o[j] : 0;
    const int n_scale = (K + kScaleBlock - 1) / kScaleBlock;
    if (lane == 0 && b < n_scale) scale[r * pitch + b] = byte;
    if (b == 0 && lane >= n_scale % 4 && lane < 4 && n_scale % 4) scale[r * pitch + n_scale / 4 * 4 + lane] = 0;
  }
}

hipError_t launch_quant_blocks(const void *x, int32_t type, int64_t rows, int64_t K, int64_t ld,
                               uint8_t *q, int64_t ldq, uint8_t *scale, hipStream_t stream) {
  const int64_t wg = (rows * ((ldq + kScaleBlock - 1) / kScaleBlock) + 3) / 4;
  const dim3 grid(static_cast<unsigned>(wg < 1 << 20 ? wg : 1 << 20));
  const char *xs = static_cast<const char *>(x);
  if (type == ULTRAEP_BF16)
    hipLaunchKernelGGL((k_quant_blocks<true>), grid, dim3(256), 0, stream, xs, rows,
                       static_cast<int32_t>(K), ld, q, ldq, scale);
  else
    hipLaunchKernelGGL((k_quant_blocks<false>), grid, dim3(256), 0, stream, xs, rows,
                       static_cast<int32_t>(K), ld, q, ldq, scale);
  return hipGetLastError();
}

}  // namespace uep
