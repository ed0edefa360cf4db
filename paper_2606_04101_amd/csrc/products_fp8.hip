// The experts' products in 8-bit floating point (e4m3) with a scale for each 128 elements,
// and the quantisation of rows to it.
#include "products_thin.hpp"

namespace uep {

hipError_t launch_expert_matmul_fp8(const uint8_t *xq, const uint8_t *xs, int64_t M,
                                    const uint8_t *wq, const uint8_t *ws, int32_t n_w, int32_t N,
                                    int32_t K, const int64_t *block_off, const int32_t *block_w,
                                    int32_t n_block, int32_t act, void *y, int32_t type,
                                    int32_t *status, hipStream_t stream) {
  auto bytes = [](const uint8_t *p) { return reinterpret_cast<const int8_t *>(p); };
  const ProductArgs a{bytes(xq), bytes(wq), bytes(xs), bytes(ws), block_off, block_w, nullptr, y,
                      status, M, static_cast<int64_t>(N) * K, n_w, N, K, n_block, act ? N / 2 : N};
  if (act == ULTRAEP_SWIGLU) choose_type<kMath8, false, ULTRAEP_SWIGLU>(a, type, stream);
  else choose_type<kMath8, false, ULTRAEP_NO_ACT>(a, type, stream);
  return hipGetLastError();
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
