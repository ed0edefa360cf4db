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

// A lane's 8 neighbouring elements as they lie in memory.
template <bool kBf16>
struct Eight {
  v4u v[kBf16 ? 1 : 2] = {};
  template <bool kOnce>
  __device__ void load(const char *p) {
#pragma unroll
    for (int i = 0; i < (kBf16 ? 1 : 2); ++i) {
      const v4u *from = reinterpret_cast<const v4u *>(p) + i;
      v[i] = kOnce ? __builtin_nontemporal_load(from) : *from;
    }
  }
  __device__ float at(int i) const {
    if (!kBf16) return __uint_as_float(v[kBf16 ? 0 : i / 4][i % 4]);
    return i % 2 ? bf16_at_high(v[0][i / 2]) : bf16_at_low(v[0][i / 2]);
  }
  // largest magnitude, as the bits of an fp32 (an infinity or a NaN is the largest)
  __device__ int largest() const {
    int m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, __float_as_int(at(i)) & 0x7FFFFFFF);
    return m;
  }
};

// A wave takes kWords times 512 elements of a row at a time, 8 a lane: 16 lanes hold a block
// of 128, and the four blocks' scales make one word.  Every element is read once.
//   The scale is a power of two, so x * 2^-e is exact and the converter's rounding to
// nearest-even is the only one.
//   Bound by memory: 131072 rows of 7168 bf16 (2.8 GB) take 486 us, 5.8 TB/s, with 7 words
// at a time (one word 518 to 543, four 506, loads that stay in the caches 543); 131072 rows
// of 2048 126 us with 4 (two 148); 40960 of 520 15 us with 2 (7 28).  Of other lengths the last 7
// are filled in part: 131072 rows of 4096 305 us, 5.3 TB/s (the least), 5120 340, 5.9, 8192 573, 5.6.  Where there are few
// waves, or a row is one word, each takes one, with loads that may stay: 2999 rows of 2888
// 7.1 us (7.9 past the caches).
template <bool kBf16, int kWords>
__global__ void __launch_bounds__(256)
k_quant_blocks(const char *__restrict__ x, int64_t rows, int32_t K, int64_t ld, uint8_t *__restrict__ q,
               int64_t ldq, uint32_t *__restrict__ scale) {
  const int lane = lane_id(), words = scale_pitch(K) / 4;
  const int first = blockIdx.y * kWords;
  constexpr int kSize = kBf16 ? 2 : 4;
  for (int64_t r = static_cast<int64_t>(blockIdx.x) * 4 + threadIdx.x / kWave; r < rows;
       r += static_cast<int64_t>(gridDim.x) * 4) {
    Eight<kBf16> f[kWords];
#pragma unroll
    for (int u = 0; u < kWords; ++u) {
      const int k = (first + u) * 512 + lane * 8;
      if (k < K) f[u].template load<(kWords > 1)>(x + (r * ld + k) * kSize);
    }
#pragma unroll
    for (int u = 0; u < kWords; ++u) {
      const int k = (first + u) * 512 + lane * 8;
      const int most = row_max(f[u].largest());
      // 448 = 1.75 * 2^8: e is the exponent - 8, one more where the mantissa is above 1.75
      const int e = max((most >> 23) - 127 - 8 + ((most & 0x7FFFFF) > 0x600000), -127);
      const bool fine = most < 0x7F800000;
      const int byte = fine ? e + 127 : 255;
      const float by = __int_as_float((127 - e) << 23);  // 2^-e
      v2u o;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        int two = __builtin_amdgcn_cvt_pk_fp8_f32(f[u].at(4 * i) * by, f[u].at(4 * i + 1) * by, 0, false);
        two = __builtin_amdgcn_cvt_pk_fp8_f32(f[u].at(4 * i + 2) * by, f[u].at(4 * i + 3) * by, two, true);
        o[i] = k >= K ? 0u : fine ? static_cast<uint32_t>(two) : 0x7F7F7F7Fu;
      }
      if (k < ldq) __builtin_nontemporal_store(o, reinterpret_cast<v2u *>(q + r * ldq + k));
      uint32_t word = 0;  // (a block past K has none)
#pragma unroll
      for (int b = 0; b < 4; ++b)
        if ((first + u) * 512 + b * kScaleBlock < K) word |= static_cast<uint32_t>(readlane(byte, b * 16)) << (8 * b);
      if (lane == 0 && first + u < words) scale[r * words + first + u] = word;
    }
  }
}

template <bool kBf16, int kWords>
static void start_quant(const char *x, int64_t rows, int64_t K, int64_t ld, uint8_t *q, int64_t ldq,
                        uint8_t *scale, hipStream_t stream) {
  const int64_t wg = (rows + 3) / 4;
  const dim3 grid(static_cast<unsigned>(wg < 1 << 20 ? wg : 1 << 20),
                  static_cast<unsigned>((ldq + 512 * kWords - 1) / (512 * kWords)));
  hipLaunchKernelGGL((k_quant_blocks<kBf16, kWords>), grid, dim3(256), 0, stream, x, rows,
                     static_cast<int32_t>(K), ld, q, ldq, reinterpret_cast<uint32_t *>(scale));
}

hipError_t launch_quant_blocks(const void *x, int32_t type, int64_t rows, int64_t K, int64_t ld,
                               uint8_t *q, int64_t ldq, uint8_t *scale, hipStream_t stream) {
  const char *xs = static_cast<const char *>(x);
  const int64_t words = (ldq + 511) / 512;
  const int at_once = words == 1 || rows * words < 1 << 15 ? 1 : words == 2 ? 2 : words <= 4 ? 4 : 7;
#define UEP_CASE(n)                                                                       \
  if (at_once == n) {                                                                     \
    if (type == ULTRAEP_BF16) start_quant<true, n>(xs, rows, K, ld, q, ldq, scale, stream); \
    else start_quant<false, n>(xs, rows, K, ld, q, ldq, scale, stream);                   \
  }
  UEP_CASE(1) UEP_CASE(2) UEP_CASE(4) UEP_CASE(7)
#undef UEP_CASE
  return hipGetLastError();
}

}  // namespace uep
