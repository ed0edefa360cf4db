// Backward pass of the combine gather: token t's output row was the sum of its
// slots' rows y weighted by their gates, so with dout its gradient
//   dy[row] = gate * dout[t],  dgate = <dout[t], y[row]>
// in one pass: each y row is read once, each dy row written once, dout once.
//
// Bound by memory: one workgroup a token, so that dgate's sums stay in it, with up
// to 8 of the token's rows' loads in flight together; y and dy pass the caches by.
// The DeepSeek-V3-shaped training layer (4096 tokens of 8 x 7168, 999 MB) takes
// 188 us, 5.3 TB/s, where a copy of 2 GiB reaches 5.0; 201 with loads and 205 with
// stores that stay in the caches.  A small batch is bound by its chain of loads: 333
// tokens of 6 x 2880 (24 MB) take 8.5 us, of which the row index, two trips of 256 threads
// over 360 chunks, the second's loads after the first's have come, and the sum.
#include "operators.hpp"

namespace uep {

constexpr int kCgRows = 8;  // slots of a token taken together

__device__ __forceinline__ void unpack8(v4u v, float (&f)[8]) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = bf16_at_low(w[i]);
    f[2 * i + 1] = bf16_at_high(w[i]);
  }
}

__device__ __forceinline__ v4u scale8(const float (&d)[8], float g) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
    w[i] = round_bf16(g * d[2 * i]) | (round_bf16(g * d[2 * i + 1]) << 16);
  return v4u{w[0], w[1], w[2], w[3]};
}

// One workgroup a token.  The tail rows n_routed .. n_rows - 1 are shared out
// evenly over the workgroups (so a long tail behind few tokens is filled by few).
template <int kThreads>
__global__ void __launch_bounds__(kThreads)
k_combine_grad(const v4u *__restrict__ dout, const v4u *__restrict__ y, int64_t n_rows,
               const float *__restrict__ gate, const int32_t *__restrict__ row_of_slot, int64_t T,
               int32_t k, int32_t nch, const int64_t *__restrict__ n_routed_p,
               v4u *__restrict__ dy, float *__restrict__ dgate, int32_t *status) {
  constexpr int kWaves = kThreads / kWave;
  __shared__ float s_dot[kWaves][kCgRows];
  const int lane = lane_id(), wave = threadIdx.x / kWave;
  int64_t n_routed = *n_routed_p;
  const bool fits = n_routed >= 0 && n_routed <= n_rows;
  if (!fits) {
    if (blockIdx.x == 0 && threadIdx.x == 0) report(status, ULTRAEP_EDATA);
    n_routed = 0;
  }
  for (int64_t t = blockIdx.x; t < T; t += gridDim.x) {
    for (int k0 = 0; k0 < k; k0 += kCgRows) {
      int row = -1;
      float g = 0.f;
      if (lane < kCgRows && k0 + lane < k) {
        row = row_of_slot[t * k + k0 + lane];
        g = gate[t * k + k0 + lane];
        if (row < -1 || row >= n_routed) {
          if (wave == 0) report(status, ULTRAEP_EDATA);
          row = -1;
        }
      }
      float dot[kCgRows] = {};
      for (int c = threadIdx.x; c < nch; c += kThreads) {
        v4u v[kCgRows];
#pragma unroll
        for (int i = 0; i < kCgRows; ++i) {
          const int r = readlane(row, i);
          if (r >= 0) v[i] = __builtin_nontemporal_load(y + static_cast<int64_t>(r) * nch + c);
        }
        float d[8];
        unpack8(dout[t * nch + c], d);
#pragma unroll
        for (int i = 0; i < kCgRows; ++i) {
          const int r = readlane(row, i);
          if (r < 0) continue;
          float f[8];
          unpack8(v[i], f);
#pragma unroll
          for (int j = 0; j < 8; ++j) dot[i] += d[j] * f[j];
          __builtin_nontemporal_store(scale8(d, readlane_f(g, i)),
                                      dy + static_cast<int64_t>(r) * nch + c);
        }
      }
      __syncthreads();
#pragma unroll
      for (int i = 0; i < kCgRows; ++i) {
        const float s = wave_sum_f(dot[i]);
        if (lane == 0) s_dot[wave][i] = s;
      }
      __syncthreads();
      if (threadIdx.x < kCgRows && k0 + static_cast<int>(threadIdx.x) < k) {
        float s = s_dot[0][threadIdx.x];
        for (int w = 1; w < kWaves; ++w) s += s_dot[w][threadIdx.x];
        dgate[t * k + k0 + threadIdx.x] = row >= 0 ? s : 0.f;
      }
    }
  }
  if (fits) {
    const int64_t tail = n_rows - n_routed, each = (tail + gridDim.x - 1) / gridDim.x;
    const int64_t r0 = n_routed + min(tail, blockIdx.x * each), r1 = min(r0 + each, n_rows);
    for (int64_t i = r0 * nch + threadIdx.x; i < r1 * nch; i += kThreads)
      __builtin_nontemporal_store(v4u{0, 0, 0, 0}, dy + i);
  }
}

hipError_t launch_combine_grad(const uint16_t *dout, const uint16_t *y, int64_t n_rows,
                               const float *gate, const int32_t *row_of_slot, int64_t T, int32_t k,
                               int32_t H, const int64_t *n_routed, uint16_t *dy, float *dgate,
                               int32_t *status, hipStream_t stream) {
  const int64_t grid = T < 1 ? 1 : T < 1 << 20 ? T : 1 << 20;
  const int32_t nch = H / 8;
#define UEP_START(threads)                                                                    \
  hipLaunchKernelGGL((k_combine_grad<threads>), dim3(static_cast<unsigned>(grid)),            \
                     dim3(threads), 0, stream, reinterpret_cast<const v4u *>(dout),           \
                     reinterpret_cast<const v4u *>(y), n_rows, gate, row_of_slot, T, k, nch,  \
                     n_routed, reinterpret_cast<v4u *>(dy), dgate, status)
  // A row of one wave's chunks leaves the other waves idle; few tokens with long rows
  // are bound by the chunks that each thread takes one after the other.
  // us with 64 / 256 / 512 threads (tokens x slots x width):
  //   16384 x 8 x 256: 31 / 56 / 95         16384 x 8 x 1024: 107 / 104 / 121
  //   16384 x 2 x 256: 16 / 37 / 68         4096 x 8 x 7168: 189 / 189 / 188
  //   16384 x 8 x 512: 55 / 61 / 103        512 x 8 x 7168: - / 26 / 26
  //   1 x 8 x 7168: 30 / 11.3 / 9.2         64 x 8 x 2048: - / 5.5 / 6.9
  //   128 x 8 x 7168: - / 13.2 / 11.1       2000 x 6 x 1024: 12.6 / 13.7 / 16.6
  if (nch <= kWave)
    UEP_START(64);
  else if (T <= 256 && nch > 512)
    UEP_START(512);
  else
    UEP_START(256);
#undef UEP_START
  return hipGetLastError();
}

}  // namespace uep
