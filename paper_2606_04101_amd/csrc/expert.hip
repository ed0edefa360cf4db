// The experts' products on 8-bit integers: the quantisation of rows, and the
// product of each dispatched block of rows with its expert's weight.
#include "operators.hpp"

namespace uep {

// ---------------------------------------------------------------- quantisation

constexpr int kQrThreads = 256;
constexpr int kQrWaves = kQrThreads / kWave;

// eight elements as fp32, from chunk c of a row
template <bool kBf16>
__device__ __forceinline__ void load8(const void *row, int64_t c, float (&f)[8]) {
  if (kBf16) {
    const v4u v = static_cast<const v4u *>(row)[c];
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = bf16_at_low(w[i]);
      f[2 * i + 1] = bf16_at_high(w[i]);
    }
  } else {
    const v4f a = static_cast<const v4f *>(row)[2 * c], b = static_cast<const v4f *>(row)[2 * c + 1];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[i] = a[i];
      f[4 + i] = b[i];
    }
  }
}

// Eight integers of a row with inverse scale inv.  The product is at most
// 127 (1 + 2^-23), so no rounding leaves [-127, 127].
__device__ __forceinline__ v2u quantise8(const float (&f)[8], float inv) {
  uint32_t w[2] = {0, 0};
#pragma unroll
  for (int i = 0; i < 8; ++i)
    w[i / 4] |= (static_cast<uint32_t>(static_cast<int>(rintf(f[i] * inv))) & 255u) << (8 * (i % 4));
  return v2u{w[0], w[1]};
}

// One wave a row, read twice (the second time from the cache).
template <bool kBf16>
__global__ void __launch_bounds__(kQrThreads)
k_quant_rows(const char *__restrict__ x, int64_t rows, int32_t nch, int64_t row_bytes,
             int8_t *__restrict__ q, int32_t nqch, float *__restrict__ scale) {
  const int lane = lane_id();
  const int64_t nw = static_cast<int64_t>(gridDim.x) * kQrWaves;
  for (int64_t r = static_cast<int64_t>(blockIdx.x) * kQrWaves + threadIdx.x / kWave; r < rows;
       r += nw) {
    const char *row = x + r * row_bytes;
    // |x| as integers: an infinity or a NaN is the largest
    int most = 0;
    for (int c = lane; c < nch; c += kWave) {
      float f[8];
      load8<kBf16>(row, c, f);
#pragma unroll
      for (int i = 0; i < 8; ++i) most = max(most, __float_as_int(f[i]) & 0x7FFFFFFF);
    }
    const float a = __int_as_float(wave_max(most));
    const bool finite = a < __builtin_inff(), live = finite && a > 0x1p-100f;
    const float inv = live ? 127.f / a : 0.f;
    if (lane == 0) scale[r] = live ? a / 127.f : finite ? 0.f : __builtin_nanf("");
    v2u *out = reinterpret_cast<v2u *>(q) + r * nqch;
    for (int c = lane; c < nqch; c += kWave) {
      v2u o{0, 0};
      if (live && c < nch) {
        float f[8];
        load8<kBf16>(row, c, f);
        o = quantise8(f, inv);
      }
      out[c] = o;
    }
  }
}

hipError_t launch_quant_rows(const void *x, int32_t type, int64_t rows, int64_t K, int64_t ld,
                             int8_t *q, int64_t ldq, float *scale, hipStream_t stream) {
  const int64_t wg = (rows + kQrWaves - 1) / kQrWaves;
  const dim3 grid(static_cast<unsigned>(wg < 65536 ? wg : 65536));
  const char *xs = static_cast<const char *>(x);
  const int32_t nch = static_cast<int32_t>(K / 8), nqch = static_cast<int32_t>(ldq / 8);
  if (type == ULTRAEP_BF16)
    hipLaunchKernelGGL((k_quant_rows<true>), grid, dim3(kQrThreads), 0, stream, xs, rows, nch, ld * 2,
                       q, nqch, scale);
  else
    hipLaunchKernelGGL((k_quant_rows<false>), grid, dim3(kQrThreads), 0, stream, xs, rows, nch,
                       ld * 4, q, nqch, scale);
  return hipGetLastError();
}

// -------------------------------------------------------------------- products

typedef int32_t v16i __attribute__((ext_vector_type(16)));

struct MatmulArgs {
  const int8_t *xq;
  const float *xs;
  const int8_t *wq;
  const float *ws;
  const int64_t *block_off;
  const int32_t *block_w;
  void *y;
  int32_t *status;
  int64_t M;
  int32_t n_w, N, K, n_block, n_out, bf16;
};

constexpr int kMmThreads = 256;
constexpr int kMmMaxBlocks = 2048;
constexpr int kMmPer = kMmMaxBlocks / kMmThreads;  // blocks a thread looks at

// Row tiles are numbered block by block.  The workgroup finds the block and the
// first row of tile `tile` by a scan over the blocks' tile counts; .rows is 0
// past the last tile.  A block that is out of order or out of [0, M], or has
// rows and no weight, has no tile.
struct RowTile {
  int64_t row;
  int32_t rows, w;
};
__device__ __forceinline__ int64_t block_rows(const MatmulArgs &a, int g, bool &bad) {
  const int64_t lo = a.block_off[g], hi = a.block_off[g + 1];
  if (lo < 0 || hi < lo || hi > a.M) {
    bad = true;
    return 0;
  }
  if (hi > lo) {
    const int w = a.block_w ? a.block_w[g] : g;
    if (w < 0 || w >= a.n_w) {
      bad = true;
      return 0;
    }
  }
  return hi - lo;
}
__device__ RowTile find_tile(const MatmulArgs &a, int64_t tile, int tile_rows) {
  __shared__ int s_wave[kMmThreads / kWave];
  __shared__ RowTile s_tile;
  const int tid = threadIdx.x, lane = lane_id(), wave = tid / kWave;
  if (tid == 0) s_tile = {0, 0, 0};
  int mine = 0;
  bool bad = false;
  for (int j = 0; j < kMmPer; ++j) {
    const int g = tid * kMmPer + j;
    if (g < a.n_block)
      mine += static_cast<int>((block_rows(a, g, bad) + tile_rows - 1) / tile_rows);
  }
  if (bad) report(a.status, ULTRAEP_EDATA);
  const int incl = wave_scan_incl(mine);
  if (lane == kWave - 1) s_wave[wave] = incl;
  __syncthreads();
  int64_t at = incl - mine;
  for (int w = 0; w < wave; ++w) at += s_wave[w];
  if (tile >= at && tile < at + mine) {
    for (int j = 0; j < kMmPer; ++j) {
      const int g = tid * kMmPer + j;
      if (g >= a.n_block) break;
      const int64_t n = block_rows(a, g, bad);
      const int64_t tiles = (n + tile_rows - 1) / tile_rows;
      if (tile < at + tiles) {
        const int64_t r = (tile - at) * tile_rows;
        s_tile = {a.block_off[g] + r, static_cast<int32_t>(n - r < tile_rows ? n - r : tile_rows),
                  a.block_w ? a.block_w[g] : g};
        break;
      }
      at += tiles;
    }
  }
  __syncthreads();
  return s_tile;
}

__device__ __forceinline__ float silu(float v) { return v / (1.f + expf(-v)); }

// Tile of 128 channels x 128 rows, K in steps of 64 bytes through LDS; four
// waves of 64 x 64 each.  The weights are the MFMA's first operand, so a lane
// holds 4 neighbouring channels of one row.  With act, channels 0..31 of each
// wave's 64 are gates and the other 32 their partners.
constexpr int kBn = 128, kBm = 128, kBk = 64;

// byte of 16-byte chunk c of tile row r in LDS, chunks exchanged so that eight
// neighbouring rows lie in all banks
__device__ __forceinline__ int lds_at(int r, int c) { return r * kBk + ((c ^ ((r >> 1) & 3)) * 16); }

template <bool kAct>
__global__ void __launch_bounds__(kMmThreads) k_matmul(MatmulArgs a, int64_t n_item, int32_t n_col) {
  __shared__ __align__(16) int8_t s_w[kBn * kBk];
  __shared__ __align__(16) int8_t s_x[kBm * kBk];
  for (int64_t item = blockIdx.x; item < n_item; item += gridDim.x) {
    const RowTile tile = find_tile(a, item / n_col, kBm);
    if (tile.rows == 0) return;  // past the last tile, as are all later items
    const int tid = threadIdx.x, lane = lane_id(), wave = tid / kWave;
    const int wn = wave & 1, wm = wave >> 1;
    const int half = kAct ? a.N / 2 : 0;
    const int n0 = static_cast<int>(item % n_col) * (kAct ? kBn / 2 : kBn);  // first output channel
    // weight row of tile row j, in range for any j
    auto weight_row = [&](int j) {
      if (!kAct) return min(n0 + j, a.N - 1);
      const int o = n0 + (j / 64) * 32 + j % 32;
      return min(o, half - 1) + (j % 64 >= 32 ? half : 0);
    };
    const int8_t *w = a.wq + static_cast<int64_t>(tile.w) * a.N * a.K;
    const int8_t *x = a.xq + tile.row * a.K;

    v16i acc[2][2] = {};
    const int nk = a.K / 16;  // 16-byte chunks of a row
    for (int k0 = 0; k0 < nk; k0 += kBk / 16) {
      __syncthreads();
  #pragma unroll
      for (int j = 0; j < kBn * kBk / 16 / kMmThreads; ++j) {
        const int i = tid + j * kMmThreads, r = i / 4, c = i % 4;
        v4i vw = {0, 0, 0, 0}, vx = {0, 0, 0, 0};
        if (k0 + c < nk) {
          vw = *reinterpret_cast<const v4i *>(w + static_cast<int64_t>(weight_row(r)) * a.K + (k0 + c) * 16);
          vx = *reinterpret_cast<const v4i *>(x + static_cast<int64_t>(min(r, tile.rows - 1)) * a.K + (k0 + c) * 16);
        }
        *reinterpret_cast<v4i *>(s_w + lds_at(r, c)) = vw;
        *reinterpret_cast<v4i *>(s_x + lds_at(r, c)) = vx;
      }
      __syncthreads();
  #pragma unroll
      for (int kk = 0; kk < kBk / 32; ++kk) {
        const int c = kk * 2 + lane / 32;
        v4i fw[2], fx[2];
  #pragma unroll
        for (int i = 0; i < 2; ++i) {
          fw[i] = *reinterpret_cast<const v4i *>(s_w + lds_at(wn * 64 + i * 32 + lane % 32, c));
          fx[i] = *reinterpret_cast<const v4i *>(s_x + lds_at(wm * 64 + i * 32 + lane % 32, c));
        }
  #pragma unroll
        for (int i = 0; i < 2; ++i)
  #pragma unroll
          for (int j = 0; j < 2; ++j)
            acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(fw[i], fx[j], acc[i][j], 0, 0, 0);
      }
    }

    // lane: row lane % 32 of a 32 x 32 part, channels 8 (i / 4) + 4 (lane / 32) + i % 4
    const float *ws = a.ws + static_cast<int64_t>(tile.w) * a.N;
  #pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int r = wm * 64 + j * 32 + lane % 32;
      if (r >= tile.rows) continue;
      const float xs = a.xs[tile.row + r];
      char *out = static_cast<char *>(a.y) + (tile.row + r) * a.n_out * (a.bf16 ? 2 : 4);
  #pragma unroll
      for (int i = 0; i < (kAct ? 1 : 2); ++i) {
  #pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int n = n0 + wn * (kAct ? 32 : 64) + i * 32 + q * 8 + lane / 32 * 4;
          if (n >= a.n_out) continue;
          float v[4];
  #pragma unroll
          for (int e = 0; e < 4; ++e) {
            v[e] = static_cast<float>(acc[i][j][q * 4 + e]) * xs * ws[n + e];
            if (kAct)
              v[e] = silu(v[e]) * (static_cast<float>(acc[1][j][q * 4 + e]) * xs * ws[half + n + e]);
          }
          if (a.bf16)
            *reinterpret_cast<v2u *>(out + n * 2) =
                v2u{round_bf16(v[0]) | (round_bf16(v[1]) << 16), round_bf16(v[2]) | (round_bf16(v[3]) << 16)};
          else
            *reinterpret_cast<v4f *>(out + n * 4) = v4f{v[0], v[1], v[2], v[3]};
        }
      }
    }
  }
}

hipError_t launch_expert_matmul(const int8_t *xq, const float *xs, int64_t M, const int8_t *wq,
                                const float *ws, int32_t n_w, int32_t N, int32_t K,
                                const int64_t *block_off, const int32_t *block_w, int32_t n_block,
                                int32_t act, void *y, int32_t type, int32_t *status,
                                hipStream_t stream) {
  const int n_out = act ? N / 2 : N;
  const MatmulArgs a{xq, xs, wq, ws, block_off, block_w, y, status, M, n_w, N, K, n_block, n_out,
                     type == ULTRAEP_BF16};
  const int bn = act ? kBn / 2 : kBn;
  // every block may end in a part of a tile
  const int64_t tiles = (M + kBm - 1) / kBm + n_block;
  const int32_t n_col = (n_out + bn - 1) / bn;
  const int64_t n_item = tiles * n_col;
  const dim3 grid(static_cast<unsigned>(n_item < 1 << 23 ? n_item : 1 << 23));
  if (act)
    hipLaunchKernelGGL((k_matmul<true>), grid, dim3(kMmThreads), 0, stream, a, n_item, n_col);
  else
    hipLaunchKernelGGL((k_matmul<false>), grid, dim3(kMmThreads), 0, stream, a, n_item, n_col);
  return hipGetLastError();
}

}  // namespace uep
