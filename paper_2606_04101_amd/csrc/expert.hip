// The experts' products on 8-bit integers: the quantisation of rows, and the
// product of each dispatched block of rows with its expert's weight.
#include <type_traits>

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
  int32_t n_w, N, K, n_block, n_out;
};

constexpr int kMmMaxBlocks = 2048;

// Row tiles are numbered block by block.  cum[g] becomes the number of tiles
// before block g, cum[n_block] that of all; a block that is out of order or out
// of [0, M], or has rows and no weight, is reported and has none.
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
template <int kThreads>
__device__ void count_tiles(const MatmulArgs &a, int tile_rows, int *cum, int *wave_sums) {
  const int tid = threadIdx.x, lane = lane_id(), wave = tid / kWave;
  const int per = (a.n_block + kThreads - 1) / kThreads;  // blocks of a thread
  int mine = 0;
  bool bad = false;
  for (int j = 0; j < per; ++j) {
    const int g = tid * per + j;
    if (g < a.n_block)
      mine += static_cast<int>((block_rows(a, g, bad) + tile_rows - 1) / tile_rows);
  }
  if (bad && blockIdx.x == 0) report(a.status, ULTRAEP_EDATA);
  const int incl = wave_scan_incl(mine);
  if (lane == kWave - 1) wave_sums[wave] = incl;
  __syncthreads();
  int at = incl - mine;
  for (int w = 0; w < wave; ++w) at += wave_sums[w];
  for (int j = 0; j < per; ++j) {
    const int g = tid * per + j;
    if (g < a.n_block) {
      cum[g] = at;
      at += static_cast<int>((block_rows(a, g, bad) + tile_rows - 1) / tile_rows);
      if (g == a.n_block - 1) cum[a.n_block] = at;
    }
  }
  __syncthreads();
}

__device__ __forceinline__ int64_t uniform(int64_t v) {
  const uint32_t lo = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(v));
  const uint32_t hi = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(v >> 32));
  return static_cast<int64_t>(static_cast<uint64_t>(hi) << 32 | lo);
}

// v, with what follows from it computed where it is used: a persistent loop would
// otherwise hold every lane's address of its rare parts in registers throughout
__device__ __forceinline__ int opaque(int v) {
  asm volatile("" : "+v"(v));
  return v;
}

// Tile `tile` < cum[n_block]: its first row, rows and weight.  Every lane must
// be active; all results are uniform.
struct RowTile {
  int64_t row;
  int32_t rows, w;
};
__device__ __forceinline__ RowTile find_tile(const MatmulArgs &a, const int *cum, int tile,
                                             int tile_rows) {
  // the last block that begins at or before the tile, among equals the last,
  // which is the one with tiles: first its run of 64 blocks, then the block
  const int lane = lane_id();
  int g = 0;
  if (a.n_block > kWave) {
    const int j = lane * kWave;
    g = (__builtin_popcountll(ballot(j < a.n_block && cum[min(j, a.n_block)] <= tile)) - 1) * kWave;
  }
  const int j = g + lane;
  g += __builtin_popcountll(ballot(j < a.n_block && cum[min(j, a.n_block)] <= tile)) - 1;
  g = __builtin_amdgcn_readfirstlane(g);
  const int64_t r = static_cast<int64_t>(tile - __builtin_amdgcn_readfirstlane(cum[g])) * tile_rows;
  const int64_t lo = uniform(a.block_off[g]), n = uniform(a.block_off[g + 1]) - lo;
  return {lo + r, __builtin_amdgcn_readfirstlane(static_cast<int>(min<int64_t>(n - r, tile_rows))),
          __builtin_amdgcn_readfirstlane(a.block_w ? a.block_w[g] : g)};
}

__device__ __forceinline__ float silu(float v) { return v / (1.f + expf(-v)); }

// 16 bytes a lane from base + off straight into LDS, lane l's at lds + 16 l.
// The wait for it is the caller's (vmcnt).
__device__ __forceinline__ void load_to_lds(const void *base, uint32_t off, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
               :
               : "s"(lds), "v"(off), "s"(base)
               : "memory");
}

// the same for 4 bytes a lane
__device__ __forceinline__ void load_word_to_lds(const void *base, uint32_t off, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2"
               :
               : "s"(lds), "v"(off), "s"(base)
               : "memory");
}
template <class T>
__device__ __forceinline__ uint32_t lds_address(T *p) {
  return static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) T *)p));
}

constexpr int kBk = 128;  // bytes of K of a step

// Output tile of kN weight rows x kM rows, K in steps of 128 bytes through two
// LDS buffers; kWn x kWm waves.  The weights are the MFMA's first operand, so a
// lane holds 4 neighbouring channels of one row.  With act, a wave's parts of 32
// weight rows alternate between gates and their partners.
template <int kN, int kM, int kWn, int kWm, bool kAct, bool kBf16>
__global__ void __launch_bounds__(64 * kWn *kWm) k_matmul(MatmulArgs a, int32_t n_col) {
  constexpr int kThreads = 64 * kWn * kWm, kWaves = kWn * kWm;
  constexpr int kFn = kN / kWn / 32, kFm = kM / kWm / 32;  // 32 x 32 parts of a wave
  constexpr int kBuf = (kN + kM) * kBk;
  constexpr int kLoads = kBuf / 1024 / kWaves;             // of a wave in a step
  constexpr int kLoadsN = kLoads * kN / (kN + kM);
  constexpr int kOut = kAct ? kN / 2 : kN;                 // channels of a tile
  constexpr int kOutW = kOut / kWn;                        // of a wave
  __shared__ __align__(1024) int8_t s_buf[2][kBuf];
  __shared__ __align__(16) int8_t s_out[kWaves][4096];
  __shared__ __align__(16) float s_scale[2][kN + kM];  // of this item and of the next
  __shared__ int s_cum[kMmMaxBlocks + 1];
  __shared__ int s_sums[kWaves];
  const int tid = threadIdx.x, lane = lane_id();
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int wn = wave % kWn, wm = wave / kWn;
  const int lr = lane & 31, hi = lane >> 5;
  const int half = a.N / 2;
  count_tiles<kThreads>(a, kM, s_cum, s_sums);
  const int n_tile = __builtin_amdgcn_readfirstlane(s_cum[a.n_block]);
  const int n_item = n_tile * n_col;  // (a y that fits the memory has fewer than 2^31)

  // the workgroups of one XCD (those of equal number modulo 8) take neighbouring
  // items, 8 row tiles by 4 column tiles at a time
  constexpr int kXcd = 8, kGroup = 8;
  const int per_xcd = gridDim.x / kXcd;  // the grid is a multiple
  const int slot = blockIdx.x % kXcd * per_xcd + blockIdx.x / kXcd;
  const uint32_t lds0 = lds_address(&s_buf[0][0]), lds_scale = lds_address(&s_scale[0][0]);
  const int steps = (a.K + kBk - 1) / kBk;
  const int tail = (a.K - (steps - 1) * kBk) / 16;  // chunks of the last step

  // an item: its rows and weight, its first channel
  RowTile tile;
  int n0;
  // byte offsets of this lane's loads: 8 rows of 8 chunks an instruction; chunk c of
  // tile row r lies at c ^ (r / 2 % 8), so that 16 neighbouring rows' lie in all banks
  const int8_t *wbase, *xbase;
  uint32_t off[kLoads];
  int turn = 1;  // which half of s_scale the item's scales are in
  const int chunk = (lane & 7) ^ ((wave & 1) * 4 + (lane >> 4));
  auto aim = [&](int item) {
    const int lane = opaque(lane_id());
    const int chunk = (lane & 7) ^ ((wave & 1) * 4 + (lane >> 4));
    const int group = item / (kGroup * n_col), rest = item - group * kGroup * n_col;
    const int high = min(kGroup, n_tile - group * kGroup);
    tile = find_tile(a, s_cum, group * kGroup + rest % high, kM);
    n0 = rest / high * kOut;
    wbase = a.wq + static_cast<int64_t>(tile.w) * a.N * a.K;
    xbase = a.xq + tile.row * a.K;
    // weight row of tile row j, in range for any j
    auto weight_row = [&](int j) {
      if (!kAct) return min(n0 + j, a.N - 1);
      return min(n0 + j / 64 * 32 + j % 32, half - 1) + (j % 64 >= 32 ? half : 0);
    };
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int j = ((i < kLoadsN ? i : i - kLoadsN) * kWaves + wave) * 8 + (lane >> 3);
      const int r = i < kLoadsN ? weight_row(j) : min(j, tile.rows - 1);
      off[i] = static_cast<uint32_t>(r) * a.K + chunk * 16;
    }
    const float *ws = a.ws + static_cast<int64_t>(tile.w) * a.N, *xs = a.xs + tile.row;
    turn ^= 1;
#pragma unroll
    for (int i = 0; i < (kN + kM) / kWave / kWaves; ++i) {
      const int j = (i * kWaves + wave) * kWave;  // the same operand for all lanes
      const int r = j < kN ? weight_row(j + lane) : min(j - kN + lane, tile.rows - 1);
      load_word_to_lds(j < kN ? ws : xs, r * 4,
                       __builtin_amdgcn_readfirstlane(lds_scale + (turn * (kN + kM) + j) * 4));
    }
  };
  // load i of a step; chunks past K (in the last step) are loaded from the step's
  // first one and not used
  auto issue = [&](int s, int i) {
    const uint32_t back = s == steps - 1 && chunk >= tail ? chunk * 16 : 0;
    load_to_lds((i < kLoadsN ? wbase : xbase) + static_cast<int64_t>(s) * kBk, off[i] - back,
                __builtin_amdgcn_readfirstlane(lds0 + (s & 1) * kBuf + (i * kWaves + wave) * 1024));
  };
  auto begin = [&](int item) {
    aim(item);
#pragma unroll
    for (int i = 0; i < kLoads; ++i) issue(0, i);
    if (steps > 1) {
#pragma unroll
      for (int i = 0; i < kLoads; ++i) issue(1, i);
    }
  };

  int item = slot;
  if (item >= n_item) return;
  begin(item);
  if (steps > 1)
    asm volatile("s_waitcnt vmcnt(%0)" : : "n"(kLoads) : "memory");
  else
    asm volatile("s_waitcnt vmcnt(0)" : : : "memory");
  while (true) {
    asm volatile("s_barrier" : : : "memory");
    v16i acc[kFn][kFm] = {};
    v4i fw[2][kFn], fx[2][kFm];
    // part f of the operands for 32 bytes kk of a step
    auto fetch = [&](int s, int kk, int f) {
      const int8_t *b = s_buf[s & 1] + ((kk * 2 + hi) ^ (lr >> 1 & 7)) * 16;
      if (f < kFn)
        fw[kk & 1][f] = *reinterpret_cast<const v4i *>(b + (wn * kFn * 32 + f * 32 + lr) * kBk);
      else
        fx[kk & 1][f - kFn] = *reinterpret_cast<const v4i *>(
            b + (kN + wm * kFm * 32 + (f - kFn) * 32 + lr) * kBk);
    };
    // One step, its first parts already in registers.  The products run in the
    // order that keeps the matrix unit fed: reads of the next parts, and at the
    // step's end the loads of the step after the next, between them.  kAhead: how
    // many steps follow, up to 2.
    auto step = [&](int s, auto ahead) {
      constexpr int kAhead = decltype(ahead)::value;
#pragma unroll
      for (int kk = 0; kk < 4; ++kk) {
        if (kk == 3)  // the next step's bytes are there, and nobody reads this step's any more
          asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" : : : "memory");
        if (kAhead == 0 && kk * 2 + 1 >= tail) {
#pragma unroll
          for (int j = 0; j < kFm; ++j)
            if (kk * 2 + hi >= tail) fx[kk & 1][j] = v4i{0, 0, 0, 0};
        }
        constexpr int kAll = kFn * kFm, kParts = kFn + kFm;
#pragma unroll
        for (int m = 0; m < kAll; ++m) {
          const int i = m / kFm, j = m % kFm;
          acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(fw[kk & 1][i], fx[kk & 1][j], acc[i][j],
                                                            0, 0, 0);
          // spread evenly over the products
          for (int f = m * kParts / kAll; f < (m + 1) * kParts / kAll; ++f) {
            if (kk < 3) fetch(s, kk + 1, f);
            else if (kAhead > 0) fetch(s + 1, 0, f);
          }
          if (kk == 3 && kAhead == 2)
            for (int f = m * kLoads / kAll; f < (m + 1) * kLoads / kAll; ++f) issue(s + 2, f);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    };

#pragma unroll
    for (int f = 0; f < kFn + kFm; ++f) fetch(0, 0, f);
    int s = 0;
    for (; s < steps - 2; ++s) step(s, std::integral_constant<int, 2>());
    if (s < steps - 1) step(s++, std::integral_constant<int, 1>());
    step(s, std::integral_constant<int, 0>());

    // the next item's first loads fly while this one's results leave
    const RowTile out = tile;
    const int nw = n0 + wn * kOutW;  // the wave's first channel
    const int was = turn;
    item += gridDim.x;
    const bool more = item < n_item;
    if (more) begin(item);

    // 32 rows x 64 channels (32 in fp32) at a time through LDS, so that a row's
    // channels leave in whole lines
    constexpr int kParts = kOutW / 32;
    const int el = opaque(lane), er = el & 31, eh = el >> 5;
    const float *scale = s_scale[was];
    int8_t *stage = s_out[wave];
#pragma unroll
    for (int j = 0; j < kFm; ++j) {
      const int r0 = (wm * kFm + j) * 32;
      const float xs = scale[kN + r0 + er];
      // the sums stay in the accumulation registers until here
#pragma unroll
      for (int i = 0; i < kFn; ++i) asm volatile("" : "+a"(acc[i][j]));
      // before the last stores: all loads, and the earlier stores, are done (and
      // nothing read from LDS is held in registers from one part to the next)
      if (j == kFm - 1) asm volatile("s_waitcnt vmcnt(0)" : : : "memory");
      else asm volatile("" : : : "memory");
#pragma unroll
      for (int i = 0; i < kParts; ++i) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int f = kAct ? 2 * i : i;
          const float *of = scale + wn * kFn * 32 + f * 32 + q * 8 + eh * 4;
          const v4f w0 = *reinterpret_cast<const v4f *>(of);
          float v[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = static_cast<float>(acc[f][j][q * 4 + e]) * xs * w0[e];
          if (kAct) {
            const v4f w1 = *reinterpret_cast<const v4f *>(of + 32);
#pragma unroll
            for (int e = 0; e < 4; ++e)
              v[e] = silu(v[e]) *
                     (static_cast<float>(acc[kAct ? f + 1 : 0][j][q * 4 + e]) * xs * w1[e]);
          }
          // 16-byte slots of the stage's 128-byte row, exchanged by the row
          if (kBf16) {
            const int at = ((i & 1) * 4 + q) ^ (er & 7);
            *reinterpret_cast<v2u *>(stage + er * 128 + at * 16 + eh * 8) =
                v2u{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
          } else {
            const int at = (q * 2 + eh) ^ (er & 7);
            *reinterpret_cast<v4f *>(stage + er * 128 + at * 16) = v4f{v[0], v[1], v[2], v[3]};
          }
        }
        if (kBf16 && (i & 1) == 0 && i + 1 < kParts) continue;
        const int c0 = nw + (kBf16 ? i / 2 * 64 : i * 32), esize = kBf16 ? 2 : 4;
        const int c = (el & 7) * (16 / esize);
#pragma unroll
        for (int p = 0; p < 4; ++p) {
          const int r = p * 8 + el / 8;
          const v4u o = *reinterpret_cast<const v4u *>(stage + r * 128 + ((el & 7) ^ (r & 7)) * 16);
          if (r0 + r < out.rows && c0 + c < min(a.n_out, nw + kOutW))
            *reinterpret_cast<v4u *>(static_cast<char *>(a.y) +
                                     ((out.row + r0 + r) * a.n_out + c0 + c) * esize) = o;
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    if (!more) return;
  }
}

template <int kN, int kM, int kWn, int kWm>
static void start_matmul(const MatmulArgs &a, bool act, bool bf16, int n_cu, hipStream_t stream) {
  const int out = act ? kN / 2 : kN;
  const int32_t n_col = (a.n_out + out - 1) / out;
  // every block may end in a part of a tile
  const int64_t items = ((a.M + kM - 1) / kM + a.n_block) * n_col;
  const dim3 grid(static_cast<unsigned>(items < n_cu ? (items + 7) / 8 * 8 : n_cu)), block(64 * kWn * kWm);
  if (act && bf16)
    hipLaunchKernelGGL((k_matmul<kN, kM, kWn, kWm, true, true>), grid, block, 0, stream, a, n_col);
  else if (act)
    hipLaunchKernelGGL((k_matmul<kN, kM, kWn, kWm, true, false>), grid, block, 0, stream, a, n_col);
  else if (bf16)
    hipLaunchKernelGGL((k_matmul<kN, kM, kWn, kWm, false, true>), grid, block, 0, stream, a, n_col);
  else
    hipLaunchKernelGGL((k_matmul<kN, kM, kWn, kWm, false, false>), grid, block, 0, stream, a, n_col);
}

hipError_t launch_expert_matmul(const int8_t *xq, const float *xs, int64_t M, const int8_t *wq,
                                const float *ws, int32_t n_w, int32_t N, int32_t K,
                                const int64_t *block_off, const int32_t *block_w, int32_t n_block,
                                int32_t act, void *y, int32_t type, int32_t *status,
                                hipStream_t stream) {
  const MatmulArgs a{xq, xs, wq, ws, block_off, block_w, y, status, M, n_w, N, K, n_block,
                     act ? N / 2 : N};
  start_matmul<256, 256, 2, 2>(a, act, type == ULTRAEP_BF16, 256, stream);
  return hipGetLastError();
}

}  // namespace uep
