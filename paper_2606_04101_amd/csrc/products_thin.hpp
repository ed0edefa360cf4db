// The floating-point products of few rows a block.  Internal header.
#pragma once

#include <cmath>

#include "products.hpp"

namespace uep {

// Few rows a block: the weight's bytes bound the call.  A workgroup takes kRows weight
// rows (with SwiGLU half of them gates, then their partners) and up to kTok rows; its waves
// share K in steps of 128 bytes in turn, each through an LDS ring of its own that kDeep
// steps fill, so no wave waits for another until they add their sums.  16 rows over 9 experts,
// N = 4096, K = 7168 in 8 bits take 48 us, 5.5 TB/s of the weights' 264 MB; one row in bf16,
// N = 4096, K = 7168: 11.4 us, 5.1 TB/s.
template <int kTok, int kRows, int kWaves, int kDeep, Math kKind, int kAct, bool kBf16>
__global__ void __launch_bounds__(64 * kWaves) k_product_thin(ProductArgs a, int32_t n_col) {
  constexpr bool kGlu = kAct == ULTRAEP_SWIGLU, kFp8 = kKind != kMath16;
  constexpr int kThreads = 64 * kWaves, kFm = kTok / 16, kFn = kRows / 16, kEsize = kFp8 ? 1 : 2;
  constexpr int kOut = kGlu ? kRows / 2 : kRows;
  constexpr int kPitch = kRows + 4;          // words of a row's sums
  constexpr int kScales = kFp8 ? 2 : 0;      // loads of a step's scales
  constexpr int kScaleAt = (kRows + kTok) * kBk;
  constexpr int kStep = kScaleAt + kScales * 256;
  constexpr int kLoadsN = kRows / 8, kLoads = (kRows + kTok) / 8;
  constexpr int kRing = kDeep * kStep;
  static_assert(kTok * kPitch * 4 <= kRing, "a wave's sums take the place of its ring");
  static_assert(kRows <= 64 && kTok <= 64, "one load takes a side's scales");
  __shared__ __align__(1024) int8_t s_ring[kWaves][kRing];
  const int tid = threadIdx.x, lane = lane_id();
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int lr = lane & 15, lc = lane >> 4;
  const int half = a.N / 2;
  RowTiles<kTok> tiles;
  tiles.count(a, reinterpret_cast<int *>(s_ring[0]), wave, kWaves);
  const int n_item = tiles.total * n_col;
  const int n_chunk = a.K * kEsize / 16, steps = (a.K * kEsize + kBk - 1) / kBk;
  const int scale_row = scale_pitch(a.K);
  const uint32_t lds0 = __builtin_amdgcn_readfirstlane(lds_address(&s_ring[wave][0]));

  for (int item = blockIdx.x; item < n_item; item += gridDim.x) {
    const RowTile tile = tiles.find(a, item / n_col);
    const int n0 = item % n_col * kOut;
    const int8_t *w = uniform(a.w + (tile.w * a.w_stride + static_cast<int64_t>(n0) * a.K) * kEsize);
    const int8_t *w2 = w + static_cast<int64_t>(half) * a.K * kEsize;  // the gates' partners
    const int8_t *x = uniform(a.x + tile.row * a.K * kEsize);
    // the weight row, after n0 (of gates or partners), and the row of a row of the tile
    auto weight_row = [&](int j) { return kGlu ? min(j % kOut, half - 1 - n0) : min(j, a.N - 1 - n0); };
    auto row = [&](int j) { return min(j, tile.rows - 1); };
    // byte offsets of this lane's rows: 8 rows of 8 chunks an instruction, chunk c of
    // row r at c ^ (r / 2 % 8)
    uint32_t off[kLoads], off_ws = 0, off_xs = 0;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int j = (i < kLoadsN ? i : i - kLoadsN) * 8 + (lane >> 3);
      off[i] = static_cast<uint32_t>(i >= kLoadsN ? row(j) : weight_row(j)) * (a.K * kEsize);
    }
    const int8_t *ws = nullptr, *xs = nullptr;
    if (kFp8) {
      ws = uniform(a.ws + (static_cast<int64_t>(tile.w) * a.N + n0) * scale_row);
      xs = uniform(a.xs + tile.row * scale_row);
      const int j = min(lane, kRows - 1);
      off_ws = static_cast<uint32_t>(weight_row(j) + (kGlu && j >= kOut ? half : 0)) * scale_row;
      off_xs = static_cast<uint32_t>(row(min(lane, kTok - 1))) * scale_row;
    }
    // step s of the wave into part `slot` of the ring; what lies past K is loaded from its
    // last chunk and not used
    const int chunk = (lane & 7) ^ (lane >> 4);
    auto issue = [&](int s, int slot) {
      const uint32_t at[2] = {min(s * 8 + chunk, n_chunk - 1) * 16u, min(s * 8 + (chunk ^ 4), n_chunk - 1) * 16u};
#pragma unroll
      for (int i = 0; i < kLoads; ++i)
        load_to_lds(i >= kLoadsN ? x : kGlu && i >= kLoadsN / 2 ? w2 : w, off[i] + at[i & 1],
                    __builtin_amdgcn_readfirstlane(lds0 + slot * kStep + i * 1024));
      if (kFp8) {  // the words that hold the step's scales
        const uint32_t word = min(s >> 2, scale_row / 4 - 1) * 4u;
        const uint32_t to = __builtin_amdgcn_readfirstlane(lds0 + slot * kStep + kScaleAt);
        load_word_to_lds(ws, off_ws + word, to);
        load_word_to_lds(xs, off_xs + word, to + 256);
      }
    };

    v4f acc[kFn][kFm] = {};
#pragma unroll
    for (int b = 0; b < kDeep; ++b) issue(wave + b * kWaves, b);
    for (int s0 = wave; s0 < steps; s0 += kDeep * kWaves) {
#pragma unroll
      for (int b = 0; b < kDeep; ++b) {
        const int s = s0 + b * kWaves;
        asm volatile("s_waitcnt vmcnt(%0)" : : "n"((kDeep - 1) * (kLoads + kScales)) : "memory");
        const int8_t *part = s_ring[wave] + b * kStep;
        v4i fw[2][kFn], fx[2][kFm];
        int sw[kFn], sx[kFm];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int at = lr * kBk + ((h * 4 + lc) ^ (lr >> 1)) * 16;
#pragma unroll
          for (int i = 0; i < kFn; ++i) fw[h][i] = *reinterpret_cast<const v4i *>(part + i * 16 * kBk + at);
#pragma unroll
          for (int j = 0; j < kFm; ++j) fx[h][j] = *reinterpret_cast<const v4i *>(part + (kRows + j * 16) * kBk + at);
        }
        if (kFp8) {
#pragma unroll
          for (int i = 0; i < kFn; ++i)
            sw[i] = *reinterpret_cast<const uint8_t *>(part + kScaleAt + (i * 16 + lr) * 4 + (s & 3));
#pragma unroll
          for (int j = 0; j < kFm; ++j)
            sx[j] = *reinterpret_cast<const uint8_t *>(part + kScaleAt + 256 + (j * 16 + lr) * 4 + (s & 3));
        }
        if (s * 8 + 8 > n_chunk) {
          // past K (or a step past the last) both sides are 0: 0 times what was loaded
          // could be a NaN
#pragma unroll
          for (int h = 0; h < 2; ++h)
            if (s * 8 + h * 4 + lc >= n_chunk) {
#pragma unroll
              for (int i = 0; i < kFn; ++i) fw[h][i] = v4i{0, 0, 0, 0};
#pragma unroll
              for (int j = 0; j < kFm; ++j) fx[h][j] = v4i{0, 0, 0, 0};
            }
          if (kFp8 && s >= steps) {  // (nor may a scale be a NaN)
#pragma unroll
            for (int i = 0; i < kFn; ++i) sw[i] = 127;
#pragma unroll
            for (int j = 0; j < kFm; ++j) sx[j] = 127;
          }
        }
        asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");  // the part is free
        issue(s + kDeep * kWaves, b);
        if constexpr (kKind == kMathWide) {
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int d = 0; d < 4; d += 2)
#pragma unroll
              for (int j = 0; j < kFm; ++j)
#pragma unroll
                for (int i = 0; i < kFn; ++i)
                  acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                      __builtin_bit_cast(v8b, widen8(fw[h][i][d], fw[h][i][d + 1], scale_value(sw[i]))),
                      __builtin_bit_cast(v8b, widen8(fx[h][j][d], fx[h][j][d + 1], scale_value(sx[j]))),
                      acc[i][j], 0, 0, 0);
        } else if constexpr (kFp8) {
#pragma unroll
          for (int j = 0; j < kFm; ++j)
#pragma unroll
            for (int i = 0; i < kFn; ++i)
              acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(
                  __builtin_shufflevector(fw[0][i], fw[1][i], 0, 1, 2, 3, 4, 5, 6, 7),
                  __builtin_shufflevector(fx[0][j], fx[1][j], 0, 1, 2, 3, 4, 5, 6, 7), acc[i][j], 0, 0, 0,
                  sw[i], 0, sx[j]);
        } else {
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int j = 0; j < kFm; ++j)
#pragma unroll
              for (int i = 0; i < kFn; ++i)
                acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                    __builtin_bit_cast(v8b, fw[h][i]), __builtin_bit_cast(v8b, fx[h][j]), acc[i][j], 0, 0, 0);
        }
      }
    }
    asm volatile("s_waitcnt vmcnt(0)" : : : "memory");

    // lane: row lr of a 16 x 16 part, weight rows 4 lc ..
    float *sums = reinterpret_cast<float *>(s_ring[wave]);
#pragma unroll
    for (int i = 0; i < kFn; ++i)
#pragma unroll
      for (int j = 0; j < kFm; ++j)
        *reinterpret_cast<v4f *>(sums + (j * 16 + lr) * kPitch + i * 16 + lc * 4) = acc[i][j];
    __syncthreads();
    for (int o = tid; o < kTok * kOut / 4; o += kThreads) {  // four channels of a row
      const int r = o / (kOut / 4), c = o % (kOut / 4) * 4, n = n0 + c;
      if (r >= tile.rows || n >= a.n_out) continue;
      auto total = [&](int at) {  // of four of the row's channels, the waves in order
        v4f sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int u = 0; u < kWaves; ++u)
          sum += *reinterpret_cast<const v4f *>(reinterpret_cast<float *>(s_ring[u]) + r * kPitch + at);
        return sum;
      };
      auto packed = [](v4f v) { return v2u{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])}; };
      v4f v = total(c);
      const int64_t m = tile.row + r;
      if (kGlu) {
        const v4f up = total(c + kOut);
        if (!kFp8 && a.pre) {
          *reinterpret_cast<v2u *>(a.pre + m * a.N + n) = packed(v);
          *reinterpret_cast<v2u *>(a.pre + m * a.N + half + n) = packed(up);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = silu(v[e]) * up[e];
      }
      char *out = static_cast<char *>(a.y) + (m * a.n_out + n) * (kBf16 ? 2 : 4);
      if (kBf16) *reinterpret_cast<v2u *>(out) = packed(v);
      else *reinterpret_cast<v4f *>(out) = v;
    }
    __syncthreads();
  }
}

// ------------------------------------------------------------------- launching

// most row tiles that M rows in n_block blocks make: every block that has rows may
// end in a part of a tile
inline int64_t most_tiles(const ProductArgs &a, int tile_rows) {
  return a.M / tile_rows + (a.M < a.n_block ? a.M : a.n_block);
}

template <int kTok, int kRows, int kWaves, int kDeep, Math kKind, int kAct, bool kBf16>
void start_thin(const ProductArgs &a, hipStream_t stream) {
  const int out = kAct == ULTRAEP_SWIGLU ? kRows / 2 : kRows;
  const int32_t n_col = (a.n_out + out - 1) / out;
  const int64_t items = most_tiles(a, kTok) * n_col;
  const dim3 grid(static_cast<unsigned>(items < 1 << 16 ? items : 1 << 16)), block(64 * kWaves);
  hipLaunchKernelGGL((k_product_thin<kTok, kRows, kWaves, kDeep, kKind, kAct, kBf16>), grid, block, 0, stream, a, n_col);
}

template <int kN, int kM, int kWn, int kWm, bool kAhead, int kRing, Math kKind, bool kTrans, int kAct, bool kBf16>
void start_product(const ProductArgs &a, int n_wg, hipStream_t stream) {
  const int out = kAct == ULTRAEP_SWIGLU ? kN / 2 : kN;
  const int32_t n_col = (a.n_out + out - 1) / out;
  const int64_t items = most_tiles(a, kM) * n_col;
  const dim3 grid(static_cast<unsigned>(items < n_wg ? (items + 7) / 8 * 8 : n_wg)), block(64 * kWn * kWm);
  hipLaunchKernelGGL((k_product<kN, kM, kWn, kWm, kAhead, kRing, kKind, kTrans, kAct, kBf16>), grid, block, 0, stream, a, n_col);
}

// four waves' worth of steps
inline bool deep_k(Math kind, int32_t K) { return static_cast<int64_t>(K) * (kind == kMath16 ? 2 : 1) >= 4096; }

// The tiles by the rounds that they would take: a round is 256 of them, one a compute unit (of
// 128 x 128 two a compute unit, 512), and its time is in thousandths of a round of 256 x 256,
// bf16 / 8 bits.  `rows`: M over the blocks, of which the host cannot know how many are empty
// (a list that is mostly empty, or an M above the rows that the blocks hold, is taken for
// small or large blocks: the result is the same but for the order of the sums of K, the
// time is not); items: estimated tiles, with a third of a tile of padding a block
// where there are several, and no fewer than blocks.  Their rounds are not taken as whole then, the
// estimate is not that near: half a round more than they fill, and of the largest tiles, whose
// last round goes by quarters where it is short, 0.175.  Over 81 calls of 5 to 32 blocks, of equal
// rows and spread ones (M = 1024 to 16384, N = 1024 to 7168, K = 512 to 7168), what this takes is 2 %
// above the best of all on average and at most a fourth; with whole rounds of half a tile of
// padding it was 4 % and at most two thirds.
//   Measured, us (256 x 256 / 128 x 128, two buffers / four / 128 x 64, four / thin 64 / 32 /
//   16; x: not run):
//   bf16, 1 block, N = 4096, K = 7168: M = 10240 485 / 519 / 618 / 827, 8192 324 / 411 / 496 / 646,
//   6144 320 / 290 / 333 / 428, 5120 218 / 288 / 274 / 344, 4096 163 / 194 / 222 / 281, 2560 143 /
//   194 / 158 / 182, 2048 144 / 99 / 113 / 142, 1024 140 / 81 / 59 / 78 / 91 / 134, 512 139 / 72 / 54 /
//   41 / 48 / 70 / x, 384 142 / 71 / 53 / 36 / 45 / 52 / 104, 256 140 / 70 / 52 / 35 / 24 / 35 / 70, 128
//   140 / 70 / 51 / 35 / 23 / 19 / 37, 64 x / x / x / 35 / 23 / 18 / 19, 16 138 / 65 / 50 / 34 / 19 / 16 / 12
//   10 blocks, the same with SwiGLU: M = 20480 998 / 1255 / 1336 / 1761, 7680 401 / 509 / 547 / 692,
//   5120 275 / 413 / 362 / 509, 2560 213 / 287 / 228 / 269, 1024 196 / 156 / 158 / 162 / 169 / 229, 640
//   x / x / x / 138 / 132 / 148 / 240, 320 x / x / x / 129 / 117 / 114 / 152, 160 x / x / x / 125 / 114 /
//   110 / 105
//   8 bits, 4 blocks, the same with SwiGLU: M = 16384 355 / 693 / 630 / 893, 4096 88 / 166 / 158 /
//   221, 2048 83 / 90 / 86 / 116, 1024 79 / 87 / 47 / 63, 512 80 / 50 / 46 / 34; 1 block: M = 512 x / x / x /
//   32 / 32 / 45 / 70, 256 x / x / x / 31 / 17 / 24 / 37, 128 x / x / x / 30 / 16 / 13 / 20, 16 x / x / x / 30 /
//   14 / 11 / 7
//   weights [K][N], 4 blocks, N = 2048, K = 4096: M = 16384 198 / 238 / 273 / 362, 4096 88 / 59 / 67 /
//   90, 2048 85 / 49 / 34 / 47, 1024 85 / 41 / 32 / 24
//   (Where the weights' bytes bound the call the choice misses the best by up to an eighth: 10
//   blocks of 6 rows, weights [K][N], take 130 us of 128 x 64 where two tiles of 128 x 128 a
//   compute unit take 114.)
// 0: 256 x 256, 1: 128 x 128, two buffers, 2: four, 3: 128 x 64, 4 to 6: thin of 64, 32, 16 rows
inline int product_tile(Math kind, bool trans, int act, int64_t M, int32_t n_block, int32_t N, int32_t K) {
  const int64_t blocks = M < n_block ? M : n_block;
  auto items = [&](int64_t tile_rows, int64_t channels) {
    const double whole = static_cast<double>((M + tile_rows - 1) / tile_rows);
    const double several = static_cast<double>(M) / tile_rows + blocks / 3.;
    return (blocks == 1 ? whole : several > blocks ? several : blocks) * ((N + channels - 1) / channels);
  };
  auto time = [&](double n, int of, int cost, double more) {
    const double rounds = n / of;
    if (blocks > 1) return cost * (rounds + more > 1 ? rounds + more : 1);
    return cost * std::ceil(rounds);
  };
  const bool k8 = kind == kMath8, large = kind != kMathWide, thin = !trans && act != ULTRAEP_SWIGLU_GRAD;
  const bool deep = deep_k(kind, K);
  const double big = items(256, 256), last = std::fmod(big, 256);
  constexpr double kNever = 1e30;
  const double times[] = {
      !large ? kNever : blocks == 1 && big > 256 && last > 0 && last <= 64 ? (big - last) / 256 * 1000 + 350 : time(big, 256, 1000, 0.175),
      k8 ? kNever : time(items(128, 128), 512, 600, 0.5),  // (8 bits: 1050 to 1100 of two of the next's)
      time(items(128, 128), 256, k8 ? 550 : 360, 0.5),
      time(items(64, 128), 256, k8 ? 370 : 250, 0.5),
      thin ? time(items(64, 64), 256, k8 ? 190 : 155, 0.5) : kNever,
      thin ? time(items(32, 64), 256, k8 ? 135 : 115, 0.5) : kNever,
      thin ? time(items(16, deep ? 32 : 64), 256, deep ? 70 : 80, 0.5) : kNever,
  };
  int best = 0;
  for (int i = 1; i < 7; ++i)
    if (times[i] < times[best]) best = i;
  return best;
}

template <Math kKind, bool kTrans, int kAct, bool kBf16>
void choose_product(const ProductArgs &a, hipStream_t stream) {
  constexpr bool k8 = kKind == kMath8, kBig = kKind != kMathWide;
  constexpr bool kThin = !kTrans && kAct != ULTRAEP_SWIGLU_GRAD;
  const bool deep = deep_k(kKind, a.K);
  const int best = product_tile(kKind, kTrans, kAct, a.M, a.n_block, a.N, a.K);
  if constexpr (kBig) {
    if (best == 0) start_product<256, 256, 2, 2, true, 2, kKind, kTrans, kAct, kBf16>(a, 256, stream);
  }
  if constexpr (!k8) {
    if (best == 1) start_product<128, 128, 2, 2, false, 2, kKind, kTrans, kAct, kBf16>(a, 512, stream);
  }
  if (best == 2) start_product<128, 128, 2, 2, false, 4, kKind, kTrans, kAct, kBf16>(a, 256, stream);
  if (best == 3) start_product<128, 64, 2, 2, false, 4, kKind, kTrans, kAct, kBf16>(a, 256, stream);
  if constexpr (kThin) {
    if (best == 4 && deep) start_thin<64, 64, 4, 2, kKind, kAct, kBf16>(a, stream);
    if (best == 4 && !deep) start_thin<64, 64, 2, 2, kKind, kAct, kBf16>(a, stream);
    if (best == 5 && deep) start_thin<32, 64, 4, 2, kKind, kAct, kBf16>(a, stream);
    if (best == 5 && !deep) start_thin<32, 64, 2, 2, kKind, kAct, kBf16>(a, stream);
    if (best == 6 && deep) start_thin<16, 32, 4, 2, kKind, kAct, kBf16>(a, stream);
    if (best == 6 && !deep) start_thin<16, 64, 2, 2, kKind, kAct, kBf16>(a, stream);
  }
}

template <Math kKind, bool kTrans, int kAct>
void choose_type(const ProductArgs &a, int32_t type, hipStream_t stream) {
  if (type == ULTRAEP_BF16) choose_product<kKind, kTrans, kAct, true>(a, stream);
  else choose_product<kKind == kMath8 ? kMathWide : kKind, kTrans, kAct, false>(a, stream);
}

}  // namespace uep
