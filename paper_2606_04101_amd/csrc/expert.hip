// The experts' products on 8-bit integers: the quantisation of rows, and the
// product of each dispatched block of rows with its expert's weight.
#include <type_traits>

#include "operators.hpp"

namespace uep {

// ---------------------------------------------------------------- quantisation

constexpr int kQrThreads = 256;
constexpr int kQrWaves = kQrThreads / kWave;

// eight elements of a row as they lie in memory
template <bool kBf16>
struct Chunk;
template <>
struct Chunk<true> {
  v4u v = {0, 0, 0, 0};
  // kOnce: not read again
  template <bool kOnce>
  __device__ void load(const void *row, int64_t c) {
    const v4u *p = static_cast<const v4u *>(row) + c;
    v = kOnce ? __builtin_nontemporal_load(p) : *p;
  }
  // largest magnitude, as the bits of an fp32 (an infinity or a NaN is the largest)
  __device__ int largest() const {
    typedef uint16_t v2h __attribute__((ext_vector_type(2)));
    v2h m = {0, 0};
#pragma unroll
    for (int i = 0; i < 4; ++i)
      m = __builtin_elementwise_max(m, __builtin_bit_cast(v2h, v[i] & 0x7FFF7FFFu));
    return static_cast<int>(max(m.x, m.y)) << 16;
  }
  __device__ float at(int i) const {
    return i % 2 ? bf16_at_high(v[i / 2]) : bf16_at_low(v[i / 2]);
  }
};
template <>
struct Chunk<false> {
  v4f v[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
  template <bool kOnce>
  __device__ void load(const void *row, int64_t c) {
    const v4f *p = static_cast<const v4f *>(row) + 2 * c;
    v[0] = kOnce ? __builtin_nontemporal_load(p) : p[0];
    v[1] = kOnce ? __builtin_nontemporal_load(p + 1) : p[1];
  }
  __device__ int largest() const {
    int m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, __float_as_int(v[i / 4][i % 4]) & 0x7FFFFFFF);
    return m;
  }
  __device__ float at(int i) const { return v[i / 4][i % 4]; }
};

// Eight integers of a row with inverse scale inv.  The product is at most
// 127 (1 + 2^-23), so no rounding leaves [-127, 127].  Added to 1.5 * 2^23 it is rounded
// to an integer, to even, which the sum's low byte holds; the product is rounded on its
// own first.
template <class C>
__device__ __forceinline__ v2u quantise8(const C &x, float inv) {
#pragma clang fp contract(off)
  uint32_t b[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) b[i] = __float_as_uint(x.at(i) * inv + 0x1.8p23f);
  v2u o;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint32_t lo = __builtin_amdgcn_perm(b[4 * i + 1], b[4 * i], 0x0C0C0400u);
    const uint32_t hi = __builtin_amdgcn_perm(b[4 * i + 3], b[4 * i + 2], 0x04000C0Cu);
    o[i] = lo | hi;
  }
  return o;
}

// scale and inverse of a row whose largest |x| is a: inv 0 where q is 0
__device__ __forceinline__ float row_scale(int most, float &inv) {
  const float a = __int_as_float(most);
  const bool finite = a < __builtin_inff(), live = finite && a > 0x1p-100f;
  inv = live ? 127.f / a : 0.f;
  return live ? a / 127.f : finite ? 0.f : __builtin_nanf("");
}

// One wave a row.  kCh > 0: the row's kCh chunks of 8 elements a lane stay in registers,
// as they lie in memory, between the maximum and the rounding, so it is read once;
// kCh = 0: longer rows, read twice.  Bound by memory: 131072 rows of 7168 bf16 (2.8 GB)
// take 476 us, 5.9 TB/s; 643 us when read twice, 583 us with the elements held as fp32
// (148 registers instead of 98), 507 us with loads that stay in the caches.
template <int kCh, bool kBf16>
__global__ void __launch_bounds__(kQrThreads)
k_quant_rows(const char *__restrict__ x, int64_t rows, int32_t nch, int64_t row_bytes,
             int8_t *__restrict__ q, int32_t nqch, float *__restrict__ scale) {
  const int lane = lane_id();
  const int64_t nw = static_cast<int64_t>(gridDim.x) * kQrWaves;
  for (int64_t r = static_cast<int64_t>(blockIdx.x) * kQrWaves + threadIdx.x / kWave; r < rows;
       r += nw) {
    const char *row = x + r * row_bytes;
    v2u *out = reinterpret_cast<v2u *>(q) + r * nqch;
    int most = 0;
    float inv;
    if constexpr (kCh > 0) {
      Chunk<kBf16> f[kCh];
#pragma unroll
      for (int u = 0; u < kCh; ++u)
        if (u * kWave + lane < nch) f[u].template load<true>(row, u * kWave + lane);
#pragma unroll
      for (int u = 0; u < kCh; ++u) most = max(most, f[u].largest());
      const float s = row_scale(wave_max(most), inv);
      if (lane == 0) scale[r] = s;
#pragma unroll
      for (int u = 0; u < kCh; ++u)
        if (u * kWave + lane < nqch)
          __builtin_nontemporal_store(inv > 0.f ? quantise8(f[u], inv) : v2u{0, 0},
                                      out + u * kWave + lane);
      for (int c = kCh * kWave + lane; c < nqch; c += kWave) out[c] = v2u{0, 0};
    } else {
      Chunk<kBf16> f;
      for (int c = lane; c < nch; c += kWave) {
        f.template load<false>(row, c);
        most = max(most, f.largest());
      }
      const float s = row_scale(wave_max(most), inv);
      if (lane == 0) scale[r] = s;
      for (int c = lane; c < nqch; c += kWave) {
        v2u o{0, 0};
        if (inv > 0.f && c < nch) {
          f.template load<true>(row, c);
          o = quantise8(f, inv);
        }
        __builtin_nontemporal_store(o, out + c);
      }
    }
  }
}

template <bool kBf16>
static void start_quant(const char *x, int64_t rows, int32_t nch, int64_t row_bytes, int8_t *q,
                        int32_t nqch, float *scale, hipStream_t stream) {
  const int64_t wg = (rows + kQrWaves - 1) / kQrWaves;
  const dim3 grid(static_cast<unsigned>(wg < 1 << 20 ? wg : 1 << 20));
#define UEP_CASE(n)                                                                              \
  if (nch <= n * kWave || n == 0) {                                                              \
    hipLaunchKernelGGL((k_quant_rows<n, kBf16>), grid, dim3(kQrThreads), 0, stream, x, rows, nch, \
                       row_bytes, q, nqch, scale);                                               \
    return;                                                                                      \
  }
  UEP_CASE(1) UEP_CASE(2) UEP_CASE(4) UEP_CASE(6) UEP_CASE(8) UEP_CASE(11) UEP_CASE(14) UEP_CASE(16)
  UEP_CASE(20) UEP_CASE(24) UEP_CASE(0)
#undef UEP_CASE
}

hipError_t launch_quant_rows(const void *x, int32_t type, int64_t rows, int64_t K, int64_t ld,
                             int8_t *q, int64_t ldq, float *scale, hipStream_t stream) {
  const char *xs = static_cast<const char *>(x);
  const int32_t nch = static_cast<int32_t>(K / 8), nqch = static_cast<int32_t>(ldq / 8);
  if (type == ULTRAEP_BF16)
    start_quant<true>(xs, rows, nch, ld * 2, q, nqch, scale, stream);
  else
    start_quant<false>(xs, rows, nch, ld * 4, q, nqch, scale, stream);
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

// v, with what follows from it computed where it is used: a persistent loop would
// otherwise hold every lane's address of its rare parts in registers throughout
__device__ __forceinline__ int opaque(int v) {
  asm volatile("" : "+v"(v));
  return v;
}

__device__ __forceinline__ int64_t readlane64(int64_t v, int l) {
  const uint32_t lo = readlane(static_cast<int>(v), l), hi = readlane(static_cast<int>(v >> 32), l);
  return static_cast<int64_t>(static_cast<uint64_t>(hi) << 32 | lo);
}

// an address that is the same in all lanes, in scalar registers
template <class T>
__device__ __forceinline__ T *uniform(T *p) {
  const uintptr_t v = reinterpret_cast<uintptr_t>(p);
  const uint32_t lo = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(v));
  const uint32_t hi = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(v >> 32));
  return reinterpret_cast<T *>(static_cast<uintptr_t>(hi) << 32 | lo);
}

// A tile of rows of one block: its first row, rows and weight.
struct RowTile {
  int64_t row;
  int32_t rows, w;
};

// Row tiles are numbered block by block.  Blocks are looked at in runs of 64, one a
// lane; a wave holds one run's blocks, and the runs' tile counts, in registers.  Where a
// block is out of order or out of [0, M], or has rows and no weight, that is reported and
// there are no tiles at all, so that what is numbered lies within M rows.  Every lane
// must be active in each call.
template <int kTileRows>
struct RowTiles {
  int64_t lo;               // this lane's block of run `run`:
  int rows, w;              //   its first row, rows, weight
  int before, tiles;        //   its tiles, and the run's before it
  int run, n_run;
  int run_before, run_tiles;  // of run `lane`
  int total;                // tiles in all

  // false (in the whole wave) if a block of run r is not sound
  __device__ bool load(const MatmulArgs &a, int r) {
    run = r;
    bool sound = true;
    const int g = r * kWave + lane_id();
    lo = 0;
    rows = w = 0;
    if (g < a.n_block) {
      lo = a.block_off[g];
      const int64_t hi = a.block_off[g + 1];
      w = a.block_w ? a.block_w[g] : g;
      sound = lo >= 0 && hi >= lo && hi <= a.M && (hi == lo || (w >= 0 && w < a.n_w));
      if (sound)
        rows = static_cast<int>(hi - lo);
      else
        report(a.status, ULTRAEP_EDATA);
    }
    tiles = rows > 0 ? (rows - 1) / kTileRows + 1 : 0;
    before = wave_scan_incl(tiles) - tiles;
    return !ballot(!sound);
  }
  // s_run: 32 words of LDS, free again after the call's last barrier
  __device__ void count(const MatmulArgs &a, int *s_run, int wave, int n_waves) {
    n_run = (a.n_block + kWave - 1) / kWave;
    if (n_run == 1) {
      const bool sound = load(a, 0);
      run_before = 0;
      total = sound ? readlane(before + tiles, kWave - 1) : 0;
      run_tiles = lane_id() == 0 ? total : 0;
      return;
    }
    for (int r = wave; r < n_run; r += n_waves) {
      const bool sound = load(a, r);
      if (lane_id() == kWave - 1) s_run[r] = sound ? before + tiles : -1;
    }
    __syncthreads();
    run_tiles = lane_id() < n_run ? s_run[lane_id()] : 0;
    __syncthreads();
    run_before = wave_scan_incl(run_tiles) - run_tiles;
    total = readlane(run_before, kWave - 1);  // (fewer than 64 runs)
    if (ballot(run_tiles < 0)) total = 0;
    run = -1;
  }
  // tile < total
  __device__ RowTile find(const MatmulArgs &a, int tile) {
    int t = tile;
    if (n_run > 1) {
      const int r = __builtin_ctzll(ballot(tile >= run_before && tile < run_before + run_tiles));
      t -= readlane(run_before, r);
      if (r != run) load(a, r);
    }
    const int l = __builtin_ctzll(ballot(t >= before && t < before + tiles));
    const int first = (t - readlane(before, l)) * kTileRows;
    return {readlane64(lo, l) + first, min(readlane(rows, l) - first, kTileRows), readlane(w, l)};
  }
};

// v / (1 + exp(-v)) by the hardware's exp2 and reciprocal: a relative error of
// (|v| + 5) 2^-24 at most for v >= -87; below, where it is under 2e-36 in magnitude, it
// becomes 0.  |v| 2^-24 is far below the rounding of the 8-bit operands; with
// expf and a division the epilogue's arithmetic costs 65 us of 3350 at 131072 x 4096 x 7168.
__device__ __forceinline__ float silu(float v) { return v * fast_rcp(1.f + fast_exp(-v)); }

// 16 bytes a lane from base + off straight into LDS, lane l's at lds + 16 l.
// The wait for it is the caller's (vmcnt).
__device__ __forceinline__ void load_to_lds(const void *base, uint32_t off, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
               :
               : "s"(lds), "v"(off), "s"(base)
               : "memory", "m0");
}

// the same for 4 bytes a lane
__device__ __forceinline__ void load_word_to_lds(const void *base, uint32_t off, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2"
               :
               : "s"(lds), "v"(off), "s"(base)
               : "memory", "m0");
}
template <class T>
__device__ __forceinline__ uint32_t lds_address(T *p) {
  return static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) T *)p));
}

constexpr int kBk = 128;  // bytes of K of a step

// Output tile of kN weight rows x kM rows, K in steps of 128 bytes through two
// LDS buffers; kWn x kWm waves, which stay and take tile after tile.  The weights
// are the matrix unit's first operand, so a lane holds 4 neighbouring channels of
// one row.  With act, a wave's parts of 32 weight rows alternate between gates and
// their partners, and a gate's sum meets its partner's in the same lane.
//   The reads of LDS bound such a tile next to the products: 4 waves of 128 x 128
// read 128 KiB of LDS a step beside 2048 cycles of products (8 waves of 128 x 64
// would read 192), and one wave a SIMD leaves it all registers: 256 for the sums.
// Loads go straight to LDS, two steps ahead, and a step has one barrier, before its
// last quarter: by then its own bytes are in registers, and the next step's have come.
// kAhead: the next tile's first two steps are loaded while the results leave.
//   Where the tiles of the last round are at most a quarter of the workgroups, these take
// quarters of them: 4608 rows of one block, N = 4096, K = 7168, act, 288 tiles for 256
// workgroups, take 144 us, with a second full round 184.  (Up to half the workgroups,
// in two rounds of quarters: 289 us for 300 at 10240 rows, but 3395 for 3370 at 131072.)
//   131072 rows of 10 blocks, N = 4096, K = 7168, act, bf16: 3.23 to 3.37 ms by the card,
// 2.38 POP/s (a library product of 8192^3 reaches 2.14 here); 32761 rows of 6 blocks,
// N = 4096, K = 1408: 210 us, 1.80 POP/s.  Bound by power: 62 % of the matrix unit's
// cycles at 1.6 GHz; with zeros as data the first takes 2.65 ms.
template <int kN, int kM, int kWn, int kWm, bool kAhead>
struct MatmulShape {
  static constexpr int kBuf = (kN + kM) * kBk, kTurns = kAhead ? 2 : 1;
  static constexpr int kWaves = kWn * kWm;
  static constexpr int kLds = 2 * kBuf + (kAhead ? kWaves * 4096 : 0);
  static constexpr int kScales = kTurns * (kN + kM);  // of this item, and of the next
  static_assert(kAhead || kWaves * 4096 <= 2 * kBuf, "results take the place of the operands");
};

// Items item, item + stride, .. below n_item, item 0 being that numbered `first`.  An
// item is a tile that `tiles` numbers, or (kPart = 2) a quarter of one, 2 x 2.
template <int kN, int kM, int kWn, int kWm, bool kAhead, int kPart, bool kAct, bool kBf16>
__device__ __forceinline__ void matmul_items(const MatmulArgs &a, int32_t n_col,
                                             RowTiles<kM * kPart> &tiles, int8_t *s_lds,
                                             float *s_scale, int first, int item, int stride,
                                             int n_item) {
  constexpr int kWaves = kWn * kWm;
  constexpr int kFn = kN / kWn / 32, kFm = kM / kWm / 32;  // 32 x 32 parts of a wave
  constexpr int kBuf = MatmulShape<kN, kM, kWn, kWm, kAhead>::kBuf;
  constexpr int kLoads = kBuf / 1024 / kWaves;             // of a wave in a step
  constexpr int kLoadsN = kLoads * kN / (kN + kM);
  constexpr int kOut = kAct ? kN / 2 : kN;                 // channels of an item
  constexpr int kOutW = kOut / kWn;                        // of a wave
  static_assert(!kAct || kFn % 2 == 0, "a wave has gates with their partners");
  const int lane = lane_id();
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int wn = wave % kWn, wm = wave / kWn;
  const int lr = lane & 31, hi = lane >> 5;
  const int half = a.N / 2, n_tile = tiles.total;
  const uint32_t lds0 = lds_address(s_lds), lds_scale = lds_address(s_scale);
  const int steps = (a.K + kBk - 1) / kBk;
  const int tail = (a.K - (steps - 1) * kBk) / 16;  // chunks of the last step

  // an item: its rows and weight, its first channel
  RowTile tile;
  int n0;
  // byte offsets of this lane's loads: 8 rows of 8 chunks an instruction; chunk c of
  // tile row r lies at c ^ (r / 2 % 8), so that 16 neighbouring rows' lie in all banks
  const int8_t *wbase, *xbase;
  uint32_t off[kLoads];
  int turn = 0;  // which part of s_scale the item's scales are in
  const int chunk = (lane & 7) ^ ((wave & 1) * 4 + (lane >> 4));
  // false for a quarter that has no rows or no channels
  auto aim = [&](int id) {
    const int item = first + id / (kPart * kPart), part = id % (kPart * kPart);
    const int lane = opaque(lane_id());
    const int chunk = (lane & 7) ^ ((wave & 1) * 4 + (lane >> 4));
    // 8 row tiles by all columns at a time
    constexpr int kGroup = 8;
    const int group = item / (kGroup * n_col), rest = item - group * kGroup * n_col;
    const int high = min(kGroup, n_tile - group * kGroup);
    tile = tiles.find(a, group * kGroup + rest % high);
    n0 = (rest / high * kPart + part / kPart) * kOut;
    if (kPart > 1) {
      tile.row += part % kPart * kM;
      tile.rows = min(tile.rows - part % kPart * kM, kM);
      if (tile.rows <= 0 || n0 >= a.n_out) return false;
    }
    wbase = uniform(a.wq + (static_cast<int64_t>(tile.w) * a.N + n0) * a.K);
    xbase = uniform(a.xq + tile.row * a.K);
    // weight row of tile row j after the tile's first (with act, among the gates or
    // among their partners), in range for any j
    auto weight_row = [&](int j) {
      return kAct ? min(j / 64 * 32 + j % 32, half - 1 - n0) : min(j, a.N - 1 - n0);
    };
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int j = ((i < kLoadsN ? i : i - kLoadsN) * kWaves + wave) * 8 + (lane >> 3);
      const int r = i < kLoadsN ? weight_row(j) : min(j, tile.rows - 1);
      off[i] = static_cast<uint32_t>(r) * a.K + chunk * 16;
    }
    const float *ws = uniform(a.ws + static_cast<int64_t>(tile.w) * a.N + n0);
    const float *xs = uniform(a.xs + tile.row);
    if (kAhead) turn ^= 1;
#pragma unroll
    for (int i = 0; i < kN + kM; i += kWaves * kWave) {
      const int j = i + wave * kWave;  // the same operand for all lanes
      if (j >= kN + kM) break;
      const int r = j >= kN ? min(j - kN + lane, tile.rows - 1)
                            : weight_row(j + lane) + (kAct && lane >= 32 ? half : 0);
      load_word_to_lds(j < kN ? ws : xs, r * 4,
                       __builtin_amdgcn_readfirstlane(lds_scale + (turn * (kN + kM) + j) * 4));
    }
    return true;
  };
  // load i of a step; chunks past K (in the last step) are loaded from the step's
  // first one and not used
  auto issue = [&](int s, int i) {
    const uint32_t back = s == steps - 1 && chunk >= tail ? chunk * 16 : 0;
    const int8_t *base = i >= kLoadsN ? xbase
                         : kAct && (i * kWaves + wave) * 8 % 64 >= 32
                             ? wbase + static_cast<int64_t>(half) * a.K
                             : wbase;
    load_to_lds(base + static_cast<int64_t>(s) * kBk, off[i] - back,
                __builtin_amdgcn_readfirstlane(lds0 + (s & 1) * kBuf + (i * kWaves + wave) * 1024));
  };
  // the first item from `item` on that has work: false if there is none
  auto begin = [&] {
    do {
      if (item >= n_item) return false;
    } while (!aim(item) && (item += stride, true));
#pragma unroll
    for (int i = 0; i < kLoads; ++i) issue(0, i);
    if (steps > 1) {
#pragma unroll
      for (int i = 0; i < kLoads; ++i) issue(1, i);
    }
    return true;
  };

  auto arrived = [&] {  // the first step's bytes are there
    if (steps > 1)
      asm volatile("s_waitcnt vmcnt(%0)" : : "n"(kLoads) : "memory");
    else
      asm volatile("s_waitcnt vmcnt(0)" : : : "memory");
  };

  if (!begin()) return;
  arrived();
  while (true) {
    asm volatile("s_barrier" : : : "memory");
    v16i acc[kFn][kFm] = {};
    v4i fw[2][kFn], fx[2][kFm];
    // part f of the operands for 32 bytes kk of a step
    auto fetch = [&](int s, int kk, int f) {
      const int8_t *b = s_lds + (s & 1) * kBuf + ((kk * 2 + hi) ^ (lr >> 1 & 7)) * 16;
      if (f < kFn)
        fw[kk & 1][f] = *reinterpret_cast<const v4i *>(b + (wn * kFn * 32 + f * 32 + lr) * kBk);
      else
        fx[kk & 1][f - kFn] = *reinterpret_cast<const v4i *>(
            b + (kN + wm * kFm * 32 + (f - kFn) * 32 + lr) * kBk);
    };
    // One step, its first parts already in registers.  The products run in the
    // order that keeps the matrix unit fed: reads of the next parts, and at the
    // step's end the loads of the step after the next, between them.  kMore: how
    // many steps follow, up to 2.
    auto step = [&](int s, auto ahead) {
      constexpr int kMore = decltype(ahead)::value;
#pragma unroll
      for (int kk = 0; kk < 4; ++kk) {
        if (kk == 3)  // the next step's bytes are there, and nobody reads this step's any more
          asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" : : : "memory");
        if (kMore == 0 && kk * 2 + 1 >= tail) {
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
            else if (kMore > 0) fetch(s + 1, 0, f);
          }
          if (kk == 3 && kMore == 2)
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

    // (kAhead) the next item's first loads fly while this one's results leave
    const RowTile out = tile;
    const int nw = n0 + wn * kOutW;  // the wave's first channel
    const int was = turn;
    item += stride;
    const bool more = kAhead && begin();

    // 32 rows x 64 channels (32 in fp32) at a time through LDS, so that a row's
    // channels leave in whole lines, past the caches (228 us for 210 at 32761 x 4096 x
    // 1408 where they stay; a quantisation of the result that follows at once reads at
    // most 67 MB 1 us slower, and the pair takes as long)
    constexpr int kParts = kOutW / 32;
    const int el = opaque(lane), er = el & 31, eh = el >> 5;
    const float *scale = s_scale + was * (kN + kM);
    int8_t *stage = s_lds + (kAhead ? 2 * kBuf : 0) + wave * 4096;
#pragma unroll
    for (int j = 0; j < kFm; ++j) {
      const int r0 = (wm * kFm + j) * 32;
      const float xs = scale[kN + r0 + er];
      // the sums stay in the accumulation registers until here
#pragma unroll
      for (int i = 0; i < kFn; ++i) asm volatile("" : "+a"(acc[i][j]));
      // before the last stores: all loads, and the earlier stores, are done (and
      // nothing read from LDS is held in registers from one part to the next)
      if (kAhead && j == kFm - 1) asm volatile("s_waitcnt vmcnt(0)" : : : "memory");
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
          const int r = p * 8 + el / 8;  // (LDS takes a wave's accesses in order)
          const v4u o = *reinterpret_cast<const v4u *>(stage + r * 128 + ((el & 7) ^ (r & 7)) * 16);
          if (r0 + r < out.rows && c0 + c < min(a.n_out, nw + kOutW))
            __builtin_nontemporal_store(
                o, reinterpret_cast<v4u *>(static_cast<char *>(a.y) +
                                           ((out.row + r0 + r) * a.n_out + c0 + c) * esize));
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    if (kAhead) {
      if (!more) return;
    } else {
      __syncthreads();
      if (!begin()) return;
      arrived();
    }
  }
}

template <int kN, int kM, int kWn, int kWm, bool kAhead, bool kAct, bool kBf16>
__global__ void __launch_bounds__(64 * kWn * kWm) k_matmul(MatmulArgs a, int32_t n_col) {
  using Shape = MatmulShape<kN, kM, kWn, kWm, kAhead>;
  __shared__ __align__(1024) int8_t s_lds[Shape::kLds];
  __shared__ __align__(16) float s_scale[Shape::kScales];
  __shared__ int s_run[32];
  RowTiles<kM> tiles;
  tiles.count(a, s_run, __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), Shape::kWaves);
  const int n_item = tiles.total * n_col;  // (fewer than 2^31: M * N < 2^38)
  // the workgroups of one XCD (those of equal number modulo 8) take neighbouring items
  constexpr int kXcd = 8;
  const int grid = gridDim.x, per_xcd = grid / kXcd;  // the grid is a multiple
  const int slot = blockIdx.x % kXcd * per_xcd + blockIdx.x / kXcd;
  int last = 0;  // tiles of the last round that are taken by quarters
  if (kAhead && n_item % grid * 4 <= grid) last = n_item % grid;
  matmul_items<kN, kM, kWn, kWm, kAhead, 1, kAct, kBf16>(a, n_col, tiles, s_lds, s_scale, 0, slot,
                                                         grid, n_item - last);
  if constexpr (kAhead) {
    __syncthreads();
    matmul_items<kN / 2, kM / 2, kWn, kWm, false, 2, kAct, kBf16>(
        a, n_col, tiles, s_lds, s_scale, n_item - last, slot, grid, last * 4);
  }
}

// Few rows a block: the weight's bytes bound the call.  A workgroup takes kRows weight
// rows (with act half of them gates, then their partners) and up to kTok rows.  Its
// waves share K in steps of 128 bytes in turn, each through an LDS ring of its own that
// kDeep steps fill, so no wave waits for another until they add their sums.  (Straight
// into registers, without LDS, neighbouring lanes would read different lines, which a
// compute unit takes at 16 bytes a cycle: 72 us where this takes 50.)  Bound by memory:
// 16 rows of 10 blocks, N = 4096, K = 7168, act: 50 us, 5.9 TB/s.  A ring of 3 steps, 8
// waves, or twice the rows take 5 to 15 % longer.
template <int kTok, int kRows, int kWaves, int kDeep, bool kAct, bool kBf16>
__global__ void __launch_bounds__(64 * kWaves) k_matmul_thin(MatmulArgs a, int32_t n_col) {
  constexpr int kThreads = 64 * kWaves, kFm = kTok / 16, kFn = kRows / 16;
  constexpr int kOut = kAct ? kRows / 2 : kRows;
  constexpr int kPitch = kRows + 4;  // words of a row's sums
  constexpr int kStep = (kRows + kTok) * kBk, kLoadsN = kRows / 8, kLoads = (kRows + kTok) / 8;
  constexpr int kRing = kDeep * kStep;
  static_assert(kTok * kPitch * 4 <= kRing, "a wave's sums take the place of its ring");
  __shared__ __align__(1024) int8_t s_ring[kWaves][kRing];
  const int tid = threadIdx.x, lane = lane_id();
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int lr = lane & 15, lc = lane >> 4;
  const int half = a.N / 2;
  RowTiles<kTok> tiles;
  tiles.count(a, reinterpret_cast<int *>(s_ring[0]), wave, kWaves);
  const int n_item = tiles.total * n_col;
  const int n_chunk = a.K / 16, steps = (a.K + kBk - 1) / kBk;
  const uint32_t lds0 = __builtin_amdgcn_readfirstlane(lds_address(&s_ring[wave][0]));

  for (int item = blockIdx.x; item < n_item; item += gridDim.x) {
    const RowTile tile = tiles.find(a, item / n_col);
    const int n0 = item % n_col * kOut;
    const int8_t *w = uniform(a.wq + (static_cast<int64_t>(tile.w) * a.N + n0) * a.K);
    const int8_t *x = uniform(a.xq + tile.row * a.K);
    // byte offsets of this lane's rows: 8 rows of 8 chunks an instruction, chunk c of
    // row r at c ^ (r / 2 % 8) as in the wide tiles
    uint32_t off[kLoads];
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int j = (i < kLoadsN ? i : i - kLoadsN) * 8 + (lane >> 3);
      const int r = i >= kLoadsN ? min(j, tile.rows - 1)
                    : kAct       ? min(j % kOut, half - 1 - n0)
                                 : min(j, a.N - 1 - n0);
      off[i] = static_cast<uint32_t>(r) * a.K;
    }
    // step s of the wave into part s % kDeep of the ring; what lies past K is loaded
    // from its last chunk and multiplied by 0
    const int chunk = (lane & 7) ^ (lane >> 4);
    auto issue = [&](int s, int slot) {
      const uint32_t at[2] = {min(s * 8 + chunk, n_chunk - 1) * 16u, min(s * 8 + (chunk ^ 4), n_chunk - 1) * 16u};
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const int8_t *base = i >= kLoadsN                   ? x
                             : kAct && i >= kLoadsN / 2 ? w + static_cast<int64_t>(half) * a.K
                                                            : w;
        load_to_lds(base, off[i] + at[i & 1],
                    __builtin_amdgcn_readfirstlane(lds0 + slot * kStep + i * 1024));
      }
    };

    v4i acc[kFn][kFm] = {};
#pragma unroll
    for (int b = 0; b < kDeep; ++b) issue(wave + b * kWaves, b);
    for (int s0 = wave; s0 < steps; s0 += kDeep * kWaves) {
#pragma unroll
      for (int b = 0; b < kDeep; ++b) {
        const int s = s0 + b * kWaves;
        asm volatile("s_waitcnt vmcnt(%0)" : : "n"((kDeep - 1) * kLoads) : "memory");
        const int8_t *part = s_ring[wave] + b * kStep;
        v4i fw[2][kFn], fx[2][kFm];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int at = lr * kBk + ((h * 4 + lc) ^ (lr >> 1)) * 16;
#pragma unroll
          for (int i = 0; i < kFn; ++i)
            fw[h][i] = *reinterpret_cast<const v4i *>(part + i * 16 * kBk + at);
#pragma unroll
          for (int j = 0; j < kFm; ++j) {
            fx[h][j] = *reinterpret_cast<const v4i *>(part + (kRows + j * 16) * kBk + at);
            if (s * 8 + h * 4 + lc >= n_chunk) fx[h][j] = v4i{0, 0, 0, 0};
          }
        }
        asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");  // the part is free
        issue(s + kDeep * kWaves, b);
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int j = 0; j < kFm; ++j)
#pragma unroll
            for (int i = 0; i < kFn; ++i)
              acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fw[h][i], fx[h][j], acc[i][j], 0, 0, 0);
      }
    }
    asm volatile("s_waitcnt vmcnt(0)" : : : "memory");

    // lane: row lr of a 16 x 16 part, weight rows 4 lc ..
    int *sums = reinterpret_cast<int *>(s_ring[wave]);
#pragma unroll
    for (int i = 0; i < kFn; ++i)
#pragma unroll
      for (int j = 0; j < kFm; ++j)
        *reinterpret_cast<v4i *>(sums + (j * 16 + lr) * kPitch + i * 16 + lc * 4) = acc[i][j];
    __syncthreads();
    const float *ws = a.ws + static_cast<int64_t>(tile.w) * a.N;
    for (int o = tid; o < kTok * kOut / 4; o += kThreads) {  // four channels of a row
      const int r = o / (kOut / 4), c = o % (kOut / 4) * 4, n = n0 + c;
      if (r >= tile.rows || n >= a.n_out) continue;
      const float xs = a.xs[tile.row + r];
      auto scaled = [&](int at, int channel) {  // four of the row's products
        v4i sum = {0, 0, 0, 0};
#pragma unroll
        for (int u = 0; u < kWaves; ++u)
          sum += *reinterpret_cast<const v4i *>(reinterpret_cast<int *>(s_ring[u]) + r * kPitch + at);
        v4f v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = static_cast<float>(sum[e]) * xs * ws[channel + e];
        return v;
      };
      v4f v = scaled(c, n);
      if (kAct) {
        const v4f up = scaled(c + kOut, half + n);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = silu(v[e]) * up[e];
      }
      char *out = static_cast<char *>(a.y) + ((tile.row + r) * a.n_out + n) * (kBf16 ? 2 : 4);
      if (kBf16)
        *reinterpret_cast<v2u *>(out) = v2u{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
      else
        *reinterpret_cast<v4f *>(out) = v;
    }
    __syncthreads();
  }
}

// most row tiles that M rows in n_block blocks make: every block that has rows may
// end in a part of a tile
static int64_t most_tiles(const MatmulArgs &a, int tile_rows) {
  return a.M / tile_rows + (a.M < a.n_block ? a.M : a.n_block);
}

#define UEP_LAUNCH_MATMUL(kernel, ...)                                                         \
  if (act && bf16)                                                                             \
    hipLaunchKernelGGL((kernel<__VA_ARGS__, true, true>), grid, block, 0, stream, a, n_col);   \
  else if (act)                                                                                \
    hipLaunchKernelGGL((kernel<__VA_ARGS__, true, false>), grid, block, 0, stream, a, n_col);  \
  else if (bf16)                                                                               \
    hipLaunchKernelGGL((kernel<__VA_ARGS__, false, true>), grid, block, 0, stream, a, n_col);  \
  else                                                                                         \
    hipLaunchKernelGGL((kernel<__VA_ARGS__, false, false>), grid, block, 0, stream, a, n_col)

template <int kTok, int kRows, int kWaves, int kDeep>
static void start_thin(const MatmulArgs &a, bool act, bool bf16, hipStream_t stream) {
  const int out = act ? kRows / 2 : kRows;
  const int32_t n_col = (a.n_out + out - 1) / out;
  const int64_t items = most_tiles(a, kTok) * n_col;
  const dim3 grid(static_cast<unsigned>(items < 1 << 16 ? items : 1 << 16)), block(64 * kWaves);
  UEP_LAUNCH_MATMUL(k_matmul_thin, kTok, kRows, kWaves, kDeep);
}

template <int kN, int kM, int kWn, int kWm, bool kAhead>
static void start_matmul(const MatmulArgs &a, bool act, bool bf16, int n_wg, hipStream_t stream) {
  const int out = act ? kN / 2 : kN;
  const int32_t n_col = (a.n_out + out - 1) / out;
  const int64_t items = most_tiles(a, kM) * n_col;
  const dim3 grid(static_cast<unsigned>(items < n_wg ? (items + 7) / 8 * 8 : n_wg)), block(64 * kWn * kWm);
  UEP_LAUNCH_MATMUL(k_matmul, kN, kM, kWn, kWm, kAhead);
}

hipError_t launch_expert_matmul(const int8_t *xq, const float *xs, int64_t M, const int8_t *wq,
                                const float *ws, int32_t n_w, int32_t N, int32_t K,
                                const int64_t *block_off, const int32_t *block_w, int32_t n_block,
                                int32_t act, void *y, int32_t type, int32_t *status,
                                hipStream_t stream) {
  const MatmulArgs a{xq, xs, wq, ws, block_off, block_w, y, status, M, n_w, N, K, n_block,
                     act ? N / 2 : N};
  const bool bf16 = type == ULTRAEP_BF16;
  // Tiles of 256 x 256 or 128 x 128 where the blocks are large, by the rounds that either
  // takes; 128 x 64 where there are few of those; else, for few rows, the kernel that
  // shares K between waves.  `rows`: M over the blocks, of which the host cannot know how
  // many are empty (a list that is mostly empty, or an M above the rows that the blocks
  // hold, is taken for small or large blocks: the result is the same, the time is not); items:
  // estimated tiles, half a tile of padding a block where there are several.
  //   Times in tenths of a round of 256 x 256: 4 for the round of its quarters, 6 for a
  // round of 128 x 128, two tiles a compute unit.
  //   Measured, us (256 x 256 / 128 x 128 / 128 x 64 / thin 64 / 32 / 16):
  //   10 blocks, N = 4096, K = 7168, act: M = 20480 590 / 646, 10240 323 / 355, 9216 315 /
  //   311, 8192 303 / 298 / 351 / 454 / 561 / 808, 6144 219 / 245, 5120 212 / 190, 3328 156 /
  //   140, 2048 109 / 127 / 139 / 152 / 182 / 250, 1024 103 / 79 / 89 / 100 / 118 / 148,
  //   512 102 / 74 / 71 / 76 / 83 / 96, 256 103 / 70 / 68 / 66 / 65 / 68, 64 98 / 67 / 65
  //   / 64 / 58 / 51
  //   1 block, the same: M = 8704 235 / 277, 8192 199 / 231, 6144 198 / 173, 4608 135 / 165,
  //   4096 102 / 116 / 159 / 204, 2048 79 / 60, 1024 75 / 43 / 50 / 53 / 70, 256
  //   75 / 37 / 34 / 18 / 22 / 26, 128 79 / 38 / 34 / 17 / 13 / 17, 16 78 / 37 / 34 / 16 / 11 / 9
  //   64 blocks, N = 1024, K = 2048: M = 8704 56 / 49, 8192 40 / 50 / 49 / 64, 4608 39 / 42, 4096
  //   38 / 29 / 33 / 44, 1024 37 / 25 / 29 / 30 / 29 / 28
  //   6 blocks, N = 4096, K = 1408: M = 20480 138 / 144, 8704 75 / 70, 8192 61 / 67 / 77, 5120
  //   50 / 44, 512 24 / 14 / 13 / 18 / 18 / 19, 256 23 / 13 / 14 / 12 / 12 / 13, 64 22 / 12 / 11
  //   / 11 / 11 / 10
  //   (The rule misses the best of a line by up to a sixth: 64 blocks of 16 rows, N = 1024,
  //   K = 2048, go to thin 32, 29, where 128 x 128 takes 25.)
  const int64_t blocks = M < n_block ? M : n_block, rows = (M + blocks - 1) / blocks;
  auto items = [&](int64_t tile_rows, int64_t channels) {
    return (blocks > 1 ? M / tile_rows + (blocks + 1) / 2 : (M + tile_rows - 1) / tile_rows) *
           ((N + channels - 1) / channels);
  };
  const int64_t big = items(256, 256), full = big / 256, last = big % 256;
  const int64_t big_time = full * 10 + (last == 0 ? 0 : full && last <= 64 ? 4 : 10);
  const int64_t mid_time = (items(128, 128) + 511) / 512 * 6;
  const bool deep = K >= 4096;  // four waves' worth of steps
  if (rows > 64 && big_time < mid_time)
    start_matmul<256, 256, 2, 2, true>(a, act, bf16, 256, stream);
  else if (rows > 56 && items(128, 128) >= 256)
    start_matmul<128, 128, 2, 2, false>(a, act, bf16, 512, stream);
  else if (rows > 32 && items(64, 128) >= 320)
    start_matmul<128, 64, 2, 1, false>(a, act, bf16, 768, stream);
  else if (rows > 32 && items(64, 64) >= 256 && deep)
    start_thin<64, 64, 4, 2>(a, act, bf16, stream);
  else if (rows > 32 && items(64, 64) >= 256)
    start_thin<64, 64, 2, 2>(a, act, bf16, stream);
  else if (rows > 12 && items(32, 64) >= 256 && deep)
    start_thin<32, 64, 4, 2>(a, act, bf16, stream);
  else if (rows > 12 && items(32, 64) >= 256)
    start_thin<32, 64, 2, 2>(a, act, bf16, stream);
  else if (deep)
    start_thin<16, 32, 4, 2>(a, act, bf16, stream);
  else
    start_thin<16, 64, 2, 2>(a, act, bf16, stream);
  return hipGetLastError();
}

}  // namespace uep
