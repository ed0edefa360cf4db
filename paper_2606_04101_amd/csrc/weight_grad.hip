// The gradient of the experts' weights: for each weight the sum, over its blocks' rows, of
// the outer products of the two sides' rows.
#include <algorithm>

#include "products.hpp"

namespace uep {

struct GradArgs {
  const int8_t *dy, *x;
  const int64_t *block_off;
  const int32_t *block_w;
  void *dw;
  int32_t *status;
  int64_t M, dw_stride;  // (dw_stride in elements)
  int32_t n_w, N, K, n_block;
  int32_t slots;  // in all so many parts of the weights' rows, dw_stride apart; 0: one a weight
};

// steps of 64 that `rows` take; a block may have 2^31 - 1
__device__ __forceinline__ int steps_of(int rows) { return rows / 64 + (rows % 64 != 0); }

// Items item, item + stride, .. below n_item: tiles of a weight's gradient, kM of its rows
// (channels n of dy) by kN of its columns (channels k of x), and of each a part of the rows
// that are summed over.  Both sides are transposed on their way from LDS.  The steps of an
// item are its blocks' rows by 64; a block's last may have fewer.  Blocks are looked at in
// runs of 64, one a lane.
template <class S, bool kBf16, bool kAdd, bool kPast>
struct GradWork {
  static constexpr uint32_t pitch = 0;
  const GradArgs &a;
  const int N, K, n_block, n_run, tn, tk, stride, n_item;
  const int64_t *const block_off;
  const int32_t *const block_w;
  const int8_t *const dy, *const x;
  int item;
  // this lane's block of run `run`: its first row, rows, weight
  int64_t lo;
  int rows, w, run;
  uint64_t mask;  // of the run's blocks of the item's weight that are still to come
  int weight, slot, n0, k0;
  const int *const first_slot;  // of each weight
  int64_t row;    // of the next step
  int remaining;  // rows of its block from there on
  int budget;     // steps of the item's part that are still to come
  bool empty;
  const int8_t *pa, *pa2, *pb, *sa, *sb;
  int left;
  uint32_t pitch_a, pitch_b;

  __device__ GradWork(const GradArgs &g, const int *slots, int first, int step, int n_tile_n, int n_tile_k, int n)
      : a(g), N(__builtin_amdgcn_readfirstlane(g.N)), K(__builtin_amdgcn_readfirstlane(g.K)),
        n_block(__builtin_amdgcn_readfirstlane(g.n_block)), n_run((n_block + kWave - 1) / kWave),
        tn(n_tile_n), tk(n_tile_k), stride(step), n_item(n), block_off(uniform(g.block_off)),
        block_w(uniform(g.block_w)), dy(uniform(g.dy)), x(uniform(g.x)), item(first), first_slot(slots) {
    pitch_a = K * 2;
    pitch_b = N * 2;
    if (n_run == 1) load(0);
  }
  __device__ void load(int r) {
    const int g = r * kWave + lane_id(), at = min(g, n_block - 1);
    lo = block_off[at];
    rows = static_cast<int>(block_off[at + 1] - lo);
    w = block_w ? block_w[at] : at;
    if (g >= n_block) rows = 0;
    run = r;
  }
  // to the first row of the item's next block; remaining 0 if there is none
  __device__ void next_block() {
    remaining = 0;
    while (!mask) {
      if (run + 1 >= n_run) return;
      load(run + 1);
      mask = ballot(w == weight && rows > 0);
    }
    const int l = __builtin_ctzll(mask);
    mask &= mask - 1;
    row = readlane64(lo, l);
    remaining = __builtin_amdgcn_readfirstlane(readlane(rows, l));
  }
  __device__ void first_block() {
    if (n_run == 1) {
      mask = ballot(w == weight && rows > 0);
    } else {
      run = -1;
      mask = 0;
    }
    next_block();
  }
  __device__ bool next_item() {
    const int of_weight = tn * tk;
    auto first_of = [&](int u) { return __builtin_amdgcn_readfirstlane(first_slot[u]); };
    int it, part = 0, parts = 1;
    while (true) {
      if (item >= n_item) return false;
      slot = item / of_weight;
      it = item - slot * of_weight;
      item += stride;
      weight = slot;
      if (a.slots == 0) break;
      if (slot >= first_of(a.n_w)) continue;
      weight = 0;
      for (int end = a.n_w; end - weight > 1;) {
        const int mid = (weight + end) / 2;
        if (first_of(mid) <= slot) weight = mid;
        else end = mid;
      }
      part = slot - first_of(weight);
      parts = first_of(weight + 1) - first_of(weight);
      break;
    }
    // 4 row tiles by all columns at a time (32768 rows of 5, 4096 x 7168: 2 1675 us, 4 1682, 6
    // 1683, 8 1730, 16 1785; 4096 x 8192: 1775, 1740, 1780, 1890, 1925)
    constexpr int kGroup = 4;
    const int group = it / (kGroup * tk), rest = it - group * kGroup * tk;
    const int high = min(kGroup, tn - group * kGroup);
    n0 = (group * kGroup + rest % high) * S::kM;
    k0 = rest / high * S::kN;
    first_block();
    budget = 1 << 30;
    if (parts > 1) {
      int steps = 0;
      static_assert(S::kStep == 64, "steps_of");
      for (; remaining > 0; next_block()) steps += steps_of(remaining);
      int skip = static_cast<int>(static_cast<int64_t>(steps) * part / parts);
      budget = static_cast<int>(static_cast<int64_t>(steps) * (part + 1) / parts) - skip;
      first_block();
      while (budget > 0 && skip >= steps_of(remaining)) {
        skip -= steps_of(remaining);
        next_block();
      }
      if (budget > 0) {
        row += static_cast<int64_t>(skip) * S::kStep;
        remaining -= skip * S::kStep;
      }
    }
    empty = !more();
    return true;
  }
  __device__ bool more() const { return remaining > 0 && budget > 0; }
  __device__ void advance() {
    pa = uniform(x + (row * K + k0) * 2);
    pb = uniform(dy + (row * N + n0) * 2);
    left = __builtin_amdgcn_readfirstlane(min(remaining, S::kStep));
    row += S::kStep;
    remaining -= left;
    --budget;
    if (remaining == 0) next_block();
  }
  __device__ int row_a(int) const { return 0; }
  __device__ int row_b(int) const { return 0; }
  __device__ bool second(int) const { return false; }
  __device__ uint32_t scale_at(int, int) const { return 0; }
  __device__ uint32_t chunk_a(int c) const { return 2 * min(c * 8, K - 8 - k0); }
  __device__ uint32_t chunk_b(int c) const { return 2 * min(c * 8, N - 8 - n0); }

  struct Out {
    int slot, n0, k0;
    bool skip;
  };
  __device__ Out out() const { return {slot, n0, k0, kAdd && empty}; }
  // Added to what is there the sums leave LDS in fp32, 4 channels a lane; a bf16 gradient
  // that is not added to leaves as such, 8.
  static constexpr bool kPacked = kBf16 && !kAdd;
  static constexpr int kLane = kPacked ? 8 : 4, kParts = S::kFn * 2 / kLane;
  static constexpr int kSize = kBf16 ? 2 : 4, kBands = S::kFm / 2;  // (of 32 rows)
  using Word = std::conditional_t<kBf16 && kAdd, v2u, v4u>;  // what a lane stores
  // (added to) what is there, of the next part while one is worked on
  struct Old {
    Word v[2][4];
  };
  struct Nothing {};
  using Early = std::conditional_t<kAdd, Old, Nothing>;
  // the address of what lane el stores of row p * 8 + el / 8 of part n; null outside
  __device__ char *place(const Out &o, int n, int p, int wn, int wm, int el) const {
    const int r = o.n0 + (wm * kBands + n / kParts) * 32 + p * 8 + el / 8;
    const int c = o.k0 + wn * S::kFn * 16 + (n % kParts * 8 + (el & 7)) * kLane;
    if (r >= N || c >= K || o.skip) return nullptr;
    const int64_t at = o.slot * a.dw_stride + static_cast<int64_t>(r) * K + c;
    return static_cast<char *>(a.dw) + at * kSize;
  }
  __device__ void keep(const Out &o, Early &k, int n, int wn, int wm) const {
    if constexpr (kAdd) {
      const int el = opaque(lane_id());
#pragma unroll
      for (int p = 0; p < 4; ++p) {
        const char *at = place(o, n, p, wn, wm, el);
        k.v[n & 1][p] = at ? *reinterpret_cast<const Word *>(at) : Word{};
      }
    }
  }
  __device__ void early(const Out &o, Early &k, int wn, int wm) const { keep(o, k, 0, wn, wm); }

  template <class Acc>
  __device__ void results(const Out &o, Early &old, Acc &acc, int8_t *lds, int wn, int wm) const {
    const Stage st(lds);
#pragma unroll
    for (int b = 0; b < kBands; ++b) {
#pragma unroll
      for (int i = 0; i < S::kFn; ++i) {
        asm volatile("" : "+a"(acc[i][2 * b]));
        asm volatile("" : "+a"(acc[i][2 * b + 1]));
      }
      // before the last stores: all loads, and the earlier stores, are done
      if (S::kAhead && b == kBands - 1) asm volatile("s_waitcnt vmcnt(0)" : : : "memory");
      else asm volatile("" : : : "memory");
#pragma unroll
      for (int i = 0; i < kParts; ++i) {
        const int n = b * kParts + i;
#pragma unroll
        for (int h = 0; h < kLane / 2; ++h)
#pragma unroll
          for (int jj = 0; jj < 2; ++jj)
            st.put(h, jj, acc[i * kLane / 2 + h][2 * b + jj], std::bool_constant<kPacked>());
        if (n + 1 < kBands * kParts) keep(o, old, n + 1, wn, wm);
#pragma unroll
        for (int p = 0; p < 4; ++p) {
          char *at = place(o, n, p, wn, wm, st.el);
          Word word;
          if constexpr (kAdd) {
            v4f v = st.get<v4f>(p);
            const Word w = old.v[n & 1][p];
#pragma unroll
            for (int e = 0; e < 4; ++e)
              v[e] += !kBf16 ? __uint_as_float(w[kBf16 ? 0 : e])
                      : e % 2 ? bf16_at_high(w[e / 2]) : bf16_at_low(w[e / 2]);
            if constexpr (kBf16) word = v2u{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
            else word = __builtin_bit_cast(v4u, v);
          } else {
            word = st.get<v4u>(p);
          }
          if (at) store_result(word, reinterpret_cast<Word *>(at), std::bool_constant<kPast>());
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  }
};

// Whether every block lies in rising order within [0, M], with a weight where it has rows;
// else that is reported.  The whole workgroup has the answer.
template <int kWaves>
__device__ __forceinline__ bool sound_blocks(const GradArgs &a, int *s_sound) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  bool sound = true;
  for (int r = wave * kWave; r < a.n_block; r += kWaves * kWave) {
    const int g = min(r + lane_id(), a.n_block - 1);
    const int64_t lo = a.block_off[g], hi = a.block_off[g + 1];
    const int w = a.block_w ? a.block_w[g] : g;
    sound &= lo >= 0 && hi >= lo && hi <= a.M && (hi == lo || (w >= 0 && w < a.n_w));
  }
  const bool all = !ballot(!sound);
  if (lane_id() == 0) s_sound[wave] = all;
  if (!all && lane_id() == 0) report(a.status, ULTRAEP_EDATA);
  __syncthreads();
  int every = 1;
#pragma unroll
  for (int u = 0; u < kWaves; ++u) every &= s_sound[u];
  return __builtin_amdgcn_readfirstlane(every);
}

constexpr int kMostParted = 256;  // weights whose rows are in parts

// The first of each weight's slots (parts of its rows), and the first that nobody has: one a
// weight and the rest by their rows, in steps of 64, so that a part's steps differ little however
// the rows are spread.  256 threads, with the same result in every workgroup.  s_steps: left with
// each weight's rows in steps of 64.
__device__ __forceinline__ void count_slots(const GradArgs &a, int *s_first, int *s_of, int *s_steps = nullptr) {
  const int tid = threadIdx.x;
  s_of[tid] = 0;
  __syncthreads();
  for (int g = tid; g < a.n_block; g += 256) {
    const int rows = static_cast<int>(a.block_off[g + 1] - a.block_off[g]);
    if (rows > 0) atomicAdd(&s_of[a.block_w ? a.block_w[g] : g], steps_of(rows));
  }
  __syncthreads();
  int total = 0, before = 0;
  for (int u = 0; u < a.n_w; ++u) total += s_of[u];
  // (the shares' roundings, 2^-22 of 2^14 in all, cannot make one more than there are)
  if (s_steps) s_steps[tid] = s_of[tid];
  const int mine = 1 + (total ? static_cast<int>(static_cast<float>(a.slots - a.n_w) * s_of[tid] / total) : 0);
  __syncthreads();
  s_of[tid] = mine;
  __syncthreads();
  for (int u = 0; u < tid && u < a.n_w; ++u) before += s_of[u];
  if (tid < a.n_w) s_first[tid] = before;
  if (tid == a.n_w - 1) s_first[a.n_w] = before + mine;
  __syncthreads();
}

// dw = dy^T x, a weight's tiles of kM rows x kN columns.  As the products bound by the matrix
// units' power, with two transposing reads more a part: 780 us at 8192^3 (1.41 PFLOP/s), 32768
// rows of 5 weights of 4096 x 7168 to fp32 in 1577 to 1722 us by the card (1.12 to 1.22): 2240 tiles are 8.75
// rounds of 256 and the fp32 results 587 MB.  Few rows a weight are bound by the results' bytes
// (2991 rows over 16 weights of 2880 x 1440, bf16: 54 us, of which the bytes take 25).
template <int kN, int kM, int kWn, int kWm, bool kAhead, bool kBf16, bool kAdd, bool kPast>
__global__ void __launch_bounds__(64 * kWn * kWm) k_weight_grad(GradArgs a, int32_t tn, int32_t tk) {
  using S = Tile<kN, kM, kWn, kWm, kAhead, 2, kMath16, true, true>;
  __shared__ __align__(1024) int8_t s_lds[S::kLds];
  static_assert(S::kThreads == 256, "slots are counted by 256 threads");
  __shared__ int s_sound[S::kWaves], s_first[kMostParted + 1];
  if (!sound_blocks<S::kWaves>(a, s_sound)) return;
  if (a.slots) count_slots(a, s_first, reinterpret_cast<int *>(s_lds));
  constexpr int kXcd = 8;  // the workgroups of one XCD take neighbouring items
  const int grid = gridDim.x, per_xcd = grid / kXcd;  // the grid is a multiple
  const int slot = blockIdx.x % kXcd * per_xcd + blockIdx.x / kXcd;
  GradWork<S, kBf16, kAdd, kPast> work(a, s_first, slot, grid, tn, tk, (a.slots ? a.slots : a.n_w) * tn * tk);
  tile_items<S>(work, s_lds);
}

// The parts' sums, in order: 4 elements a thread.  (Added to what is there: a weight without
// rows is not touched, -0 + 0 would be 0.)
template <bool kBf16>
__global__ void __launch_bounds__(256)
k_weight_grad_sum(GradArgs a, const v4f *from, int64_t of_weight, int32_t accumulate) {
  __shared__ int s_sound[4], s_first[kMostParted + 1], s_of[256], s_steps[256];
  if (!sound_blocks<4>(a, s_sound)) return;
  count_slots(a, s_first, s_of, s_steps);
  const int64_t all = of_weight * a.n_w, step = static_cast<int64_t>(gridDim.x) * 256;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < all; i += step) {
    const int weight = static_cast<int>(i / of_weight), last = s_first[weight + 1];
    if (accumulate && s_steps[weight] == 0) continue;
    const int64_t e = i % of_weight;
    v4f v = from[s_first[weight] * of_weight + e];
    for (int p = s_first[weight] + 1; p < last; ++p) v += from[p * of_weight + e];
    const int64_t at = weight * a.dw_stride + e * 4;
    if (kBf16) {
      v2u *to = reinterpret_cast<v2u *>(static_cast<uint16_t *>(a.dw) + at);
      if (accumulate) {
        const v2u w = *to;
        v += v4f{bf16_at_low(w.x), bf16_at_high(w.x), bf16_at_low(w.y), bf16_at_high(w.y)};
      }
      *to = v2u{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
    } else {
      v4f *to = reinterpret_cast<v4f *>(static_cast<float *>(a.dw) + at);
      *to = accumulate ? *to + v : v;
    }
  }
}

// Slots, over all weights: where the weights' tiles would not fill the card, so many that they
// do, of 512 rows at least; and, where they would fill little more than that, of 2048 rows, so that
// one weight with most of the rows does not hold up the call.  No more with fewer rows.
static int32_t row_slots(int64_t M, int32_t N, int32_t K, int32_t n_w) {
  const int64_t of_weight = int64_t((N + 127) / 128) * ((K + 127) / 128), tiles = n_w * of_weight;
  if (n_w > kMostParted || tiles > 384) return 0;
  const int64_t fill = std::min({512 / tiles, M / (int64_t(n_w) * 512), int64_t(64)}) * n_w;
  const int64_t spread = std::min({1024 / of_weight, M / 2048, int64_t(64) * n_w});
  const int64_t slots = std::max(fill, spread);
  return static_cast<int32_t>(slots > n_w ? slots : 0);
}

size_t weight_grad_ws_bytes(int64_t M, int32_t N, int32_t K, int32_t n_w) {
  const int64_t slots = row_slots(M, N, K, n_w);
  return slots ? static_cast<size_t>(slots) * N * K * 4 : 16;
}

template <int kN, int kM, int kWn, int kWm, bool kAhead, bool kBf16, bool kAdd, bool kPast>
static void start_grad(const GradArgs &a, int n_wg, hipStream_t stream) {
  const int32_t tn = (a.N + kM - 1) / kM, tk = (a.K + kN - 1) / kN;
  const int64_t items = int64_t(a.slots ? a.slots : a.n_w) * tn * tk;
  const dim3 grid(static_cast<unsigned>(items < n_wg ? (items + 7) / 8 * 8 : n_wg)), block(64 * kWn * kWm);
  hipLaunchKernelGGL((k_weight_grad<kN, kM, kWn, kWm, kAhead, kBf16, kAdd, kPast>), grid, block, 0, stream, a, tn, tk);
}

// Tiles of 256 x 256 or, two a compute unit, of 128 x 128, by the rounds that either takes, in
// twentieths of a round of the first; the second where a weight has few rows, so that the
// results' bytes bound the call, and it pads less or its stores fill lines together.  Measured, us (256 / 128; fp32 results):
//   5 weights, N = 4096, K = 7168: M = 16384 855 / 1004; N = 7168, K = 2048: M = 16384 441 / 504,
//   1024 79 / 74; 4 weights, N = K = 2048: M = 32768 197 / 247, 8192 60 / 67, 1024 20.5 / 20.6; 2
//   weights, K = 2048, M = 8192: N = 2048 94 / 64, 1024 67 / 49, 512 43 / 32; 8 weights, K = 1024,
//   M = 8192: N = 2048 37 / 37, 1024 31 / 21; 64 weights, N = 1024, K = 2048: M = 4096 91 / 104; 16
//   weights, N = 2880, K = 1440: M = 2000 69 / 56 (bf16 results 48 / 40)
//   Out of a cache that holds no results yet: 16 weights, N = 2880, K = 1440: M = 8192 113 / 104, 2991
//   to bf16 76 / 54; 6 of 4096 x 1408, M = 2048 to bf16 46 / 40; 10 of 4096 x 7168, M = 4096 353 / 391
//   Rows of no whole lines, to bf16: 6 weights, N = 5584, K = 3048, M = 277 127 / 63; K = 3040, M = 1024
//   77 / 70; 6 of 4096 x 1440, M = 2048 46 / 41
static bool large_tiles(const GradArgs &a, bool bf16) {
  auto tiles = [&](int64_t n, int64_t k) {
    return int64_t(a.slots ? a.slots : a.n_w) * ((a.N + n - 1) / n) * ((a.K + k - 1) / k);
  };
  const int64_t big = (tiles(256, 256) + 255) / 256 * 20, mid = (tiles(128, 128) + 511) / 512 * 13;
  const bool lines = a.K * (bf16 ? 2 : 4) % 128 == 0;  // the smaller tiles' stores may fill them together
  const bool few = a.M < int64_t(768) * a.n_w && (!lines || tiles(128, 128) < 4 * tiles(256, 256));
  return big < mid && !few;
}
template <bool kBf16, bool kAdd>
static void choose_grad(const GradArgs &a, hipStream_t stream) {
  if (large_tiles(a, kBf16)) return start_grad<256, 256, 2, 2, true, kBf16, kAdd, true>(a, 256, stream);
  // Stores as by_halves chooses them; here by instances, since small calls feel the longer
  // code (31 rows, 160 x 160 5.0 us, with both kinds 5.2).  What is added to has just been read, and
  // parts are read again at once: through the caches (added to, either takes the same; 2535 rows,
  // 96 x 224 in parts 14.2, past them 15.0).
  if constexpr (!kAdd)
    if (a.slots == 0 && whole_halves(a.dw, (a.K | a.dw_stride) * (kBf16 ? 2 : 4)))
      return start_grad<128, 128, 2, 2, false, kBf16, kAdd, true>(a, 512, stream);
  start_grad<128, 128, 2, 2, false, kBf16, kAdd, false>(a, 512, stream);
}

hipError_t launch_expert_weight_grad(const uint16_t *dy, const uint16_t *x, int64_t M, int32_t N,
                                     int32_t K, const int64_t *block_off, const int32_t *block_w,
                                     int32_t n_block, int32_t n_w, int64_t dw_stride,
                                     int32_t accumulate, void *dw, int32_t type, void *ws,
                                     int32_t *status, hipStream_t stream) {
  GradArgs a{reinterpret_cast<const int8_t *>(dy), reinterpret_cast<const int8_t *>(x), block_off, block_w, dw, status,
             M, dw_stride, n_w, N, K, n_block, 0};
  const bool bf16 = type == ULTRAEP_BF16;
  const int32_t slots = ws ? row_slots(M, N, K, n_w) : 0;
  if (slots) {
    GradArgs part = a;
    const int64_t of_weight = int64_t(N) * K;
    part.dw = ws;
    part.dw_stride = of_weight;
    a.slots = part.slots = slots;
    choose_grad<false, false>(part, stream);
    const int64_t wg = (of_weight / 4 * n_w + 255) / 256;
    const dim3 grid(static_cast<unsigned>(wg < 2048 ? wg : 2048));
    if (bf16) hipLaunchKernelGGL((k_weight_grad_sum<true>), grid, dim3(256), 0, stream, a, static_cast<const v4f *>(ws), of_weight / 4, accumulate);
    else hipLaunchKernelGGL((k_weight_grad_sum<false>), grid, dim3(256), 0, stream, a, static_cast<const v4f *>(ws), of_weight / 4, accumulate);
  } else if (accumulate) {
    if (bf16) choose_grad<true, true>(a, stream);
    else choose_grad<false, true>(a, stream);
  } else {
    if (bf16) choose_grad<true, false>(a, stream);
    else choose_grad<false, false>(a, stream);
  }
  return hipGetLastError();
}

}  // namespace uep

// Whether a call takes tiles of 256 x 256, for the tests (host only): parts, whether it has a
// workspace
extern "C" int uep_weight_grad_large(int64_t M, int32_t N, int32_t K, int32_t n_w, int32_t type, int32_t parts) {
  const int32_t slots = parts ? uep::row_slots(M, N, K, n_w) : 0;
  uep::GradArgs a{};
  a.M = M, a.N = N, a.K = K, a.n_w = n_w, a.slots = slots;
  return uep::large_tiles(a, type == ULTRAEP_BF16 && !slots);
}
