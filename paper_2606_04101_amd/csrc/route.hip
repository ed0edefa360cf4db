// The router of an MoE layer: top-k ids and gates from the logits, the
// statistics of its balance loss, the loss, and the logits' gradient.
//
// A row of 16 lanes, or a whole wave, takes one token.  Its E logits lie across
// the lanes in id order: with groups, 2^n lanes share a group and each holds kVpl
// neighbouring experts of it; without, all lanes share the one group.  So a
// group's sum of two largest keys is a merge over neighbouring lanes.  Where a
// group does not fill its lanes, the ends of them are holes: an expert's place
// among lanes and holes is its slot, of the same order as the ids.
//
// A call reads little (4096 tokens of 256 experts: 4 MB), so instructions and the
// chain of loads bound it, and launches: ids, gates and statistics of those 4096
// tokens, by groups, take 8.4 us, their sums over the workgroups 2.8, the loss 2.5, the
// gradient 4.8; 16384 tokens of 128 experts 9.4, 3.8, 1.8; one token of 256 4.6.  Prompts are
// bound by instructions: 65536 tokens of 256 in groups take 36 us, 47 with statistics, where
// their 71 MB take 14.
#include "operators.hpp"

namespace uep {

constexpr int kRtThreads = 256;
constexpr int kRtWaves = kRtThreads / kWave;
constexpr int kRtMaxE = 1024;
constexpr float kInf = __builtin_inff();

struct RouteArgs {
  const void *logits;
  int64_t T, ld;
  const float *bias;
  const uint8_t *mask;
  int32_t *topk;
  float *gate;
  int32_t E, k, sigmoid, renorm, n_group, top_group;
  int32_t group_lanes;  // lanes of a group, a power of two
  int32_t wide;         // all lanes that have experts have kVpl, in aligned chunks
  int32_t wide_bias;    // and so with the bias
  // the top_group groups spread over all lanes: lanes of one, a power of two, and slots
  // of such a lane, a multiple of 4; 0 slots: they stay where they are
  int32_t pick_lanes, pick;
  float scale;
  int64_t seq, chunk, n_chunk;
  int32_t *counts;  // outputs, or the workspace's partials if n_chunk > 1
  float *prob_sum;
  int32_t *tokens;
  int32_t *status;
};

template <bool kBf16>
__device__ __forceinline__ float load_logit(const void *row, int e) {
  if (kBf16) return bf16_at_low(static_cast<const uint16_t *>(row)[e]);
  return static_cast<const float *>(row)[e];
}

// elements that a lane with kVpl of them loads at once: 16 bytes, or 8 in bf16
constexpr int chunk_of(int vpl, bool bf16) { return bf16 && vpl % 8 == 0 ? 8 : 4; }

// kC logits from element e on, together: aligned
template <int kC, bool kBf16>
__device__ __forceinline__ void load_chunk(const void *row, int64_t e, float *z) {
  if constexpr (kBf16) {
    typedef uint32_t raw __attribute__((ext_vector_type(kC / 2)));
    const raw v = *reinterpret_cast<const raw *>(static_cast<const uint16_t *>(row) + e);
#pragma unroll
    for (int i = 0; i < kC; ++i) z[i] = i % 2 ? bf16_at_high(v[i / 2]) : bf16_at_low(v[i / 2]);
  } else {
#pragma unroll
    for (int c = 0; c < kC; c += 4) {
      const v4f v = *reinterpret_cast<const v4f *>(static_cast<const float *>(row) + e + c);
#pragma unroll
      for (int i = 0; i < 4; ++i) z[c + i] = v[i];
    }
  }
}

// A lane's logits, neighbours in the row, -inf past the n it has.
template <int kVpl, bool kBf16>
__device__ __forceinline__ void load_logits(const void *row, int base, int n, bool wide,
                                            float (&z)[kVpl]) {
  constexpr int kC = chunk_of(kVpl, kBf16);
  if constexpr (kVpl % kC == 0) {
    if (wide) {
#pragma unroll
      for (int i = 0; i < kVpl; ++i) z[i] = -kInf;
      if (n > 0) {
#pragma unroll
        for (int c = 0; c < kVpl; c += kC) load_chunk<kC, kBf16>(row, base + c, z + c);
      }
      return;
    }
  }
  // (not 2 * kVpl scalar registers of comparisons held throughout a loop)
  asm volatile("" : "+v"(n));
#pragma unroll
  for (int i = 0; i < kVpl; ++i) z[i] = i < n ? load_logit<kBf16>(row, base + i) : -kInf;
}

// fp32 as an integer of the same order (-0 as +0)
__device__ __forceinline__ int order_of(float v) {
  const int i = __float_as_int(v + 0.f);
  return i ^ ((i >> 31) & 0x7FFFFFFF);
}

// the two largest of two pairs
__device__ __forceinline__ void merge_two(float &a1, float &a2, float b1, float b2) {
  a2 = larger(__builtin_amdgcn_fmed3f(a1, b1, -kInf), larger(a2, b2));
  a1 = larger(a1, b1);
}

// the lanes of this lane's token among those of a ballot, its first one at bit 0
template <int kLanes>
__device__ __forceinline__ uint64_t mine(uint64_t bits) {
  if (kLanes == kWave) return bits;
  return bits >> (lane_id() & ~(kLanes - 1)) & ((uint64_t(1) << (kLanes % kWave)) - 1);
}

// LDS writes of a wave's lanes before this are seen by its reads after it
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// The k largest keys by taking out the largest k times: a tie goes to the lowest
// lane and there to the lowest element, which is the lower id.  slots[j]: the j-th.
template <int kLanes, int kVpl>
__device__ void select_by_rounds(float (&key)[kVpl], int k, int *slots) {
  const int l = lane_id() % kLanes;
  for (int j = 0; j < k; ++j) {
    float m = key[0];
#pragma unroll
    for (int i = 1; i < kVpl; ++i) m = larger(m, key[i]);
    const float best = lanes_max<kLanes>(m);
    const bool can = m == best && best > -kInf;
    const uint64_t who = ballot(can);
    if (!who) break;
    const bool own = can && l == __builtin_ctzll(mine<kLanes>(who) | uint64_t(1) << 63);
    const float wanted = own ? best : __builtin_nanf("");
    int at = -1;
#pragma unroll
    for (int i = kVpl - 1; i >= 0; --i) at = key[i] == wanted ? i : at;
#pragma unroll
    for (int i = 0; i < kVpl; ++i) key[i] = at == i ? -kInf : key[i];
    if (own) slots[j] = l * kVpl + at;
  }
}

// The same for a token in 16 lanes, k <= 16, where few keys are likely to be among the
// k largest: a key below the k-th largest of the lanes' largest keys is not.  What is left
// (of 256 random keys 11, k = 8) goes to LDS, and each finds its place by counting those
// ahead of it.  False (in the whole wave) where more than 32 are left.
//   key   this lane's n keys, of slots from, from + 1 ..
//   row   the token's keys in LDS by slot;  left: 32 pairs of words in LDS
constexpr int kMostLeft = 32;
template <int kVpl>
__device__ bool select_by_rank(const float (&key)[kVpl], int n, int from, int k, const float *row,
                               int64_t *left, int *slots) {
  const int l = lane_id() % 16;
  float m = -kInf;
#pragma unroll
  for (int c = 0; c < kVpl; c += 4)
    if (c < n) {
#pragma unroll
      for (int i = c; i < c + 4; ++i) m = larger(m, key[i]);
    }
  int above = 0;  // lanes whose largest is larger
#define UEP_TURN(i) above += dpp_f<0x120 + i>(m) > m;  // row_ror
  UEP_TURN(1) UEP_TURN(2) UEP_TURN(3) UEP_TURN(4) UEP_TURN(5) UEP_TURN(6) UEP_TURN(7) UEP_TURN(8)
  UEP_TURN(9) UEP_TURN(10) UEP_TURN(11) UEP_TURN(12) UEP_TURN(13) UEP_TURN(14) UEP_TURN(15)
#undef UEP_TURN
  // (at least the type's lowest value, so that no -inf is left)
  const float least = larger(-lanes_max<16>(above < k ? -m : -kInf), -__FLT_MAX__);
  uint32_t mask = 0;  // of the keys that are left
#pragma unroll
  for (int c = 0; c < kVpl; c += 4)
    if (c < n) {
#pragma unroll
      for (int i = c; i < c + 4; ++i) mask |= key[i] >= least ? 1u << i : 0u;
    }
  const int some = __popc(mask);
  int at = some;  // inclusive sum over the row
  at += __builtin_amdgcn_update_dpp(0, at, 0x111, 0xF, 0xF, false);
  at += __builtin_amdgcn_update_dpp(0, at, 0x112, 0xF, 0xF, false);
  at += __builtin_amdgcn_update_dpp(0, at, 0x114, 0xF, 0xF, false);
  at += __builtin_amdgcn_update_dpp(0, at, 0x118, 0xF, 0xF, false);
  const int total = lanes_max<16>(at), most = wave_max(total);
  if (most > kMostLeft) return false;
  int *left_slot = reinterpret_cast<int *>(left) + 2 * (at - some);
  while (ballot(mask != 0)) {
    if (mask) {
      *left_slot = from + __builtin_ctz(mask);
      left_slot += 2;
      mask &= mask - 1;
    }
  }
  wave_sync();
  // (key, lower slot first) as one number
  int64_t v[2] = {INT64_MIN, INT64_MIN};
#pragma unroll
  for (int u = 0; u < 2; ++u)
    if (u * 16 < most) {
      if (u * 16 + l < total) {
        const int slot = reinterpret_cast<int *>(left)[2 * (u * 16 + l)];
        v[u] = static_cast<int64_t>(order_of(row[slot])) << 32 | static_cast<uint32_t>(~slot);
      }
      wave_sync();
      left[u * 16 + l] = v[u];
    }
  wave_sync();
  int place[2] = {0, 0};
#pragma unroll 8
  for (int j = 0; j < most; ++j) place[0] += left[j] > v[0];
  if (v[0] != INT64_MIN && place[0] < k) slots[place[0]] = static_cast<int>(~static_cast<uint32_t>(v[0]));
  if (most > 16) {
#pragma unroll 8
    for (int j = 0; j < most; ++j) place[1] += left[j] > v[1];
    if (v[1] != INT64_MIN && place[1] < k) slots[place[1]] = static_cast<int>(~static_cast<uint32_t>(v[1]));
  }
  return true;
}

// a lane's values into its part of a row in LDS
template <int kVpl>
__device__ __forceinline__ void put_lane(float *row, int l, const float (&v)[kVpl]) {
  if constexpr (kVpl % 4 == 0) {
#pragma unroll
    for (int i = 0; i < kVpl; i += 4)
      *reinterpret_cast<v4f *>(row + l * kVpl + i) = v4f{v[i], v[i + 1], v[i + 2], v[i + 3]};
  } else {
#pragma unroll
    for (int i = 0; i < kVpl; ++i) row[l * kVpl + i] = v[i];
  }
}

// 16 experts a lane without statistics would take 186 registers; held to 168, with 4 words
// spilled, a SIMD has three waves instead of two.  us with 168 and 186: 65536 tokens of 256
// experts in groups 36 and 44, without groups 26 and 34, 16384 in groups 13.0 and 13.9, 4096
// 6.5 and 6.3.
template <int kLanes, int kVpl, bool kBf16, bool kStats>
__global__ void __launch_bounds__(kRtThreads, kLanes == 16 && kVpl == 16 && !kStats ? 3 : 1)
k_route(RouteArgs a) {
  constexpr int kTok = kWave / kLanes;  // tokens of a wave
  constexpr int kParts = kRtWaves * kTok;
  constexpr int kSlots = kLanes * kVpl;
  // a token's logits, and its keys, by slot; at the end the parts' sums of the scores
  __shared__ __align__(16) float s_row[kParts * kSlots];
  __shared__ __align__(16) float s_key[kLanes == 16 ? kParts * kSlots : 1];
  __shared__ int64_t s_left[kLanes == 16 ? kParts * kMostLeft : 1];
  __shared__ int s_slots[kRtWaves][kWave];
  __shared__ int s_count[kStats ? kSlots : 1];
  __shared__ int s_tokens;
  const int wave = threadIdx.x / kWave, l = lane_id() % kLanes, part = threadIdx.x / kLanes;
  const int gsz = a.E / a.n_group;
  const int group = l / a.group_lanes, sub = l - group * a.group_lanes;
  const int base = group * gsz + sub * kVpl;
  const int n_mine = group < a.n_group ? min(max(gsz - sub * kVpl, 0), kVpl) : 0;
  const int hole = a.group_lanes * kVpl - gsz;  // slots of a group without expert
  const bool by_score = a.sigmoid && (a.bias || a.n_group > 1);

  if (kStats) {
    for (int e = threadIdx.x; e < a.E; e += kRtThreads) s_count[e] = 0;
    if (threadIdx.x == 0) s_tokens = 0;
    __syncthreads();
  }
  float bias[kVpl] = {};
  if (a.bias) {
    load_logits<kVpl, false>(a.bias, base, n_mine, a.wide_bias, bias);
    float odd = 0.f;  // a NaN if a bias is no finite number
#pragma unroll
    for (int i = 0; i < kVpl; ++i) {
      bias[i] = i < n_mine ? bias[i] : 0.f;
      odd = fmaf(bias[i], 0.f, odd);
    }
    if (ballot(odd != 0.f)) {  // no key is to be a NaN, also where +inf meets a logit of -inf
      bool nan = false;
#pragma unroll
      for (int i = 0; i < kVpl; ++i) {
        const bool bad = bias[i] != bias[i];
        nan |= bad;
        bias[i] = bad ? -kInf : fminf(bias[i], __FLT_MAX__);
      }
      if (nan && blockIdx.x == 0) report(a.status, ULTRAEP_EDATA);
    }
  }
  float acc[kVpl] = {};
  int n_tokens = 0;
  float *z_row = s_row + part * kSlots;
  float *key_row = kLanes == 16 ? s_key + part * kSlots : nullptr;

  const int64_t seg = blockIdx.x / a.n_chunk;
  const int64_t t0 = seg * a.seq + (blockIdx.x - seg * a.n_chunk) * a.chunk;
  const int64_t t1 = min(min(t0 + a.chunk, (seg + 1) * a.seq), a.T);
  // (all of a wave's tokens are taken together, so every lane goes through all of this)
  for (int64_t tw = t0 + wave * kTok; tw < t1; tw += kParts) {
    const int64_t t = tw + (kTok > 1 ? lane_id() / kLanes : 0);
    const bool here = t < t1;
    const char *row = static_cast<const char *>(a.logits) + (here ? t : tw) * a.ld * (kBf16 ? 2 : 4);
    float z[kVpl];
    load_logits<kVpl, kBf16>(row, base, n_mine, a.wide, z);
    bool on = here && (!a.mask || a.mask[t] != 0);
    float top = -kInf, sum_z = 0.f;  // the sum is a NaN if a logit is (and cannot overflow)
#pragma unroll
    for (int i = 0; i < kVpl; ++i) {
      top = larger(top, z[i]);
      sum_z = fmaf(z[i], 0x1p-12f, sum_z);
    }
    if (mine<kLanes>(ballot(!(sum_z < kInf))) && on) {
      if (l == 0) report(a.status, ULTRAEP_EDATA);
      on = false;
    }
    top = lanes_max<kLanes>(top);
    on = on && top > -kInf;
    if (!ballot(on)) {
      if (here && l < a.k) {
        a.topk[t * a.k + l] = -1;
        a.gate[t * a.k + l] = 0.f;
      }
      continue;
    }
    put_lane<kVpl>(z_row, l, z);

    float s[kVpl];  // scores (sigmoid)
    if (a.sigmoid && (by_score || kStats)) {
#pragma unroll
      for (int i = 0; i < kVpl; ++i) s[i] = sigmoid(z[i]);
    }
    float key[kVpl];  // -inf: not to be chosen
#pragma unroll
    for (int i = 0; i < kVpl; ++i) key[i] = (by_score && z[i] > -kInf ? s[i] : z[i]) + bias[i];
    if (kLanes == 16) put_lane<kVpl>(key_row, l, key);
    bool keep = on;
    if (a.n_group > 1) {
      float m1 = -kInf, m2 = -kInf;
#pragma unroll
      for (int i = 0; i < kVpl; ++i) {
        m2 = __builtin_amdgcn_fmed3f(m1, m2, key[i]);
        m1 = larger(m1, key[i]);
      }
      if (a.group_lanes > 1) merge_two(m1, m2, dpp_f<0xB1>(m1), dpp_f<0xB1>(m2));
      if (a.group_lanes > 2) merge_two(m1, m2, dpp_f<0x4E>(m1), dpp_f<0x4E>(m2));
      if (a.group_lanes > 4) merge_two(m1, m2, dpp_f<0x141>(m1), dpp_f<0x141>(m2));
      if (a.group_lanes > 8) merge_two(m1, m2, dpp_f<0x140>(m1), dpp_f<0x140>(m2));
      for (int d = 16; d < a.group_lanes; d *= 2)
        merge_two(m1, m2, __shfl_xor(m1, d), __shfl_xor(m2, d));
      const float score = m2 > -kInf ? m1 + m2 : -kInf;  // (-inf, not a NaN, of +inf alone)
      int before = 0, top = a.top_group;  // groups ahead of this lane's
      if constexpr (kLanes == 16) {
        // their lanes: of a larger score, or of the same one and in front of this group
        const int mine = order_of(group < a.n_group ? score : -kInf);
        int at = l;  // (not 15 of the comparisons below held throughout the loop)
        asm volatile("" : "+v"(at));
#define UEP_TURN(i) before += dpp_i<0x120 + i>(mine) >= mine + (at < i);  // row_ror
        UEP_TURN(1) UEP_TURN(2) UEP_TURN(3) UEP_TURN(4) UEP_TURN(5) UEP_TURN(6) UEP_TURN(7)
        UEP_TURN(8) UEP_TURN(9) UEP_TURN(10) UEP_TURN(11) UEP_TURN(12) UEP_TURN(13) UEP_TURN(14)
        UEP_TURN(15)
#undef UEP_TURN
        before -= sub;
        top *= a.group_lanes;
      } else {
        for (int g = 0; g < a.n_group; ++g) {
          const float o = readlane_f(score, g * a.group_lanes);
          before += o > score || (o == score && g < group);
        }
      }
      keep = keep && group < a.n_group && before < top;
    }

    int *slots = &s_slots[wave][lane_id() - l];
    slots[l] = -1;
    bool done = false;
    if constexpr (kLanes == 16) {
      float some[kVpl];
      if (a.pick > 0) {  // the groups that are left, over all lanes: pick keys a lane
        uint32_t left = static_cast<uint32_t>(mine<16>(ballot(keep && sub == 0)));
        const int nth = l / a.pick_lanes;
        for (int j = 0; j < nth; ++j) left &= left - 1;
        const int from = (left ? __builtin_ctz(left) * kVpl : 0) + (l - nth * a.pick_lanes) * a.pick;
        const bool has = nth < a.top_group && left;
        wave_sync();
#pragma unroll
        for (int c = 0; c < kVpl; c += 4)
          if (c < a.pick) {
            const v4f v = *reinterpret_cast<const v4f *>(key_row + (has ? from : 0) + c);
#pragma unroll
            for (int i = 0; i < 4; ++i) some[c + i] = has ? v[i] : -kInf;
          }
        done = select_by_rank<kVpl>(some, a.pick, from, a.k, key_row, s_left + part * kMostLeft, slots);
      } else {
#pragma unroll
        for (int i = 0; i < kVpl; ++i) some[i] = keep ? key[i] : -kInf;
        done = select_by_rank<kVpl>(some, kVpl, l * kVpl, a.k, key_row, s_left + part * kMostLeft, slots);
      }
    }
    if (!done) {
#pragma unroll
      for (int i = 0; i < kVpl; ++i) key[i] = keep ? key[i] : -kInf;
      select_by_rounds<kLanes, kVpl>(key, a.k, slots);
    }
    wave_sync();
    const int slot = l < a.k ? slots[l] : -1;
    // ids fill from the front: without a first one (every best group held only
    // -inf and lone experts) the token has none
    on = on && slots[0] >= 0;
    const float my_z = slot >= 0 ? z_row[slot] : -kInf;
    int my_id = slot;
    if (hole > 0 && slot >= 0) my_id -= slot / (a.group_lanes * kVpl) * hole;

    // scores over all experts: u = s / exp(c), c so that no u of weight vanishes
    float g = 0.f;
    if (a.sigmoid) {
      if (a.renorm) {
        const float c = lanes_max<kLanes>(slot >= 0 ? fminf(my_z, 0.f) : -kInf);
        const float u = slot >= 0 ? sigmoid_over(my_z, c) : 0.f;
        g = u * fast_rcp(lanes_sum<kLanes>(u));
      } else {
        g = slot >= 0 ? sigmoid(my_z) : 0.f;
      }
    } else if (a.renorm) {
      const float c = lanes_max<kLanes>(my_z);
      const float u = slot >= 0 ? exp_neg(my_z - c) : 0.f;
      g = u * fast_rcp(lanes_sum<kLanes>(u));
    }
    if (kStats || (!a.sigmoid && !a.renorm)) {
      float u[kVpl], sum = 0.f, c = 0.f;
      if (!a.sigmoid) {
        c = on ? top : 0.f;
#pragma unroll
        for (int i = 0; i < kVpl; ++i) u[i] = exp_neg(z[i] - c);
      } else if (ballot(on && top < -60.f)) {
        c = on ? fminf(top, 0.f) : 0.f;
#pragma unroll
        for (int i = 0; i < kVpl; ++i) u[i] = sigmoid_over(z[i], c);
      } else {
#pragma unroll
        for (int i = 0; i < kVpl; ++i) u[i] = s[i];
      }
#pragma unroll
      for (int i = 0; i < kVpl; ++i) sum += u[i];
      sum = lanes_sum<kLanes>(sum);
      const float inv = on ? fast_rcp(sum) : 0.f;
      if (kStats) {
#pragma unroll
        for (int i = 0; i < kVpl; ++i) acc[i] += on ? u[i] * inv : 0.f;
        n_tokens += on;
      }
      if (!a.sigmoid && !a.renorm) g = slot >= 0 ? exp_neg(my_z - c) * inv : 0.f;
    }
    if (here && l < a.k) {
      a.topk[t * a.k + l] = my_id;
      a.gate[t * a.k + l] = slot >= 0 ? g * a.scale : 0.f;
      if (kStats && slot >= 0) atomicAdd(&s_count[my_id], 1);
    }
    wave_sync();
  }

  if (kStats) {
    put_lane<kVpl>(z_row, l, acc);
    if (l == 0 && n_tokens) atomicAdd(&s_tokens, n_tokens);
    __syncthreads();
    for (int e = threadIdx.x; e < a.E; e += kRtThreads) {
      const int slot = e + (hole > 0 ? e / gsz * hole : 0);
      float p = 0.f;
#pragma unroll
      for (int w = 0; w < kParts; ++w) p += s_row[w * kSlots + slot];
      a.prob_sum[static_cast<int64_t>(blockIdx.x) * a.E + e] = p;
      a.counts[static_cast<int64_t>(blockIdx.x) * a.E + e] = s_count[e];
    }
    if (threadIdx.x == 0) a.tokens[blockIdx.x] = s_tokens;
  }
}

// A sequence's partials, 8 experts a workgroup: 128 threads an expert take the chunks in
// turn, and their sums are added over lanes 8 apart, then over waves in order.  The
// first workgroup of a sequence also sums its tokens.
constexpr int kRsThreads = 1024, kRsExperts = 8, kRsTurns = kRsThreads / kRsExperts;
__global__ void __launch_bounds__(kRsThreads)
k_route_sum(const int32_t *__restrict__ part_c, const float *__restrict__ part_p,
            const int32_t *__restrict__ part_n, int64_t n_chunk, int32_t E, int32_t n_eb,
            int32_t *__restrict__ counts, float *__restrict__ prob_sum,
            int32_t *__restrict__ tokens) {
  constexpr int kWaves = kRsThreads / kWave;
  __shared__ float s_p[kWaves][kRsExperts];
  __shared__ int s_c[kWaves][kRsExperts];
  const int64_t seg = blockIdx.x / n_eb;
  const int eb = static_cast<int>(blockIdx.x - seg * n_eb);
  const int i = threadIdx.x % kRsExperts, turn = threadIdx.x / kRsExperts;
  const int e = min(eb * kRsExperts + i, E - 1);
  float p = 0.f;
  int c = 0;
#pragma unroll 8
  for (int64_t j = turn; j < n_chunk; j += kRsTurns) {
    p += part_p[(seg * n_chunk + j) * E + e];
    c += part_c[(seg * n_chunk + j) * E + e];
  }
#pragma unroll
  for (int d = kRsExperts; d < kWave; d *= 2) {
    p += __shfl_xor(p, d);
    c += __shfl_xor(c, d);
  }
  const int wave = threadIdx.x / kWave;
  if (lane_id() < kRsExperts) {
    s_p[wave][i] = p;
    s_c[wave][i] = c;
  }
  if (eb == 0 && wave == kWaves - 1) {
    int n = 0;
#pragma unroll 8
    for (int64_t j = lane_id(); j < n_chunk; j += kWave) n += part_n[seg * n_chunk + j];
    n = wave_sum(n);
    if (lane_id() == 0) tokens[seg] = n;
  }
  __syncthreads();
  if (turn == 0 && eb * kRsExperts + i < E) {
    p = s_p[0][i];
    c = s_c[0][i];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) {
      p += s_p[w][i];
      c += s_c[w][i];
    }
    prob_sum[seg * E + e] = p;
    counts[seg * E + e] = c;
  }
}

// Workgroups past the first write the coefficients; the first sums the loss, in
// 64 bits and one order.
constexpr int kBlThreads = 1024;
__device__ __forceinline__ float loss_coef(int c, int f, int n, float unit) {
  return f > 0 && n > 0 ? unit * static_cast<float>(c) / (static_cast<float>(f) * static_cast<float>(n)) : 0.f;
}
__global__ void __launch_bounds__(kBlThreads)
k_balance_loss(const int32_t *__restrict__ counts, const int32_t *__restrict__ load_tokens,
               const float *__restrict__ prob_sum, const int32_t *__restrict__ tokens, int64_t n,
               int32_t E, float unit, float *__restrict__ loss, float *__restrict__ coef) {
  __shared__ double s_part[kBlThreads / kWave];
  if (blockIdx.x > 0) {
    for (int64_t i = static_cast<int64_t>(blockIdx.x - 1) * kBlThreads + threadIdx.x; i < n;
         i += static_cast<int64_t>(gridDim.x - 1) * kBlThreads)
      coef[i] = loss_coef(counts[i], load_tokens[i / E], tokens[i / E], unit);
    return;
  }
  double sum = 0.0;
  for (int64_t i = threadIdx.x; i < n; i += kBlThreads)
    sum += static_cast<double>(loss_coef(counts[i], load_tokens[i / E], tokens[i / E], unit)) *
           prob_sum[i];
  for (int d = 1; d < kWave; d *= 2) sum += __shfl_xor(sum, d);
  if (lane_id() == 0) s_part[threadIdx.x / kWave] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < kBlThreads / kWave; ++w) sum += s_part[w];
    *loss = static_cast<float>(sum);
  }
}

struct RouteGradArgs {
  const void *logits;
  void *dlogits;
  int64_t T, ld, seq;
  const uint8_t *mask;
  const int32_t *topk;
  const float *dgate, *coef, *dloss;
  int32_t E, k, sigmoid, renorm;
  int32_t wide, wide_coef;  // aligned chunks, the last one whole
  float scale;
  int32_t *status;
};

// The lanes of a token take chunks of its experts in turn, so that a load or store of
// theirs is of neighbouring bytes (no order among the experts matters here): element i
// of lane l is expert at(i).  `past` where there is none.
constexpr int spread_chunk(int lanes, int vpl, bool bf16) {
  return lanes == kWave && vpl % 8 == 0 && bf16 ? 8 : 4;
}
template <int kLanes, int kC>
__device__ __forceinline__ int spread_at(int i) {
  return (i / kC * kLanes + lane_id() % kLanes) * kC + i % kC;
}
template <int kLanes, int kVpl, int kC, bool kBf16>
__device__ __forceinline__ void load_spread(const void *row, int E, bool wide, float past,
                                            float (&z)[kVpl]) {
#pragma unroll
  for (int c = 0; c < kVpl; c += kC) {
    const int e = spread_at<kLanes, kC>(c);
#pragma unroll
    for (int i = 0; i < kC; ++i) z[c + i] = past;
    if (wide) {
      if (e < E) load_chunk<kC, kBf16>(row, e, z + c);
    } else {
#pragma unroll
      for (int i = 0; i < kC; ++i)
        if (e + i < E) z[c + i] = load_logit<kBf16>(row, e + i);
    }
  }
}

// Sum over a token's experts of chunk sums s, in an order that is the same with 16 lanes
// and with 64 for up to 256 experts in chunks of 4: chunks 16 apart first, then the
// lanes of a row.  So a token's gradient does not depend on how many others there are.
template <int kLanes, int n>
__device__ __forceinline__ float spread_sum(float (&s)[n]) {
  static_assert(n <= 4);
#pragma unroll
  for (int c = 1; c < n; c += 2) s[c - 1] += s[c];
  float v = n > 2 ? s[0] + s[2] : s[0];
  if (kLanes == kWave) {
    const v2u r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(r.x) + __uint_as_float(r.y);
    const v2u h = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(h.x) + __uint_as_float(h.y);
  }
  return lanes_sum<16>(v);
}

// With w the balance loss's gradient by p and d the gates' by the chosen scores' logits:
//   softmax  dz = p (w - <w, p>) + d,  sigmoid  dz = p (1 - s) (w - <w, p>) + d
// and without renorm a softmax gate is a p of its own, so scale * dgate joins w.
template <int kLanes, int kVpl, bool kBf16>
__global__ void __launch_bounds__(kRtThreads) k_route_grad(RouteGradArgs a) {
  // (the same roundings with 16 lanes and with 64: fused only where it says so)
#pragma clang fp contract(off)
  constexpr int kTok = kWave / kLanes, kParts = kRtWaves * kTok, kSlots = kLanes * kVpl;
  constexpr int kC = spread_chunk(kLanes, kVpl, kBf16);
  __shared__ __align__(16) float s_d[kParts * kSlots];  // a token's d, by expert
  const int wave = threadIdx.x / kWave, l = lane_id() % kLanes, part = threadIdx.x / kLanes;
  const float dloss = a.dloss ? *a.dloss : 1.f;
  float *d_row = s_d + part * kSlots;
  for (int64_t tw = static_cast<int64_t>(blockIdx.x) * kParts + wave * kTok; tw < a.T;
       tw += static_cast<int64_t>(gridDim.x) * kParts) {
    const int64_t t = tw + (kTok > 1 ? lane_id() / kLanes : 0);
    const bool here = t < a.T;
    const int64_t at = (here ? t : tw) * a.ld * (kBf16 ? 2 : 4);
    const char *row = static_cast<const char *>(a.logits) + at;
    char *out = static_cast<char *>(a.dlogits) + at;
    float z[kVpl], w[kVpl] = {};
    load_spread<kLanes, kVpl, kC, kBf16>(row, a.E, a.wide, -kInf, z);
    if (a.coef) {
      const float *coef = a.coef + (here ? t : tw) / a.seq * a.E;
      load_spread<kLanes, kVpl, kC, false>(coef, a.E, a.wide_coef, 0.f, w);
    }
    bool on = here && (!a.mask || a.mask[t] != 0);
    int id = -1;
    float dg = 0.f, my_z = -kInf;
    if (here && l < a.k) {
      id = a.topk[t * a.k + l];
      if (id < -1 || id >= a.E) {
        report(a.status, ULTRAEP_EDATA);
        id = -1;
      }
      if (id >= 0) {
        my_z = load_logit<kBf16>(row, id);
        if (a.dgate) dg = a.dgate[t * a.k + l] * a.scale;
      }
    }
    float top = -kInf, sum_z = 0.f;  // the sum is a NaN if a logit is (and cannot overflow)
#pragma unroll
    for (int i = 0; i < kVpl; ++i) {
      top = larger(top, z[i]);
      sum_z = fmaf(z[i], 0x1p-12f, sum_z);
      w[i] *= dloss;
    }
    if (mine<kLanes>(ballot(!(sum_z < kInf))) && on) {
      if (l == 0) report(a.status, ULTRAEP_EDATA);
      on = false;
    }
    top = lanes_max<kLanes>(top);
    on = on && top > -kInf && (mine<kLanes>(ballot(id >= 0)) & 1);

    // the chosen: this lane's is lane l's
    const bool chosen = on && my_z > -kInf;
    const Sigmoid score = sigmoid_both(my_z);
    const float not_s = a.sigmoid ? score.rest : 1.f;
    float d;
    if (a.renorm) {
      const float c = lanes_max<kLanes>(chosen ? (a.sigmoid ? fminf(my_z, 0.f) : my_z) : -kInf);
      const float u = !chosen ? 0.f : a.sigmoid ? sigmoid_over(my_z, c) : exp_neg(my_z - c);
      const float us = lanes_sum<kLanes>(u);
      const float q = us > 0.f ? u * fast_rcp(us) : 0.f;
      d = q * (dg - lanes_sum<kLanes>(dg * q)) * not_s;
    } else {
      d = a.sigmoid ? score.s * not_s * dg : dg;
    }
    const float zero[kVpl] = {};
    put_lane<kVpl>(d_row, l, zero);
    wave_sync();
    if (chosen) atomicAdd(d_row + id, d);
    wave_sync();
    const bool joins_w = !a.sigmoid && !a.renorm;

    // (1 - s is 1 where all scores are so low that only their ratios can be told)
    const bool low = on && a.sigmoid && top < -60.f;
    const float c = on ? top : 0.f;
    float p[kVpl], sum[kVpl / kC] = {}, dots[kVpl / kC] = {};
    if (a.sigmoid) {  // p: s (1 - s) from here on
      const bool some_low = ballot(low) != 0;
#pragma unroll
      for (int i = 0; i < kVpl; ++i) {
        const Sigmoid of = sigmoid_both(z[i]);
        float s = of.s;
        p[i] = of.s * of.rest;
        if (some_low) {
          const float over = sigmoid_over(z[i], c);
          s = low ? over : s;
          p[i] = low ? over : p[i];
        }
        sum[i / kC] += s;
        dots[i / kC] = fmaf(w[i], s, dots[i / kC]);
      }
    } else {
#pragma unroll
      for (int i = 0; i < kVpl; ++i) {
        p[i] = exp_neg(z[i] - c);
        sum[i / kC] += p[i];
        if (joins_w) w[i] += d_row[spread_at<kLanes, kC>(i)];
        dots[i / kC] = fmaf(w[i], p[i], dots[i / kC]);
      }
    }
    const float inv = fast_rcp(spread_sum<kLanes>(sum));
    const float dot = spread_sum<kLanes>(dots) * inv;
    float dz[kVpl];
#pragma unroll
    for (int i = 0; i < kVpl; ++i) {
      const float of = joins_w ? 0.f : d_row[spread_at<kLanes, kC>(i)];
      dz[i] = on ? fmaf(p[i] * inv, w[i] - dot, of) : 0.f;
    }
    wave_sync();
    if (!here) continue;
#pragma unroll
    for (int c = 0; c < kVpl; c += kC) {
      const int e = spread_at<kLanes, kC>(c);
      if (a.wide) {
        if (e >= a.E) continue;
        if constexpr (kBf16) {
          typedef uint32_t raw __attribute__((ext_vector_type(kC / 2)));
          raw o;
#pragma unroll
          for (int i = 0; i < kC / 2; ++i) o[i] = pack_bf16(dz[c + 2 * i], dz[c + 2 * i + 1]);
          *reinterpret_cast<raw *>(out + e * 2) = o;
        } else {
          *reinterpret_cast<v4f *>(out + e * 4) = v4f{dz[c], dz[c + 1], dz[c + 2], dz[c + 3]};
        }
      } else {
#pragma unroll
        for (int i = 0; i < kC; ++i) {
          if (e + i >= a.E) continue;
          if (kBf16) reinterpret_cast<uint16_t *>(out)[e + i] = static_cast<uint16_t>(round_bf16(dz[c + i]));
          else reinterpret_cast<float *>(out)[e + i] = dz[c + i];
        }
      }
    }
  }
}

constexpr int64_t kRtChunk = 16;  // a workgroup's tokens are a multiple of it
static int64_t route_wg(const ultraep_router &r) { return r.E > 64 ? 512 : 1024; }

RouteShape route_shape(int64_t T, const ultraep_router &r) {
  RouteShape s;
  s.seq = r.seq_len > 0 && r.seq_len < T ? r.seq_len : T > 0 ? T : 1;
  s.n_seg = T > 0 ? (T + s.seq - 1) / s.seq : 1;
  // Workgroups of at least 16 tokens, about as many as run at once (two a compute unit,
  // four with few experts): more make more partials, fewer take turns.  With 1024 and 512
  // of them, us with the sums, one sequence: E = 256, T = 16384 23.5 and 18.6, 65536 50.0 and
  // 45.6; E = 128, T = 16384 16.1 and 13.0; E = 64, T = 16384 10.7 and 10.6, 65536 19.4 and 24.3.
  const int64_t n_wg = route_wg(r);
  s.chunk = (T + n_wg - 1) / n_wg;
  s.chunk = s.chunk < kRtChunk ? kRtChunk : (s.chunk + kRtChunk - 1) / kRtChunk * kRtChunk;
  s.n_chunk = (s.seq + s.chunk - 1) / s.chunk;
  return s;
}

static size_t partial_bytes(int64_t n, const ultraep_router &r) {
  return n > 0 ? static_cast<size_t>(n) * (2 * static_cast<size_t>(r.E) + 1) * 4 : 4;
}

size_t route_ws_need(int64_t T, const ultraep_router &r) {
  const RouteShape s = route_shape(T, r);
  return partial_bytes(s.n_chunk > 1 ? s.n_seg * s.n_chunk : 0, r);
}

// At least what any T' <= T needs, so that a workspace for the largest batch does for all:
// the partials of T' alone fall where its chunk grows (E = 256: 512 at 16384 tokens, 342 at
// 16385).  With n workgroups aimed at, a chunk c >= 16 and c >= T' / n: one sequence has at
// most min(n, ceil(T' / 16)) chunks.  Several of L tokens, cut where c < L, are s = ceil(T' / L)
// <= n, and s * ceil(L / c) < (T' / L + 1) (L / c + 1) <= n + 1 + T' / L + n L / T' <= 2 n + 2,
// and at most s * ceil(L / 16).  Neither bound falls with T.
size_t route_ws_bytes(int64_t T, const ultraep_router &r) {
  const RouteShape s = route_shape(T, r);
  if (s.seq <= kRtChunk) return partial_bytes(0, r);
  const int64_t n = route_wg(r), most = s.n_seg == 1 ? n : 2 * n + 2;
  const int64_t small = s.n_seg * ((s.seq + kRtChunk - 1) / kRtChunk);
  return partial_bytes(small < most ? small : most, r);
}

template <bool kBf16, bool kStats>
static void start_route(int lanes, int vpl, dim3 grid, hipStream_t stream, const RouteArgs &a) {
#define UEP_CASE(m, n)                                                                         \
  if (lanes == m && vpl == n) {                                                                \
    hipLaunchKernelGGL((k_route<m, n, kBf16, kStats>), grid, dim3(kRtThreads), 0, stream, a);  \
    return;                                                                                    \
  }
  UEP_CASE(16, 4) UEP_CASE(16, 8) UEP_CASE(16, 12) UEP_CASE(16, 16) UEP_CASE(16, 24)
  if constexpr (kStats) {  // (a wave takes a token of so many experts otherwise)
    UEP_CASE(16, 32)
  }
  UEP_CASE(64, 1) UEP_CASE(64, 2) UEP_CASE(64, 4) UEP_CASE(64, 8) UEP_CASE(64, 16) UEP_CASE(64, 32)
#undef UEP_CASE
}

hipError_t launch_route(const void *logits, int32_t type, int64_t T, int64_t ld,
                        const ultraep_router &r, const float *bias, const uint8_t *mask,
                        int32_t *topk, float *gate, int32_t *counts, float *prob_sum,
                        int32_t *tokens, void *ws, int32_t *status, hipStream_t stream) {
  const RouteShape s = route_shape(T, r);
  const int n_group = r.n_group > 0 ? r.n_group : 1, gsz = r.E / n_group;
  // experts of a lane when a token takes `lanes`, and the lanes of a group
  int group_lanes = 0;
  auto spread = [&](int lanes) {
    group_lanes = lanes;
    while (group_lanes * n_group > lanes) group_lanes /= 2;
    return group_lanes ? (gsz + group_lanes - 1) / group_lanes : 1 << 30;
  };
  int lanes = 16, vpl = r.k <= 16 ? spread(16) : 1 << 30;
  // A wave a token where 2048 of them, two a SIMD, are all there are and no statistics are
  // wanted: us of E = 256 with groups, 16 and 64 lanes a token: T = 1 5.3 and 4.6, 2048 6.4
  // and 5.9, 4096 6.5 and 7.8, 65536 36 and 71 (with statistics 47 and 124); E = 64: 1 3.6 and
  // 3.2, 4096 4.2 and 4.9, 65536 16 and 35.  Rows of over 24 experts a lane have one wave a
  // SIMD: E = 512, T = 65536 98 and 75 (with statistics 99 and 142).
  const bool stats = counts != nullptr;
  if (vpl > (stats ? 32 : 24) || (!stats && T <= 2048)) {
    lanes = kWave;
    vpl = spread(kWave);
  }
  if (lanes == 16) vpl = vpl <= 16 ? (vpl + 3) / 4 * 4 : (vpl + 7) / 8 * 8;
  else vpl = vpl <= 1 ? 1 : 1 << (32 - __builtin_clz(vpl - 1));
  const int esize = type == ULTRAEP_BF16 ? 2 : 4;
  const int chunk = chunk_of(vpl, type == ULTRAEP_BF16);
  const bool full = gsz % vpl == 0;
  const bool wide = full && vpl % chunk == 0 && ld % chunk == 0 &&
                    reinterpret_cast<uintptr_t>(logits) % (chunk * esize) == 0;
  const bool wide_bias = full && vpl % 4 == 0 && reinterpret_cast<uintptr_t>(bias) % 16 == 0;
  int pick_lanes = 16;
  while (n_group > 1 && pick_lanes * r.top_group > 16) pick_lanes /= 2;
  int pick = 0;
  if (lanes == 16 && n_group > 1 && pick_lanes > 0 && vpl * group_lanes % (4 * pick_lanes) == 0)
    pick = vpl * group_lanes / pick_lanes;
  RouteArgs a{logits, T, ld, bias, mask, topk, gate, r.E, r.k, r.score == ULTRAEP_SIGMOID, r.renorm,
              n_group, r.top_group, group_lanes, wide, wide_bias, pick_lanes, pick, r.scale, s.seq, s.chunk, s.n_chunk, counts,
              prob_sum, tokens, status};
  if (!stats) {  // no partials to keep few
    a.seq = T;
    a.chunk = kRtThreads / lanes;
    a.n_chunk = (T + a.chunk - 1) / a.chunk;
  }
  const int64_t n_wg = stats ? s.n_seg * s.n_chunk : a.n_chunk;
  if (stats && s.n_chunk > 1) {
    a.prob_sum = static_cast<float *>(ws);
    a.counts = reinterpret_cast<int32_t *>(a.prob_sum + n_wg * r.E);
    a.tokens = a.counts + n_wg * r.E;
  }
  const dim3 grid(static_cast<unsigned>(n_wg));
  if (type == ULTRAEP_BF16) {
    if (stats) start_route<true, true>(lanes, vpl, grid, stream, a);
    else start_route<true, false>(lanes, vpl, grid, stream, a);
  } else {
    if (stats) start_route<false, true>(lanes, vpl, grid, stream, a);
    else start_route<false, false>(lanes, vpl, grid, stream, a);
  }
  if (stats && s.n_chunk > 1) {
    const int n_eb = (r.E + kRsExperts - 1) / kRsExperts;
    hipLaunchKernelGGL(k_route_sum, dim3(static_cast<unsigned>(s.n_seg * n_eb)), dim3(kRsThreads), 0,
                       stream, a.counts, a.prob_sum, a.tokens, s.n_chunk, r.E, n_eb, counts, prob_sum,
                       tokens);
  }
  return hipGetLastError();
}

hipError_t launch_balance_loss(const int32_t *counts, const int32_t *load_tokens,
                               const float *prob_sum, const int32_t *tokens, int64_t n_seg,
                               const ultraep_router &r, float alpha, float *loss, float *coef,
                               hipStream_t stream) {
  const int64_t n = n_seg * r.E;
  const float unit = n_seg > 0 ? static_cast<float>(static_cast<double>(alpha) * r.E /
                                                    (static_cast<double>(n_seg) * r.k))
                               : 0.f;
  const int64_t wg = (n + kBlThreads - 1) / kBlThreads;
  hipLaunchKernelGGL(k_balance_loss, dim3(1 + static_cast<unsigned>(wg < 2048 ? wg : 2048)),
                     dim3(kBlThreads), 0, stream, counts, load_tokens, prob_sum, tokens, n, r.E, unit,
                     loss, coef);
  return hipGetLastError();
}

hipError_t launch_route_grad(const void *logits, int32_t type, int64_t T, int64_t ld,
                             const ultraep_router &r, const uint8_t *mask, const int32_t *topk,
                             const float *dgate, const float *coef, const float *dloss,
                             void *dlogits, int32_t *status, hipStream_t stream) {
  const RouteShape s = route_shape(T, r);
  // A wave a token for many experts or few tokens, where it shortens the chain; else its
  // idle lanes and its sums over 64 lanes cost more.  us with 16 and 64 lanes, fp32:
  //   E = 256: T = 1 5.0 and 3.1, 3000 6.4 and 4.4, 6144 8.0 and 6.7, 8192 8.3 and 8.2, 16384
  //   11.6 and 12.6, 65536 40 and 39; E = 128: 512 3.9 and 3.5, 3000 4.1 and 4.2, 6144 4.6 and
  //   5.7, 16384 7.2 and 11.5; E = 384: 16384 19 and 18; E = 512: 2048 10.1 and 4.9, 16384 27
  //   and 19, 65536 103 and 71
  // (16 lanes of neighbouring experts, whose loads lie 16 to 64 bytes apart, take 16 us at
  // 16384 x 256 and 12.3 at 16384 x 192 in bf16, where chunks in turn take 11.0 and 7.1.)
  const int lanes = r.E > 256 || r.k > 16 || T <= (r.E > 128 ? 6144 : 2048) ? kWave : 16;
  int vpl = (r.E + lanes - 1) / lanes;
  vpl = lanes == 16 ? (vpl + 3) / 4 * 4 : vpl <= 4 ? 4 : vpl <= 8 ? 8 : 16;
  const int esize = type == ULTRAEP_BF16 ? 2 : 4, chunk = spread_chunk(lanes, vpl, type == ULTRAEP_BF16);
  auto wide = [&](const void *p, int bytes, int64_t pitch) {
    return r.E % chunk == 0 && pitch % chunk == 0 && reinterpret_cast<uintptr_t>(p) % bytes == 0;
  };
  const RouteGradArgs a{logits, dlogits, T, ld, s.seq, mask, topk, dgate, coef, dloss, r.E, r.k,
                        r.score == ULTRAEP_SIGMOID, r.renorm,
                        wide(logits, chunk * esize, ld) && wide(dlogits, chunk * esize, ld),
                        wide(coef, 16, r.E), r.scale, status};
  const int64_t parts = kRtThreads / lanes, wg = (T + parts - 1) / parts;
  const dim3 grid(static_cast<unsigned>(wg < 1 << 16 ? wg : 1 << 16));
#define UEP_CASE(m, n)                                                                             \
  if (lanes == m && vpl == n) {                                                                    \
    if (type == ULTRAEP_BF16)                                                                      \
      hipLaunchKernelGGL((k_route_grad<m, n, true>), grid, dim3(kRtThreads), 0, stream, a);        \
    else                                                                                           \
      hipLaunchKernelGGL((k_route_grad<m, n, false>), grid, dim3(kRtThreads), 0, stream, a);       \
    return hipGetLastError();                                                                      \
  }
  UEP_CASE(16, 4) UEP_CASE(16, 8) UEP_CASE(16, 12) UEP_CASE(16, 16) UEP_CASE(64, 4)
  UEP_CASE(64, 8) UEP_CASE(64, 16)
#undef UEP_CASE
  return hipErrorInvalidValue;
}

}  // namespace uep
