// The router of an MoE layer: top-k ids and gates from the logits, the
// statistics of its balance loss, the loss, and the logits' gradient.
//
// One wave takes one token.  Its E logits lie across the lanes in id order:
// with groups, 2^n lanes share a group and each holds VPL neighbouring experts
// of it; without, all 64 lanes share the one group.  So a group's sum of two
// largest keys is a merge over neighbouring lanes, a tie goes to the lowest
// lane and there to the lowest element, and nothing is sorted: k times the
// largest key of the wave is found and taken out.
#include "operators.hpp"

namespace uep {

constexpr int kRtThreads = 256;
constexpr int kRtWaves = kRtThreads / kWave;
constexpr int kRtMaxE = 1024;
constexpr float kInf = __builtin_inff();

// where a lane's experts lie
struct RouteLanes {
  int32_t lanes;  // lanes of a group, a power of two
  int32_t vpl;    // experts of a lane
};

static RouteLanes route_lanes(int32_t E, int32_t n_group) {
  int lanes = kWave;
  while (lanes * n_group > kWave) lanes /= 2;
  const int gsz = E / n_group;
  return {lanes, (gsz + lanes - 1) / lanes};
}

struct RouteArgs {
  const void *logits;
  int64_t T, ld;
  const float *bias;
  const uint8_t *mask;
  int32_t *topk;
  float *gate;
  int32_t E, k, sigmoid, renorm, n_group, top_group, lanes;
  float scale;
  int64_t seq, chunk, n_chunk;
  int32_t *counts;   // outputs, or the workspace's partials if n_chunk > 1
  float *prob_sum;
  int32_t *tokens;
  int32_t *status;
};

template <bool kBf16>
__device__ __forceinline__ float load_logit(const void *row, int e) {
  if (kBf16) return bf16_at_low(static_cast<const uint16_t *>(row)[e]);
  return static_cast<const float *>(row)[e];
}

// fp32 as an integer of the same order (-0 as +0)
__device__ __forceinline__ int order_of(float v) {
  const int i = __float_as_int(v + 0.f);
  return i ^ ((i >> 31) & 0x7FFFFFFF);
}

// the two largest of two pairs
__device__ __forceinline__ void merge_two(float &a1, float &a2, float b1, float b2) {
  a2 = fmaxf(fminf(a1, b1), fmaxf(a2, b2));
  a1 = fmaxf(a1, b1);
}

template <int kVpl, bool kBf16, bool kStats>
__global__ void __launch_bounds__(kRtThreads) k_route(RouteArgs a) {
  __shared__ float s_prob[kStats ? kRtWaves * kRtMaxE : 1];
  __shared__ int s_count[kStats ? kRtMaxE : 1];
  __shared__ int s_tokens;
  const int lane = lane_id(), wave = threadIdx.x / kWave;
  const int gsz = a.E / a.n_group;
  const int group = lane / a.lanes, sub = lane - group * a.lanes;
  const int base = group * gsz + sub * kVpl;
  const int n_mine = group < a.n_group ? min(max(gsz - sub * kVpl, 0), kVpl) : 0;
  const bool by_score = a.sigmoid && (a.bias || a.n_group > 1);

  if (kStats) {
    for (int e = threadIdx.x; e < a.E; e += kRtThreads) s_count[e] = 0;
    if (threadIdx.x == 0) s_tokens = 0;
    __syncthreads();
  }
  float bias[kVpl];
#pragma unroll
  for (int i = 0; i < kVpl; ++i) bias[i] = a.bias && i < n_mine ? a.bias[base + i] : 0.f;
  float acc[kVpl] = {};
  int n_tokens = 0;

  const int64_t seg = blockIdx.x / a.n_chunk;
  const int64_t t0 = seg * a.seq + (blockIdx.x - seg * a.n_chunk) * a.chunk;
  const int64_t t1 = min(min(t0 + a.chunk, (seg + 1) * a.seq), a.T);
  for (int64_t t = t0 + wave; t < t1; t += kRtWaves) {
    const char *row = static_cast<const char *>(a.logits) + t * a.ld * (kBf16 ? 2 : 4);
    float z[kVpl];
    bool bad = false;
    float top = -kInf;
#pragma unroll
    for (int i = 0; i < kVpl; ++i) {
      z[i] = i < n_mine ? load_logit<kBf16>(row, base + i) : -kInf;
      bad |= !(z[i] < kInf);
      top = fmaxf(top, z[i]);
    }
    top = wave_max_f(top);
    bool on = !a.mask || a.mask[t] != 0;
    if (on && ballot(bad)) {
      if (lane == 0) report(a.status, ULTRAEP_EDATA);
      on = false;
    }
    on = on && top > -kInf;
    if (!on) {
      if (lane < a.k) {
        a.topk[t * a.k + lane] = -1;
        a.gate[t * a.k + lane] = 0.f;
      }
      continue;
    }

    int key[kVpl];
    {
      float f[kVpl];
#pragma unroll
      for (int i = 0; i < kVpl; ++i) f[i] = (by_score ? sigmoid(z[i]) : z[i]) + bias[i];
      bool keep = true;
      if (a.n_group > 1) {
        float m1 = -kInf, m2 = -kInf;
#pragma unroll
        for (int i = 0; i < kVpl; ++i) merge_two(m1, m2, z[i] > -kInf ? f[i] : -kInf, -kInf);
        for (int d = 1; d < a.lanes; d *= 2)
          merge_two(m1, m2, __shfl_xor(m1, d), __shfl_xor(m2, d));
        const float score = m1 + m2;
        int before = 0;  // groups ahead of this lane's
        for (int g = 0; g < a.n_group; ++g) {
          const float o = readlane_f(score, g * a.lanes);
          before += o > score || (o == score && g < group);
        }
        keep = before < a.top_group;
      }
#pragma unroll
      for (int i = 0; i < kVpl; ++i)
        key[i] = keep && z[i] > -kInf ? order_of(f[i]) : INT32_MIN;
    }

    // lane j ends up with the j-th id and its logit
    int my_id = -1;
    float my_z = -kInf;
    for (int j = 0; j < a.k; ++j) {
      int m = key[0];
#pragma unroll
      for (int i = 1; i < kVpl; ++i) m = max(m, key[i]);
      const int best = wave_max(m);
      if (best == INT32_MIN) break;
      const int owner = __builtin_ctzll(ballot(m == best));
      int at = 0;
      float v = z[0];
#pragma unroll
      for (int i = kVpl - 1; i >= 0; --i)
        if (key[i] == best) {
          at = i;
          v = z[i];
        }
      const int id = readlane(base + at, owner);
      v = readlane_f(v, owner);
      if (lane == j) {
        my_id = id;
        my_z = v;
      }
      if (lane == owner) {
#pragma unroll
        for (int i = 0; i < kVpl; ++i)
          if (i == at) key[i] = INT32_MIN;
      }
    }

    // ids fill from the front: without a first one (every best group held only
    // -inf and lone experts) the token has none
    on = readlane(my_id, 0) >= 0;

    // scores over all experts: u = s / exp(c), c so that no u of weight vanishes
    float g = 0.f;
    if (a.sigmoid) {
      if (a.renorm) {
        const float c = wave_max_f(my_id >= 0 ? fminf(my_z, 0.f) : -kInf);
        const float u = my_id >= 0 ? expf(fminf(my_z, 0.f) - c) / (1.f + expf(-fabsf(my_z))) : 0.f;
        g = u / wave_sum_f(u);
      } else {
        g = my_id >= 0 ? sigmoid(my_z) : 0.f;
      }
    } else if (a.renorm) {
      const float c = wave_max_f(my_z);
      const float u = my_id >= 0 ? expf(my_z - c) : 0.f;
      g = u / wave_sum_f(u);
    }
    if (on && (kStats || (!a.sigmoid && !a.renorm))) {
      const float c = a.sigmoid ? fminf(top, 0.f) : top;
      float u[kVpl], sum = 0.f;
#pragma unroll
      for (int i = 0; i < kVpl; ++i) {
        u[i] = a.sigmoid ? expf(fminf(z[i], 0.f) - c) / (1.f + expf(-fabsf(z[i]))) : expf(z[i] - c);
        sum += u[i];
      }
      const float inv = 1.f / wave_sum_f(sum);
#pragma unroll
      for (int i = 0; i < kVpl; ++i) acc[i] += u[i] * inv;
      if (!a.sigmoid && !a.renorm) g = my_id >= 0 ? expf(my_z - c) * inv : 0.f;
      ++n_tokens;
    }
    if (lane < a.k) {
      a.topk[t * a.k + lane] = my_id;
      a.gate[t * a.k + lane] = my_id >= 0 ? g * a.scale : 0.f;
      if (kStats && my_id >= 0) atomicAdd(&s_count[my_id], 1);
    }
  }

  if (kStats) {
#pragma unroll
    for (int i = 0; i < kVpl; ++i)
      if (i < n_mine) s_prob[wave * kRtMaxE + base + i] = acc[i];
    if (lane == 0) atomicAdd(&s_tokens, n_tokens);
    __syncthreads();
    for (int e = threadIdx.x; e < a.E; e += kRtThreads) {
      float p = 0.f;
#pragma unroll
      for (int w = 0; w < kRtWaves; ++w) p += s_prob[w * kRtMaxE + e];
      a.prob_sum[static_cast<int64_t>(blockIdx.x) * a.E + e] = p;
      a.counts[static_cast<int64_t>(blockIdx.x) * a.E + e] = s_count[e];
    }
    if (threadIdx.x == 0) a.tokens[blockIdx.x] = s_tokens;
  }
}

// A sequence's partials, 16 experts a workgroup: 64 threads an expert take the chunks in
// turn, then the 64 sums are added in order of the thread.  The first workgroup of a
// sequence also sums its tokens.
constexpr int kRsThreads = 1024, kRsExperts = 16, kRsTurns = kRsThreads / kRsExperts;
__global__ void __launch_bounds__(kRsThreads)
k_route_sum(const int32_t *__restrict__ part_c, const float *__restrict__ part_p,
            const int32_t *__restrict__ part_n, int64_t n_chunk, int32_t E, int32_t n_eb,
            int32_t *__restrict__ counts, float *__restrict__ prob_sum,
            int32_t *__restrict__ tokens) {
  __shared__ float s_p[kRsTurns][kRsExperts];
  __shared__ int s_c[kRsTurns][kRsExperts];
  const int64_t seg = blockIdx.x / n_eb;
  const int eb = static_cast<int>(blockIdx.x - seg * n_eb);
  const int i = threadIdx.x % kRsExperts, turn = threadIdx.x / kRsExperts;
  const int e = eb * kRsExperts + i;
  float p = 0.f;
  int c = 0;
  if (e < E)
    for (int64_t j = turn; j < n_chunk; j += kRsTurns) {
      p += part_p[(seg * n_chunk + j) * E + e];
      c += part_c[(seg * n_chunk + j) * E + e];
    }
  s_p[turn][i] = p;
  s_c[turn][i] = c;
  if (eb == 0 && threadIdx.x >= kRsThreads - kWave) {  // the last wave
    int n = 0;
    for (int64_t j = lane_id(); j < n_chunk; j += kWave) n += part_n[seg * n_chunk + j];
    n = wave_sum(n);
    if (lane_id() == 0) tokens[seg] = n;
  }
  __syncthreads();
  if (turn == 0 && e < E) {
    for (int w = 1; w < kRsTurns; ++w) {
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
  float scale;
  int32_t *status;
};

// One wave a token, lane l holds experts l * VPL ..  With w the balance loss's
// gradient by p and d the gates' by the chosen scores' logits:
//   softmax  dz = p (w - <w, p>) + d,  sigmoid  dz = p (1 - s) (w - <w, p>) + d
// and without renorm a softmax gate is a p of its own, so scale * dgate joins w.
template <int kVpl, bool kBf16>
__global__ void __launch_bounds__(kRtThreads) k_route_grad(RouteGradArgs a) {
  const int lane = lane_id();
  const int base = lane * kVpl;
  const int n_mine = min(max(a.E - base, 0), kVpl);
  const float dloss = a.dloss ? *a.dloss : 1.f;
  const int64_t nw = static_cast<int64_t>(gridDim.x) * kRtWaves;
  for (int64_t t = static_cast<int64_t>(blockIdx.x) * kRtWaves + threadIdx.x / kWave; t < a.T;
       t += nw) {
    const char *row = static_cast<const char *>(a.logits) + t * a.ld * (kBf16 ? 2 : 4);
    char *out = static_cast<char *>(a.dlogits) + t * a.ld * (kBf16 ? 2 : 4);
    float z[kVpl];
    bool bad = false;
    float top = -kInf;
#pragma unroll
    for (int i = 0; i < kVpl; ++i) {
      z[i] = i < n_mine ? load_logit<kBf16>(row, base + i) : -kInf;
      bad |= !(z[i] < kInf);
      top = fmaxf(top, z[i]);
    }
    top = wave_max_f(top);
    bool on = !a.mask || a.mask[t] != 0;
    int id = -1;
    float dg = 0.f;
    if (lane < a.k) {
      id = a.topk[t * a.k + lane];
      if (id < -1 || id >= a.E) {
        report(a.status, ULTRAEP_EDATA);
        id = -1;
      }
      if (id >= 0 && a.dgate) dg = a.dgate[t * a.k + lane] * a.scale;
    }
    if (on && ballot(bad)) {
      if (lane == 0) report(a.status, ULTRAEP_EDATA);
      on = false;
    }
    on = on && top > -kInf && readlane(id, 0) >= 0;
    float dz[kVpl] = {};
    if (on) {
      const float c = a.sigmoid ? fminf(top, 0.f) : top;
      float p[kVpl], w[kVpl], sum = 0.f;
#pragma unroll
      for (int i = 0; i < kVpl; ++i) {
        p[i] = a.sigmoid ? expf(fminf(z[i], 0.f) - c) / (1.f + expf(-fabsf(z[i]))) : expf(z[i] - c);
        sum += p[i];
      }
      const float inv = 1.f / wave_sum_f(sum);
      const int64_t at = t / a.seq * a.E;
#pragma unroll
      for (int i = 0; i < kVpl; ++i) {
        p[i] *= inv;
        w[i] = a.coef && i < n_mine ? dloss * a.coef[at + base + i] : 0.f;
      }
      float d = dg;  // what joins the chosen expert's w or dz
      float my_z = id >= 0 ? load_logit<kBf16>(row, id) : -kInf;
      if (my_z == -kInf) {
        d = 0.f;
      } else if (a.sigmoid) {
        d *= 1.f - sigmoid(my_z);
      }
      if (a.renorm) {
        const float cc = wave_max_f(a.sigmoid ? (my_z > -kInf ? fminf(my_z, 0.f) : -kInf) : my_z);
        float u = 0.f;
        if (my_z > -kInf)
          u = a.sigmoid ? expf(fminf(my_z, 0.f) - cc) / (1.f + expf(-fabsf(my_z))) : expf(my_z - cc);
        const float us = wave_sum_f(u);
        const float q = us > 0.f ? u / us : 0.f;
        const float mean = wave_sum_f(dg * q);
        d = q * (dg - mean);
        if (a.sigmoid) d *= my_z > -kInf ? 1.f - sigmoid(my_z) : 0.f;
      } else if (a.sigmoid) {
        d *= my_z > -kInf ? sigmoid(my_z) : 0.f;
      }
      const bool joins_w = !a.sigmoid && !a.renorm;
      for (int j = 0; j < a.k; ++j) {
        const int e = readlane(id, j);
        const float v = readlane_f(d, j);
        if (e < 0) continue;
#pragma unroll
        for (int i = 0; i < kVpl; ++i)
          if (base + i == e) {
            if (joins_w) w[i] += v;
            else dz[i] += v;
          }
      }
      float dot = 0.f;
#pragma unroll
      for (int i = 0; i < kVpl; ++i) dot += w[i] * p[i];
      dot = wave_sum_f(dot);
#pragma unroll
      for (int i = 0; i < kVpl; ++i) {
        float v = p[i] * (w[i] - dot);
        if (a.sigmoid) v *= 1.f - sigmoid(z[i]);
        dz[i] = z[i] > -kInf ? dz[i] + v : 0.f;
      }
    }
#pragma unroll
    for (int i = 0; i < kVpl; ++i)
      if (i < n_mine) {
        if (kBf16) reinterpret_cast<uint16_t *>(out)[base + i] = static_cast<uint16_t>(round_bf16(dz[i]));
        else reinterpret_cast<float *>(out)[base + i] = dz[i];
      }
  }
}

RouteShape route_shape(int64_t T, const ultraep_router &r) {
  RouteShape s;
  s.seq = r.seq_len > 0 ? r.seq_len : (T > 0 ? T : 1);
  if (s.seq > T && T > 0) s.seq = T;
  s.n_seg = T > 0 ? (T + s.seq - 1) / s.seq : 1;
  // about 512 workgroups, and no partials where one workgroup has few tokens anyway
  s.chunk = (T + 511) / 512;
  s.chunk = s.chunk < 4 ? 4 : (s.chunk + 3) / 4 * 4;
  if (s.seq <= 16) s.chunk = 16;
  s.n_chunk = (s.seq + s.chunk - 1) / s.chunk;
  return s;
}

size_t route_ws_bytes(int64_t T, const ultraep_router &r) {
  const RouteShape s = route_shape(T, r);
  if (s.n_chunk <= 1) return 4;
  return static_cast<size_t>(s.n_seg) * s.n_chunk * (2 * static_cast<size_t>(r.E) + 1) * 4;
}

template <bool kBf16, bool kStats>
static void start_route(int vpl, dim3 grid, hipStream_t stream, const RouteArgs &a) {
#define UEP_CASE(n)                                                                            \
  if (vpl <= n) {                                                                              \
    hipLaunchKernelGGL((k_route<n, kBf16, kStats>), grid, dim3(kRtThreads), 0, stream, a);     \
    return;                                                                                    \
  }
  UEP_CASE(1) UEP_CASE(2) UEP_CASE(4) UEP_CASE(8) UEP_CASE(16) UEP_CASE(32)
#undef UEP_CASE
}

hipError_t launch_route(const void *logits, int32_t type, int64_t T, int64_t ld,
                        const ultraep_router &r, const float *bias, const uint8_t *mask,
                        int32_t *topk, float *gate, int32_t *counts, float *prob_sum,
                        int32_t *tokens, void *ws, int32_t *status, hipStream_t stream) {
  const RouteShape s = route_shape(T, r);
  const int n_group = r.n_group > 0 ? r.n_group : 1;
  const RouteLanes l = route_lanes(r.E, n_group);
  RouteArgs a{logits, T, ld, bias, mask, topk, gate, r.E, r.k, r.score == ULTRAEP_SIGMOID, r.renorm,
              n_group, r.top_group, l.lanes, r.scale, s.seq, s.chunk, s.n_chunk, counts, prob_sum,
              tokens, status};
  const bool stats = counts != nullptr;
  const int64_t n_wg = s.n_seg * s.n_chunk;
  if (stats && s.n_chunk > 1) {
    a.prob_sum = static_cast<float *>(ws);
    a.counts = reinterpret_cast<int32_t *>(a.prob_sum + n_wg * r.E);
    a.tokens = a.counts + n_wg * r.E;
  }
  const dim3 grid(static_cast<unsigned>(n_wg));
  if (type == ULTRAEP_BF16) {
    if (stats) start_route<true, true>(l.vpl, grid, stream, a);
    else start_route<true, false>(l.vpl, grid, stream, a);
  } else {
    if (stats) start_route<false, true>(l.vpl, grid, stream, a);
    else start_route<false, false>(l.vpl, grid, stream, a);
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
  const RouteGradArgs a{logits, dlogits, T, ld, s.seq, mask, topk, dgate, coef, dloss, r.E, r.k,
                        r.score == ULTRAEP_SIGMOID, r.renorm, r.scale, status};
  const int vpl = (r.E + kWave - 1) / kWave;
  const int64_t wg = (T + kRtWaves - 1) / kRtWaves;
  const dim3 grid(static_cast<unsigned>(wg < 16384 ? wg : 16384));
#define UEP_CASE(n)                                                                               \
  if (vpl <= n) {                                                                                 \
    if (type == ULTRAEP_BF16)                                                                     \
      hipLaunchKernelGGL((k_route_grad<n, true>), grid, dim3(kRtThreads), 0, stream, a);          \
    else                                                                                          \
      hipLaunchKernelGGL((k_route_grad<n, false>), grid, dim3(kRtThreads), 0, stream, a);         \
    return hipGetLastError();                                                                     \
  }
  UEP_CASE(1) UEP_CASE(2) UEP_CASE(4) UEP_CASE(8) UEP_CASE(16)
#undef UEP_CASE
  return hipErrorInvalidValue;
}

}  // namespace uep
