// Routing to experts for CDNA4 (gfx950): the choice of experts with its
// weights, their gradient, and the plan that sorts (token, slot) by expert.
//
// A wave holds a token: lane i has the V consecutive experts from V i on, so
// that the lowest lane of a ballot is the lowest expert among equals, and a
// token's logits are one coalesced read. The choice is top_k rounds of a
// maximum over the wave (DPP, no LDS) and one ballot.
//
// Which experts are chosen has to be the choice of exact values, not of their
// fp32 roundings. Where the logits order the values (no bias), they are
// compared themselves. Else values are computed in fp32, whose error is bounded
// below (kTolAbs, kTolRel); a token with two neighbours in the order of the
// choice closer than that is done again in fp64. Some tokens in a thousand are,
// where scores are spread like a trained router's.
#include "ciera_expert.h"
#include "ciera_expert_dev.h"

namespace ciera {

namespace {

constexpr uint32_t kWaves = 4;  // tokens per workgroup
constexpr float kInf = __builtin_inff();

// |fp32 value - exact value| <= kTolAbs + kTolRel |value|. expf is within 1 ulp
// of its argument's exponential, and its argument (l, or l - max, rounded
// once: relative 2^-24 of a number x) moves it by |x| 2^-24; s (1 - s) |x| <=
// 0.28 and p |log p| <= 0.37 bound what that does to a score. The sum of up to
// 1024 exponentials is off by at most 2^-24 (16 values in a lane, 6 steps)
// relative to it: 22 half ulps; the division adds 1.5 ulp. Together below (0.37
// + 1 + 22 / 2 + 1.5) 2^-23 of a score of at most 1, and 2^-24 of the value for
// the bias's addition.
constexpr float kTolAbs = 14 * 0x1p-23f;
constexpr float kTolRel = 0x1p-23f;

__device__ __forceinline__ float exp_of(float x) { return expf(x); }
__device__ __forceinline__ double exp_of(double x) { return exp(x); }

template <typename T, int V>
__device__ __forceinline__ void load_logits(const RouteArgs &a, uint64_t row,
                                            uint32_t lane, float (&l)[V]) {
  const typename T::Raw *p =
      static_cast<const typename T::Raw *>(a.logits) + row * a.row_stride;
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const uint32_t e = lane * V + j;
    l[j] = e < a.n_experts ? T::to_float(p[e]) : -kInf;
  }
}

// Groups that take part, as a mask: the top_groups groups of highest rank
// among the n_groups groups of `key`. `close`: whether the border between them
// is within tol. `shared` holds 64 V values of this wave.
template <typename K, int V>
__device__ __forceinline__ uint64_t choose_groups(const RouteArgs &a,
                                                  const K (&key)[V],
                                                  uint32_t lane, K *shared,
                                                  float tol_abs, float tol_rel,
                                                  bool &close) {
  const uint32_t S = a.n_experts / a.n_groups;
#pragma unroll
  for (int j = 0; j < V; ++j) shared[lane * V + j] = key[j];
  wave_order();
  K one = -kInf, two = -kInf;
  if (lane < a.n_groups) {
    for (uint32_t i = 0; i < S; ++i) {
      const K v = shared[lane * S + i];
      const K low = v < one ? v : one;
      one = larger(one, v);
      two = larger(two, low);
    }
  }
  K rank_by = one;
  if ((a.flags & CIERA_ROUTE_GROUP_TOP_TWO) && two > -kInf) rank_by = one + two;
  uint32_t rank = 0;
  for (uint32_t g = 0; g < a.n_groups; ++g) {
    const K v = lane_of(rank_by, int(g));
    rank += (v > rank_by || (v == rank_by && g < lane)) ? 1u : 0u;
  }
  const bool kept = lane < a.n_groups && rank < a.top_groups;
  const K least = -wave_max(kept ? -rank_by : K(-kInf));
  const K most = wave_max(lane < a.n_groups && !kept ? rank_by : K(-kInf));
  const K size = larger(larger(least, -least), larger(most, -most));
  close = most > -kInf && least - most <= 4 * (tol_abs + tol_rel * size);
  return __ballot(kept);
}

// One token's choice. Lane s < top_k gets the expert of slot s in `id` (-1:
// none). Returns false where two values are too close for K.
template <typename K, int V>
__device__ __forceinline__ bool choose(const RouteArgs &a, K (&key)[V],
                                       uint32_t lane, K *shared, float tol_abs,
                                       float tol_rel, int &id) {
  if (a.top_groups < a.n_groups) {
    bool close;
    const uint64_t groups =
        choose_groups(a, key, lane, shared, tol_abs, tol_rel, close);
    if (close && tol_abs > 0) return false;
    const uint32_t S = a.n_experts / a.n_groups;
    uint32_t g = lane * V / S, r = lane * V - g * S;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      if (g >= 64 || !((groups >> g) & 1)) key[j] = -kInf;
      if (++r == S) r = 0, ++g;
    }
  }
  id = -1;
  K before = kInf;
  // one round more than slots: the first that is left out must not be close
  const uint32_t rounds = a.top_k + (tol_abs > 0 ? 1 : 0);
  for (uint32_t s = 0; s < rounds; ++s) {
    K best = key[0];
    int at = 0;
#pragma unroll
    for (int j = 1; j < V; ++j)
      if (key[j] > best) best = key[j], at = j;
    const K m = wave_max(best);
    if (m == -kInf) break;
    if (tol_abs > 0 && s > 0) {
      const K size = larger(larger(before, -before), larger(m, -m));
      if (before - m <= 2 * (tol_abs + tol_rel * size)) return false;
    }
    before = m;
    const int first = __builtin_ctzll(__ballot(best == m));
    const int j = __builtin_amdgcn_readlane(at, first);
    if (s < a.top_k && lane == s) id = first * V + j;
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (int(lane) == first && i == j) key[i] = -kInf;
  }
  return true;
}

// The values that the choice compares, in K.
template <typename K, int V>
__device__ __forceinline__ void values_of(const RouteArgs &a,
                                          const float (&l)[V], float top,
                                          uint32_t lane, K (&key)[V]) {
  if (a.flags & CIERA_ROUTE_SIGMOID) {
#pragma unroll
    for (int j = 0; j < V; ++j) key[j] = K(1) / (K(1) + exp_of(-K(l[j])));
  } else {
    K sum = 0;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      key[j] = exp_of(K(l[j]) - K(top));
      sum += key[j];
    }
    sum = wave_sum(sum);
#pragma unroll
    for (int j = 0; j < V; ++j) key[j] /= sum;
  }
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const uint32_t e = lane * V + j;
    const float b = a.bias && e < a.n_experts ? a.bias[e] : 0.0f;
    const bool live = l[j] > -kInf && fabsf(b) < kInf;
    key[j] = live ? key[j] + K(b) : K(-kInf);
  }
}

template <typename T, int V>
__global__ void __launch_bounds__(64 * kWaves) route_kernel(RouteArgs a) {
  __shared__ double shared[kWaves][64 * V];
  const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint32_t token = blockIdx.x * kWaves + wave;
  if (token >= a.n_tokens) return;
  float l[V];
  load_logits<T, V>(a, token, lane, l);
  float top = l[0];
  bool fine = l[0] < kInf;  // neither NaN nor +inf
#pragma unroll
  for (int j = 1; j < V; ++j) {
    top = fmaxf(top, l[j]);
    fine = fine && l[j] < kInf;
  }
  const uint64_t out = uint64_t(token) * a.top_k + lane;
  if (__ballot(!fine)) {
    if (lane < a.top_k) {
      a.ids[out] = -1;
      a.weights[out] = __builtin_nanf("");
    }
    return;
  }
  top = wave_max(top);
  const bool all_groups = a.top_groups == a.n_groups;
  const bool by_logit =
      !a.bias && (all_groups || !(a.flags & CIERA_ROUTE_GROUP_TOP_TWO));
  int id = -1;
  if (top > -kInf) {
    float key[V];
    bool sure;
    if (by_logit) {
#pragma unroll
      for (int j = 0; j < V; ++j) key[j] = l[j];
      sure = choose(a, key, lane, reinterpret_cast<float *>(shared[wave]),
                    0.0f, 0.0f, id);
    } else {
      values_of(a, l, top, lane, key);
      sure = choose(a, key, lane, reinterpret_cast<float *>(shared[wave]),
                    kTolAbs, kTolRel, id);
    }
    if (!sure) {
      double wide[V];
      values_of(a, l, top, lane, wide);
      choose(a, wide, lane, shared[wave], 0.0f, 0.0f, id);
    }
  }
  // the weights, from the chosen logits
  const typename T::Raw *row =
      static_cast<const typename T::Raw *>(a.logits) + token * a.row_stride;
  const bool chosen = id >= 0;
  const float mine = chosen ? T::to_float(row[id]) : -kInf;
  float w;
  if (a.flags & CIERA_ROUTE_NORMALIZE) {
    // softmax's own sum cancels. Below -30, where 1 + e^l rounds to 1, sigmoids
    // go as exponentials too; relative to the largest they cannot vanish.
    const float high = wave_max(mine);
    float p = 0;
    if ((a.flags & CIERA_ROUTE_SIGMOID) && high > -30.0f)
      p = chosen ? 1.0f / (1.0f + expf(-mine)) : 0.0f;
    else
      p = chosen ? expf(mine - high) : 0.0f;
    w = p / wave_sum(p);
  } else if (a.flags & CIERA_ROUTE_SIGMOID) {
    w = 1.0f / (1.0f + expf(-mine));
  } else {
    float sum = 0;
#pragma unroll
    for (int j = 0; j < V; ++j) sum += l[j] > -kInf ? expf(l[j] - top) : 0.0f;
    sum = wave_sum(sum);
    w = expf(mine - top) / sum;
  }
  if (lane < a.top_k) {
    a.ids[out] = id;
    a.weights[out] = chosen ? w * a.scale : 0.0f;
  }
}

// ------------------------------------------------------------- gradient ----
// With c = scale and the chosen set fixed:
//   softmax normalised   d_i = w_i (g_i - sum_j w_j g_j / c)
//   softmax              d_e = p_e (c g_e [chosen] - c sum_j p_j g_j)
//   sigmoid normalised   d_i = w_i (1 - s_i) (g_i - sum_j w_j g_j / c)
//   sigmoid              d_i = c s_i (1 - s_i) g_i
// (d_i for the chosen; 0 elsewhere). Only the plain softmax reads the whole
// row.
template <typename T, int V>
__global__ void __launch_bounds__(64 * kWaves)
    route_backward_kernel(RouteBackArgs a) {
  const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint32_t token = blockIdx.x * kWaves + wave;
  if (token >= a.n_tokens) return;
  const typename T::Raw *row = static_cast<const typename T::Raw *>(a.logits) +
                               uint64_t(token) * a.row_stride;
  typename T::Raw *d_row = static_cast<typename T::Raw *>(a.d_logits) +
                           uint64_t(token) * a.d_row_stride;
  const bool sigmoid = a.flags & CIERA_ROUTE_SIGMOID;
  const bool normal = a.flags & CIERA_ROUTE_NORMALIZE;
  int id = -1;
  float g = 0;
  if (lane < a.top_k) {
    id = a.ids[uint64_t(token) * a.top_k + lane];
    g = a.d_weights[uint64_t(token) * a.top_k + lane] * a.scale;
  }
  const bool chosen = uint32_t(id) < a.n_experts;
  if (!chosen) id = -1;
  const float mine = chosen ? T::to_float(row[id]) : -kInf;
  float d = 0;  // of this lane's slot
  float l[V], spread = 0, top = 0, sum = 1;
  const bool whole = !sigmoid && !normal;
  if (whole) {
    top = -kInf;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const uint32_t e = lane * V + j;
      l[j] = e < a.n_experts ? T::to_float(row[e]) : -kInf;
      top = l[j] > top || l[j] != l[j] ? l[j] : top;
    }
    // a NaN stays the maximum's choice of no lane: the sum carries it instead
    top = wave_max(top == top ? top : -kInf);
    sum = 0;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      l[j] = l[j] == -kInf ? 0.0f : expf(l[j] - top);
      sum += l[j];
    }
    sum = wave_sum(sum);
    const float p = chosen && sum != 0 ? expf(mine - top) / sum : 0.0f;
    d = p * g;
    spread = wave_sum(d);
  } else if (normal) {
    const float high = wave_max(mine);
    const bool as_exp = !sigmoid || high <= -30.0f;
    const float s = sigmoid ? 1.0f / (1.0f + expf(-mine)) : 0.0f;
    float p = 0;
    if (chosen && high != -kInf) p = as_exp ? expf(mine - high) : s;
    const float all = wave_sum(p);
    const float w = all == 0 ? 0.0f : p / all;
    const float mean = wave_sum(chosen ? w * g : 0.0f);
    d = chosen ? w * (1.0f - s) * (g - mean) : 0.0f;
  } else {
    const float s = 1.0f / (1.0f + expf(-mine));
    d = chosen ? s * (1.0f - s) * g : 0.0f;
  }
  float o[V];
#pragma unroll
  for (int j = 0; j < V; ++j) o[j] = whole ? -(l[j] / sum) * spread : 0.0f;
  if (whole && !(sum > 0)) {  // every logit is -inf, or one is NaN
#pragma unroll
    for (int j = 0; j < V; ++j) o[j] = sum != sum ? sum : 0.0f;
  }
  for (uint32_t s = 0; s < a.top_k; ++s) {
    const int e = __builtin_amdgcn_readlane(id, int(s));
    const float v = lane_of(d, int(s));
#pragma unroll
    for (int j = 0; j < V; ++j)
      if (e == int(lane * V + j)) o[j] += v;
  }
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const uint32_t e = lane * V + j;
    if (e < a.n_experts) d_row[e] = T::from_float(o[j]);
  }
}

// ----------------------------------------------------------------- plan ----
// A stable counting sort. Tiles of kPlanTile pairs are counted, the counts
// scanned expert by expert, and every tile places its pairs: each wave takes a
// run of the tile, and among 64 pairs those of the same expert are found by
// ballots over the bits of the id. Up to one tile is sorted by one workgroup in
// one launch. Nothing depends on the order in which waves run.
constexpr uint32_t kPlanThreads = 512;
constexpr uint32_t kPlanWaves = kPlanThreads / 64;
constexpr uint32_t kPlanRun = kPlanTile / kPlanWaves;  // pairs per wave

__device__ __forceinline__ uint32_t expert_of(const PlanArgs &a, uint32_t i,
                                              uint32_t end) {
  if (i >= end) return a.n_experts;
  const uint32_t e = uint32_t(a.ids[i]) - a.first_expert;
  return e < a.n_experts ? e : a.n_experts;
}

// Lanes that hold the same e, by its low `bits` bits.
__device__ __forceinline__ uint64_t same_as(uint32_t e, uint32_t bits) {
  uint64_t same = ~0ull;
  for (uint32_t b = 0; b < bits; ++b) {
    const uint64_t set = __ballot((e >> b) & 1);
    same &= (e >> b) & 1 ? set : ~set;
  }
  return same;
}

__global__ void __launch_bounds__(kPlanThreads)
    plan_count_kernel(PlanArgs a, uint32_t tiles) {
  __shared__ uint32_t count[CIERA_MAX_EXPERTS + 1];
  for (uint32_t e = threadIdx.x; e <= a.n_experts; e += kPlanThreads)
    count[e] = 0;
  __syncthreads();
  const uint32_t from = blockIdx.x * kPlanTile;
  for (uint32_t i = threadIdx.x; i < kPlanTile; i += kPlanThreads)
    atomicAdd(&count[expert_of(a, from + i, a.n_pairs)], 1u);
  __syncthreads();
  for (uint32_t e = threadIdx.x; e < a.n_experts; e += kPlanThreads)
    a.counts[uint64_t(e) * tiles + blockIdx.x] = count[e];
}

// The counts' running sum in place: where each tile's first row of each expert
// is; counts[n_experts * tiles] gets the total.
__global__ void __launch_bounds__(1024)
    plan_scan_kernel(PlanArgs a, uint32_t tiles) {
  __shared__ uint32_t wave_total[16];
  const uint32_t n = a.n_experts * tiles;
  const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint32_t base = 0;
  for (uint32_t from = 0; from < n; from += 1024) {
    const uint32_t i = from + threadIdx.x;
    const uint32_t c = i < n ? a.counts[i] : 0;
    uint32_t total;
    uint32_t before = wave_prefix(c, lane, total);
    if (lane == 0) wave_total[wave] = total;
    __syncthreads();
    uint32_t all = 0;
#pragma unroll
    for (uint32_t w = 0; w < 16; ++w) {
      if (w < wave) before += wave_total[w];
      all += wave_total[w];
    }
    __syncthreads();
    if (i < n) {
      a.counts[i] = base + before;
      if (i % tiles == 0) a.offsets[i / tiles] = int32_t(base + before);
    }
    base += all;
  }
  if (threadIdx.x == 0) {
    a.counts[n] = base;
    a.offsets[a.n_experts] = int32_t(base);
  }
}

template <bool ONE>
__global__ void __launch_bounds__(kPlanThreads)
    plan_place_kernel(PlanArgs a, uint32_t tiles, uint32_t bits) {
  // where the next pair of each expert goes, for every wave of the tile
  __shared__ uint32_t next[kPlanWaves][CIERA_MAX_EXPERTS];
  __shared__ uint32_t part[kPlanWaves + 1];
  const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (uint32_t e = threadIdx.x; e < a.n_experts; e += kPlanThreads)
#pragma unroll
    for (uint32_t w = 0; w < kPlanWaves; ++w) next[w][e] = 0;
  __syncthreads();
  const uint32_t tile = blockIdx.x * kPlanTile;
  const uint32_t tile_end = tile + kPlanTile < a.n_pairs ? tile + kPlanTile
                                                         : a.n_pairs;
  const uint32_t from = tile + wave * kPlanRun;
  uint32_t mine[kPlanRun / 64];
#pragma unroll
  for (uint32_t r = 0; r < kPlanRun / 64; ++r) {
    mine[r] = expert_of(a, from + r * 64 + lane, tile_end);
    if (mine[r] < a.n_experts) atomicAdd(&next[wave][mine[r]], 1u);
  }
  __syncthreads();
  uint32_t total;
  if constexpr (ONE) {
    // the workgroup's own scan over experts: each thread's experts are
    // consecutive
    constexpr uint32_t kPer = CIERA_MAX_EXPERTS / kPlanThreads;
    uint32_t c[kPer], sum = 0;
#pragma unroll
    for (uint32_t j = 0; j < kPer; ++j) {
      const uint32_t e = threadIdx.x * kPer + j;
      c[j] = 0;
      if (e < a.n_experts)
#pragma unroll
        for (uint32_t w = 0; w < kPlanWaves; ++w) c[j] += next[w][e];
      sum += c[j];
    }
    uint32_t wave_all;
    uint32_t before = wave_prefix(sum, lane, wave_all);
    if (lane == 0) part[wave] = wave_all;
    __syncthreads();
    total = 0;
#pragma unroll
    for (uint32_t w = 0; w < kPlanWaves; ++w) {
      if (w < wave) before += part[w];
      total += part[w];
    }
#pragma unroll
    for (uint32_t j = 0; j < kPer; ++j) {
      const uint32_t e = threadIdx.x * kPer + j;
      if (e < a.n_experts) {
        a.offsets[e] = int32_t(before);
        uint32_t at = before;
#pragma unroll
        for (uint32_t w = 0; w < kPlanWaves; ++w) {
          const uint32_t n = next[w][e];
          next[w][e] = at;
          at += n;
        }
        before += c[j];
      }
    }
    if (threadIdx.x == 0) a.offsets[a.n_experts] = int32_t(total);
  } else {
    total = a.counts[uint64_t(a.n_experts) * tiles];
    for (uint32_t e = threadIdx.x; e < a.n_experts; e += kPlanThreads) {
      uint32_t at = a.counts[uint64_t(e) * tiles + blockIdx.x];
#pragma unroll
      for (uint32_t w = 0; w < kPlanWaves; ++w) {
        const uint32_t n = next[w][e];
        next[w][e] = at;
        at += n;
      }
    }
  }
  __syncthreads();
#pragma unroll
  for (uint32_t r = 0; r < kPlanRun / 64; ++r) {
    const uint32_t i = from + r * 64 + lane, e = mine[r];
    const uint64_t same = same_as(e, bits);
    const uint64_t below = same & ((1ull << lane) - 1);
    uint32_t at = 0;
    if (e < a.n_experts) at = next[wave][e] + __popcll(below);
    wave_order();
    if (e < a.n_experts && below == 0) next[wave][e] = at + __popcll(same);
    wave_order();
    if (i < tile_end) {
      a.position[i] = e < a.n_experts ? int32_t(at) : -1;
      if (e < a.n_experts) a.source[at] = int32_t(i);
      if (i >= total) a.source[i] = -1;
    }
  }
}

__global__ void plan_empty_kernel(int32_t *offsets, uint32_t n) {
  for (uint32_t i = threadIdx.x; i < n; i += blockDim.x) offsets[i] = 0;
}

template <typename T>
hipError_t route_typed(const RouteArgs &a, hipStream_t s) {
  const dim3 grid((a.n_tokens + kWaves - 1) / kWaves), block(64 * kWaves);
  if (a.n_experts <= 64)
    route_kernel<T, 1><<<grid, block, 0, s>>>(a);
  else if (a.n_experts <= 128)
    route_kernel<T, 2><<<grid, block, 0, s>>>(a);
  else if (a.n_experts <= 256)
    route_kernel<T, 4><<<grid, block, 0, s>>>(a);
  else
    route_kernel<T, 16><<<grid, block, 0, s>>>(a);
  return hipGetLastError();
}

template <typename T>
hipError_t route_back_typed(const RouteBackArgs &a, hipStream_t s) {
  const dim3 grid((a.n_tokens + kWaves - 1) / kWaves), block(64 * kWaves);
  if (a.n_experts <= 64)
    route_backward_kernel<T, 1><<<grid, block, 0, s>>>(a);
  else if (a.n_experts <= 128)
    route_backward_kernel<T, 2><<<grid, block, 0, s>>>(a);
  else if (a.n_experts <= 256)
    route_backward_kernel<T, 4><<<grid, block, 0, s>>>(a);
  else
    route_backward_kernel<T, 16><<<grid, block, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_route(const RouteArgs &a, hipStream_t s) {
  return a.dtype == CIERA_DT_BF16   ? route_typed<Bf16>(a, s)
         : a.dtype == CIERA_DT_FP16 ? route_typed<Fp16>(a, s)
                                    : route_typed<Fp32>(a, s);
}

hipError_t launch_route_backward(const RouteBackArgs &a, hipStream_t s) {
  return a.dtype == CIERA_DT_BF16   ? route_back_typed<Bf16>(a, s)
         : a.dtype == CIERA_DT_FP16 ? route_back_typed<Fp16>(a, s)
                                    : route_back_typed<Fp32>(a, s);
}

hipError_t launch_route_plan(const PlanArgs &a, hipStream_t s) {
  if (a.n_pairs == 0) {
    plan_empty_kernel<<<1, 64, 0, s>>>(a.offsets, a.n_experts + 1);
    return hipGetLastError();
  }
  const uint32_t tiles = uint32_t(plan_tiles(a.n_pairs));
  uint32_t bits = 0;  // that tell n_experts + 1 ids apart
  while ((a.n_experts >> bits) != 0) ++bits;
  if (tiles == 1) {
    plan_place_kernel<true><<<1, kPlanThreads, 0, s>>>(a, tiles, bits);
    return hipGetLastError();
  }
  plan_count_kernel<<<tiles, kPlanThreads, 0, s>>>(a, tiles);
  plan_scan_kernel<<<1, 1024, 0, s>>>(a, tiles);
  plan_place_kernel<false><<<tiles, kPlanThreads, 0, s>>>(a, tiles, bits);
  return hipGetLastError();
}

}  // namespace ciera
