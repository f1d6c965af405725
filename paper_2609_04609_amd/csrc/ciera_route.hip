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
// below (kTol...); a token with two neighbours in the order of the choice
// closer than that is done again in fp64. Some tokens in a thousand are, where
// scores are spread like a trained router's.
//
// Vector instructions bound it, not memory: the choice of 8 of 256 with a bias
// and groups takes 690 a wave. Keys are whole numbers in the floats' order, whose
// maximum takes the other lane's value within the instruction; float maxima,
// which quiet NaN first and move lanes apart, took 960. 32768 fp32 tokens of that
// kind: 43 us (57 with float keys, and unsorted ones); 16384 bf16 tokens, 8 of 64:
// 8.5 us; 8 of 256 with a bias, no groups: 21 us.
#include <type_traits>

#include "ciera_expert.h"
#include "ciera_expert_dev.h"

namespace ciera {

namespace {

constexpr uint32_t kWaves = 4;  // tokens per workgroup
constexpr float kInf = __builtin_inff();

// |fp32 value - exact value| <= tol + kTolRel |value|. v_exp_f32 is within 1 ulp
// (2^-23); its argument x log2(e) is rounded twice (the product and the constant), and
// x = l - max once, which moves the exponential by at most 1.5 |x| 2^-23 of itself.
//   sigmoid  s = 1 / (1 + e^-l): the exponential's error counts s (1 - s) <= 1/4 fold,
//            s (1 - s) |l| <= 0.28, and the sum and the reciprocal are off by 1.5
//            ulp: (0.25 + 1.5 * 0.28 + 1.5) 2^-23
//   softmax  of at most the largest score p: |x| p e^x <= 0.37 p; the sum of up
//            to 1024 exponentials (16 in a lane, 6 steps) by at most 22 half ulps, the
//            reciprocal and the product by 1.5: (1 + 1.5 * 0.37 + 11 + 1.5) p 2^-23
// and the bias's addition by half an ulp of the value.
constexpr float kTolSigmoid = 3 * 0x1p-23f, kTolSoftmax = 15 * 0x1p-23f;
constexpr float kTolRel = 0x1p-23f;

__device__ __forceinline__ float exp_of(float x) {
  return __builtin_amdgcn_exp2f(x * 1.44269504088896340736f);
}
__device__ __forceinline__ double exp_of(double x) { return exp(x); }
__device__ __forceinline__ float one_over(float x) {
  return __builtin_amdgcn_rcpf(x);
}
__device__ __forceinline__ double one_over(double x) { return 1 / x; }

// V consecutive logits a lane; `vec`: they may be read at once.
template <typename T, int V>
__device__ __forceinline__ void load_logits(const typename T::Raw *row,
                                            uint32_t n_experts, bool vec,
                                            uint32_t lane, float (&l)[V]) {
  typename T::Raw raw[V];
  if (vec) {
    if (lane * V < n_experts)
      __builtin_memcpy(raw, __builtin_assume_aligned(row + lane * V,
                                                     V * T::kBytes < 16
                                                         ? V * T::kBytes : 16),
                       V * T::kBytes);
#pragma unroll
    for (int j = 0; j < V; ++j)
      l[j] = lane * V < n_experts ? T::to_float(raw[j]) : -kInf;
  } else {
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const uint32_t e = lane * V + j;
      l[j] = e < n_experts ? T::to_float(row[e]) : -kInf;
    }
  }
}

// A value's place in the order as a whole number; 0: out of the choice.
template <typename K>
using Order = std::conditional_t<sizeof(K) == 4, uint32_t, uint64_t>;

// The two largest of two pairs (one >= two).
template <typename O>
__device__ __forceinline__ void merge_two(O &one, O &two, O other_one,
                                          O other_two) {
  const O low = one < other_one ? one : other_one;
  one = larger(one, other_one);
  two = larger(larger(two, other_two), low);
}

// Whether neighbours in the order, values of K that are each within tol_abs +
// tol_rel |value| of what they stand for, could stand in the other order.
template <typename K>
__device__ __forceinline__ bool too_close(K above, K below, float parts,
                                          float tol_abs, float tol_rel) {
  const K size = larger(larger(above, -above), larger(below, -below));
  return above - below <= 2 * parts * (tol_abs + tol_rel * size);
}

// Keep the top_groups groups of highest rank; the keys of others become 0.
// Returns whether the border between them is closer than K tells apart. Groups
// of V, 2 V ... 16 V experts are reduced within a row of lanes; other
// sizes go through `shared`, 64 V keys of this wave, a lane a group.
template <typename K, int V>
__device__ __forceinline__ bool choose_groups(const RouteArgs &a,
                                              Order<K> (&key)[V], uint32_t lane,
                                              Order<K> *shared, float tol_abs,
                                              float tol_rel) {
  using O = Order<K>;
  const uint32_t S = a.n_experts / a.n_groups;
  const uint32_t lanes = S / V;
  const bool in_row = S % V == 0 && (lanes & (lanes - 1)) == 0 && lanes <= 16;
  O one = 0, two = 0;
  if (in_row) {
    one = key[0];
#pragma unroll
    for (int j = 1; j < V; ++j) merge_two(one, two, key[j], O(0));
    if (lanes >= 2)
      merge_two(one, two, dpp_or_zero<kDppPair>(one),
                dpp_or_zero<kDppPair>(two));
    if (lanes >= 4)
      merge_two(one, two, dpp_or_zero<kDppQuad>(one),
                dpp_or_zero<kDppQuad>(two));
    if (lanes >= 8)
      merge_two(one, two, dpp_or_zero<kDppHalfMirror>(one),
                dpp_or_zero<kDppHalfMirror>(two));
    if (lanes >= 16)
      merge_two(one, two, dpp_or_zero<kDppMirror>(one),
                dpp_or_zero<kDppMirror>(two));
  } else {
#pragma unroll
    for (int j = 0; j < V; ++j) shared[lane * V + j] = key[j];
    wave_order();
    if (lane < a.n_groups)
      for (uint32_t i = 0; i < S; ++i)
        merge_two(one, two, shared[lane * S + i], O(0));
  }
  O rank_by = one;
  if ((a.flags & CIERA_ROUTE_GROUP_TOP_TWO) && two != 0)
    rank_by = to_order(from_order(one) + from_order(two));
  // group g's rank is in lane g * step
  const uint32_t step = in_row ? lanes : 1, mine = lane / step;
  uint32_t rank = 0;
  for (uint32_t g = 0; g < a.n_groups; ++g) {
    const O v = lane_of(rank_by, int(g * step));
    rank += (v > rank_by || (v == rank_by && g < mine)) ? 1u : 0u;
  }
  const bool kept = mine < a.n_groups && rank < a.top_groups;
  if (in_row) {
#pragma unroll
    for (int j = 0; j < V; ++j) key[j] = kept ? key[j] : O(0);
  } else {
    const uint64_t groups = __ballot(kept);
    uint32_t g = lane * V / S, r = lane * V - g * S;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      if (g >= 64 || !((groups >> g) & 1)) key[j] = 0;
      if (++r == S) r = 0, ++g;
    }
  }
  if (tol_abs == 0) return false;
  const O least = ~wave_max(kept ? O(~rank_by) : O(0));
  const O most = wave_max(mine < a.n_groups && !kept ? rank_by : O(0));
  // a group's rank has up to two values' errors
  return most != 0 && too_close(K(from_order(least)), K(from_order(most)), 2,
                                tol_abs, tol_rel);
}

// One token's choice. Lane s < top_k gets the expert of slot s in `id` (-1:
// none). Returns false where two values are too close for K. Up to four keys
// a lane are sorted first (the lower index ahead among equals), so that a round
// looks at the lanes' first ones alone; `order` holds their places, two bits each.
template <typename K, int V>
__device__ __forceinline__ bool choose(const RouteArgs &a, Order<K> (&key)[V],
                                       uint32_t lane, Order<K> *shared,
                                       float tol_abs, float tol_rel, int &id) {
  using O = Order<K>;
  if (a.top_groups < a.n_groups &&
      choose_groups<K, V>(a, key, lane, shared, tol_abs, tol_rel))
    return false;
  id = -1;
  constexpr bool kSorted = V <= 4;
  uint32_t order = 0;
  if constexpr (kSorted && V > 1) {
    uint32_t at[V];
#pragma unroll
    for (int j = 0; j < V; ++j) at[j] = j;
    const auto in_turn = [&](int x, int y) {
      const bool swap = key[y] > key[x] || (key[y] == key[x] && at[y] < at[x]);
      const O k = key[x];
      const uint32_t i = at[x];
      key[x] = swap ? key[y] : k;
      key[y] = swap ? k : key[y];
      at[x] = swap ? at[y] : i;
      at[y] = swap ? i : at[y];
    };
    if constexpr (V == 2) {
      in_turn(0, 1);
    } else {
      in_turn(0, 1), in_turn(2, 3), in_turn(0, 2), in_turn(1, 3), in_turn(1, 2);
    }
#pragma unroll
    for (int j = 0; j < V; ++j) order |= at[j] << (2 * j);
  }
  // one round more than slots: the first that is left out must not be close
  const uint32_t rounds = a.top_k + (tol_abs > 0 ? 1 : 0);
  O chosen = 0;  // lane s: the key of round s
  bool close = false;
  for (uint32_t s = 0; s < rounds; ++s) {
    O best = key[0];
    uint32_t at = order & 3;
    if constexpr (!kSorted) {
      at = 0;
#pragma unroll
      for (int j = 1; j < V; ++j)
        if (key[j] > best) best = key[j], at = j;
    }
    const O m = wave_max(best);
    if (m == 0) break;
    const uint32_t first = __builtin_ctzll(__ballot(best == m));
    const uint32_t j = __builtin_amdgcn_readlane(at, int(first));
    if (lane == s) {
      chosen = m;
      id = int(first * V + j);
    }
    if (s == 64)  // no lane's round
      close = too_close(K(from_order(lane_of(chosen, 63))), K(from_order(m)), 1,
                        tol_abs, tol_rel);
    const bool taken = lane == first;
    if constexpr (kSorted) {
#pragma unroll
      for (int i = 0; i + 1 < V; ++i) key[i] = taken ? key[i + 1] : key[i];
      key[V - 1] = taken ? O(0) : key[V - 1];
      order = taken ? order >> 2 : order;
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (taken && uint32_t(i) == j) key[i] = 0;
    }
  }
  if (lane >= a.top_k) id = -1;
  if (tol_abs == 0) return true;
  // a round's value against the one before
  const O before = __shfl_up(chosen, 1, 64);
  close = close ||
          (lane > 0 && chosen != 0 &&
           too_close(K(from_order(before)), K(from_order(chosen)), 1, tol_abs,
                     tol_rel));
  return __ballot(close) == 0;
}

// The values that the choice compares, computed in K; returns tol.
template <typename K, int V>
__device__ __forceinline__ float values_of(const RouteArgs &a,
                                           const float (&l)[V], float top,
                                           uint32_t lane, Order<K> (&key)[V]) {
  float tol = kTolSigmoid;
  K v[V];
  if (a.flags & CIERA_ROUTE_SIGMOID) {
#pragma unroll
    for (int j = 0; j < V; ++j) v[j] = one_over(K(1) + exp_of(-K(l[j])));
  } else {
    K sum = 0;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      v[j] = exp_of(K(l[j]) - K(top));
      sum += v[j];
    }
    sum = one_over(wave_sum(sum));  // the largest score
    tol = kTolSoftmax * float(sum);
#pragma unroll
    for (int j = 0; j < V; ++j) v[j] *= sum;
  }
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const uint32_t e = lane * V + j;
    const float b = a.bias && e < a.n_experts ? a.bias[e] : 0.0f;
    const bool live = l[j] > -kInf && fabsf(b) < kInf;
    key[j] = live ? to_order(v[j] + K(b)) : Order<K>(0);
  }
  return tol;
}

template <typename T, int V>
__global__ void __launch_bounds__(64 * kWaves)
    route_kernel(RouteArgs a, bool vec) {
  __shared__ uint64_t shared[kWaves][64 * V];
  const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint32_t token = blockIdx.x * kWaves + wave;
  if (token >= a.n_tokens) return;
  float l[V];
  load_logits<T, V>(static_cast<const typename T::Raw *>(a.logits) +
                        token * a.row_stride,
                    a.n_experts, vec, lane, l);
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
    uint32_t key[V];
    uint32_t *const room = reinterpret_cast<uint32_t *>(shared[wave]);
    bool sure;
    if (by_logit) {
#pragma unroll
      for (int j = 0; j < V; ++j) key[j] = l[j] > -kInf ? to_order(l[j]) : 0u;
      sure = choose<float, V>(a, key, lane, room, 0.0f, 0.0f, id);
    } else {
      const float tol = values_of<float, V>(a, l, top, lane, key);
      sure = choose<float, V>(a, key, lane, room, tol, kTolRel, id);
    }
    if (!sure) {
      uint64_t wide[V];
      values_of<double, V>(a, l, top, lane, wide);
      choose<double, V>(a, wide, lane, shared[wave], 0.0f, 0.0f, id);
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
    route_backward_kernel(RouteBackArgs a, bool vec) {
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
    load_logits<T, V>(row, a.n_experts, vec, lane, l);
    top = -kInf;
#pragma unroll
    for (int j = 0; j < V; ++j) top = l[j] > top || l[j] != l[j] ? l[j] : top;
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
// A stable counting sort. Tiles of kPlanTile pairs are counted, every expert's
// counts scanned by a wave, and every tile places its pairs behind the experts
// before (it scans their totals itself): each wave takes a run of the tile, and
// among 64 pairs those of the same expert are found by ballots over the bits of
// the id. Up to one tile is sorted by one workgroup in one launch. Nothing depends on
// the order in which waves run.
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

// A wave an expert: its counts' running sum in place, where the tile's first row
// is among the expert's, and its total behind all experts' counts.
__global__ void __launch_bounds__(256)
    plan_scan_kernel(PlanArgs a, uint32_t tiles) {
  constexpr uint32_t kAtOnce = 8;
  const uint32_t lane = threadIdx.x & 63;
  const uint32_t e = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (e >= a.n_experts) return;
  uint32_t *const row = a.counts + uint64_t(e) * tiles;
  uint32_t base = 0;
  for (uint32_t from = lane; from - lane < tiles; from += 64 * kAtOnce) {
    uint32_t c[kAtOnce];
#pragma unroll
    for (uint32_t j = 0; j < kAtOnce; ++j)
      c[j] = from + 64 * j < tiles ? row[from + 64 * j] : 0;
#pragma unroll
    for (uint32_t j = 0; j < kAtOnce; ++j) {
      uint32_t total;
      const uint32_t before = wave_prefix(c[j], total);
      if (from + 64 * j < tiles) row[from + 64 * j] = base + before;
      base += total;
    }
  }
  if (lane == 0) a.counts[uint64_t(a.n_experts) * tiles + e] = base;
}

template <bool ONE>
__global__ void __launch_bounds__(kPlanThreads)
    plan_place_kernel(PlanArgs a, uint32_t tiles, uint32_t bits) {
  // where the next pair of each expert goes, for every wave of the tile
  __shared__ uint32_t next[kPlanWaves][CIERA_MAX_EXPERTS];
  __shared__ uint32_t part[kPlanWaves];
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
  // Every workgroup scans the experts' totals; each thread's are consecutive.
  constexpr uint32_t kPer = CIERA_MAX_EXPERTS / kPlanThreads;
  uint32_t c[kPer], sum = 0;
#pragma unroll
  for (uint32_t j = 0; j < kPer; ++j) {
    const uint32_t e = threadIdx.x * kPer + j;
    c[j] = 0;
    if (e < a.n_experts) {
      if constexpr (ONE) {
#pragma unroll
        for (uint32_t w = 0; w < kPlanWaves; ++w) c[j] += next[w][e];
      } else {
        c[j] = a.counts[uint64_t(a.n_experts) * tiles + e];
      }
    }
    sum += c[j];
  }
  uint32_t wave_all;
  uint32_t before = wave_prefix(sum, wave_all);
  if (lane == 0) part[wave] = wave_all;
  __syncthreads();
  uint32_t total = 0;
#pragma unroll
  for (uint32_t w = 0; w < kPlanWaves; ++w) {
    if (w < wave) before += part[w];
    total += part[w];
  }
#pragma unroll
  for (uint32_t j = 0; j < kPer; ++j) {
    const uint32_t e = threadIdx.x * kPer + j;
    if (e < a.n_experts) {
      if (blockIdx.x == 0) a.offsets[e] = int32_t(before);
      uint32_t at = before;
      if constexpr (!ONE) at += a.counts[uint64_t(e) * tiles + blockIdx.x];
#pragma unroll
      for (uint32_t w = 0; w < kPlanWaves; ++w) {
        const uint32_t n = next[w][e];
        next[w][e] = at;
        at += n;
      }
      before += c[j];
    }
  }
  if (blockIdx.x == 0 && threadIdx.x == 0)
    a.offsets[a.n_experts] = int32_t(total);
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

// Whether V values of a row may be read at once at places that are multiples of V.
bool whole_reads(const void *p, uint64_t stride, uint32_t n, uint32_t V,
                 uint32_t bytes) {
  const uint32_t align = V * bytes < 16 ? V * bytes : 16;
  return n % V == 0 && stride * bytes % align == 0 &&
         reinterpret_cast<uintptr_t>(p) % align == 0;
}

template <typename T, int V>
hipError_t route_wide(const RouteArgs &a, hipStream_t s) {
  route_kernel<T, V><<<dim3((a.n_tokens + kWaves - 1) / kWaves),
                       dim3(64 * kWaves), 0, s>>>(
      a, whole_reads(a.logits, a.row_stride, a.n_experts, V, T::kBytes));
  return hipGetLastError();
}
template <typename T>
hipError_t route_typed(const RouteArgs &a, hipStream_t s) {
  return a.n_experts <= 64    ? route_wide<T, 1>(a, s)
         : a.n_experts <= 128 ? route_wide<T, 2>(a, s)
         : a.n_experts <= 256 ? route_wide<T, 4>(a, s)
                              : route_wide<T, 16>(a, s);
}

template <typename T, int V>
hipError_t route_back_wide(const RouteBackArgs &a, hipStream_t s) {
  route_backward_kernel<T, V><<<dim3((a.n_tokens + kWaves - 1) / kWaves),
                                dim3(64 * kWaves), 0, s>>>(
      a, whole_reads(a.logits, a.row_stride, a.n_experts, V, T::kBytes));
  return hipGetLastError();
}
template <typename T>
hipError_t route_back_typed(const RouteBackArgs &a, hipStream_t s) {
  return a.n_experts <= 64    ? route_back_wide<T, 1>(a, s)
         : a.n_experts <= 128 ? route_back_wide<T, 2>(a, s)
         : a.n_experts <= 256 ? route_back_wide<T, 4>(a, s)
                              : route_back_wide<T, 16>(a, s);
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
  plan_scan_kernel<<<(a.n_experts + 3) / 4, 256, 0, s>>>(a, tiles);
  plan_place_kernel<false><<<tiles, kPlanThreads, 0, s>>>(a, tiles, bits);
  return hipGetLastError();
}

}  // namespace ciera
