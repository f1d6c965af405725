// Routing to experts for CDNA4 (gfx950): the choice of experts with its
// weights, their gradient, and the plan that sorts (token, slot) by expert.
//
// A team of lanes holds a token, a wave or, for many tokens, 16 lanes: lane i
// has the V consecutive experts from V i on, so that the lowest lane of a ballot
// is the lowest expert among equals, and a token's logits are one coalesced read. The
// choice is top_k rounds of a maximum over the team (DPP, no LDS) and one ballot.
//
// Which experts are chosen has to be the choice of exact values, not of their
// fp32 roundings. Where the logits order the values (no bias), they are
// compared themselves. Else values are computed in fp32, whose error is bounded
// below (kTol...); a token with two neighbours in the order of the choice
// closer than that, equals among them, is done again in fp64, by a whole wave. Of fp32
// logits, or with biases that differ, some tokens in a thousand are; of 16-bit logits
// with a zero bias, whose scores are often equal, a third (32768 tokens, best 4 of 8
// groups: 22 us and 50).
//
// Vector instructions bound it, not memory. Keys are whole numbers in the floats'
// order, whose maximum takes the other lane's value within the instruction (float
// maxima quiet NaN first and move lanes apart), and what a round costs a wave, a
// wave of four teams pays once for four tokens. 32768 fp32 tokens, 8 of 256 with a
// bias and groups: 23 us (37 a wave per token, 57 with float keys; their bytes
// take 8); bf16 tokens, 8 of 256: 12.7 us, 8 of 64: 6.8 us.
#include <type_traits>

#include "ciera_expert.h"
#include "ciera_expert_dev.h"

namespace ciera {

namespace {

constexpr uint32_t kWaves = 4;  // of a workgroup
// Tokens from which four share a wave, that the card's 1024 SIMDs still have a
// wave each. 8 of 256 with a bias and groups, us a wave per token and per four:
// 1024 tokens 8.7 and 10.1, 4096 10.6 and 10.3, 32768 37 and 23; 8 of 64: 3.3 and
// 3.5, 4.0 and 3.7, 13.4 and 6.8.
constexpr uint32_t kRowTokens = 4096;
constexpr float kInf = __builtin_inff();

// |fp32 value - exact value| <= tol + kTolRel |value|. v_exp_f32 is within 1 ulp
// (2^-23); its argument x log2(e) is rounded twice (the product and the constant), and
// x = l - max once, which moves the exponential by at most 1.5 |x| 2^-23 of itself.
//   sigmoid  s = 1 / (1 + e^-l): the exponential's error counts s (1 - s) <= 1/4 fold,
//            s (1 - s) |l| <= 0.28, and the sum and the reciprocal are off by 1.5
//            ulp: (0.25 + 1.5 * 0.28 + 1.5) 2^-23
//   softmax  of the largest score p. The exponential of x <= 0 by (1 + 1.5 |x|) e^x <=
//            1.08 of p; the reciprocal of the sum and the product by 1.5; the sum by its
//            V + log2 L additions (V in a lane, then the team's steps), half an ulp
//            each, and by its exponentials', weighted by the scores: 1 + 1.5 times the
//            mean |x|. That is the entropy and the largest score's logarithm, the most
//            for one of n experts ahead of equal ones: t - 1 with (n - 1) e^-t = t - 1.
// and the bias's addition by half an ulp of the value.
constexpr float kTolSigmoid = 3 * 0x1p-23f;
template <int V, int L>
constexpr float softmax_tol() {
  constexpr int n = V * L, steps = V + (L == 64 ? 6 : 4);
  constexpr float mean = n <= 64 ? 2.4f : n <= 128 ? 2.9f : n <= 256 ? 3.4f : 4.5f;
  return (1.08f + 1.5f + 0.5f * steps + 1 + 1.5f * mean) * 0x1p-23f;
}
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
__device__ __forceinline__ void load_logits(const void *values,
                                            uint32_t n_experts, bool vec,
                                            uint32_t lane, float (&l)[V]) {
  const auto *row = static_cast<const typename T::Raw *>(values);
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

// c ? a : b of values. Written out, the choice between two elements of an array
// is one between their addresses, and the array is searched.
template <typename O>
__device__ __forceinline__ O either(bool c, O a, O b) {
  return c ? a : b;
}

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
__device__ __forceinline__ bool too_close(K above, K below, float tol_abs,
                                          float tol_rel) {
  const K size = larger(larger(above, -above), larger(below, -below));
  return above - below <= 2 * (tol_abs + tol_rel * size);
}

// A team of L lanes, 64 or 16 (a row), holds a token; `lane` counts in the team.
template <int L, typename O>
__device__ __forceinline__ O team_max(O x) {
  if constexpr (L == 64)
    return wave_max(x);
  else
    return row_max(x);
}
template <int L, typename K>
__device__ __forceinline__ K team_sum(K x) {
  if constexpr (L == 64)
    return wave_sum(x);
  else
    return row_sum(x);
}
// the team's lanes with p
template <int L>
__device__ __forceinline__ auto team_bits(bool p) {
  if constexpr (L == 64)
    return uint64_t(__ballot(p));
  else
    return uint32_t(__ballot(p) >> (threadIdx.x & 48)) & 0xFFFFu;
}
// x of the team's lane i
template <int L, typename O>
__device__ __forceinline__ O team_lane(O x, uint32_t i) {
  if constexpr (L == 64)
    return lane_of(x, int(i));
  else
    return __shfl(x, int(i), L);
}

// Whether groups of S experts are whole lanes of a row, 1, 2, 4 ... 16 of them.
__device__ inline bool groups_in_row(uint32_t S, uint32_t V) {
  const uint32_t lanes = S / V;
  return S % V == 0 && (lanes & (lanes - 1)) == 0 && lanes <= 16;
}

// Keep the top_groups groups of highest rank; the keys of others become 0.
// Returns whether the border between them is closer than K tells apart. Groups
// in a row are reduced there, as are all of whole lanes for teams of 16; others, for
// teams of 64, go through `shared`, 64 V keys of this wave, a lane a group.
template <typename K, int V, int L>
__device__ __forceinline__ bool choose_groups(const RouteArgs &a,
                                              Order<K> (&key)[V], uint32_t lane,
                                              Order<K> *shared, bool inexact,
                                              float tol_abs, float tol_rel) {
  using O = Order<K>;
  const uint32_t S = a.n_experts / a.n_groups;
  const uint32_t lanes = S / V;
  const bool in_row = L == 16 || groups_in_row(S, V);
  O one = 0, two = 0;
  if (L == 16 && (lanes & (lanes - 1)) != 0) {
    // of another number of lanes of a team of 16: one after the other
    O mine_one = key[0], mine_two = 0;
#pragma unroll
    for (int j = 1; j < V; ++j) merge_two(mine_one, mine_two, key[j], O(0));
    const uint32_t from = lane / lanes * lanes;
    for (uint32_t i = 0; i < lanes; ++i)
      merge_two(one, two, team_lane<L>(mine_one, from + i),
                team_lane<L>(mine_two, from + i));
  } else if (in_row) {
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
  const bool two_values = a.flags & CIERA_ROUTE_GROUP_TOP_TWO;
  if (two_values && two != 0)
    rank_by = to_order(from_order(one) + from_order(two));
  // group g's rank is in lane g * step
  const uint32_t step = in_row ? lanes : 1, mine = lane / step;
  uint32_t rank = 0;
  for (uint32_t g = 0; g < a.n_groups; ++g) {
    const O v = team_lane<L>(rank_by, g * step);
    rank += uint32_t((v > rank_by) | ((v == rank_by) & (g < mine)));
  }
  const bool kept = mine < a.n_groups && rank < a.top_groups;
  if (in_row) {
#pragma unroll
    for (int j = 0; j < V; ++j) key[j] = either(kept, key[j], O(0));
  } else {
    const uint64_t groups = __ballot(kept);
    uint32_t g = lane * V / S, r = lane * V - g * S;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      if (g >= 64 || !((groups >> g) & 1)) key[j] = 0;
      if (++r == S) r = 0, ++g;
    }
  }
  if (!inexact) return false;
  // A rank is off by its values' errors, each relative to that value (they may cancel
  // in the sum), and its own rounding. `off` is twice that, which covers the rounding of
  // the rank's ends; where it is no number nothing is sure.
  const bool sum = two_values && two != 0, live = one != 0;
  const K f1 = from_order(one), f2 = sum ? from_order(two) : K(0);
  const K off = 2 * ((sum ? 2 : 1) * K(tol_abs) +
                     K(tol_rel) * (larger(f1, -f1) + larger(f2, -f2)));
  const bool known = off < K(kInf);
  const O low = to_order(known ? from_order(rank_by) - off : -K(kInf));
  const O high = to_order(known ? from_order(rank_by) + off : K(kInf));
  const O least = ~team_max<L>(kept && live ? O(~low) : O(0));
  const O most = team_max<L>(mine < a.n_groups && !kept && live ? high : O(0));
  return least <= most;
}

// One token's choice. Lane s < top_k gets the expert of slot s in `id` (-1:
// none). Returns false where two values, if inexact, are too close. A lane's keys are
// sorted first in runs of up to four (the lower index ahead among equals), so that
// a round looks at the runs' first ones alone; `order` holds the indexes of a
// run, a byte each. `slot`: L words of this team.
template <typename K, int V, int L>
__device__ __forceinline__ bool choose(const RouteArgs &a, Order<K> (&key)[V],
                                       uint32_t lane, Order<K> *shared,
                                       uint32_t *slot, bool inexact,
                                       float tol_abs, float tol_rel, int &id) {
  using O = Order<K>;
  bool close = false;
  if (a.top_groups < a.n_groups)
    close = choose_groups<K, V, L>(a, key, lane, shared, inexact, tol_abs,
                                      tol_rel);
  constexpr int kRun = V < 4 ? V : 4, kRuns = V / kRun;
  uint32_t order[kRuns];
#pragma unroll
  for (int r = 0; r < kRuns; ++r) {
    uint32_t at[kRun];
#pragma unroll
    for (int j = 0; j < kRun; ++j) at[j] = r * kRun + j;
    const auto in_turn = [&](int x) {
      const O k = key[r * kRun + x], n = key[r * kRun + x + 1];
      const uint32_t i = at[x], m = at[x + 1];
      const bool swap = n > k;
      key[r * kRun + x] = either(swap, n, k);
      key[r * kRun + x + 1] = either(swap, k, n);
      at[x] = either(swap, m, i);
      at[x + 1] = either(swap, i, m);
    };
    // neighbours alone change places, so equals keep their order
    if constexpr (kRun == 2) {
      in_turn(0);
    } else if constexpr (kRun == 4) {
      in_turn(0), in_turn(2), in_turn(1), in_turn(0), in_turn(2), in_turn(1);
    }
    order[r] = 0;
#pragma unroll
    for (int j = 0; j < kRun; ++j) order[r] |= at[j] << (8 * j);
  }
  // one round more than slots: the first that is left out must not be close
  const uint32_t rounds = a.top_k + (inexact ? 1 : 0);
  O chosen = 0, last = 0;  // lane s: the key of round s; the last round's
  for (uint32_t s = 0; s < rounds; ++s) {
    O best = key[0];
    uint32_t at = order[0], from = 0;
#pragma unroll
    for (int r = 1; r < kRuns; ++r) {
      const bool more = key[r * kRun] > best;
      best = either(more, key[r * kRun], best);
      at = either(more, order[r], at);
      from = either(more, uint32_t(r), from);
    }
    last = team_max<L>(best);
    if (__ballot(last != 0) == 0) break;
    const auto who = team_bits<L>(best == last);
    const bool first = (who & (~who + 1)) == decltype(who)(1) << lane;
    const bool taken = (last != 0) & first;
    if (taken & (s < a.top_k)) slot[s] = lane * V + (at & 0xFF);
    chosen = either(lane == s, last, chosen);
#pragma unroll
    for (int r = 0; r < kRuns; ++r) {
      const bool here = taken & (kRuns == 1 || from == uint32_t(r));
#pragma unroll
      for (int i = r * kRun; i + 1 < (r + 1) * kRun; ++i)
        key[i] = either(here, key[i + 1], key[i]);
      key[(r + 1) * kRun - 1] = either(here, O(0), key[(r + 1) * kRun - 1]);
      order[r] = either(here, order[r] >> 8, order[r]);
    }
  }
  wave_order();
  id = lane < a.top_k && chosen != 0 ? int(slot[lane]) : -1;
  if (!inexact) return true;
  // a round's value against the one before; that of round L is in no lane
  const O before = __shfl_up(chosen, 1, L);
  if (lane > 0 && chosen != 0)
    close |= too_close(K(from_order(before)), K(from_order(chosen)), tol_abs,
                       tol_rel);
  if (a.top_k == L && lane == L - 1 && last != 0)
    close |= too_close(K(from_order(chosen)), K(from_order(last)), tol_abs,
                       tol_rel);
  return team_bits<L>(close) == 0;
}

// The values that the choice compares, computed in K; returns tol.
template <typename K, int V, int L>
__device__ __forceinline__ float values_of(const RouteArgs &a,
                                           const float (&l)[V], float top,
                                           uint32_t lane, bool vec_bias,
                                           Order<K> (&key)[V]) {
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
    sum = one_over(team_sum<L>(sum));  // the largest score
    tol = softmax_tol<V, L>() * float(sum);
#pragma unroll
    for (int j = 0; j < V; ++j) v[j] *= sum;
  }
  float b[V];
  if (a.bias) {
    load_logits<Fp32, V>(a.bias, a.n_experts, vec_bias, lane, b);
  } else {
#pragma unroll
    for (int j = 0; j < V; ++j) b[j] = 0;
  }
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const bool live = (l[j] > -kInf) & (fabsf(b[j]) < kInf);
    key[j] = live ? to_order(v[j] + K(b[j])) : Order<K>(0);
  }
  return tol;
}

template <typename T, int V, int L>
__global__ void __launch_bounds__(64 * kWaves)
    route_kernel(RouteArgs a, bool vec, bool vec_bias) {
  constexpr int kTeams = 64 / L;
  constexpr int kWide = V / kTeams;  // experts a lane of a whole wave
  __shared__ uint64_t shared[kWaves][64 * kWide];
  __shared__ uint32_t slots[kWaves][64];
  const uint32_t wave = threadIdx.x >> 6, lane = threadIdx.x & (L - 1);
  const uint32_t team = (threadIdx.x & 63) / L;
  const uint32_t mine_token = (blockIdx.x * kWaves + wave) * kTeams + team;
  if (mine_token - team >= a.n_tokens) return;
  // a team without a token does the last one again
  const bool real = mine_token < a.n_tokens;
  const uint32_t token = real ? mine_token : a.n_tokens - 1;
  const typename T::Raw *const row =
      static_cast<const typename T::Raw *>(a.logits) +
      uint64_t(token) * a.row_stride;
  uint32_t *const slot = slots[wave] + team * L;
  float l[V];
  load_logits<T, V>(row, a.n_experts, vec, lane, l);
  float top = l[0];
  bool fine = l[0] < kInf;  // neither NaN nor +inf
#pragma unroll
  for (int j = 1; j < V; ++j) {
    top = fmaxf(top, l[j]);
    fine &= l[j] < kInf;
  }
  fine = team_bits<L>(!fine) == 0;
  top = from_order(team_max<L>(to_order(top)));
  const bool all_groups = a.top_groups == a.n_groups;
  const bool by_logit =
      !a.bias && (all_groups || !(a.flags & CIERA_ROUTE_GROUP_TOP_TWO));
  int id = -1;
  uint32_t key[V];
  uint32_t *const room = reinterpret_cast<uint32_t *>(shared[wave]);
  float tol = 0;
  if (by_logit) {
#pragma unroll
    for (int j = 0; j < V; ++j) key[j] = l[j] > -kInf ? to_order(l[j]) : 0u;
  } else {
    tol = values_of<float, V, L>(a, l, top, lane, vec_bias, key);
  }
  const bool sure = choose<float, V, L>(a, key, lane, room, slot, !by_logit,
                                        tol, kTolRel, id);
  if (!by_logit) {
    // again in fp64, a token after the other, the whole wave on each
    for (uint64_t again = __ballot(!sure && fine && real && lane == 0);
         again != 0; again &= again - 1) {
      const int at = __builtin_ctzll(again);
      const uint64_t its = __builtin_amdgcn_readlane(token, at);
      const uint32_t all = threadIdx.x & 63;
      float wide_l[kWide];
      uint64_t wide[kWide];
      load_logits<T, kWide>(static_cast<const typename T::Raw *>(a.logits) +
                                its * a.row_stride,
                            a.n_experts, vec, all, wide_l);
      values_of<double, kWide, 64>(a, wide_l, lane_of(top, at), all, vec_bias,
                                   wide);
      int its_id;
      wave_order();
      choose<double, kWide, 64>(a, wide, all, shared[wave], slots[wave], false,
                                0.0f, 0.0f, its_id);
      its_id = __shfl(its_id, int(lane), 64);
      if (int(team) == at / L) id = its_id;
    }
  }
  // the weights, from the chosen logits
  const bool chosen = id >= 0;
  const float mine = chosen ? T::to_float(row[id]) : -kInf;
  float w;
  if (a.flags & CIERA_ROUTE_NORMALIZE) {
    // softmax's own sum cancels. Below -30, where 1 + e^l rounds to 1, sigmoids
    // go as exponentials too; relative to the largest they cannot vanish.
    const float high = from_order(team_max<L>(to_order(mine)));
    float p = 0;
    if ((a.flags & CIERA_ROUTE_SIGMOID) && high > -30.0f)
      p = chosen ? 1.0f / (1.0f + expf(-mine)) : 0.0f;
    else
      p = chosen ? expf(mine - high) : 0.0f;
    w = p / team_sum<L>(p);
  } else if (a.flags & CIERA_ROUTE_SIGMOID) {
    w = 1.0f / (1.0f + expf(-mine));
  } else {
    float sum = 0;
#pragma unroll
    for (int j = 0; j < V; ++j) sum += l[j] > -kInf ? expf(l[j] - top) : 0.0f;
    sum = team_sum<L>(sum);
    w = expf(mine - top) / sum;
  }
  if (real && lane < a.top_k) {
    const uint64_t out = uint64_t(token) * a.top_k + lane;
    a.ids[out] = fine ? id : -1;
    a.weights[out] = !fine ? __builtin_nanf("") : chosen ? w * a.scale : 0.0f;
  }
}

// ------------------------------------------------------------- gradient ----
// With c = scale and the chosen set fixed:
//   softmax normalised   d_i = w_i (g_i - sum_j w_j g_j / c)
//   softmax              d_e = p_e (c g_e [chosen] - c sum_j p_j g_j)
//   sigmoid normalised   d_i = w_i (1 - s_i) (g_i - sum_j w_j g_j / c)
//   sigmoid              d_i = c s_i (1 - s_i) g_i
// (d_i for the chosen; 0 elsewhere). Only the plain softmax reads the whole
// row. 1 - s is computed beside s: subtracted from 1, an s close to it leaves nothing (l
// = 16: 6% off, from 17 on 0). So it is with the largest share m, which
// alone can near 1: what it takes from itself is left out on both sides,
//   g_m - sum_j w_j g_j / c  =  g_m (1 - w_m / c) - sum_{j != m} w_j g_j / c
// with 1 - w_m / c as the sum of the others' shares (of all other experts' scores where
// weights are not renormalised). An m that is named twice has the other slot among them.
// s and 1 - s of a sigmoid from the exponential that does not grow
__device__ __forceinline__ void sigmoid_of(float l, float &s, float &off) {
  const float e = expf(-fabsf(l)), large = 1.0f / (1.0f + e);
  s = l >= 0 ? large : e * large;
  off = l >= 0 ? e * large : large;
}

template <typename T, int V, int L>
__global__ void __launch_bounds__(64 * kWaves)
    route_backward_kernel(RouteBackArgs a, bool vec, bool vec_out) {
  const uint32_t lane = threadIdx.x & (L - 1);
  const uint32_t token = blockIdx.x * (64 / L * kWaves) + threadIdx.x / L;
  if (token >= a.n_tokens) return;  // a whole team
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
  if (!chosen) {  // adds nothing, whatever its gradient is
    id = -1;
    g = 0;
  }
  const float mine = chosen ? T::to_float(row[id]) : -kInf;
  float d = 0;  // of this lane's slot
  float l[V], spread = 0, sum = 1;
  int top_id = -1;  // whole: the expert of the largest score, if it is chosen
  const bool whole = !sigmoid && !normal;
  if (whole) {
    load_logits<T, V>(row, a.n_experts, vec, lane, l);
    float top = -kInf;
#pragma unroll
    for (int j = 0; j < V; ++j) top = l[j] > top || l[j] != l[j] ? l[j] : top;
    // a NaN stays the maximum's choice of no lane: the sum carries it instead
    top = from_order(team_max<L>(to_order(top == top ? top : -kInf)));
    const auto who =
        team_bits<L>(chosen && mine == top && fabsf(top) < kInf);
    const uint32_t m = who ? uint32_t(__builtin_ctzll(who)) : 0u;
    if (who) top_id = int(team_lane<L>(uint32_t(id), m));
    float others = 0;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const bool out = l[j] == -kInf || int(lane * V + j) == top_id;
      l[j] = out ? 0.0f : expf(l[j] - top);
      others += l[j];
    }
    others = team_sum<L>(others);
    sum = others + (who ? 1.0f : 0.0f);  // e^0
    const float p = chosen && sum != 0 ? expf(mine - top) / sum : 0.0f;
    d = p * g;
    spread = team_sum<L>(d);
    const bool is_top = who && lane == m;
    const float rest = team_sum<L>(is_top ? 0.0f : d);
    if (is_top) d = p * (g * (others / sum) - rest);
  } else if (normal) {
    const float high = from_order(team_max<L>(to_order(mine)));
    const auto who = team_bits<L>(chosen && mine == high);
    const bool is_top = who && lane == uint32_t(__builtin_ctzll(who));
    const bool as_exp = !sigmoid || high <= -30.0f;
    float s = 0, off = 1;
    if (sigmoid) sigmoid_of(mine, s, off);
    float p = 0;
    if (chosen && high != -kInf) p = as_exp ? expf(mine - high) : s;
    const float all = team_sum<L>(p), others = team_sum<L>(is_top ? 0.0f : p);
    const float w = all == 0 ? 0.0f : p / all;
    const float wg = chosen ? w * g : 0.0f;
    const float mean = team_sum<L>(wg), rest = team_sum<L>(is_top ? 0.0f : wg);
    const float from_mean =
        !is_top ? g - mean : all == 0 ? 0.0f : g * (others / all) - rest;
    d = chosen ? w * off * from_mean : 0.0f;
  } else {
    float s, off;
    sigmoid_of(mine, s, off);
    d = chosen ? s * off * g : 0.0f;
  }
  float o[V];
#pragma unroll
  for (int j = 0; j < V; ++j) o[j] = whole ? -(l[j] / sum) * spread : 0.0f;
  if (whole && !(sum > 0)) {  // every logit is -inf, or one is NaN
#pragma unroll
    for (int j = 0; j < V; ++j) o[j] = sum != sum ? sum : 0.0f;
  }
  for (uint32_t s = 0; s < a.top_k; ++s) {
    const int e = int(team_lane<L>(uint32_t(id), s));
    const float v = team_lane<L>(d, s);
#pragma unroll
    for (int j = 0; j < V; ++j)
      if (e == int(lane * V + j)) o[j] += v;
  }
  typename T::Raw raw[V];
#pragma unroll
  for (int j = 0; j < V; ++j) raw[j] = T::from_float(o[j]);
  if (vec_out) {
    if (lane * V < a.n_experts)
      __builtin_memcpy(
          __builtin_assume_aligned(d_row + lane * V,
                                   V * T::kBytes < 16 ? V * T::kBytes : 16),
          raw, V * T::kBytes);
  } else {
#pragma unroll
    for (int j = 0; j < V; ++j)
      if (lane * V + j < a.n_experts) d_row[lane * V + j] = raw[j];
  }
}

// ----------------------------------------------------------------- plan ----
// A stable counting sort. Tiles of pairs are counted, every expert's
// counts scanned by a wave, and every tile places its pairs behind the experts
// before (it scans their totals itself): each wave takes a run of the tile, and
// among 64 pairs those of the same expert are found by ballots over the bits of
// the id. Up to 2048 pairs are sorted by one workgroup in one launch (8 pairs 2.8 us,
// 2048 4.8). Nothing depends on the order in which waves run.
constexpr uint32_t kPlanThreads = 512;
constexpr uint32_t kPlanWaves = kPlanThreads / 64;

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

template <uint32_t TILE>
__global__ void __launch_bounds__(kPlanThreads)
    plan_count_kernel(PlanArgs a, uint32_t tiles) {
  __shared__ uint32_t count[CIERA_MAX_EXPERTS + 1];
  for (uint32_t e = threadIdx.x; e <= a.n_experts; e += kPlanThreads)
    count[e] = 0;
  __syncthreads();
  const uint32_t from = blockIdx.x * TILE;
#pragma unroll
  for (uint32_t i = threadIdx.x; i < TILE; i += kPlanThreads)
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

template <bool ONE, uint32_t TILE>
__global__ void __launch_bounds__(kPlanThreads)
    plan_place_kernel(PlanArgs a, uint32_t tiles, uint32_t bits) {
  // where the next pair of each expert goes, for every wave of the tile
  __shared__ uint32_t next[kPlanWaves][CIERA_MAX_EXPERTS];
  __shared__ uint32_t part[kPlanWaves];
  constexpr uint32_t kRun = TILE / kPlanWaves;  // pairs per wave
  const uint32_t lane = threadIdx.x & 63;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  for (uint32_t e = threadIdx.x; e < a.n_experts; e += kPlanThreads)
#pragma unroll
    for (uint32_t w = 0; w < kPlanWaves; ++w) next[w][e] = 0;
  __syncthreads();
  const uint32_t tile = blockIdx.x * TILE;
  const uint32_t tile_end = tile + TILE < a.n_pairs ? tile + TILE : a.n_pairs;
  // alone, all waves share few pairs
  const uint32_t run =
      ONE ? (a.n_pairs + kPlanThreads - 1) / kPlanThreads * 64 : kRun;
  const uint32_t from = tile + wave * run;
  const uint32_t end = from + run < tile_end ? from + run : tile_end;
  uint32_t mine[kRun / 64];
#pragma unroll
  for (uint32_t r = 0; r < kRun / 64; ++r) {
    mine[r] = expert_of(a, from + r * 64 + lane, end);
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
  for (uint32_t r = 0; r < kRun / 64; ++r) {
    if (from + r * 64 >= end) break;  // the whole wave
    const uint32_t i = from + r * 64 + lane, e = mine[r];
    const uint64_t same = same_as(e, bits);
    const uint64_t below = same & ((1ull << lane) - 1);
    uint32_t at = 0;
    if (e < a.n_experts) at = next[wave][e] + __popcll(below);
    wave_order();
    if (e < a.n_experts && below == 0) next[wave][e] = at + __popcll(same);
    wave_order();
    if (i < end) {
      a.position[i] = e < a.n_experts ? int32_t(at) : -1;
      if (e < a.n_experts) a.source[at] = int32_t(i);
      if (i >= total) a.source[i] = -1;
    }
  }
}

__global__ void plan_empty_kernel(int32_t *offsets, uint32_t n) {
  for (uint32_t i = threadIdx.x; i < n; i += blockDim.x) offsets[i] = 0;
}

template <uint32_t TILE>
hipError_t plan_tiled(const PlanArgs &a, uint32_t tiles, uint32_t bits,
                      hipStream_t s) {
  plan_count_kernel<TILE><<<tiles, kPlanThreads, 0, s>>>(a, tiles);
  plan_scan_kernel<<<(a.n_experts + 3) / 4, 256, 0, s>>>(a, tiles);
  plan_place_kernel<false, TILE><<<tiles, kPlanThreads, 0, s>>>(a, tiles, bits);
  return hipGetLastError();
}

// Whether V values of a row may be read at once at places that are multiples of V.
bool whole_reads(const void *p, uint64_t stride, uint32_t n, uint32_t V,
                 uint32_t bytes) {
  const uint32_t align = V * bytes < 16 ? V * bytes : 16;
  return n % V == 0 && stride * bytes % align == 0 &&
         reinterpret_cast<uintptr_t>(p) % align == 0;
}

template <typename T, int V, int L>
hipError_t route_wide(const RouteArgs &a, hipStream_t s) {
  constexpr uint32_t kTokens = kWaves * (64 / L);  // per workgroup
  route_kernel<T, V, L><<<dim3((a.n_tokens + kTokens - 1) / kTokens),
                          dim3(64 * kWaves), 0, s>>>(
      a, whole_reads(a.logits, a.row_stride, a.n_experts, V, T::kBytes),
      whole_reads(a.bias, 0, a.n_experts, V, 4));
  return hipGetLastError();
}
// Whether V experts a lane in teams of 16 hold the tokens.
bool in_rows(const RouteArgs &a, uint32_t V) {
  return a.n_experts <= 16 * V && a.top_k <= 16 && a.n_tokens >= kRowTokens &&
         (a.top_groups == a.n_groups || a.n_experts / a.n_groups % V == 0);
}
template <typename T>
hipError_t route_typed(const RouteArgs &a, hipStream_t s) {
  return in_rows(a, 4)        ? route_wide<T, 4, 16>(a, s)
         : in_rows(a, 8)      ? route_wide<T, 8, 16>(a, s)
         : in_rows(a, 16)     ? route_wide<T, 16, 16>(a, s)
         : a.n_experts <= 64  ? route_wide<T, 1, 64>(a, s)
         : a.n_experts <= 128 ? route_wide<T, 2, 64>(a, s)
         : a.n_experts <= 256 ? route_wide<T, 4, 64>(a, s)
                              : route_wide<T, 16, 64>(a, s);
}

template <typename T, int V, int L>
hipError_t route_back_wide(const RouteBackArgs &a, hipStream_t s) {
  constexpr uint32_t kTokens = kWaves * (64 / L);
  route_backward_kernel<T, V, L>
      <<<dim3((a.n_tokens + kTokens - 1) / kTokens), dim3(64 * kWaves), 0, s>>>(
          a, whole_reads(a.logits, a.row_stride, a.n_experts, V, T::kBytes),
          whole_reads(a.d_logits, a.d_row_stride, a.n_experts, V, T::kBytes));
  return hipGetLastError();
}
template <typename T>
hipError_t route_back_typed(const RouteBackArgs &a, hipStream_t s) {
  const bool rows = a.top_k <= 16 && a.n_tokens >= kRowTokens;
  return rows && a.n_experts <= 64    ? route_back_wide<T, 4, 16>(a, s)
         : rows && a.n_experts <= 128 ? route_back_wide<T, 8, 16>(a, s)
         : rows && a.n_experts <= 256 ? route_back_wide<T, 16, 16>(a, s)
         : a.n_experts <= 64          ? route_back_wide<T, 1, 64>(a, s)
         : a.n_experts <= 128         ? route_back_wide<T, 2, 64>(a, s)
         : a.n_experts <= 256         ? route_back_wide<T, 4, 64>(a, s)
                                      : route_back_wide<T, 16, 64>(a, s);
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
    plan_place_kernel<true, kPlanOne>
        <<<1, kPlanThreads, 0, s>>>(a, tiles, bits);
    return hipGetLastError();
  }
  return plan_tile(a.n_pairs) == 1024 ? plan_tiled<1024>(a, tiles, bits, s)
                                      : plan_tiled<2048>(a, tiles, bits, s);
}

}  // namespace ciera
