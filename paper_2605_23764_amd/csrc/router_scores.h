// Routing by scores: the selection of moe_route_scores (its backward and the balance bias: scores_backward.h).
//
//   l: logits, NaN as -inf;  s = sigmoid(l), or softmax over all E;  key[e] = s[e] + bias[e], -inf where l[e] = -inf or the sum is NaN
//   the experts in n_group groups of E / n_group: a group's score is its best key + its second best (0 without a living one); the
//   topk_group best groups stay (ties: the lowest);  the k largest keys in them (ties: the lowest expert)
//   w[j] = scale * s[j] / (renormalize ? sum of the selected s : 1), 0 / 0 = 0
//
// Scores, keys and weights are in 64 bits: between two experts whose keys differ by less than a rounding to 32 bits, the rounding would
// decide, and with a bias the order of the logits does not (8192 tokens of 256 experts have a few such pairs; every implementation would
// select others).  Weights are rounded once.
#pragma once
#include "route_select.h"
#include "scores_math.h"

namespace moe {

constexpr int kMaxGroups = 16;             // a lane of the token's row to a group

struct ScoreParams {
  const float* bias;     // [E] or null
  int sigmoid;           // 0: softmax
  int n_group, topk_group, per_group;
  int renorm;
  float scale;
};

// Monotone map double -> uint64, NaN as -inf; every value's key is above 0.
__device__ __forceinline__ uint64_t double_order_key(double v) {
  if (v != v) v = -__builtin_huge_val();
  const uint64_t u = __builtin_bit_cast(uint64_t, v == 0.0 ? 0.0 : v);
  return (u >> 63) ? ~u : (u | (1ull << 63));
}
__device__ __forceinline__ double double_from_order_key(uint64_t k) {
  return __builtin_bit_cast(double, (k >> 63) ? k & ~(1ull << 63) : ~k);
}

// Over the 16 lanes of a DPP row, in all of them.
template <typename OP> __device__ __forceinline__ uint64_t row_reduce_u64(uint64_t v, OP op) {
#define MOE_STEP(ctrl)                                                                                                          \
  {                                                                                                                             \
    const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)v, ctrl, 0xf, 0xf, false);                      \
    const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(v >> 32), ctrl, 0xf, 0xf, false);              \
    v = op(v, (uint64_t)hi << 32 | lo);                                                                                         \
  }
  MOE_STEP(0xB1) MOE_STEP(0x4E) MOE_STEP(0x141) MOE_STEP(0x140)
#undef MOE_STEP
  return v;
}
__device__ __forceinline__ uint64_t row_max_u64(uint64_t v) {
  return row_reduce_u64(v, [](uint64_t a, uint64_t b) { return a > b ? a : b; });
}
__device__ __forceinline__ double row_sum_f64(double v) {
  return __builtin_bit_cast(double, row_reduce_u64(__builtin_bit_cast(uint64_t, v), [](uint64_t a, uint64_t b) {
    return __builtin_bit_cast(uint64_t, __builtin_bit_cast(double, a) + __builtin_bit_cast(double, b));
  }));
}

// Four tokens by one wave, one per 16-lane row, as route_select; the keys of the wave's tokens also stand in LDS, where a lane per group
// finds the group's two best (s_keys: 4 E words, used with more than one group).
template <int KP, bool GROUPS>
__device__ __forceinline__ void route_scores_select(const RouteParams& p, const ScoreParams& sc, int t_first, int lane, const uint32_t (&order)[KP],
                                                    int32_t* s_idx, float* s_val, uint64_t* s_keys) {
  const int row = lane >> 4, s = lane & 15, e0 = s * KP;
  float l[KP];
#pragma unroll
  for (int i = 0; i < KP; ++i) l[i] = order[i] ? float_from_order_key(order[i]) : -__builtin_huge_valf();   // 0: no expert there
  float m = 0.f;
  double inv = 1.0;
  if (!sc.sigmoid) {
    uint32_t top = order[0];
#pragma unroll
    for (int i = 1; i < KP; ++i) top = order[i] > top ? order[i] : top;
    m = float_from_order_key(row_max_u32(top));
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < KP; ++i) sum += exp_below(l[i], m);
    sum = row_sum_f64(sum);
    inv = sum > 0.0 ? 1.0 / sum : 0.0;
  }
  auto score = [&](float v) __attribute__((always_inline)) { return sc.sigmoid ? sigmoid64(v) : exp_below(v, m) * inv; };
  uint64_t key[KP];
#pragma unroll
  for (int i = 0; i < KP; ++i) {
    const double b = sc.bias && e0 + i < p.E ? (double)sc.bias[e0 + i] : 0.0;
    const double v = l[i] == -__builtin_huge_valf() ? -__builtin_huge_val() : score(l[i]) + b;
    key[i] = e0 + i < p.E ? double_order_key(v) : 0ull;
  }
  if constexpr (GROUPS) {
    uint64_t* mine = s_keys + row * p.E;
#pragma unroll
    for (int i = 0; i < KP; ++i)
      if (e0 + i < p.E) mine[e0 + i] = key[i];
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    uint64_t group = 0;                                          // of group s; 0: no such group
    if (s < sc.n_group) {
      uint64_t best = 0, second = 0;
      int at = s;                                                // lanes start at different banks
      while (at >= sc.per_group) at -= sc.per_group;
      for (int i = 0; i < sc.per_group; ++i) {
        const uint64_t v = mine[s * sc.per_group + at];
        second = v > best ? best : (v > second ? v : second);
        best = v > best ? v : best;
        at = at + 1 == sc.per_group ? 0 : at + 1;
      }
      const double b1 = double_from_order_key(best), b2 = second ? double_from_order_key(second) : 0.0;
      group = double_order_key(b1 + (b2 == -__builtin_huge_val() ? 0.0 : b2));
    }
    uint32_t keep = 0;
    for (int j = 0; j < sc.topk_group; ++j) {
      const uint64_t best = row_max_u64(group);
      const int first = __builtin_ctz((uint32_t)(__ballot(group == best) >> (row * 16)) & 0xFFFFu);
      keep |= 1u << first;
      if (s == first) group = 0;
    }
    int g = e0 / sc.per_group, left = (g + 1) * sc.per_group - e0;
#pragma unroll
    for (int i = 0; i < KP; ++i) {
      if (!((keep >> g) & 1)) key[i] = 0;
      if (--left == 0) { ++g; left = sc.per_group; }
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");       // the next four tokens' keys go to the same place
    __builtin_amdgcn_wave_barrier();
  }
  for (int j = 0; j < p.k; ++j) {
    uint64_t local = key[0];
    float val = l[0];
    int li = 0;
#pragma unroll
    for (int i = 1; i < KP; ++i)
      if (key[i] > local) { local = key[i]; val = l[i]; li = i; }
    const uint64_t best = row_max_u64(local);
    const uint32_t in_row = (uint32_t)(__ballot(local == best) >> (row * 16)) & 0xFFFFu;
    const bool winner = s == __builtin_ctz(in_row);
#pragma unroll
    for (int i = 0; i < KP; ++i)
      if (winner && i == li) key[i] = 0;
    if (winner) {
      s_idx[row * kMaxK + j] = e0 + li;
      s_val[row * kMaxK + j] = val;
    }
  }
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  const int t = t_first + row;
  const bool slot = s < p.k;
  const int idx = slot ? s_idx[row * kMaxK + s] : 0;
  const double ps = slot ? score(s_val[row * kMaxK + s]) : 0.0;
  const double sum = row_sum_f64(ps);
  if (t < p.T && slot) {
    p.topk_idx[(size_t)t * p.k + s] = idx;
    p.topk_w[(size_t)t * p.k + s] = (float)((double)sc.scale * (sc.renorm ? (sum > 0.0 ? ps / sum : 0.0) : ps));
  }
}

// The selection as route_chunk and route_one call it.  s_keys: the workgroup's, 4 kMaxE words per wave.
template <bool GROUPS> struct SelectScores {
  const ScoreParams& sc;
  uint64_t* s_keys;
  template <int KP>
  __device__ __forceinline__ void operator()(const RouteParams& p, int t_first, int lane, uint32_t (&key)[KP], int32_t* s_idx, float* s_val) const {
    route_scores_select<KP, GROUPS>(p, sc, t_first, lane, key, s_idx, s_val, s_keys + (threadIdx.x / kWave) * (kRouteTokensPerWave * kMaxE));
  }
};

}  // namespace moe
