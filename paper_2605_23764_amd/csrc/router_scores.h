// Routing by scores: the selection of moe_route_scores (its backward and the balance bias: scores_backward.h).
//
//   l: logits, NaN as -inf;  s = sigmoid(l), or softmax over all E;  key[e] = s[e] + bias[e], -inf where l[e] = -inf or the sum is NaN
//   the experts in n_group groups of E / n_group: a group's score is its best key + its second best (0 without a living one); the
//   topk_group best groups stay (ties: the lowest);  the k largest keys in them (ties: the lowest expert)
//   w[j] = scale * s[j] / (renormalize ? sum of the selected s : 1), 0 / 0 = 0
//
// Scores, keys and weights are in 64 bits: between two experts whose keys differ by less than a rounding to 32 bits, the rounding would
// decide, and with a bias the order of the logits does not (8192 tokens of 256 experts have a few such pairs; every implementation would
// select others).  Weights are rounded once.  Keys, and groups' sums of them, are rounded to 44 bits, and the lowest 8 are the expert's
// number, so that one maximum finds the key, the expert and the lowest of equals.
//
// Bound by instructions and their latency: about 30 in 64 bits per expert for its score, and a round of the selection is a maximum over the
// token's lanes' first keys (each lane sorts its own, by a network of maxima and minima), behind which the winner takes its next from LDS
// (moved up in registers instead, and groups scored by a loop over their experts: 8192 x 256 21.6 us, so 18.4).  Groups of whole lanes are
// scored from the lanes' two best, joined; others by that loop.  What is done per expert is a loop on the token's keys in LDS where a lane
// has more than four, for the code's length: a line of it that no wave has run yet costs some 300 clocks.  A token takes 16 lanes up to 128 experts, 32 beyond, of twice as many waves, and 64 in a launch of up to 16 tokens,
// a wave to each.  8192 tokens of 256 experts in 8 groups, k = 8: 18.4 us, without groups 17, where their logits' 8.4 MB take 1.6; 30001
// tokens of 64 experts in 4 groups, k = 6: 17.4 (in another form 17.8, and 28.0 with the LDS that 256 need).
#pragma once
#include "route_select.h"
#include "scores_math.h"

namespace moe {

struct ScoreParams {
  const float* bias;     // [E] or null
  int sigmoid;           // 0: softmax
  int n_group, topk_group, per_group, group_mul;   // (e * group_mul) >> 16 = e / per_group for e < 256
  int renorm;
  float scale;
};

// A key, rounded to 44 bits, with its number n below 256 in the lowest 8: larger keys are larger, and of equal ones those with the lower number.
// (Rounded, not cut off: two scores that add up to 1 do so still.)
constexpr double kKeyDead = -1e301;        // an expert that comes behind all others, a group without a living one
constexpr double kKeyNone = -1e308;        // nothing there
__device__ __forceinline__ double key_with(double v, int n) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v) + 128;
  const uint32_t hi = (uint32_t)(u >> 32);
  const uint32_t low = (int32_t)hi < 0 ? (uint32_t)n : 255u - (uint32_t)n;
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | (((uint32_t)u & ~255u) | low));
}
__device__ __forceinline__ int key_number(double v) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  const int low = (int)(u & 255u);
  return (int32_t)(u >> 32) < 0 ? low : 255 - low;
}
__device__ __forceinline__ double key_without(double v) { return __builtin_bit_cast(double, __builtin_bit_cast(uint64_t, v) & ~255ull); }

// The value of the lane that `CTRL` names: kLane1, its neighbour's; then, once lanes of one such set hold the same, that of the other two, four, eight.
constexpr int kLane1 = 0xB1, kLane2 = 0x4E, kLane4 = 0x141, kLane8 = 0x140;
template <int CTRL> __device__ __forceinline__ double lane_value(double v) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)u, CTRL, 0xf, 0xf, false);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(u >> 32), CTRL, 0xf, 0xf, false);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
// Over the LPT lanes of a token, in all of them.
template <int LPT, typename OP> __device__ __forceinline__ double lanes_reduce(double v, OP op) {
  v = op(v, lane_value<kLane1>(v));
  v = op(v, lane_value<kLane2>(v));
  v = op(v, lane_value<kLane4>(v));
  v = op(v, lane_value<kLane8>(v));
  if constexpr (LPT >= 32) {
    auto join = [&](auto a, auto b) __attribute__((always_inline)) {
      v = op(__builtin_bit_cast(double, (uint64_t)(uint32_t)b[0] << 32 | (uint32_t)a[0]),
             __builtin_bit_cast(double, (uint64_t)(uint32_t)b[1] << 32 | (uint32_t)a[1]));
    };
    uint64_t u = __builtin_bit_cast(uint64_t, v);
    join(__builtin_amdgcn_permlane16_swap((uint32_t)u, (uint32_t)u, false, false),
         __builtin_amdgcn_permlane16_swap((uint32_t)(u >> 32), (uint32_t)(u >> 32), false, false));
    if constexpr (LPT == 64) {
      u = __builtin_bit_cast(uint64_t, v);
      join(__builtin_amdgcn_permlane32_swap((uint32_t)u, (uint32_t)u, false, false),
           __builtin_amdgcn_permlane32_swap((uint32_t)(u >> 32), (uint32_t)(u >> 32), false, false));
    }
  }
  return v;
}
template <int LPT> __device__ __forceinline__ double lanes_max(double v) {
  return lanes_reduce<LPT>(v, [](double a, double b) { return __builtin_fmax(a, b); });
}
template <int LPT> __device__ __forceinline__ double lanes_sum(double v) {
  return lanes_reduce<LPT>(v, [](double a, double b) { return a + b; });
}

// Descending, by Batcher's odd-even merges (Batcher, 1968).
template <int N> __device__ __forceinline__ void sort_keys(double (&v)[N]) {
#pragma unroll
  for (int p = 1; p < N; p *= 2)
#pragma unroll
    for (int k = p; k >= 1; k /= 2)
#pragma unroll
      for (int j = k % p; j + k < N; j += 2 * k)
#pragma unroll
        for (int i = 0; i < k; ++i)
          if (i + j + k < N && (i + j) / (2 * p) == (i + j + k) / (2 * p)) {
            const double a = v[i + j], b = v[i + j + k];
            v[i + j] = __builtin_fmax(a, b);
            v[i + j + k] = __builtin_fmin(a, b);
          }
}

// Words of LDS of a wave whose lanes have KP experts: a word beside each lane's, so that the lanes' lie in all banks.
constexpr int slot_words(int kp) { return kWave * (kp + 1); }
// 64 / LPT tokens from t_first on by one wave, LPT lanes to each, KP experts to a lane (LPT KP >= E).
template <int LPT, int KP, bool GROUPS>
__device__ __forceinline__ void route_scores_select(const RouteParams& p, const ScoreParams& sc, int t_first, int lane, int32_t* s_idx, double* slots) {
  constexpr int kUnroll = KP <= 4 ? KP : 1;
  const int row = lane / LPT, s = lane % LPT, e0 = s * KP, n = p.E - e0, tok = t_first + row;
  const float none = -__builtin_huge_valf();
  double* mine = slots + row * (LPT * (KP + 1));
  auto at = [](int e) __attribute__((always_inline)) { return e + e / KP; };
  float l[KP];                                                   // -inf where the lane has no expert
  {
    const float* logits = p.logits + (size_t)min(tok, p.T - 1) * p.E;   // tokens past the end repeat the last one
    if (KP >= 4 && (p.E & 3) == 0) {
#pragma unroll
      for (int i = 0; i + 3 < KP; i += 4) __builtin_memcpy(l + i, logits + min(e0 + i, p.E - 4), 16);
    } else {
#pragma unroll
      for (int i = 0; i < KP; ++i) l[i] = logits[min(e0 + i, p.E - 1)];
    }
#pragma unroll
    for (int i = 0; i < KP; ++i)
      if (i >= n || l[i] != l[i]) l[i] = none;
  }
  auto settled = []() __attribute__((always_inline)) {           // a wave's LDS accesses, seen by its other lanes
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  };
  float m = none;
#pragma unroll
  for (int i = 0; i < KP; ++i) {
    m = __builtin_fmaxf(m, l[i]);
    mine[at(e0) + i] = (double)l[i];                             // where there is no expert, too
  }
  // scores, -1 for the dead; softmax: not yet over their sum
  double inv = 1.0;
  if (sc.sigmoid) {
#pragma unroll kUnroll
    for (int i = 0; i < KP; ++i) {
      const float v = (float)mine[at(e0) + i];
      mine[at(e0) + i] = v == none ? -1.0 : sigmoid64(v);
    }
  } else {
    m = (float)lanes_max<LPT>((double)m);
    double sum = 0.0;
#pragma unroll kUnroll
    for (int i = 0; i < KP; ++i) {
      const float v = (float)mine[at(e0) + i];
      const double t = exp_below(v, m);
      sum += t;
      mine[at(e0) + i] = v == none ? -1.0 : t;
    }
    sum = lanes_sum<LPT>(sum);
    inv = sum > 0.0 ? reciprocal64(sum) : 0.0;                   // a living row's sum is 1 .. E
  }
  // keys
  float next = sc.bias ? sc.bias[min(e0, p.E - 1)] : 0.f;
#pragma unroll kUnroll
  for (int i = 0; i < KP; ++i) {
    const float b = next;
    if (sc.bias) next = sc.bias[min(e0 + i + 1, p.E - 1)];
    const double t = mine[at(e0) + i];
    double v = __builtin_fmax(__builtin_fmin(t * inv + (double)b, 1e300), -1e300);
    v = t < 0.0 || b != b || b == none ? kKeyDead : v;
    mine[at(e0) + i] = key_with(v, e0 + i);
  }
  settled();
  double key[KP];
#pragma unroll
  for (int i = 0; i < KP; ++i) {
    const double v = mine[at(e0) + i];
    key[i] = i < n ? v : kKeyNone;
  }
  // a group's score of its two best keys, whose own numbers go from the sum; kKeyDead stays below every living group
  auto group_key = [](double best, double second, int g) __attribute__((always_inline)) {
    return key_with(best < -1e300 ? kKeyDead : key_without(best) + (second < -1e300 ? 0.0 : key_without(second)), g);
  };
  // lanes of a group; 0 where groups begin or end inside a lane's experts, or are no power of two up to 16 of them
  const int whole = sc.per_group / KP, lanes = sc.per_group % KP == 0 && (whole & (whole - 1)) == 0 && whole <= 16 ? whole : 0;
  if (GROUPS && lanes == 0) {                                    // lane s for group s
    double group = kKeyNone;
    if (s < sc.n_group) {
      double best = kKeyNone, second = kKeyNone;
      int e = s * sc.per_group;
#pragma unroll 2
      for (int i = 0; i < sc.per_group; ++i, ++e) {
        const double v = mine[at(e)];
        second = __builtin_fmax(second, __builtin_fmin(best, v));
        best = __builtin_fmax(best, v);
      }
      group = group_key(best, second, s);
    }
    uint32_t keep = 0;
    for (int j = 0; j < sc.topk_group; ++j) {
      const double best = lanes_max<LPT>(group);
      keep |= 1u << key_number(best);
      if (group == best) group = kKeyNone;
    }
#pragma unroll
    for (int i = 0; i < KP; ++i)
      if (!((keep >> (((uint32_t)(e0 + i) * (uint32_t)sc.group_mul) >> 16)) & 1)) key[i] = kKeyNone;
  }
  sort_keys(key);
  double top = key[0];
  if (GROUPS && lanes != 0) {                                    // every lane for its own group
    double best = top, second = KP > 1 ? key[KP > 1 ? 1 : 0] : kKeyNone;
    auto join = [&](double b, double c) __attribute__((always_inline)) {
      second = __builtin_fmax(__builtin_fmin(best, b), __builtin_fmax(second, c));
      best = __builtin_fmax(best, b);
    };
    if (lanes >= 2) join(lane_value<kLane1>(best), lane_value<kLane1>(second));
    if (lanes >= 4) join(lane_value<kLane2>(best), lane_value<kLane2>(second));
    if (lanes >= 8) join(lane_value<kLane4>(best), lane_value<kLane4>(second));
    if (lanes >= 16) join(lane_value<kLane8>(best), lane_value<kLane8>(second));
    double group = n > 0 ? group_key(best, second, ((uint32_t)e0 * (uint32_t)sc.group_mul) >> 16) : kKeyNone;
    bool stays = false;
    for (int j = 0; j < sc.topk_group; ++j)
      if (group == lanes_max<LPT>(group)) {
        stays = true;
        group = kKeyNone;
      }
    top = stays ? top : kKeyNone;
  }
  // the lane's keys behind its first, and none behind them, for the rounds to come
  double* rest = mine + at(e0);
  if constexpr (KP > 1) {
#pragma unroll
    for (int i = 1; i < KP; ++i) rest[i - 1] = key[i];
    rest[KP - 1] = kKeyNone;
  }
  double chosen = kKeyNone;                                      // of slot s
  for (int j = 0; j < p.k; ++j) {
    const double best = lanes_max<LPT>(top);
    chosen = s == j ? best : chosen;
    if (top == best) {
      if constexpr (KP == 1) top = kKeyNone;
      else top = *rest++;
    }
  }
  const bool slot = s < p.k;
  const int idx = slot ? key_number(chosen) : 0;
  if (slot) s_idx[row * kMaxK + s] = idx;
  float val = p.logits[(size_t)min(tok, p.T - 1) * p.E + idx];
  if (!slot || val != val) val = none;
  const double ps = sc.sigmoid ? sigmoid64(val) : exp_below(val, m) * inv;
  const double sum = lanes_sum<LPT>(slot ? ps : 0.0);
  if (tok < p.T && slot) {
    p.topk_idx[(size_t)tok * p.k + s] = idx;
    p.topk_w[(size_t)tok * p.k + s] = (float)((double)sc.scale * (sc.renorm ? (sum > 0.0 ? ps / sum : 0.0) : ps));
  }
  settled();                                                     // the next tokens' go to the same places
}

// The selection as route_chunk calls it: LPT lanes per token and KP experts per lane as with_score_lanes has them.  s_slots: slot_words per wave.
template <bool GROUPS, int LPT, int KP> struct SelectScores {
  const ScoreParams& sc;
  double* s_slots;
  __device__ __forceinline__ void tokens(const RouteParams& p, int t0, int32_t* s_idx, float*) const {
    constexpr int kTokens = kWave / LPT;
    const int wave = threadIdx.x / kWave, n_waves = blockDim.x / kWave;
#pragma unroll 1
    for (int i = wave * kTokens; i < kSub && t0 + i < p.T; i += n_waves * kTokens)
      route_scores_select<LPT, KP, GROUPS>(p, sc, t0 + i, lane_id(), s_idx + i * kMaxK, s_slots + wave * slot_words(KP));
  }
};
// The selection as route_one calls it, for as many tokens as it has waves: a wave to each.
constexpr int kFewSlotWords = slot_words(kMaxE / kWave);
template <bool GROUPS> struct SelectScoresFew {
  const ScoreParams& sc;
  double* s_slots;
  __device__ __forceinline__ void few(const RouteParams& p, int wave, int lane, int32_t* s_idx, float*) const {
    if (wave >= p.T) return;
    auto one = [&](auto kp) __attribute__((always_inline)) {
      route_scores_select<kWave, decltype(kp)::value, GROUPS>(p, sc, wave, lane, s_idx + wave * kMaxK, s_slots + wave * kFewSlotWords);
    };
    if (p.E <= 64) one(std::integral_constant<int, 1>{});
    else if (p.E <= 128) one(std::integral_constant<int, 2>{});
    else one(std::integral_constant<int, 4>{});
  }
};

// f(lanes per token, experts per lane, threads per workgroup) for E experts.
template <typename F> void with_score_lanes(int E, F&& f) {
  typedef std::integral_constant<int, 16> L16;
  typedef std::integral_constant<int, 512> W8;
  if (E <= 16) f(L16{}, std::integral_constant<int, 1>{}, W8{});
  else if (E <= 32) f(L16{}, std::integral_constant<int, 2>{}, W8{});
  else if (E <= 64) f(L16{}, std::integral_constant<int, 4>{}, W8{});
  else if (E <= 128) f(L16{}, std::integral_constant<int, 8>{}, W8{});
  else f(std::integral_constant<int, 32>{}, std::integral_constant<int, 8>{}, std::integral_constant<int, 1024>{});
}

}  // namespace moe
