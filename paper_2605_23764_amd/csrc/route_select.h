// Top-k and softmax of a token's logits (paper Section 2.2: routing): the selection itself, which the routing kernels (route.h) and the
// 4-bit experts of few tokens (experts_w4.h) share.
#pragma once
#include <type_traits>

#include "common.h"

namespace moe {

struct RouteParams {
  const float* logits;   // [T,E]
  int32_t* topk_idx;     // [T,k]
  float* topk_w;         // [T,k]
  int32_t* counts;       // [E_local]
  int32_t* offsets;      // [E_local+1]
  int32_t* row_of;       // [T,k]
  int32_t* token_of;     // [R_max]
  int32_t* slot_of;      // [R_max]
  int32_t* chunk_cnt;    // [n_sub, E_local]  histogram of every 32-token sub-chunk
  TileMap tiles;
  int T, E, E_local, expert_base, k;
  int n_sub;     // ceil(T / kSub) histogram rows
  int subs;      // sub-chunks that a rank workgroup takes
  int BM;        // M-tile row capacity of the plain wide shape
  int wide_max;  // rows a single wide M tile can take (>= BM: the bf16 kernels feed one more row block per wave row from registers)
  int tall;      // row capacity of a tall M tile (0 = the kernels have no tall shape)
  int granule;   // an expert's rows are dealt to its tiles in units of this many rows
};

// Monotone map float -> uint32 (larger float = larger key); -0.0 and NaN are
// canonicalised first (-0.0 ties with +0.0, NaN ranks as -inf).
__device__ __forceinline__ uint32_t float_order_key(float v) {
  if (v != v) v = -__builtin_huge_valf();
  if (v == 0.0f) v = 0.0f;
  uint32_t u = __builtin_bit_cast(uint32_t, v);
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}
__device__ __forceinline__ float float_from_order_key(uint32_t k) {
  uint32_t u = (k & 0x80000000u) ? (k & 0x7FFFFFFFu) : ~k;
  return __builtin_bit_cast(float, u);
}

// Reductions over the 16 lanes of a DPP row (butterfly: every lane ends up with the
// result): quad_perm [1,0,3,2] and [2,3,0,1], then the 8-lane and 16-lane mirrors.
#define MOE_DPP_ROW_STEPS(OP)  \
  OP(0xB1) OP(0x4E) OP(0x141) OP(0x140)
__device__ __forceinline__ uint32_t row_max_u32(uint32_t v) {
#define MOE_STEP(ctrl)                                                                               \
  {                                                                                                  \
    const uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, ctrl, 0xf, 0xf, false);      \
    v = o > v ? o : v;                                                                               \
  }
  MOE_DPP_ROW_STEPS(MOE_STEP)
#undef MOE_STEP
  return v;
}
__device__ __forceinline__ float row_sum_f32(float v) {
#define MOE_STEP(ctrl) v += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), ctrl, 0xf, 0xf, false));
  MOE_DPP_ROW_STEPS(MOE_STEP)
#undef MOE_STEP
  return v;
}
#undef MOE_DPP_ROW_STEPS

constexpr int kRouteTokensPerWave = 4;    // one token per 16-lane row
constexpr int kRouteKeys = kMaxE / 16;    // experts per lane, at most

// Logits of the wave's four tokens as order-preserving keys: lane s of row r holds
// experts KP s .. KP s + KP - 1 of token t_first + r (0 = absent).
template <int KP>
__device__ __forceinline__ void route_load(const RouteParams& p, int t_first, int lane, uint32_t (&key)[KP]) {
  const int t = min(t_first + (lane >> 4), p.T - 1);   // tokens past the end repeat the last one; results are not stored
  const float* row = p.logits + (size_t)t * p.E;
  const int e0 = (lane & 15) * KP;
  if (KP >= 4 && (p.E & 3) == 0) {
#pragma unroll
    for (int i = 0; i + 3 < KP; i += 4) {
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
      const bool in = e0 + i < p.E;
      if (in) v = *reinterpret_cast<const float4*>(row + e0 + i);
      key[i + 0] = in ? float_order_key(v.x) : 0u;
      key[i + 1] = in ? float_order_key(v.y) : 0u;
      key[i + 2] = in ? float_order_key(v.z) : 0u;
      key[i + 3] = in ? float_order_key(v.w) : 0u;
    }
  } else {
#pragma unroll
    for (int i = 0; i < KP; ++i) key[i] = e0 + i < p.E ? float_order_key(row[e0 + i]) : 0u;
  }
}

// Top-k of four tokens by one wave, one token per 16-lane row, so every reduction
// step serves four tokens.  Each round: a lane's best remaining key (lowest
// position among equals), the row maximum, the lowest lane of the row that holds
// it (expert ids grow with the lane, then with the position), and that lane
// retires the key and files (id, logit) as slot j in LDS.  Afterwards lane s < k of
// a row picks up slot s and the row computes the softmax over the k selected logits.
// s_idx / s_val: [4][kMaxK] words of LDS for this wave.
template <int KP>
__device__ __forceinline__ void route_select(const RouteParams& p, int t_first, int lane, uint32_t (&key)[KP],
                                             int32_t* s_idx, float* s_val) {
  const int row = lane >> 4, s = lane & 15;
  for (int j = 0; j < p.k; ++j) {
    uint32_t local = key[0];
    int li = 0;
#pragma unroll
    for (int i = 1; i < KP; ++i)
      if (key[i] > local) { local = key[i]; li = i; }
    const uint32_t best = row_max_u32(local);
    const uint64_t bal = __ballot(local == best);
    const uint32_t in_row = (uint32_t)(bal >> (row * 16)) & 0xFFFFu;
    const bool winner = s == __builtin_ctz(in_row);   // in_row != 0: the row maximum is some lane's local maximum
#pragma unroll
    for (int i = 0; i < KP; ++i)
      if (winner && i == li) key[i] = 0u;
    if (winner) {
      s_idx[row * kMaxK + j] = s * KP + li;
      s_val[row * kMaxK + j] = float_from_order_key(best);
    }
  }
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  // softmax over the k selected logits; slot 0 holds the maximum
  const int t = t_first + row;
  const bool slot = s < p.k;
  const float val = slot ? s_val[row * kMaxK + s] : 0.f;
  const int idx = slot ? s_idx[row * kMaxK + s] : 0;
  const float m = s_val[row * kMaxK];
  const float pj = slot ? expf(val - m) : 0.f;
  const float sum = row_sum_f32(pj);
  if (t < p.T && slot) {
    p.topk_idx[(size_t)t * p.k + s] = idx;
    p.topk_w[(size_t)t * p.k + s] = pj / sum;
  }
}

// f(number of experts per lane) for E experts: the least of 1, 2, 4, 8, 16 that holds them.  A round of the selection walks a
// lane's experts, so with 16 to a lane for any E its cost was that of 256 experts
// (16 experts, T = 65..256: a layer of H = 2048 66.8 -> 64.4 us, 80 -> 77.7; a training step of T = 777, 24 experts 114.9 -> 112.2).
template <typename F>
__device__ __forceinline__ void with_route_keys(int E, F&& f) {
  static_assert(kRouteKeys == 16, "cases");
  if (E <= 16) f(std::integral_constant<int, 1>{});
  else if (E <= 32) f(std::integral_constant<int, 2>{});
  else if (E <= 64) f(std::integral_constant<int, 4>{});
  else if (E <= 128) f(std::integral_constant<int, 8>{});
  else f(std::integral_constant<int, 16>{});
}

}  // namespace moe
