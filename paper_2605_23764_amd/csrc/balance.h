// The router's balance loss with per-expert counts, and the gradient of the logits.
//
//   p[t,:] = softmax over all E logits of token t;  over the n tokens that the mask leaves:
//   c_e = selections of expert e, f_e = c_e / (k n), P_e = sum_t p[t,e] / n;   loss = coef * E * sum_e f_e P_e
//   dlogits[t,e] = dloss * coef * E / n * p[t,e] * (f_e - sum_e' f_e' p[t,e'])          (tokens of the mask)
//                + [e = topk_idx[t,j]] w[t,j] * (dw[t,j] - sum_i w[t,i] dw[t,i])        (softmax over the k selected logits)
// The counts carry no gradient.  A row without a finite logit (all -inf) has p = 0.
//
// Bound by the logits: read once forward, read and written once backward (the softmax is made again: four logits per lane, no trip
// through memory for p).  At the sizes of a router (T = 8192, E = 256: 8 MB) that is 1.5 us of HBM, so latency decides: a token takes
// the fewest lanes that hold it (a power of two, so a wave has 1 .. 64 tokens in hand), everything that kBalAhead tokens need is
// requested before the first of them is worked on, and the lanes per token are a template parameter.  Sums over tokens are kept in
// registers along a workgroup's strided tokens, then joined in a fixed order: over the wave, over the workgroup, over the workgroups
// (second launch); one workgroup does few tokens alone, in one launch.  T = 8192, E = 256: 7.0 us, the join 5.1, the backward 7.4.
#pragma once
#include "rows.h"

namespace moe {

constexpr int kBalThreads = 1024;
constexpr int kBalMaxParts = 128;          // workgroups of the first launch, at most: what one workgroup joins afterwards (T = 8192: 64 +2 us, 256 +3)
constexpr int kBalAhead = 4;               // tokens per group of lanes under way together (2: +0.5 us)
// Tokens x lanes that one workgroup does alone, in one launch: two turns (E = 256: T = 128 11.3 -> 9.9 us, E = 64: T = 512 10.6 -> 9.2; with
// four turns T = 256 11.2 -> 17.6).
constexpr int kBalOneLanes = 2 * kBalAhead * kBalThreads;
constexpr int kRouterThreads = 256;        // the backward's
constexpr int kRouterAhead = 2;            // (1: +0.5 us)

struct BalanceParams {
  const float* logits;           // [T, E]
  const int32_t* topk_idx;       // [T, k]
  const uint8_t* mask;           // [T], null: every token counts
  int32_t* counts;               // [E + 1]: selections per expert, tokens that count
  float* prob_sum;               // [E]
  float* loss;                   // [1]
  u32x2* part;                   // [parts][kMaxE + 1] {sum of probabilities, selections}; behind them {-, tokens}
  float coef;
  int T, E, k, parts;
};

struct RouterBackwardParams {
  const float* logits;
  const int32_t* topk_idx;
  const float *topk_w, *dtopk_w; // null (both): no gradient by way of the routing weights
  const uint8_t* mask;
  const int32_t* counts;         // [E + 1], null: no balance loss
  const float* dloss;            // [1], null: 1
  float* dlogits;
  float coef;
  int T, E, k;
};

// Over the L lanes of a token, in all of them.
template <int L, typename OP> __device__ __forceinline__ float token_reduce(float v, OP op) {
#define MOE_STEP(ctrl) v = op(v, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), ctrl, 0xf, 0xf, false)))
  if constexpr (L >= 2) MOE_STEP(0xB1);
  if constexpr (L >= 4) MOE_STEP(0x4E);
  if constexpr (L >= 8) MOE_STEP(0x141);
  if constexpr (L >= 16) MOE_STEP(0x140);
#undef MOE_STEP
  if constexpr (L >= 32) {
    const auto r = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, v), __builtin_bit_cast(uint32_t, v), false, false);
    v = op(__builtin_bit_cast(float, (uint32_t)r[0]), __builtin_bit_cast(float, (uint32_t)r[1]));
  }
  if constexpr (L >= 64) {
    const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, v), __builtin_bit_cast(uint32_t, v), false, false);
    v = op(__builtin_bit_cast(float, (uint32_t)r[0]), __builtin_bit_cast(float, (uint32_t)r[1]));
  }
  return v;
}
template <int L> __device__ __forceinline__ float token_sum(float v) { return token_reduce<L>(v, [](float a, float b) { return a + b; }); }
// What a lane has of a token: four logits, and the slots l, l + L, ... (k <= E <= 4 L: four at most, one if a token has 16 lanes).
// Everything is requested at addresses that are there, whatever the lane needs of it, so that nothing waits before the first use.
template <int L> struct RouterToken {
  static constexpr int kSlots = L >= kMaxK ? 1 : 4;
  float q[4];
  int id[kSlots];
  float w[kSlots], dw[kSlots];
  uint8_t mask;
};

// TAIL: E % 4 != 0.  WEIGHTS: with the routing weights and their gradient.
template <int L, bool TAIL, bool WEIGHTS, typename P>
__device__ __forceinline__ void token_request(RouterToken<L>& x, const P& p, long t, int l) {
  t = min(t, (long)p.T - 1);
  x.mask = (p.mask ? p.mask : reinterpret_cast<const uint8_t*>(p.topk_idx))[t];   // without a mask: some byte, not looked at
  const float* row = p.logits + (size_t)t * p.E;
  if (!TAIL) {
    __builtin_memcpy(x.q, row + (l * 4 < p.E ? l * 4 : 0), 16);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) x.q[i] = row[min(l * 4 + i, p.E - 1)];
  }
#pragma unroll
  for (int j = 0; j < RouterToken<L>::kSlots; ++j) {
    const size_t at = (size_t)t * p.k + min(l + j * L, p.k - 1);
    x.id[j] = p.topk_idx[at];
    if constexpr (WEIGHTS) {
      x.w[j] = p.topk_w[at];
      x.dw[j] = p.dtopk_w[at];
    }
  }
}
// Whether slot j of the lane is one, with an expert.
template <int L> __device__ __forceinline__ bool token_slot(const RouterToken<L>& x, int j, int l, int E, int k) {
  return l + j * L < k && (uint32_t)x.id[j] < (uint32_t)E;
}

// Logits to probabilities (0 past E, and in rows without a finite logit; a NaN makes all of its row NaN).
template <int L, bool TAIL> __device__ __forceinline__ void token_softmax(float (&q)[4], int e0, int E) {
  const float none = -__builtin_huge_valf();
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (e0 + (TAIL ? i : 0) >= E) q[i] = none;
  float m = __builtin_fmaxf(__builtin_fmaxf(q[0], q[1]), __builtin_fmaxf(q[2], q[3]));   // passes over NaN
  m = token_reduce<L>(m, [](float a, float b) { return __builtin_fmaxf(a, b); });
  m = m == none ? 0.f : m;                                       // exp(-inf - 0) = 0
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    q[i] = expf(q[i] - m);
    s += q[i];
  }
  s = token_sum<L>(s);
  const float inv = s == 0.f ? 0.f : 1.0f / s;
#pragma unroll
  for (int i = 0; i < 4; ++i) q[i] *= inv;
}

// counts, prob_sum and the loss from the sums; e: this thread's expert.  s: a word per wave.
__device__ __forceinline__ void balance_finish(const BalanceParams& p, int e, int c, float prob, int n, float* s) {
  float part = 0.f;
  if (e < p.E) {
    p.counts[e] = c;
    p.prob_sum[e] = prob;
    part = (float)c * prob;
  }
  if (e < kMaxE) {                                               // whole waves: the experts are the first threads'
    part = token_sum<kWave>(part);
    if (lane_id() == 0) s[threadIdx.x / kWave] = part;
  }
  __syncthreads();
  if (e == 0) {
    float sum = 0.f;
    for (int w = 0; w < kMaxE / kWave; ++w) sum += s[w];
    p.counts[p.E] = n;
    // coef E sum_e (c_e / (k n)) (prob_e / n); no tokens: no loss
    p.loss[0] = n > 0 ? p.coef * (float)p.E * (sum / ((float)p.k * (float)n * (float)n)) : 0.f;
  }
}

template <int L, bool TAIL> __global__ __launch_bounds__(kBalThreads) void balance_kernel(BalanceParams p) {
  constexpr int kWaves = kBalThreads / kWave, kPer = kBalThreads / L;
  __shared__ int s_n[kMaxE + 1];
  __shared__ float s_p[kWaves][4 * L];
  __shared__ float s_w[kWaves];
  const int g = threadIdx.x / L, l = threadIdx.x & (L - 1);
  if (threadIdx.x <= kMaxE) s_n[threadIdx.x] = 0;
  __syncthreads();
  float acc[4] = {0.f, 0.f, 0.f, 0.f};
  const long step = (long)gridDim.x * kPer;
  for (long t = (long)blockIdx.x * kPer + g; t < p.T; t += kBalAhead * step) {
    RouterToken<L> x[kBalAhead];
#pragma unroll
    for (int u = 0; u < kBalAhead; ++u) token_request<L, TAIL, false>(x[u], p, t + u * step, l);
#pragma unroll
    for (int u = 0; u < kBalAhead; ++u) {
      token_softmax<L, TAIL>(x[u].q, l * 4, p.E);
      if (t + u * step >= p.T || (p.mask && x[u].mask == 0)) continue;       // all lanes of a token together
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[i] += x[u].q[i];
#pragma unroll
      for (int j = 0; j < RouterToken<L>::kSlots; ++j)
        if (token_slot<L>(x[u], j, l, p.E, p.k)) atomicAdd(&s_n[x[u].id[j]], 1);   // whole numbers: no order to keep
      if (l == 0) atomicAdd(&s_n[kMaxE], 1);
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
#pragma unroll
    for (int o = L; o < kWave; o <<= 1) acc[i] += __shfl_xor(acc[i], o);
    if (lane_id() < L) s_p[threadIdx.x / kWave][l * 4 + i] = acc[i];
  }
  __syncthreads();
  const int e = threadIdx.x;
  float prob = 0.f;
  if (e < p.E)
#pragma unroll
    for (int w = 0; w < kWaves; ++w) prob += s_p[w][e];
  if (gridDim.x == 1) {
    balance_finish(p, e, e < p.E ? s_n[e] : 0, prob, s_n[kMaxE], s_w);
    return;
  }
  if (e < p.E || e == kMaxE) p.part[(size_t)blockIdx.x * (kMaxE + 1) + e] = u32x2{__builtin_bit_cast(uint32_t, prob), (uint32_t)s_n[e]};
}

// Joins the workgroups' sums: every fourth of them per 256 threads, all requested together.
__global__ __launch_bounds__(1024) void balance_join_kernel(BalanceParams p) {
  __shared__ float s_p[4][kMaxE], s_w[16];
  __shared__ int s_n[4][kMaxE];
  const int e = threadIdx.x & (kMaxE - 1), quarter = threadIdx.x / kMaxE;
  int n = 0;                                                     // the first wave counts the tokens
  if (threadIdx.x < kWave)
    for (int i = threadIdx.x; i < p.parts; i += kWave) n += (int)p.part[(size_t)i * (kMaxE + 1) + kMaxE][1];
  float prob = 0.f;
  int c = 0;
  if (e < p.E) {
    u32x2 v[kBalMaxParts / 4];
#pragma unroll
    for (int i = 0; i < kBalMaxParts / 4; ++i) v[i] = p.part[(size_t)min(quarter + 4 * i, p.parts - 1) * (kMaxE + 1) + e];
#pragma unroll
    for (int i = 0; i < kBalMaxParts / 4; ++i) {
      const bool there = quarter + 4 * i < p.parts;
      prob += there ? __builtin_bit_cast(float, v[i][0]) : 0.f;
      c += there ? (int)v[i][1] : 0;
    }
  }
  s_p[quarter][e] = prob;
  s_n[quarter][e] = c;
  for (int o = 1; o < kWave; o <<= 1) n += __shfl_xor(n, o);
  __syncthreads();
  float pt = 0.f;
  int ct = 0;
  if (quarter == 0)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      pt += s_p[i][e];
      ct += s_n[i][e];
    }
  balance_finish(p, quarter == 0 ? e : kMaxE, ct, pt, n, s_w);
}

template <int L, bool TAIL, bool WEIGHTS> __global__ __launch_bounds__(kRouterThreads) void router_backward_kernel(RouterBackwardParams p) {
  constexpr int kWaves = kRouterThreads / kWave, kPer = kRouterThreads / L;
  __shared__ float s_row[WEIGHTS ? kWaves : 1][kMaxE];           // the rows of a wave's tokens: 64 / L rows of 4 L
  const int g = threadIdx.x / L, l = threadIdx.x & (L - 1), e0 = l * 4;
  float* row = s_row[WEIGHTS ? threadIdx.x / kWave : 0] + (lane_id() / L) * (4 * L);
  float f[4] = {0.f, 0.f, 0.f, 0.f}, c = 0.f;
  int cnt[4] = {0, 0, 0, 0}, tokens = 0;
  float dloss = 1.f;
  if (p.counts) {
    tokens = p.counts[p.E];
#pragma unroll
    for (int i = 0; i < 4; ++i) cnt[i] = p.counts[min(e0 + i, p.E)];
    if (p.dloss) dloss = p.dloss[0];
  }
  const long step = (long)gridDim.x * kPer;
  bool first = true;
  for (long t = (long)blockIdx.x * kPer + g; t < p.T; t += kRouterAhead * step) {
    RouterToken<L> x[kRouterAhead];
#pragma unroll
    for (int u = 0; u < kRouterAhead; ++u) token_request<L, TAIL, WEIGHTS>(x[u], p, t + u * step, l);
    if (first) {                                                 // behind the first tokens' requests
      first = false;
      if (tokens > 0) {
        c = p.coef * (float)p.E / (float)tokens * dloss;
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = (float)cnt[i] / ((float)p.k * (float)tokens);
      }
    }
#pragma unroll
    for (int u = 0; u < kRouterAhead; ++u) {
      if (t + u * step >= p.T) break;
      float d[4];
      token_softmax<L, TAIL>(x[u].q, e0, p.E);
      float fp = 0.f;
#pragma unroll
      for (int i = 0; i < 4; ++i) fp += f[i] * x[u].q[i];
      fp = token_sum<L>(fp);
#pragma unroll
      for (int i = 0; i < 4; ++i) d[i] = p.counts && (!p.mask || x[u].mask) ? c * x[u].q[i] * (f[i] - fp) : 0.f;
      if constexpr (WEIGHTS) {
        // the slots' shares go to their experts' lanes through LDS (one wave's own, in order)
        constexpr int kSlots = RouterToken<L>::kSlots;
        float dot = 0.f;
#pragma unroll
        for (int j = 0; j < kSlots; ++j) dot += l + j * L < p.k ? x[u].w[j] * x[u].dw[j] : 0.f;
        dot = token_sum<L>(dot);
#pragma unroll
        for (int i = 0; i < 4; ++i) row[e0 + i] = 0.f;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
        for (int j = 0; j < kSlots; ++j)
          if (token_slot<L>(x[u], j, l, p.E, p.k)) row[x[u].id[j]] = x[u].w[j] * (x[u].dw[j] - dot);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
        for (int i = 0; i < 4; ++i) d[i] += row[e0 + i];
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      }
      float* out = p.dlogits + (size_t)(t + u * step) * p.E;
      if (!TAIL) {
        if (e0 < p.E) __builtin_memcpy(out + e0, d, 16);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (e0 + i < p.E) out[e0 + i] = d[i];
      }
    }
  }
}

}  // namespace moe
