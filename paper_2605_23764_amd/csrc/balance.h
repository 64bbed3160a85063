// The router's balance loss with per-expert counts, and the gradient of the logits.
//
//   p[t,:] = softmax over all E logits of token t;  over the n tokens that the mask leaves:
//   c_e = selections of expert e, f_e = c_e / (k n), P_e = sum_t p[t,e] / n;   loss = coef * E * sum_e f_e P_e
//   dlogits[t,e] = dloss * coef * E / n * p[t,e] * (f_e - sum_e' f_e' p[t,e'])          (tokens of the mask)
//                + [e = topk_idx[t,j]] w[t,j] * (dw[t,j] - sum_i w[t,i] dw[t,i])        (softmax over the k selected logits)
// The counts carry no gradient.  A row without a finite logit (all -inf) has p = 0.
//
// Bound by the logits: read once forward, read and written once backward (the softmax is made again: four logits per lane, no trip
// through memory for p).  A token takes the fewest lanes that hold it (power of two), so a wave has 1 .. 64 tokens in hand.  Sums over
// tokens are kept in registers along a workgroup's strided tokens, then joined in a fixed order: over the wave, over the
// workgroup, over the workgroups (second launch); one workgroup does few tokens alone, in one launch.
#pragma once
#include "rows.h"

namespace moe {

constexpr int kBalThreads = 512;
constexpr int kBalMaxParts = 128;          // workgroups of the first launch, at most
constexpr int kBalOneT = 64;               // tokens that one workgroup does alone

struct BalanceParams {
  const float* logits;           // [T, E]
  const int32_t* topk_idx;       // [T, k]
  const uint8_t* mask;           // [T], null: every token counts
  int32_t* counts;               // [E + 1]: selections per expert, tokens that count
  float* prob_sum;               // [E]
  float* loss;                   // [1]
  int32_t* part_n;               // [parts][kMaxE + 1]
  float* part_p;                 // [parts][kMaxE]
  float coef;
  int T, E, k, lanes, parts;
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
  int T, E, k, lanes;
};

// Lanes per token: four logits each.
template <typename OP> __device__ __forceinline__ float token_reduce(float v, int L, OP op) {
#define MOE_STEP(ctrl) v = op(v, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), ctrl, 0xf, 0xf, false)))
  if (L >= 2) MOE_STEP(0xB1);
  if (L >= 4) MOE_STEP(0x4E);
  if (L >= 8) MOE_STEP(0x141);
  if (L >= 16) MOE_STEP(0x140);
#undef MOE_STEP
  if (L >= 32) {
    const auto r = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, v), __builtin_bit_cast(uint32_t, v), false, false);
    v = op(__builtin_bit_cast(float, (uint32_t)r[0]), __builtin_bit_cast(float, (uint32_t)r[1]));
  }
  if (L >= 64) {
    const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, v), __builtin_bit_cast(uint32_t, v), false, false);
    v = op(__builtin_bit_cast(float, (uint32_t)r[0]), __builtin_bit_cast(float, (uint32_t)r[1]));
  }
  return v;
}
__device__ __forceinline__ float token_sum(float v, int L) { return token_reduce(v, L, [](float a, float b) { return a + b; }); }
// a NaN on either side stays
__device__ __forceinline__ float token_max(float v, int L) {
  return token_reduce(v, L, [](float a, float b) { return a != a || a > b ? a : b; });
}

// Softmax of the logits e0 .. e0 + 3 of this lane (0 past E, and in rows without a finite logit).
__device__ __forceinline__ void token_softmax(const float* row, int e0, int E, int L, float (&q)[4]) {
  const float none = -__builtin_huge_valf();
  if (e0 + 4 <= E) {
    __builtin_memcpy(q, row + e0, 16);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) q[i] = e0 + i < E ? row[e0 + i] : none;
  }
  float m = q[0];
#pragma unroll
  for (int i = 1; i < 4; ++i) m = m != m || m > q[i] ? m : q[i];
  m = token_max(m, L);
  const bool empty = m == none;
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    q[i] = empty ? 0.f : expf(q[i] - m);
    s += q[i];
  }
  s = token_sum(s, L);
  const float inv = empty ? 0.f : 1.0f / s;
#pragma unroll
  for (int i = 0; i < 4; ++i) q[i] *= inv;
}

// Sum of v over the workgroup's threads, in all of them.
__device__ __forceinline__ float workgroup_sum(float v, float* s) {
  v = token_sum(v, kWave);
  if (lane_id() == 0) s[threadIdx.x / kWave] = v;
  __syncthreads();
  float t = 0.f;
  for (int w = 0; w < (int)blockDim.x / kWave; ++w) t += s[w];
  return t;
}

// counts, prob_sum and the loss from the sums; e = threadIdx.x.  s: a word per wave.
__device__ __forceinline__ void balance_finish(const BalanceParams& p, int e, int c, float prob, int n, float* s) {
  float part = 0.f;
  if (e < p.E) {
    p.counts[e] = c;
    p.prob_sum[e] = prob;
    part = (float)c * prob;
  }
  const float sum = workgroup_sum(part, s);
  if (e == 0) {
    p.counts[p.E] = n;
    // coef E sum_e (c_e / (k n)) (prob_e / n); no tokens: no loss
    p.loss[0] = n > 0 ? p.coef * (float)p.E * (sum / ((float)p.k * (float)n * (float)n)) : 0.f;
  }
}

__global__ __launch_bounds__(kBalThreads) void balance_kernel(BalanceParams p) {
  constexpr int kWaves = kBalThreads / kWave;
  __shared__ int s_n[kMaxE + 1];
  __shared__ float s_p[kWaves][kMaxE];
  __shared__ float s_w[kWaves];
  const int L = p.lanes, per = kBalThreads / L;
  const int g = threadIdx.x / L, l = threadIdx.x & (L - 1), e0 = l * 4;
  for (int i = threadIdx.x; i <= kMaxE; i += kBalThreads) s_n[i] = 0;
  __syncthreads();
  float acc[4] = {0.f, 0.f, 0.f, 0.f};
  const long first = (long)blockIdx.x * per, step = (long)gridDim.x * per;
  for (long t = first + g; t < p.T; t += step) {
    if (p.mask && p.mask[t] == 0) continue;                      // all lanes of a token together
    float q[4];
    token_softmax(p.logits + (size_t)t * p.E, e0, p.E, L, q);
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[i] += q[i];
    for (int j = l; j < p.k; j += L) {
      const int id = p.topk_idx[(size_t)t * p.k + j];
      if (id >= 0 && id < p.E) atomicAdd(&s_n[id], 1);           // whole numbers: no order to keep
    }
    if (l == 0) atomicAdd(&s_n[kMaxE], 1);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    for (int o = L; o < kWave; o <<= 1) acc[i] += __shfl_xor(acc[i], o);
    if (lane_id() < L && e0 + i < kMaxE) s_p[threadIdx.x / kWave][e0 + i] = acc[i];
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
  if (e < p.E) {
    p.part_p[(size_t)blockIdx.x * kMaxE + e] = prob;
    p.part_n[(size_t)blockIdx.x * (kMaxE + 1) + e] = s_n[e];
  }
  if (e == kMaxE) p.part_n[(size_t)blockIdx.x * (kMaxE + 1) + kMaxE] = s_n[kMaxE];
}

// Joins the workgroups' sums: a quarter of them per 256 threads.
__global__ __launch_bounds__(1024) void balance_join_kernel(BalanceParams p) {
  __shared__ float s_p[4][kMaxE];
  __shared__ int s_n[4][kMaxE], s_tok[4];
  __shared__ float s_w[16];
  const int e = threadIdx.x & (kMaxE - 1), quarter = threadIdx.x / kMaxE;
  float prob = 0.f;
  int c = 0, n = 0;
  if (e < p.E) {
#pragma unroll 8
    for (int i = quarter; i < p.parts; i += 4) {
      prob += p.part_p[(size_t)i * kMaxE + e];
      c += p.part_n[(size_t)i * (kMaxE + 1) + e];
    }
  }
  if (e == 0) {
    for (int i = quarter; i < p.parts; i += 4) n += p.part_n[(size_t)i * (kMaxE + 1) + kMaxE];
    s_tok[quarter] = n;
  }
  s_p[quarter][e] = prob;
  s_n[quarter][e] = c;
  __syncthreads();
  const bool mine = quarter == 0 && e < p.E;
  float pt = 0.f;
  int ct = 0;
  if (mine)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      pt += s_p[i][e];
      ct += s_n[i][e];
    }
  balance_finish(p, quarter == 0 ? e : kMaxE + (int)threadIdx.x, ct, pt, s_tok[0] + s_tok[1] + s_tok[2] + s_tok[3], s_w);
}

__global__ __launch_bounds__(kBalThreads) void router_backward_kernel(RouterBackwardParams p) {
  constexpr int kWaves = kBalThreads / kWave;
  __shared__ float s_row[kWaves][kMaxE];                         // the rows of a wave's tokens: 64 / L rows of 4 L
  const int L = p.lanes, per = kBalThreads / L;
  const int g = threadIdx.x / L, l = threadIdx.x & (L - 1), e0 = l * 4;
  float* row = s_row[threadIdx.x / kWave] + (lane_id() / L) * (4 * L);
  float f[4] = {0.f, 0.f, 0.f, 0.f}, c = 0.f;
  if (p.counts) {
    const float n = (float)p.counts[p.E];
    if (n > 0.f) {
      c = p.coef * (float)p.E / n * (p.dloss ? p.dloss[0] : 1.f);
#pragma unroll
      for (int i = 0; i < 4; ++i) f[i] = e0 + i < p.E ? (float)p.counts[e0 + i] / ((float)p.k * n) : 0.f;
    }
  }
  const long first = (long)blockIdx.x * per, step = (long)gridDim.x * per;
  for (long t = first + g; t < p.T; t += step) {
    float d[4] = {0.f, 0.f, 0.f, 0.f};
    if (p.counts && (!p.mask || p.mask[t] != 0)) {
      float q[4];
      token_softmax(p.logits + (size_t)t * p.E, e0, p.E, L, q);
      float fp = 0.f;
#pragma unroll
      for (int i = 0; i < 4; ++i) fp += f[i] * q[i];
      fp = token_sum(fp, L);
#pragma unroll
      for (int i = 0; i < 4; ++i) d[i] = c * q[i] * (f[i] - fp);
    }
    if (p.topk_w) {
      // lane l has the slots l, l + L, ...; their shares go to their experts' lanes through LDS (one wave's own, in order)
      float dot = 0.f;
      for (int j = l; j < p.k; j += L) dot += p.topk_w[(size_t)t * p.k + j] * p.dtopk_w[(size_t)t * p.k + j];
      dot = token_sum(dot, L);
#pragma unroll
      for (int i = 0; i < 4; ++i) row[e0 + i] = 0.f;
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      for (int j = l; j < p.k; j += L) {
        const int id = p.topk_idx[(size_t)t * p.k + j];
        if (id >= 0 && id < p.E) row[id] = p.topk_w[(size_t)t * p.k + j] * (p.dtopk_w[(size_t)t * p.k + j] - dot);
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
      for (int i = 0; i < 4; ++i) d[i] += row[e0 + i];
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
    float* out = p.dlogits + (size_t)t * p.E;
    if (e0 + 4 <= p.E) {
      __builtin_memcpy(out + e0, d, 16);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (e0 + i < p.E) out[e0 + i] = d[i];
    }
  }
}

}  // namespace moe
