// The backward of the routing by scores (router_scores.h), and the step of its balance bias.
#pragma once
#include "balance.h"
#include "scores_math.h"

namespace moe {

// Gradient of the logits.  With w' = the weights over scale (the selected scores, renormalised or not), d = sum over slots of w' dw:
//   sigmoid:              dl[j] = scale * w'[j] * (renorm ? dw[j] - d : dw[j]) * (1 - s[j]) at the selected experts
//   softmax, renormalised dl[j] = scale * w'[j] * (dw[j] - d) at the selected experts (what the sum over all E takes off is 0)
//   softmax               dl[e] = scale * s[e] * ([e selected] dw - d)
// plus dadd.  Slots in 64 bits (a lane has one, or up to four where a token has fewer than 16 lanes); the softmax over all E, whose
// result is rounded to 32 bits anyway, in 32.  Bound by dadd and dlogits (and the softmax's logits) as router_backward_kernel is: 8192 tokens of
// 256 experts, sigmoid 6.0 us, softmax 7.0 (from a graph).
struct ScoresBackwardParams {
  const float* logits;           // [T, E]
  const int32_t* topk_idx;       // [T, k]
  const float* dtopk_w;          // [T, k]
  const float* dadd;             // [T, E] or null; may be dlogits
  float* dlogits;                // [T, E]; may be logits
  int renorm;
  float scale;
  int T, E, k;
};

template <int L, bool TAIL, bool FULL> __global__ __launch_bounds__(kRouterThreads) void scores_backward_kernel(ScoresBackwardParams p) {
  // FULL: softmax, which needs the row's maximum (and, not renormalised, its sum); else sigmoid
  constexpr int kPer = kRouterThreads / L, kSlots = RouterToken<L>::kSlots;
  __shared__ float s_row[kPer][4 * L];
  const int g = threadIdx.x / L, l = threadIdx.x & (L - 1), e0 = l * 4;
  float* row = s_row[g];
  const float none = -__builtin_huge_valf();
  for (long t = (long)blockIdx.x * kPer + g; t < p.T; t += (long)gridDim.x * kPer) {
    const float* q = p.logits + (size_t)t * p.E;
    float d[4] = {0.f, 0.f, 0.f, 0.f}, x[4];
    const float* add = p.dadd ? p.dadd + (size_t)t * p.E : nullptr;
    if (!TAIL) {
      if (add && e0 < p.E) __builtin_memcpy(d, add + e0, 16);
      if (FULL) __builtin_memcpy(x, q + (e0 < p.E ? e0 : 0), 16);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (add && e0 + i < p.E) d[i] = add[e0 + i];
        if (FULL) x[i] = q[min(e0 + i, p.E - 1)];
      }
    }
    int id[kSlots];
    float dw[kSlots], lv[kSlots];
#pragma unroll
    for (int j = 0; j < kSlots; ++j) {
      const bool on = l + j * L < p.k;
      id[j] = on ? p.topk_idx[(size_t)t * p.k + l + j * L] : -1;
      dw[j] = on ? p.dtopk_w[(size_t)t * p.k + l + j * L] : 0.f;
      const bool in = (uint32_t)id[j] < (uint32_t)p.E;
      id[j] = in ? id[j] : -1;
      lv[j] = in ? q[id[j]] : none;
      if (lv[j] != lv[j]) lv[j] = none;
      if (lv[j] == none) dw[j] = 0.f;      // no part, whatever it holds: not even 0 * NaN
    }
    float m = none, sum = 0.f;
    if (FULL) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (e0 + i >= p.E || x[i] != x[i]) x[i] = none;
        m = __builtin_fmaxf(m, x[i]);
      }
      m = token_reduce<L>(m, [](float a, float b) { return __builtin_fmaxf(a, b); });
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[i] = x[i] == none ? 0.f : x[i] == m ? 1.f : expf(x[i] - m);
        sum += x[i];
      }
      sum = token_sum<L>(sum);
    }
    // the slots: selected scores (softmax: without the division by the row's sum, which is the same for all).  Where they are renormalised they
    // come times 2^500, which the division takes off again: far below zero their sum is subnormal, and its reciprocal would overflow.
    const double up = p.renorm ? 0x1p500 : 1.0;
    double ps[kSlots], total = 0.0, dot = 0.0;
#pragma unroll
    for (int j = 0; j < kSlots; ++j) {
      ps[j] = id[j] < 0 ? 0.0 : up * (FULL ? exp_below(lv[j], m) : sigmoid64(lv[j]));
      total += ps[j];
      dot += ps[j] * (double)dw[j];
    }
#pragma unroll
    for (int o = 1; o < L; o <<= 1) {
      total += __shfl_xor(total, o);
      dot += __shfl_xor(dot, o);
    }
    // w'[j] = ps[j] * norm
    const double norm = p.renorm ? (total > 0.0 ? 1.0 / total : 0.0) : !FULL ? 1.0 : (sum > 0.f ? 1.0 / (double)sum : 0.0);
    dot *= norm;                                                 // sum of w' dw
#pragma unroll
    for (int i = 0; i < 4; ++i) row[e0 + i] = 0.f;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
    for (int j = 0; j < kSlots; ++j)
      if (id[j] >= 0) {
        double v = (double)p.scale * ps[j] * norm * ((double)dw[j] - (p.renorm ? dot : 0.0));
        if (!FULL) v *= sigmoid64(-lv[j]);
        __hip_atomic_fetch_add(row + id[j], (float)v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WAVEFRONT);   // an expert may be there twice
      }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    const float off = FULL && !p.renorm ? (float)((double)p.scale * norm * dot) : 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) d[i] += FULL && !p.renorm ? row[e0 + i] - x[i] * off : row[e0 + i];
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    float* out = p.dlogits + (size_t)t * p.E;
    if (!TAIL) {
      if (e0 < p.E) __builtin_memcpy(out + e0, d, 16);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (e0 + i < p.E) out[e0 + i] = d[i];
    }
  }
}

// bias[e] += rate * sign(mean - counts[e]), decided in whole numbers: sum of counts against E counts[e].
__global__ __launch_bounds__(kMaxE) void bias_update_kernel(const int32_t* counts, int E, float rate, const float* bias, float* out) {
  __shared__ long long s_sum[kMaxE / kWave];
  const int e = threadIdx.x;
  const long long c = e < E ? counts[e] : 0;
  long long sum = c;
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) sum += __shfl_xor(sum, o);
  if (lane_id() == 0) s_sum[e / kWave] = sum;
  __syncthreads();
  sum = 0;
#pragma unroll
  for (int w = 0; w < kMaxE / kWave; ++w) sum += s_sum[w];
  if (e < E) out[e] = bias[e] + (sum > E * c ? rate : sum < E * c ? -rate : 0.f);
}

}  // namespace moe
