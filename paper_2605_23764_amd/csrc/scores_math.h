// Scores in 64 bits, as the routing by scores and its backward take them.
#pragma once
#include "common.h"

namespace moe {

// exp(l - m) with exp(x - x) = 1 for infinities too, 0 where l = -inf
__device__ __forceinline__ double exp_below(float l, float m) { return l == m ? (l == -__builtin_huge_valf() ? 0.0 : 1.0) : exp((double)l - (double)m); }
__device__ __forceinline__ double sigmoid64(float l) { return 1.0 / (1.0 + exp(-(double)l)); }

}  // namespace moe
