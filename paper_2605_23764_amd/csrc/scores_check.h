// Arguments of the routing by scores, checked alike by its entry points.
#pragma once
#include <cmath>

#include "../../include/moe_ffn.h"

namespace moe {

// k: experts per token
inline int check_scores(const MoeScores* s, int E, int k) {
  if (!s || (s->score != MOE_SCORE_SOFTMAX && s->score != MOE_SCORE_SIGMOID) || (s->renormalize != 0 && s->renormalize != 1) ||
      !std::isfinite(s->scale))
    return MOE_ERR_INVALID_ARG;
  if (s->n_group < 1 || s->n_group > 16 || E % s->n_group || s->topk_group < 1 || s->topk_group > s->n_group ||
      k > s->topk_group * (E / s->n_group))
    return MOE_ERR_UNSUPPORTED_SHAPE;
  return MOE_OK;
}

}  // namespace moe
