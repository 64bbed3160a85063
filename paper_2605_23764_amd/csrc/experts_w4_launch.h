// The grouped products with 4-bit weights (experts_w4.hip) as moe_ffn.hip launches them.
#pragma once
#include <stdint.h>

namespace moe {

struct W4Launch {
  const void* x;
  const int32_t* gather;         // token of each row; null: x holds the rows in tiles
  const void *q, *scale;
  const int32_t* offsets;
  void* out;
  int E_local, K, N;
  int experts;                   // experts with rows, at most
  int rows;                      // of an expert, on average
};

// swiglu: N bf16 columns from N gate and N up columns, in tiles; otherwise rows of N fp32.  Returns a MoeStatus, as the next two.
__attribute__((visibility("hidden"))) int launch_experts_w4(const W4Launch& l, bool swiglu, void* stream);

// Token rows of K in the tiles that the products read fastest.
__attribute__((visibility("hidden"))) int launch_tiles_w4(const void* x, const int32_t* token_of, const int32_t* offsets, void* tiles, int E_local,
                                                          int K, void* stream);

// Combine of fp32 rows into bf16 [T,H].
__attribute__((visibility("hidden"))) int launch_combine_w4(const float* y, const int32_t* row_of, const float* topk_w, void* out, int T, int H,
                                                            int k, void* stream);

}  // namespace moe
