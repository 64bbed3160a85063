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
  int experts;                   // experts with rows, expected
  int rows;                      // of an expert, on average
  // The routed form (T up to kW4MaxRoutedT, rows up to kW4FewRows, k <= E_local): no routing launch has run, `gather` and `offsets`
  // are null; GEMM-1 leaves topk_idx, topk_w and row_of, a row is token * k + slot, activations between the two are rows, not tiles.
  const float* logits;           // null: not routed
  int32_t* topk_idx;
  float* topk_w;
  int32_t* row_of;
  int32_t* meta;                 // MetaWord, of which GEMM-1 clears the status
  int T, E, expert_base, k;
};
constexpr int kW4MaxRoutedT = 16, kW4FewRows = 8;

// swiglu: N bf16 columns from N gate and N up columns, in tiles; otherwise rows of N fp32.  Returns a MoeStatus, as the next two.
__attribute__((visibility("hidden"))) int launch_experts_w4(const W4Launch& l, bool swiglu, void* stream);

// Token rows of K in the tiles that the products read fastest.
__attribute__((visibility("hidden"))) int launch_tiles_w4(const void* x, const int32_t* token_of, const int32_t* offsets, void* tiles, int E_local,
                                                          int K, void* stream);

// Combine of fp32 rows into bf16 [T,H].
__attribute__((visibility("hidden"))) int launch_combine_w4(const float* y, const int32_t* row_of, const float* topk_w, void* out, int T, int H,
                                                            int k, void* stream);

}  // namespace moe
