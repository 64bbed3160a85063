// Host side of the 4-bit experts: the quantiser's entry point and the launches of the two products (moe_ffn_forward_w4 itself, with
// routing and Combine around them, is in moe_ffn.hip).
#include "../../include/moe_ffn.h"

#include "device_cus.h"
#include "experts_w4.h"
#include "experts_w4_launch.h"

using namespace moe;

namespace moe {

template <int RT, int NB, bool SWIGLU, bool ROUTED> static void launch(W4Params p, int E_local, hipStream_t s) {
  p.n_items = p.N / w4_columns(NB, SWIGLU);
  const unsigned grid = (unsigned)E_local * (unsigned)p.n_items + (ROUTED && SWIGLU ? 1 : 0);
  hipLaunchKernelGGL((experts_w4_kernel<RT, NB, SWIGLU, ROUTED>), dim3(grid), dim3(kW4Waves * kWave), 0, s, p);
}

int launch_experts_w4(const W4Launch& l, bool swiglu, void* stream) {
  W4Params p{};
  p.x = static_cast<const __bf16*>(l.x); p.gather = l.gather;
  p.q = static_cast<const uint8_t*>(l.q); p.scale = static_cast<const uint8_t*>(l.scale);
  p.offsets = l.offsets; p.out = l.out;
  p.K = l.K; p.N = l.N; p.cols = swiglu ? 2 * l.N : l.N;
  // 32 rows at a time where experts have more than 8 on average (T = 100, 10 of 24 experts, k = 3: 28 -> 24 us); otherwise 16, which
  // leaves room for more waves, and the few experts above read their weights again.  Items of four column blocks, whose activations
  // are fetched half as often, as long as there are two of them per CU (32 tokens, H = 7168, I = 2048, 32 of 256 experts: 117 -> 97
  // us; 64 tokens, H = 2048, I = 1408, 16 experts: 47 -> 38; but one token there 20.8 -> 22.7).
  const bool rows32 = l.rows > kW4FewRows, wide = (long)l.experts * (l.N / w4_columns(4, swiglu)) >= 2 * device_cus();
  hipStream_t s = static_cast<hipStream_t>(stream);
  auto with_blocks = [&](auto rt, auto nb, auto routed) {
    if (swiglu) launch<rt.value, nb.value, true, routed.value>(p, l.E_local, s);
    else launch<rt.value, nb.value, false, routed.value>(p, l.E_local, s);
  };
  auto with_rows = [&](auto rt, auto routed) {
    if (wide) with_blocks(rt, std::integral_constant<int, 4>{}, routed);
    else with_blocks(rt, std::integral_constant<int, 2>{}, routed);
  };
  if (l.logits) {
    p.route.logits = l.logits; p.route.topk_idx = l.topk_idx; p.route.topk_w = l.topk_w; p.route.row_of = l.row_of; p.route.tiles.meta = l.meta;
    p.route.T = l.T; p.route.E = l.E; p.route.E_local = l.E_local; p.route.expert_base = l.expert_base; p.route.k = l.k;
    with_rows(std::integral_constant<int, 1>{}, std::true_type{});
  } else if (rows32) {
    with_rows(std::integral_constant<int, 2>{}, std::false_type{});
  } else {
    with_rows(std::integral_constant<int, 1>{}, std::false_type{});
  }
  return hipGetLastError() == hipSuccess ? MOE_OK : MOE_ERR_LAUNCH;
}

int launch_tiles_w4(const void* x, const int32_t* token_of, const int32_t* offsets, void* tiles, int E_local, int K, void* stream) {
  hipLaunchKernelGGL(tiles_w4_kernel, dim3(E_local, 32), dim3(256), 0, static_cast<hipStream_t>(stream), static_cast<const __bf16*>(x),
                     token_of, offsets, static_cast<__bf16*>(tiles), K);
  return hipGetLastError() == hipSuccess ? MOE_OK : MOE_ERR_LAUNCH;
}

int launch_combine_w4(const float* y, const int32_t* row_of, const float* topk_w, void* out, int T, int H, int k, void* stream) {
  const long want = (long)T * ((H + 2047) / 2048);
  hipLaunchKernelGGL(combine_w4_kernel, dim3((unsigned)(want < (1 << 16) ? want : 1 << 16)), dim3(256), 0, static_cast<hipStream_t>(stream), y,
                     row_of, topk_w, static_cast<__bf16*>(out), T, H, k);
  return hipGetLastError() == hipSuccess ? MOE_OK : MOE_ERR_LAUNCH;
}

}  // namespace moe

extern "C" int moe_quantize_w4(int32_t E_local, int32_t K, int32_t N, int dtype, const void* d_w, void* d_q, void* d_scale,
                               void* stream) {
  if (dtype != MOE_F32 && dtype != MOE_BF16) return MOE_ERR_INVALID_ARG;
  if (E_local < 1 || E_local > kMaxE || K < 32 || K % 32 || N < 1 || K > (1 << 19) || N > (1 << 19)) return MOE_ERR_UNSUPPORTED_SHAPE;
  for (const void* p : {d_w, (const void*)d_q, (const void*)d_scale})
    if (!p || (reinterpret_cast<uintptr_t>(p) & 15)) return MOE_ERR_INVALID_ARG;
  const long blocks = (long)E_local * (K / 32) * N, want = (blocks + 255) / 256;
  const dim3 grid((unsigned)(want < (1 << 20) ? want : 1 << 20));
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (dtype == MOE_BF16)
    hipLaunchKernelGGL(quantize_w4_kernel<__bf16>, grid, dim3(256), 0, s, static_cast<const __bf16*>(d_w), static_cast<uint8_t*>(d_q),
                       static_cast<uint8_t*>(d_scale), blocks, K / 32, N);
  else
    hipLaunchKernelGGL(quantize_w4_kernel<float>, grid, dim3(256), 0, s, static_cast<const float*>(d_w), static_cast<uint8_t*>(d_q),
                       static_cast<uint8_t*>(d_scale), blocks, K / 32, N);
  return hipGetLastError() == hipSuccess ? MOE_OK : MOE_ERR_LAUNCH;
}
