// Host side of the 4-bit experts: the quantiser's entry point and the launches of the two products (moe_ffn_forward_w4 itself, with
// routing and Combine around them, is in moe_ffn.hip).
#include "../../include/moe_ffn.h"

#include "experts_w4.h"
#include "experts_w4_launch.h"

using namespace moe;

namespace moe {

int launch_experts_w4(const W4Launch& l, bool swiglu, void* stream) {
  W4Params p{};
  p.x = static_cast<const __bf16*>(l.x); p.gather = l.gather;
  p.q = static_cast<const uint8_t*>(l.q); p.scale = static_cast<const uint8_t*>(l.scale);
  p.offsets = l.offsets; p.out = l.out;
  p.K = l.K; p.N = l.N; p.cols = swiglu ? 2 * l.N : l.N; p.n_items = swiglu ? l.N / 16 : l.N / 32;
  const dim3 grid((unsigned)l.E_local * (unsigned)p.n_items), block(kW4Waves * kWave);
  if (swiglu) hipLaunchKernelGGL(experts_w4_kernel<true>, grid, block, 0, static_cast<hipStream_t>(stream), p);
  else hipLaunchKernelGGL(experts_w4_kernel<false>, grid, block, 0, static_cast<hipStream_t>(stream), p);
  return hipGetLastError() == hipSuccess ? MOE_OK : MOE_ERR_LAUNCH;
}

int launch_combine_w4(const float* y, const int32_t* row_of, const float* topk_w, void* out, int T, int H, int k, void* stream) {
  const long want = ((long)T * (H / 8) + 255) / 256;
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
