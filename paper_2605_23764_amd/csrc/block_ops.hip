// Host side of the operators around the layer (include/moe_ffn.h): layer norm, dropout with residual, balance loss, the router's
// backward and that of the routing by scores with its bias.  Argument checks and launches on the caller's stream; nothing here allocates or synchronises.
#include "../../include/moe_ffn.h"

#include <math.h>

#include <algorithm>

#include "balance.h"
#include "device_cus.h"
#include "layer_norm.h"
#include "scores_backward.h"
#include "scores_check.h"

using namespace moe;

namespace {

bool aligned(const void* p, uintptr_t n = 16) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
// present and aligned
bool good(const void* p) { return p && aligned(p); }
int launched() { return hipGetLastError() == hipSuccess ? MOE_OK : MOE_ERR_LAUNCH; }
int ceil_div(long a, long b) { return (int)((a + b - 1) / b); }

int check_rows(int T, int H, int dtype) {
  if (dtype != MOE_F32 && dtype != MOE_BF16) return MOE_ERR_INVALID_ARG;
  if (T < 0 || H < 1 || H > (1 << 18)) return MOE_ERR_UNSUPPORTED_SHAPE;
  return MOE_OK;
}

// p: the nearest multiple of 2^-16
int check_drop(float p, const uint64_t* rng, DropParams& d) {
  if (!(p >= 0.f && p <= 1.f)) return MOE_ERR_INVALID_ARG;
  d.thr = (uint32_t)lrint((double)p * 65536.0);
  d.scale = d.thr < 65536 ? (float)(65536.0 / (65536.0 - d.thr)) : 0.f;
  d.rng = rng;
  if (d.thr && !(rng && aligned(rng, 8))) return MOE_ERR_INVALID_ARG;
  return MOE_OK;
}

// Lanes per row: as many as its vectors, up to a wave in powers of two from 8, beyond in whole waves.
int row_group(int H) {
  const int vecs = ceil_div(H, 8);
  if (vecs > kWave) return ceil_div(vecs, kWave) * kWave;
  int g = 8;
  while (g < vecs) g *= 2;
  return g;
}

// Workgroups of a launch that could have one per row: a launch holds 2^32 work-items at most, so the kernels walk on in strides.
unsigned row_grid(long want) { return (unsigned)(want < (1 << 20) ? want : 1 << 20); }

// dtype x short last vector
template <typename F> void with_row_form(int dtype, int H, F&& f) {
  auto tail = [&](auto t) {
    if (H % 8) f(t, std::true_type{});
    else f(t, std::false_type{});
  };
  if (dtype == MOE_BF16) tail(__bf16{});
  else tail(float{});
}

// Arrays that are read or written once: by way of the caches or not.
template <typename T, typename F> void with_caching(int rows, int H, F&& f) {
  if ((size_t)rows * H * sizeof(T) > kNormNtBytes) f(std::true_type{});
  else f(std::false_type{});
}

// One vector per lane up to a wave's worth, two beyond.  A launch has the workgroups that run at a time (about 21 waves per CU by their
// registers; 7, 14 and 28 waves of them: within 0.3 % of each other), which walk on in strides.
template <bool FUSED> int run_norm_forward(NormForwardParams p, int dtype, hipStream_t s) {
  with_row_form(dtype, p.H, [&](auto t, auto tail) {
    using T = decltype(t);
    const int vecs = ceil_div(p.H, 8);
    if (p.H > kRowMaxH) {
      hipLaunchKernelGGL((norm_forward_long_kernel<T, tail.value, FUSED>), dim3(row_grid(p.T)), dim3(1024), 0, s, p);
      return;
    }
    p.group = vecs <= kWave ? row_group(p.H) : ceil_div(vecs, 2 * kWave) * kWave;
    const int rows = p.group > kWave ? 1 : 256 / p.group, threads = p.group * rows;
    const int most = device_cus() * (1536 / threads), want = ceil_div(p.T, rows);   // up to 512 threads
    const dim3 grid(want < most ? want : most);
    with_caching<T>(p.T, p.H, [&](auto nt) {
      if (vecs <= kWave) hipLaunchKernelGGL((norm_forward_kernel<T, 1, tail.value, FUSED, nt.value>), grid, dim3(threads), 0, s, p);
      else hipLaunchKernelGGL((norm_forward_kernel<T, 2, tail.value, FUSED, nt.value>), grid, dim3(threads), 0, s, p);
    });
  });
  return launched();
}

int norm_parts(int T) { return T < kNormMaxParts ? T : kNormMaxParts; }

// Whether arrays of n bytes share any.
bool overlap(const void* a, const void* b, size_t n) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x < y + n && y < x + n;
}

template <bool FUSED> int run_norm_backward(NormBackwardParams p, int dtype, void* dgamma, void* dbeta, hipStream_t s) {
  const bool sums = dgamma || dbeta;
  const size_t bytes = (size_t)p.T * p.H * (dtype == MOE_BF16 ? 2 : 4);
  const bool in_place = overlap(p.dx, p.dy, bytes) || overlap(p.dx, p.x, bytes) ||
                        (FUSED && (overlap(p.dv, p.dy, bytes) || overlap(p.dv, p.x, bytes)));
  if (!sums) p.part = nullptr;
  p.inv_h = 1.0f / (float)p.H;
  with_row_form(dtype, p.H, [&](auto t, auto tail) {
    using T = decltype(t);
    int parts = 0;
    if (sums && p.T > 0 && p.T <= kNormFewRows && bytes <= kNormFewBytes && p.H <= kRowMaxH) {
      p.part = nullptr;
      p.dgamma = dgamma; p.dbeta = dbeta;
      p.group = row_group(p.H);
      p.groups = kNormFewLanes / p.group;
      p.row_groups = ceil_div(p.T, p.groups);
      const auto few = norm_backward_few_kernel<T, tail.value, FUSED>;
      const int rows = p.row_groups, columns = ceil_div(p.H, kWave);
      const dim3 lanes(p.group * p.groups);
      if (in_place) {                                            // the columns' sums before anything lies over what they read
        p.row_groups = 0;
        hipLaunchKernelGGL(few, dim3(columns), lanes, 0, s, p);
        p.row_groups = rows;
      }
      hipLaunchKernelGGL(few, dim3(in_place ? rows : rows + columns), lanes, 0, s, p);
      return;
    }
    if (p.T > 0 && p.H > kRowMaxH) {
      if (sums) {                                                // ahead of the launch that writes dx, which may be dy or x
        parts = norm_parts(p.T) < 64 ? norm_parts(p.T) : 64;
        hipLaunchKernelGGL((norm_columns_long_kernel<T, tail.value>), dim3(ceil_div(p.H, 2048), parts), dim3(256), 0, s, p);
      }
      hipLaunchKernelGGL((norm_backward_long_kernel<T, tail.value, FUSED>), dim3(row_grid(p.T)), dim3(1024), 0, s, p);
    } else if (p.T > 0) {
      p.group = row_group(p.H);
      const int cus = std::min(device_cus(), kNormMaxParts);
      // a workgroup per CU, of as many rows at a time as 1024 threads hold, fewer where that leaves CUs without rows
      p.groups = 1024 / p.group;
      while (p.groups > 1 && p.groups * p.group > kWave && p.T < cus * p.groups) p.groups /= 2;
      const int want = ceil_div(p.T, p.groups);
      parts = std::min(want, cus);
      const size_t lds = p.groups > 1 ? (size_t)p.groups * p.group * 64 : 0;
      with_caching<T>(p.T, p.H, [&](auto nt) {
        hipLaunchKernelGGL((norm_backward_kernel<T, tail.value, FUSED, nt.value>), dim3(parts), dim3(p.group * p.groups), lds, s, p);
      });
    }
    if (sums)
      hipLaunchKernelGGL(norm_columns_kernel<T>, dim3(ceil_div(p.H, kWave), 2), dim3(1024), 0, s, p.part, parts, p.H, dgamma, dbeta);
  });
  return launched();
}

int run_drop_add(DropAddParams p, int dtype, hipStream_t s) {
  int g = 8;
  while (g < kDropGroup && g * 8 * kDropItems < p.H) g *= 2;
  p.group = g;
  const unsigned grid = row_grid((long)ceil_div(p.T, 256 / g) * ceil_div(p.H, g * 8 * kDropItems));
  with_row_form(dtype, p.H, [&](auto t, auto tail) {
    with_caching<decltype(t)>(p.T, p.H, [&](auto nt) {
      hipLaunchKernelGGL((drop_add_kernel<decltype(t), tail.value, nt.value>), dim3(grid), dim3(256), 0, s, p);
    });
  });
  return launched();
}

// Lanes per token (four experts each, a power of two) x E % 4 != 0
template <typename F> void with_token_form(int E, F&& f) {
  auto tail = [&](auto lanes) {
    if (E % 4) f(lanes, std::true_type{});
    else f(lanes, std::false_type{});
  };
  if (E <= 4) tail(std::integral_constant<int, 1>{});
  else if (E <= 8) tail(std::integral_constant<int, 2>{});
  else if (E <= 16) tail(std::integral_constant<int, 4>{});
  else if (E <= 32) tail(std::integral_constant<int, 8>{});
  else if (E <= 64) tail(std::integral_constant<int, 16>{});
  else if (E <= 128) tail(std::integral_constant<int, 32>{});
  else tail(std::integral_constant<int, 64>{});
}

int check_router(int T, int E, int k) {
  return T < 0 || k < 1 || k > kMaxK || E < k || E > kMaxE ? MOE_ERR_UNSUPPORTED_SHAPE : MOE_OK;
}

}  // namespace

extern "C" {

int moe_layer_norm_workspace_bytes(int32_t T, int32_t H, size_t* bytes) {
  const int st = check_rows(T, H, MOE_F32);
  if (st != MOE_OK) return st;
  if (!bytes) return MOE_ERR_INVALID_ARG;
  *bytes = (size_t)(T > 0 ? norm_parts(T) : 1) * 2 * H * 4;
  return MOE_OK;
}

int moe_layer_norm_forward(int32_t T, int32_t H, int dtype, const void* d_x, const void* d_gamma, const void* d_beta, float eps,
                           void* d_y, float* d_mean, float* d_rstd, void* stream) {
  const int st = check_rows(T, H, dtype);
  if (st != MOE_OK) return st;
  if (!(eps >= 0.f) || isinf(eps)) return MOE_ERR_INVALID_ARG;
  if (T == 0) return MOE_OK;
  if (!good(d_x) || !good(d_y) || !aligned(d_gamma) || !aligned(d_beta) || !aligned(d_mean) || !aligned(d_rstd))
    return MOE_ERR_INVALID_ARG;
  NormForwardParams p{};
  p.x = d_x; p.gamma = d_gamma; p.beta = d_beta; p.y = d_y; p.mean = d_mean; p.rstd = d_rstd;
  p.eps = eps; p.T = T; p.H = H;
  return run_norm_forward<false>(p, dtype, static_cast<hipStream_t>(stream));
}

int moe_dropout_add_layer_norm_forward(int32_t T, int32_t H, int dtype, const void* d_v, const void* d_residual, float p,
                                       const uint64_t* d_rng, const void* d_gamma, const void* d_beta, float eps, void* d_z, void* d_y,
                                       float* d_mean, float* d_rstd, void* stream) {
  int st = check_rows(T, H, dtype);
  if (st != MOE_OK) return st;
  NormForwardParams q{};
  if ((st = check_drop(p, d_rng, q.drop)) != MOE_OK) return st;
  if (!(eps >= 0.f) || isinf(eps)) return MOE_ERR_INVALID_ARG;
  if (T == 0) return MOE_OK;
  if (!good(d_v) || !good(d_z) || !good(d_y) || d_z == d_y || !aligned(d_residual) || !aligned(d_gamma) || !aligned(d_beta) ||
      !aligned(d_mean) || !aligned(d_rstd))
    return MOE_ERR_INVALID_ARG;
  q.v = d_v; q.x = d_residual; q.gamma = d_gamma; q.beta = d_beta; q.z = d_z; q.y = d_y; q.mean = d_mean; q.rstd = d_rstd;
  q.eps = eps; q.T = T; q.H = H;
  return run_norm_forward<true>(q, dtype, static_cast<hipStream_t>(stream));
}

}  // extern "C"

// Both backward entry points.
static int norm_backward(bool fused, int32_t T, int32_t H, int dtype, const void* dy, const void* x, const void* gamma, const float* mean,
                         const float* rstd, const void* dres, const DropParams& drop, void* dx, void* dv, void* dgamma, void* dbeta,
                         void* ws, size_t ws_bytes, void* stream) {
  if (!aligned(dgamma) || !aligned(dbeta)) return MOE_ERR_INVALID_ARG;
  if (T > 0) {
    if (!good(dy) || !good(x) || !good(mean) || !good(rstd) || !good(dx) || !aligned(gamma) || !aligned(dres)) return MOE_ERR_INVALID_ARG;
    if (fused && (!good(dv) || dv == dx)) return MOE_ERR_INVALID_ARG;
    if (dgamma || dbeta) {
      size_t need = 0;
      const int st = moe_layer_norm_workspace_bytes(T, H, &need);
      if (st != MOE_OK) return st;
      if (!good(ws)) return MOE_ERR_INVALID_ARG;
      if (ws_bytes < need) return MOE_ERR_WORKSPACE_TOO_SMALL;
    }
  }
  NormBackwardParams p{};
  p.dy = dy; p.x = x; p.gamma = gamma; p.dres = dres; p.mean = mean; p.rstd = rstd; p.dx = dx; p.dv = dv;
  p.part = static_cast<float*>(ws); p.drop = drop; p.T = T; p.H = H;
  hipStream_t s = static_cast<hipStream_t>(stream);
  return fused ? run_norm_backward<true>(p, dtype, dgamma, dbeta, s) : run_norm_backward<false>(p, dtype, dgamma, dbeta, s);
}

extern "C" {

int moe_layer_norm_backward(int32_t T, int32_t H, int dtype, const void* d_dy, const void* d_x, const void* d_gamma,
                            const float* d_mean, const float* d_rstd, const void* d_dres, void* d_dx, void* d_dgamma, void* d_dbeta,
                            void* d_workspace, size_t workspace_bytes, void* stream) {
  const int st = check_rows(T, H, dtype);
  if (st != MOE_OK) return st;
  return norm_backward(false, T, H, dtype, d_dy, d_x, d_gamma, d_mean, d_rstd, d_dres, DropParams{}, d_dx, nullptr, d_dgamma, d_dbeta,
                       d_workspace, workspace_bytes, stream);
}

int moe_dropout_add_layer_norm_backward(int32_t T, int32_t H, int dtype, const void* d_dy, const void* d_z, const void* d_gamma,
                                        const float* d_mean, const float* d_rstd, const void* d_dres, float p, const uint64_t* d_rng,
                                        void* d_dz, void* d_dv, void* d_dgamma, void* d_dbeta, void* d_workspace, size_t workspace_bytes,
                                        void* stream) {
  int st = check_rows(T, H, dtype);
  if (st != MOE_OK) return st;
  DropParams drop{};
  if ((st = check_drop(p, d_rng, drop)) != MOE_OK) return st;
  return norm_backward(true, T, H, dtype, d_dy, d_z, d_gamma, d_mean, d_rstd, d_dres, drop, d_dz, d_dv, d_dgamma, d_dbeta, d_workspace,
                       workspace_bytes, stream);
}

int moe_dropout_add_forward(int32_t T, int32_t H, int dtype, const void* d_v, const void* d_residual, float p, const uint64_t* d_rng,
                            void* d_out, void* stream) {
  int st = check_rows(T, H, dtype);
  if (st != MOE_OK) return st;
  DropAddParams q{};
  if ((st = check_drop(p, d_rng, q.drop)) != MOE_OK) return st;
  if (T == 0) return MOE_OK;
  if (!good(d_v) || !good(d_out) || !aligned(d_residual)) return MOE_ERR_INVALID_ARG;
  q.v = d_v; q.res = d_residual; q.out = d_out; q.T = T; q.H = H;
  return run_drop_add(q, dtype, static_cast<hipStream_t>(stream));
}

int moe_dropout_add_backward(int32_t T, int32_t H, int dtype, const void* d_dout, float p, const uint64_t* d_rng, void* d_dv,
                             void* stream) {
  return moe_dropout_add_forward(T, H, dtype, d_dout, nullptr, p, d_rng, d_dv, stream);   // the residual's gradient is dout itself
}

int moe_balance_workspace_bytes(int32_t T, int32_t E, size_t* bytes) {
  const int st = check_router(T, E, 1);
  if (st != MOE_OK) return st;
  if (!bytes) return MOE_ERR_INVALID_ARG;
  *bytes = (size_t)kBalMaxParts * (kMaxE + 1) * 8;
  return MOE_OK;
}

int moe_balance_forward(int32_t T, int32_t E, int32_t k, const float* d_logits, const int32_t* d_topk_idx, const uint8_t* d_mask,
                        float coef, int32_t* d_counts, float* d_prob_sum, float* d_loss, void* d_workspace, size_t workspace_bytes,
                        void* stream) {
  int st = check_router(T, E, k);
  if (st != MOE_OK) return st;
  if (!good(d_counts) || !good(d_prob_sum) || !good(d_loss) || !good(d_workspace)) return MOE_ERR_INVALID_ARG;
  if (T > 0 && (!good(d_logits) || !good(d_topk_idx))) return MOE_ERR_INVALID_ARG;
  size_t need = 0;
  moe_balance_workspace_bytes(T, E, &need);
  if (workspace_bytes < need) return MOE_ERR_WORKSPACE_TOO_SMALL;
  BalanceParams p{};
  p.logits = d_logits; p.topk_idx = d_topk_idx; p.mask = d_mask; p.counts = d_counts; p.prob_sum = d_prob_sum; p.loss = d_loss;
  p.part = static_cast<u32x2*>(d_workspace);
  p.coef = coef; p.T = T; p.E = E; p.k = k;
  hipStream_t s = static_cast<hipStream_t>(stream);
  with_token_form(E, [&](auto lanes, auto tail) {
    const int want = ceil_div(T, kBalThreads / lanes.value);
    p.parts = (long)T * lanes.value <= kBalOneLanes ? 1 : want < kBalMaxParts ? want : kBalMaxParts;
    hipLaunchKernelGGL((balance_kernel<lanes.value, tail.value>), dim3(p.parts), dim3(kBalThreads), 0, s, p);
  });
  if (p.parts > 1) hipLaunchKernelGGL(balance_join_kernel, dim3(1), dim3(1024), 0, s, p);
  return launched();
}

int moe_router_backward(int32_t T, int32_t E, int32_t k, const float* d_logits, const int32_t* d_topk_idx, const float* d_topk_w,
                        const float* d_dtopk_w, const uint8_t* d_mask, float coef, const int32_t* d_counts, const float* d_dloss,
                        float* d_dlogits, void* stream) {
  int st = check_router(T, E, k);
  if (st != MOE_OK) return st;
  if (!d_topk_w != !d_dtopk_w) return MOE_ERR_INVALID_ARG;
  if (T == 0) return MOE_OK;
  if (!good(d_logits) || !good(d_topk_idx) || !good(d_dlogits) || !aligned(d_topk_w) || !aligned(d_dtopk_w) || !aligned(d_counts) ||
      !aligned(d_dloss))
    return MOE_ERR_INVALID_ARG;
  RouterBackwardParams p{};
  p.logits = d_logits; p.topk_idx = d_topk_idx; p.topk_w = d_topk_w; p.dtopk_w = d_dtopk_w; p.mask = d_mask; p.counts = d_counts;
  p.dloss = d_dloss; p.dlogits = d_dlogits; p.coef = coef; p.T = T; p.E = E; p.k = k;
  hipStream_t s = static_cast<hipStream_t>(stream);
  with_token_form(E, [&](auto lanes, auto tail) {
    const int want = ceil_div(T, kRouterThreads / lanes.value * kRouterAhead);
    const dim3 grid(want < 2048 ? want : 2048);
    if (p.topk_w) hipLaunchKernelGGL((router_backward_kernel<lanes.value, tail.value, true>), grid, dim3(kRouterThreads), 0, s, p);
    else hipLaunchKernelGGL((router_backward_kernel<lanes.value, tail.value, false>), grid, dim3(kRouterThreads), 0, s, p);
  });
  return launched();
}

int moe_route_scores_backward(int32_t T, int32_t E, int32_t k, const MoeScores* scores, const float* d_logits, const int32_t* d_topk_idx,
                              const float* d_dtopk_w, const float* d_dadd, float* d_dlogits, void* stream) {
  int st = check_router(T, E, k);
  if (st != MOE_OK || (st = check_scores(scores, E, k)) != MOE_OK) return st;
  if (T == 0) return MOE_OK;
  if (!good(d_logits) || !good(d_topk_idx) || !good(d_dtopk_w) || !aligned(d_dadd) || !good(d_dlogits)) return MOE_ERR_INVALID_ARG;
  ScoresBackwardParams p{};
  p.logits = d_logits; p.topk_idx = d_topk_idx; p.dtopk_w = d_dtopk_w; p.dadd = d_dadd; p.dlogits = d_dlogits;
  p.renorm = scores->renormalize; p.scale = scores->scale;
  p.T = T; p.E = E; p.k = k;
  hipStream_t s = static_cast<hipStream_t>(stream);
  with_token_form(E, [&](auto lanes, auto tail) {
    const int want = ceil_div(T, kRouterThreads / lanes.value);
    const dim3 grid(want < 2048 ? want : 2048);
    if (scores->score == MOE_SCORE_SIGMOID) hipLaunchKernelGGL((scores_backward_kernel<lanes.value, tail.value, false>), grid, dim3(kRouterThreads), 0, s, p);
    else hipLaunchKernelGGL((scores_backward_kernel<lanes.value, tail.value, true>), grid, dim3(kRouterThreads), 0, s, p);
  });
  return launched();
}

int moe_bias_update(int32_t E, const int32_t* d_counts, float rate, const float* d_bias, float* d_bias_out, void* stream) {
  if (E < 1 || E > kMaxE) return MOE_ERR_UNSUPPORTED_SHAPE;
  if (!isfinite(rate) || !good(d_counts) || !good(d_bias) || !good(d_bias_out)) return MOE_ERR_INVALID_ARG;
  hipLaunchKernelGGL(bias_update_kernel, dim3(1), dim3(kMaxE), 0, static_cast<hipStream_t>(stream), d_counts, E, rate, d_bias, d_bias_out);
  return launched();
}

}  // extern "C"
