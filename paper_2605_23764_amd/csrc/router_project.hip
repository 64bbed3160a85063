// Host side of the router's projection (include/moe_ffn.h): argument checks and launches on the caller's stream.
#include "../../include/moe_ffn.h"

#include <algorithm>

#include "router_project.h"

using namespace moe;

namespace {

constexpr int kProjMaxE = 256;
constexpr int kProjWorkgroups = 512;       // two per CU
constexpr int kProjMaxSplits = 256;

bool aligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
bool good(const void* p) { return p && aligned(p); }
int ceil_div(long a, long b) { return (int)((a + b - 1) / b); }
int launched() { return hipGetLastError() == hipSuccess ? MOE_OK : MOE_ERR_LAUNCH; }

int check(int T, int H, int E, int dtype) {
  if (dtype != MOE_F32 && dtype != MOE_BF16) return MOE_ERR_INVALID_ARG;
  if (T < 0 || H < 1 || H > (1 << 18) || E < 1 || E > kProjMaxE) return MOE_ERR_UNSUPPORTED_SHAPE;
  // a launch holds 2^32 work-items at most
  if ((size_t)ceil_div(T, kProjTile) * ceil_div(std::max(H, E), kProjTile) >= ((size_t)1 << 24)) return MOE_ERR_UNSUPPORTED_SHAPE;
  return MOE_OK;
}

// Columns of a tile: 32 for up to as many experts.
int tile_cols(int cols) { return cols <= 32 ? 32 : kProjTile; }

// k's per workgroup and workgroups along k of a product of rows x cols over K.
struct Split { int k, n; };
Split split_of(int rows, int cols, int K) {
  const long tiles = (long)ceil_div(rows, kProjTile) * ceil_div(cols, tile_cols(cols));
  const int want = (int)std::max<long>(1, std::min<long>(kProjMaxSplits, kProjWorkgroups / std::max<long>(tiles, 1)));
  Split s;
  s.k = ceil_div(ceil_div(K, want), kProjK) * kProjK;
  s.n = ceil_div(K, s.k);
  return s;
}
// Experts in pairs, and the bytes of both sides' pairs.
int pad_pairs(int E) { return ceil_div(E, 32) * 32; }
constexpr int kProjRows = 1 << 21;         // rows of dx at a time: 32-bit offsets into their pairs of up to 1 KB
size_t pairs_bytes(int T, int H, int E) { return ((size_t)std::min(T, kProjRows) + H) * pad_pairs(E) * 4; }
size_t part_bytes(const Split& s, int rows, int cols) { return s.n > 1 ? (size_t)s.n * rows * cols * 4 : 0; }

int join(const float* part, int splits, size_t n, float* out, hipStream_t s) {
  if (splits > 0 && splits <= 8 && n % 4 == 0)
    hipLaunchKernelGGL(project_join4_kernel, dim3((unsigned)((n / 4 + 255) / 256)), dim3(256), 0, s, part, splits, n / 4, out);
  else if (splits <= 16)
    hipLaunchKernelGGL(project_join_kernel<4>, dim3((unsigned)((n + 63) / 64)), dim3(256), 0, s, part, splits, n, out);
  else
    hipLaunchKernelGGL(project_join_kernel<16>, dim3((unsigned)((n + 15) / 16)), dim3(256), 0, s, part, splits, n, out);
  return launched();
}

template <typename TP, bool KCP, int NP, int NQ, int TN> int run_sums(ProjParams p, float* out, void* ws, hipStream_t s) {
  const Split sp = split_of(p.rows, p.cols, p.K);
  p.k_split = sp.k;
  p.splits = sp.n;
  p.tj = ceil_div(p.cols, TN);
  p.part = sp.n > 1 ? static_cast<float*>(ws) : out;
  hipLaunchKernelGGL((project_kernel<TP, KCP, NP, float, false, NQ, TN, void>), dim3((unsigned)ceil_div(p.rows, kProjTile) * p.tj * p.splits),
                     dim3(kProjThreads), 0, s, p);
  if (sp.n == 1) return launched();
  return join(p.part, sp.n, (size_t)p.rows * p.cols, out, s);
}
// P in the storage type, k-contiguous or not, against fp32 row-contiguous.
template <bool KCP> int run_sums(const ProjParams& p, int dtype, float* out, void* ws, hipStream_t s) {
  if (p.cols <= 32) return dtype == MOE_BF16 ? run_sums<__bf16, KCP, 1, 3, 32>(p, out, ws, s) : run_sums<float, KCP, 3, 3, 32>(p, out, ws, s);
  return dtype == MOE_BF16 ? run_sums<__bf16, KCP, 1, 3, 128>(p, out, ws, s) : run_sums<float, KCP, 3, 3, 128>(p, out, ws, s);
}

}  // namespace

extern "C" {

int moe_router_project_workspace_bytes(int32_t T, int32_t H, int32_t E, size_t* bytes) {
  const int st = check(T, H, E, MOE_F32);
  if (st != MOE_OK) return st;
  if (!bytes) return MOE_ERR_INVALID_ARG;
  *bytes = T == 0 ? 16 : std::max({pairs_bytes(T, H, E), part_bytes(split_of(T, E, H), T, E), part_bytes(split_of(H, E, T), H, E)});
  return MOE_OK;
}

int moe_router_project(int32_t T, int32_t H, int32_t E, int dtype, const void* d_x, const float* d_w, float* d_logits, void* d_workspace,
                       size_t workspace_bytes, void* stream) {
  const int st = check(T, H, E, dtype);
  if (st != MOE_OK || T == 0) return st;
  if (!good(d_x) || !good(d_w) || !good(d_logits) || !good(d_workspace)) return MOE_ERR_INVALID_ARG;
  size_t need = 0;
  moe_router_project_workspace_bytes(T, H, E, &need);
  if (workspace_bytes < need) return MOE_ERR_WORKSPACE_TOO_SMALL;
  ProjParams p{};
  p.P = d_x; p.Q = d_w;
  p.ld_p = H; p.ld_q = E;
  p.rows = T; p.cols = E; p.K = H;
  hipStream_t s = static_cast<hipStream_t>(stream);
  return run_sums<true>(p, dtype, d_logits, d_workspace, s);
}

int moe_router_project_backward(int32_t T, int32_t H, int32_t E, int dtype, const float* d_dlogits, const void* d_x, const float* d_w,
                                const void* d_dres, void* d_dx, float* d_dw, void* d_workspace, size_t workspace_bytes, void* stream) {
  int st = check(T, H, E, dtype);
  if (st != MOE_OK) return st;
  if (!aligned(d_dx) || !aligned(d_dw) || !aligned(d_dres)) return MOE_ERR_INVALID_ARG;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (T == 0) {
    if (!d_dw) return MOE_OK;
    return join(nullptr, 0, (size_t)H * E, d_dw, s);   // sums over nothing
  }
  if (!d_dx && !d_dw) return MOE_OK;
  if (!good(d_dlogits) || (d_dx && !good(d_w)) || (d_dw && !good(d_x)) || !good(d_workspace)) return MOE_ERR_INVALID_ARG;
  size_t need = 0;
  moe_router_project_workspace_bytes(T, H, E, &need);
  if (workspace_bytes < need) return MOE_ERR_WORKSPACE_TOO_SMALL;
  if (d_dw) {
    ProjParams p{};                        // ahead of dx, which may be x
    p.P = d_x; p.Q = d_dlogits;
    p.ld_p = H; p.ld_q = E;
    p.rows = H; p.cols = E; p.K = T;
    st = run_sums<false>(p, dtype, d_dw, d_workspace, s);
    if (st != MOE_OK) return st;
  }
  if (d_dx) {
    ProjParams p{};
    p.rows = T; p.cols = H;
    p.tj = ceil_div(H, kProjTile);
    p.add = d_dres; p.out = d_dx;
    if (dtype == MOE_BF16) {
      const int Ep = pad_pairs(E);
      char* pairs = static_cast<char*>(d_workspace);               // W's, then dlogits'
      p.Q = pairs;
      p.P = pairs + (size_t)H * Ep * 4;
      for (int t0 = 0; t0 < T; t0 += kProjRows) {
        const int n = std::min(T - t0, kProjRows), w_rows = t0 ? 0 : H;
        hipLaunchKernelGGL(project_pairs_kernel, dim3((unsigned)(((size_t)n + w_rows) * (Ep / 8) / 256 + 1)), dim3(256), 0, s, d_w, w_rows,
                           d_dlogits + (size_t)t0 * E, n, E, Ep, pairs + (size_t)(H - w_rows) * Ep * 4);
        p.rows = n;
        p.add = d_dres ? static_cast<const uint16_t*>(d_dres) + (size_t)t0 * H : nullptr;
        p.out = static_cast<uint16_t*>(d_dx) + (size_t)t0 * H;
        const size_t tiles = (size_t)ceil_div(n, kProjTile) * p.tj;
        hipLaunchKernelGGL(project_dx_kernel, dim3((unsigned)((tiles + 7) / 8 * 8)), dim3(256), 0, s, p, Ep);
        if (T - t0 <= kProjRows) break;
      }
    } else {
      p.P = d_dlogits; p.Q = d_w;
      p.ld_p = p.ld_q = p.K = E;
      p.k_split = ceil_div(E, kProjK) * kProjK;
      p.splits = 1;
      hipLaunchKernelGGL((project_kernel<float, true, 3, float, true, 3, 128, float>), dim3((unsigned)((size_t)ceil_div(T, kProjTile) * p.tj)),
                         dim3(kProjThreads), 0, s, p);
    }
    st = launched();
  }
  return st;
}

}  // extern "C"
