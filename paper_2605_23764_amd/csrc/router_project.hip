// Host side of the router's projection (include/moe_ffn.h): argument checks and launches on the caller's stream.
#include "../../include/moe_ffn.h"

#include <math.h>

#include <algorithm>

#include "router_project.h"

using namespace moe;

namespace {

constexpr int kProjMaxE = 256;
constexpr int kProjCUs = 256;              // the card's, not asked for: workspace sizes follow from it, whichever device is current when they are asked
constexpr int kProjTiles = 48;             // of 128 columns, at least
constexpr int kProjMaxSplits = 256;

bool aligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
bool good(const void* p) { return p && aligned(p); }
int ceil_div(long a, long b) { return (int)((a + b - 1) / b); }
int launched() { return hipGetLastError() == hipSuccess ? MOE_OK : MOE_ERR_LAUNCH; }

int check(int T, int H, int E, int dtype) {
  if (dtype != MOE_F32 && dtype != MOE_BF16) return MOE_ERR_INVALID_ARG;
  if (T < 0 || H < 1 || H > (1 << 18) || E < 1 || E > kProjMaxE) return MOE_ERR_UNSUPPORTED_SHAPE;
  // a launch holds 2^32 work-items at most
  if ((size_t)ceil_div(T, kProjTile) * ceil_div(std::max(H, E), 64) >= ((size_t)1 << 24)) return MOE_ERR_UNSUPPORTED_SHAPE;
  return MOE_OK;
}

// Columns of a tile: as many as there are where that is up to 64, which leaves none of a tile's empty (4096 x 2048 x 64: 128 columns 21.4 and 24.2 us
// forward and for dW, 64 18.6 and 21.2).  Above, 128 in bf16 with enough such tiles (8192 x 7168 x 256: 94 and 102, with 64 116 and 143; but 1024 x 4096 x
// 128 27 and 24, with 64 22 and 19), and 64 in fp32, whose three pieces of 128 columns leave a CU one workgroup (8192 x 7168 x 256: 217 and 244, with
// 64 195 and 205).
int tile_cols(int rows, int cols, int dtype) {
  if (cols <= 32) return 32;
  return cols <= 64 || dtype == MOE_F32 || (long)ceil_div(rows, kProjTile) * ceil_div(cols, kProjTile) < kProjTiles ? 64 : 128;
}

// k's per workgroup and workgroups along k of a product of rows x cols over K: two workgroups to a CU, but no more than pay.  A step of a
// workgroup takes about as long as the whole chip takes to write 2^20 partial sums and read them again, so s splits cost steps / s + s rows cols / 2^20,
// least at the root of the quotient (128 x 7168 x 256, bf16: with two to a CU, 112 splits, 17.6 us, with 58 14.4; its dW 16.2 and 8.6).  What is left
// of two to a CU by that, but leaves most CUs one, is one each (4096 x 2048 x 64: dW in 352 workgroups 21.5 us, in 256 15.9).
int splits_wanted(int rows, int cols, int K, int dtype) {
  const int tiles = (int)std::min<long>((long)ceil_div(rows, kProjTile) * ceil_div(cols, tile_cols(rows, cols, dtype)), 1 << 20);
  const double most = sqrt((double)ceil_div(K, kProjK) * (1 << 20) / ((double)rows * cols));
  int want = std::min({kProjMaxSplits, 2 * kProjCUs / tiles, (int)std::min(most + 0.5, 1e6)});
  if (want * tiles < kProjCUs * 3 / 2) want = std::min(want, kProjCUs / tiles);
  return std::max(want, 1);
}
struct Split { int k, n; };
Split split_of(int rows, int cols, int K, int dtype) {
  Split s;
  s.k = ceil_div(ceil_div(K, splits_wanted(rows, cols, K, dtype)), kProjK) * kProjK;
  s.n = ceil_div(K, s.k);
  return s;
}

// Bytes of the partial sums of a call with T tokens and of every one with fewer: a program allocates for its largest call, and fewer tokens may
// have more sums (8192 x 7168 x 256 33.5 MB, of 32768 tokens 29.4).  s splits, by split_of:
//   logits  s T E values.  s is at most kProjMaxSplits, the steps of H, and the root above, rounded; times T E each of them grows with T.  It is at most
//           2 kProjCUs / tiles, too, and T / tiles at most kProjTile / (tiles of 128 columns): the same for every T
//   dW      s H E values.  splits_wanted and the steps of T, which s does not exceed, grow with T
size_t logits_part_bound(int T, int H, int E) {
  const double n = (double)T * E, steps = ceil_div(H, kProjK);
  const double tile_bound = 2.0 * kProjCUs * kProjTile / ceil_div(E, kProjTile) * E;
  const double most = sqrt(steps * (1 << 20) * n) + 0.5 * n;
  const double values = std::min({kProjMaxSplits * n, steps * n, most, tile_bound});
  return (size_t)ceil(values) * 4;
}
size_t dw_part_bound(int T, int H, int E, int dtype) {
  const int n = std::min(splits_wanted(H, E, T, dtype), ceil_div(T, kProjK));
  return n > 1 ? (size_t)n * H * E * 4 : 0;
}

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
  const Split sp = split_of(p.rows, p.cols, p.K, sizeof(TP) == 2 ? MOE_BF16 : MOE_F32);
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
  const int tn = tile_cols(p.rows, p.cols, dtype);
  if (tn == 32) return dtype == MOE_BF16 ? run_sums<__bf16, KCP, 1, 3, 32>(p, out, ws, s) : run_sums<float, KCP, 3, 3, 32>(p, out, ws, s);
  if (tn == 64) return dtype == MOE_BF16 ? run_sums<__bf16, KCP, 1, 3, 64>(p, out, ws, s) : run_sums<float, KCP, 3, 3, 64>(p, out, ws, s);
  return run_sums<__bf16, KCP, 1, 3, 128>(p, out, ws, s);
}

}  // namespace

extern "C" {

int moe_router_project_workspace_bytes(int32_t T, int32_t H, int32_t E, size_t* bytes) {
  const int st = check(T, H, E, MOE_F32);
  if (st != MOE_OK) return st;
  if (!bytes) return MOE_ERR_INVALID_ARG;
  *bytes = T == 0 ? 16 : std::max({(size_t)16, logits_part_bound(T, H, E), dw_part_bound(T, H, E, MOE_F32), dw_part_bound(T, H, E, MOE_BF16)});
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
    p.P = d_dlogits; p.Q = d_w;
    p.ld_p = p.ld_q = p.K = E;
    p.rows = T; p.cols = H;
    p.k_split = ceil_div(E, kProjK) * kProjK;
    p.splits = 1;
    p.tj = ceil_div(H, 64);
    p.add = d_dres; p.out = d_dx;
    const dim3 grid((unsigned)((size_t)ceil_div(T, kProjTile) * p.tj)), threads(kProjThreads);
    if (dtype == MOE_BF16) hipLaunchKernelGGL((project_kernel<float, true, 2, float, true, 2, 64, __bf16>), grid, threads, 0, s, p);
    else hipLaunchKernelGGL((project_kernel<float, true, 3, float, true, 3, 64, float>), grid, threads, 0, s, p);
    st = launched();
  }
  return st;
}

}  // extern "C"
