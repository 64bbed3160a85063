// Host side of the orthogonal updates (include/moe_ffn.h): argument checks, the scales of the matrices in between, launches on the
// caller's stream.  Nothing here allocates or synchronises.
#include "../../include/moe_ffn.h"

#include <math.h>

#include <algorithm>

#include "device_cus.h"
#include "newton_schulz.h"

using namespace moe;

namespace {


constexpr int kMaxSteps = 16;
// Matrices are worked on in groups whose workspace stays below this, one at least: enough tiles at a time for the whole chip.
constexpr size_t kNsGroupBytes = (size_t)4 << 30;
constexpr int kNsMaxShares = 256;          // partial tiles of a product's remainder
constexpr int kNsSmallSteps = 40;          // K steps of a tile of 64 x 64 where tiles of 128 x 128 could share them
constexpr int kNsShareSteps = 4, kNsMaxSplits = 8;   // K steps of a share, at least; shares of a tile, at most

bool aligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
bool good(const void* p) { return p && aligned(p); }
int pad(int v) { return (v + kNsPad - 1) / kNsPad * kNsPad; }
size_t align_up(size_t v) { return (v + 255) / 256 * 256; }

int check_matrices(int B, int M, int N, int dtype) {
  if (dtype != MOE_F32 && dtype != MOE_BF16) return MOE_ERR_INVALID_ARG;
  if (B < 0 || M < 1 || N < 1 || M > (1 << 18) || N > (1 << 18)) return MOE_ERR_UNSUPPORTED_SHAPE;
  const double s = pad(std::min(M, N)), l = pad(std::max(M, N));
  if (s * l * (dtype == MOE_F32 ? 4 : 2) >= 4294967296.0 || s > (1 << 15)) return MOE_ERR_UNSUPPORTED_SHAPE;   // 32-bit offsets inside a matrix
  if ((double)B * M * N * 4 > 9.0e18) return MOE_ERR_UNSUPPORTED_SHAPE;
  return MOE_OK;
}

// Matrices of a group, and a group's workspace.
struct Plan {
  int B, M, N, Sp, Lp, group;
  size_t x_bytes, a_bytes;                 // of one matrix
  size_t x, a, part, share, total;                // X and its transpose, two of each; A and B
};
Plan make_plan(int B, int M, int N, int dtype) {
  Plan p{};
  p.B = B; p.M = M; p.N = N;
  p.Sp = pad(std::min(M, N));
  p.Lp = pad(std::max(M, N));
  const size_t value = dtype == MOE_F32 ? 4 : 2;   // fp16, or pairs of it
  p.x_bytes = (size_t)p.Sp * p.Lp * value;
  p.a_bytes = (size_t)p.Sp * p.Sp * value;
  const size_t per = 4 * p.x_bytes + 2 * p.a_bytes + kNsMaxParts * 8;
  const int most = (int)std::min<size_t>(std::max<size_t>(kNsGroupBytes / per, 1), 1 << 14);
  const int groups = std::max(1, (B + most - 1) / most);
  p.group = std::max(1, (B + groups - 1) / groups);
  size_t off = 0;
  auto take = [&](size_t bytes) { const size_t o = off; off += align_up(bytes); return o; };
  // of as many matrices as a group can have: groups of more matrices may be smaller, and a program allocates for its largest call
  const size_t room = std::max(1, std::min(B, most));
  p.x = take(4 * p.x_bytes * room);
  p.a = take(2 * p.a_bytes * room);
  p.part = take((size_t)kNsMaxParts * 8 * room);
  p.share = take((size_t)kNsMaxShares * 128 * 128 * 4);
  p.total = off;
  return p;
}

// Coefficients of each step and the scales that follow from how large singular values can become.
struct Steps {
  int n;
  float c[kMaxSteps][3];
  int ex, ea[kMaxSteps], eb[kMaxSteps];    // stored: X 2^ex, A 2^ea, B 2^eb
};
int floor_log2(double v) { return (int)floor(log2(v)); }
// pairs: scales of pairs of fp16 (newton_schulz.h).  false: the coefficients let singular values grow out of bounds
bool make_steps(Steps& s, int n, const float* coefs, int S, int L, bool pairs) {
  static const float usual[3] = {3.4445f, -4.7750f, 2.0315f};
  s.n = n;
  s.ex = floor_log2((double)L) / 2;
  double top = 1.0, largest = 1.0;         // largest singular value possible, now and in any step
  for (int i = 0; i < n; ++i) {
    for (int j = 0; j < 3; ++j) {
      s.c[i][j] = coefs ? coefs[3 * i + j] : usual[j];
      if (!isfinite(s.c[i][j])) return false;
    }
    const double a = s.c[i][0], b = s.c[i][1], c = s.c[i][2];
    const double t = top * top;            // of A: its eigenvalues lie in [0, t], those of B are q there
    auto q = [&](double v) { return fabs(a + b * v + c * v * v); };
    double qmax = std::max(q(0.0), q(t));
    if (c != 0.0 && -b / (2 * c) > 0.0 && -b / (2 * c) < t) qmax = std::max(qmax, q(-b / (2 * c)));
    auto p = [&](double v) { return v > 0.0 && v < t ? sqrt(v) * q(v) : 0.0; };   // p(s) = s q(s^2), at v = s^2
    double pmax = top * q(t);
    if (c != 0.0) {                        // p'(s) = a + 3 b v + 5 c v^2
      const double d = 9 * b * b - 20 * a * c;
      if (d >= 0.0) pmax = std::max(pmax, std::max(p((-3 * b + sqrt(d)) / (10 * c)), p((-3 * b - sqrt(d)) / (10 * c))));
    } else if (b != 0.0) {
      pmax = std::max(pmax, p(-a / (3 * b)));
    }
    // entries are at most the largest singular value; 2^15 leaves a factor of two for roundings
    s.ea[i] = pairs ? 14 - (int)ceil(log2(t)) : std::min(floor_log2(S), 15 - (int)ceil(log2(t)));
    s.eb[i] = pairs ? 14 - (int)ceil(log2(std::max(qmax, 1e-6))) : std::min(floor_log2(S), 15 - (int)ceil(log2(std::max(qmax, 1e-6))));
    top = std::max(pmax, 1e-3) * 1.0001;
    if (!(qmax <= 1024.0) || !(top <= 32.0)) return false;
    largest = std::max(largest, top);
  }
  if (pairs) s.ex = 14 - (int)ceil(log2(largest));
  return true;
}

struct Update {
  const void* g;
  const float* m;
  float* m_out;
  const void* w;
  float* master;
  void* out;
  float mu, w_keep, w_step, eps;
  int nesterov;
};

// Tiles of 128 x 128 from p.first on, p.tiles of them, with fewer than one to a CU left over at the end of whole rounds.  A remainder that
// would leave half of the CUs idle is dealt out along k as well and joined by a second launch (4 matrices of 1408 x 2048 in fp32, 264 tiles for A: 256 of
// them 53 us, the 8 left over 9 + 6; all in one launch with two workgroups to a CU 81).  Up to a tile per CU four stages, beyond two and
// two workgroups (2048 x 2048 bf16 with four everywhere 308 us, so 306; 10 of 704 x 1088 in fp32 575 and 529).
template <int EPI, bool SPLIT, typename T, bool QUARTERS> void run_tiles128(NsGemmParams p, int cus, hipStream_t s) {
  auto grid = [](int n) { return dim3((unsigned)((n + 7) / 8 * 8)); };
  const int n_steps = p.K * (SPLIT ? 4 : 2) / 128, first = p.first, tiles = p.tiles;
  const int rest = tiles % cus;
  p.splits = rest ? std::min({std::min(cus, kNsMaxShares) / rest, n_steps / kNsShareSteps, kNsMaxSplits}) : 0;
  if (p.splits < 2) p.splits = 0;
  p.tiles = p.splits ? tiles - rest : tiles;
  if (p.tiles > 0) {
    if (p.tiles <= cus) hipLaunchKernelGGL((ns_gemm128_kernel<EPI, SPLIT, T, QUARTERS, 4, false>), grid(p.tiles), dim3(256), 0, s, p);
    else hipLaunchKernelGGL((ns_gemm128_kernel<EPI, SPLIT, T, QUARTERS, 2, false>), grid(p.tiles), dim3(256), 0, s, p);
  }
  if (p.splits) {
    p.first = first + p.tiles;
    p.tiles = rest;
    hipLaunchKernelGGL((ns_gemm128_kernel<EPI, SPLIT, T, QUARTERS, 4, true>), grid(rest * p.splits), dim3(256), 0, s, p);
    hipLaunchKernelGGL((ns_join_kernel<EPI, SPLIT, T, QUARTERS>), dim3(8 * rest), dim3(64), 0, s, p);
  }
}

// One product of every matrix of the group.  Whole rounds of tiles of 256 x 256, one to a CU, as long as they fill the chip: half the operand bytes of
// those of 128 x 128 (the next X of 4 x 4096 x 7168 in bf16 822 us, 1.17 PFLOP/s, with 128 x 128 1073; of 4 x 4096 x 4096 in fp32 1273, 1.30 PFLOP/s of
// its three products, with 128 x 128 1487).  What is left over, and everything of a product with too few of them, as tiles of 128 x 128; a small
// product, whose launches wait for each other's latency and not for the matrix cores, as tiles of 64 x 64 as long as two to a CU hold all (all steps
// of one matrix in bf16: 200 x 330 105 us with 128 x 128, 71 with 64 x 64; 512 x 512 146 and 87; 1024 x 1024 233 and 132; 1408 x 1408 277 and 160; but
// 4 of 1024 x 2048, 544 tiles for A, 279 and 335), unless the sums are long and so few that shares of them pay (256 x 4096: 113 and 147).
// Tiles count as whole ones however much of them lies past a matrix's sides: many matrices of sides below 256 go through 256 x 256 all the same.
template <int EPI, typename T> void run_product(NsGemmParams p, int cus, hipStream_t s) {
  constexpr bool SPLIT = sizeof(T) == 4, SYM = ns_symmetric(EPI);
  auto tiles = [&](int side) {
    const int ti = (p.rows + side - 1) / side, tj = (p.cols + side - 1) / side;
    return p.n * (SYM ? ti * (ti + 1) / 2 : ti * tj);
  };
  p.first = 0;
  const int whole = tiles(256), rest = whole % cus;
  if (whole >= cus) {
    const bool quarters = rest > 0 && 2 * rest <= cus;
    p.tiles = quarters ? whole - rest : whole;
    if constexpr (SPLIT) {
      hipLaunchKernelGGL((ns_gemm256_pairs_kernel<EPI, T>), dim3((unsigned)((p.tiles + 7) / 8 * 8)), dim3(256), 0, s, p);
    } else {
      auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(cus), dim3(kGemmThreads), 0, s, p); };
      const bool vec = p.N % 4 == 0;
      if constexpr (EPI != kNsOut) launch(ns_gemm256_kernel<EPI, T, void, true>);
      else if (p.master) launch(vec ? ns_gemm256_kernel<EPI, T, float, true> : ns_gemm256_kernel<EPI, T, float, false>);
      else if (p.w) launch(vec ? ns_gemm256_kernel<EPI, T, T, true> : ns_gemm256_kernel<EPI, T, T, false>);
      else launch(vec ? ns_gemm256_kernel<EPI, T, void, true> : ns_gemm256_kernel<EPI, T, void, false>);
    }
    if (quarters) {
      p.first = 4 * p.tiles;
      p.tiles = 4 * rest;
      run_tiles128<EPI, SPLIT, T, true>(p, cus, s);
    }
    return;
  }
  const int small = tiles(64), steps = p.K * (SPLIT ? 4 : 2) / 128;
  if (small <= 2 * cus && (steps <= kNsSmallSteps || 2 * small > cus)) {
    p.tiles = small;
    hipLaunchKernelGGL((ns_gemm64_kernel<EPI, SPLIT, T>), dim3((unsigned)((small + 7) / 8 * 8)), dim3(128), 0, s, p);
    return;
  }
  p.tiles = tiles(128);
  run_tiles128<EPI, SPLIT, T, false>(p, cus, s);
}

template <typename T> int run_update(const Plan& L, const Steps& st, const Update& u, char* ws, hipStream_t stream) {
  constexpr bool SPLIT = sizeof(T) == 4;
  const bool wide = L.M <= L.N;
  const int cus = device_cus() / 8 * 8;
  for (int e0 = 0; e0 < L.B; e0 += L.group) {
    const int n = std::min(L.group, L.B - e0);
    const size_t first = (size_t)e0 * L.M * L.N;
    // the group's arrays: X short x long and long x short, two of each; A; B
    auto x_of = [&](int i) { return ws + L.x + (size_t)i * L.group * L.x_bytes; };
    char *xs = x_of(0), *xl = x_of(1), *xs_next = x_of(2), *xl_next = x_of(3);
    char *A = ws + L.a, *Bm = A + (size_t)L.group * L.a_bytes;

    NsPrepParams q{};
    q.g = static_cast<const T*>(u.g) + first;
    q.m = u.m ? u.m + first : nullptr;
    q.m_out = u.m_out ? u.m_out + first : nullptr;
    q.mu = u.mu; q.nesterov = u.nesterov;
    q.part = reinterpret_cast<double*>(ws + L.part);
    q.parts = (int)std::min<size_t>(kNsMaxParts, ((size_t)L.M * L.N + 2047) / 2048);
    q.scale = ldexpf(1.f, st.ex);
    q.eps = u.eps;
    q.X = wide ? xs : xl;
    q.XT = wide ? xl : xs;
    q.stride = (long)L.x_bytes;
    q.M = L.M; q.N = L.N; q.Mp = wide ? L.Sp : L.Lp; q.Np = wide ? L.Lp : L.Sp; q.n = n;
    hipLaunchKernelGGL(ns_norm_kernel<T>, dim3((unsigned)(n * q.parts)), dim3(256), 0, stream, q);
    hipLaunchKernelGGL((ns_first_kernel<T, SPLIT>), dim3((unsigned)n * (q.Mp / 64) * (q.Np / 64)), dim3(256), 0, stream, q);

    for (int i = 0; i < st.n; ++i) {
      NsGemmParams p{};
      p.n = n;
      p.part = reinterpret_cast<float*>(ws + L.share);
      p.rows = p.cols = L.Sp;
      p.ld_c = p.ld_ct = L.Sp;
      p.c_stride = p.a_stride = (long)L.a_bytes;
      // A = X X^T
      p.P = p.Q = xs; p.C = p.CT = A;
      p.p_stride = p.q_stride = (long)L.x_bytes;
      p.K = L.Lp;
      p.s_acc = ldexpf(1.f, st.ea[i] - 2 * st.ex);
      run_product<kNsGram, T>(p, cus, stream);
      // B = a I + b A + c A^2
      p.P = p.Q = p.A = A; p.C = p.CT = Bm;
      p.p_stride = p.q_stride = (long)L.a_bytes;
      p.K = L.Sp;
      p.s_acc = ldexpf(st.c[i][2], st.eb[i] - 2 * st.ea[i]);
      p.s_a = ldexpf(st.c[i][1], st.eb[i] - st.ea[i]);
      p.diag = ldexpf(st.c[i][0], st.eb[i]);
      run_product<kNsPoly, T>(p, cus, stream);
      if (i + 1 < st.n) {
        // X <- B X, and its transpose
        p.P = Bm; p.Q = xl; p.C = xs_next; p.CT = xl_next;
        p.q_stride = p.c_stride = (long)L.x_bytes;
        p.cols = L.Lp;
        p.ld_c = L.Lp; p.ld_ct = L.Sp;
        p.s_acc = ldexpf(1.f, -st.eb[i]);
        run_product<kNsNext, T>(p, cus, stream);
        std::swap(xs, xs_next);
        std::swap(xl, xl_next);
      } else {
        // the caller's side up: M x N
        p.P = wide ? Bm : xl; p.Q = wide ? xl : Bm;
        p.p_stride = (long)(wide ? L.a_bytes : L.x_bytes);
        p.q_stride = (long)(wide ? L.x_bytes : L.a_bytes);
        p.rows = wide ? L.Sp : L.Lp; p.cols = wide ? L.Lp : L.Sp;
        p.s_acc = ldexpf(1.f, -st.eb[i] - st.ex);
        p.w = u.w ? static_cast<const T*>(u.w) + first : nullptr;
        p.master = u.master ? u.master + first : nullptr;
        p.out = static_cast<T*>(u.out) + first;
        p.w_keep = u.w_keep; p.w_step = u.w_step;
        p.M = L.M; p.N = L.N;
        run_product<kNsOut, T>(p, cus, stream);
      }
    }
    if (hipGetLastError() != hipSuccess) return MOE_ERR_LAUNCH;
  }
  return MOE_OK;
}

int check_call(const Plan& L, void* ws, size_t ws_bytes) {
  if (!good(ws)) return MOE_ERR_INVALID_ARG;
  return ws_bytes < L.total ? MOE_ERR_WORKSPACE_TOO_SMALL : MOE_OK;
}

int run(const Plan& L, int dtype, const Steps& st, const Update& u, void* ws, void* stream) {
  char* w = static_cast<char*>(ws);
  hipStream_t s = static_cast<hipStream_t>(stream);
  return dtype == MOE_BF16 ? run_update<__bf16>(L, st, u, w, s) : run_update<float>(L, st, u, w, s);
}

// Whether arrays of a and b bytes share any.
bool overlap(const void* x, size_t a, const void* y, size_t b) {
  const uintptr_t p = reinterpret_cast<uintptr_t>(x), q = reinterpret_cast<uintptr_t>(y);
  return x && y && p < q + b && q < p + a;
}

}  // namespace

extern "C" {

int moe_muon_workspace_bytes(int32_t B, int32_t M, int32_t N, int dtype, size_t* bytes) {
  const int st = check_matrices(B, M, N, dtype);
  if (st != MOE_OK) return st;
  if (!bytes) return MOE_ERR_INVALID_ARG;
  *bytes = make_plan(B, M, N, dtype).total;
  return MOE_OK;
}

int moe_orthogonalize(int32_t B, int32_t M, int32_t N, int dtype, const void* d_u, int32_t steps, const float* coefs, float eps,
                      void* d_out, void* d_workspace, size_t workspace_bytes, void* stream) {
  int st = check_matrices(B, M, N, dtype);
  if (st != MOE_OK) return st;
  Steps s;
  if (steps < 1 || steps > kMaxSteps || !(eps > 0.f) || isinf(eps) || !make_steps(s, steps, coefs, std::min(M, N), std::max(M, N), dtype == MOE_F32))
    return MOE_ERR_INVALID_ARG;
  if (B == 0) return MOE_OK;
  if (!good(d_u) || !good(d_out)) return MOE_ERR_INVALID_ARG;
  const size_t bytes = (size_t)B * M * N * (dtype == MOE_BF16 ? 2 : 4);
  if (d_out != d_u && overlap(d_out, bytes, d_u, bytes)) return MOE_ERR_INVALID_ARG;
  const Plan L = make_plan(B, M, N, dtype);
  if ((st = check_call(L, d_workspace, workspace_bytes)) != MOE_OK) return st;
  Update u{};
  u.g = d_u; u.out = d_out; u.eps = eps;
  return run(L, dtype, s, u, d_workspace, stream);
}

int moe_muon_step(int32_t B, int32_t M, int32_t N, int dtype, const void* d_g, const float* d_m, const void* d_w, float* d_master,
                  float mu, int32_t nesterov, float lr, float weight_decay, float scale, int32_t steps, const float* coefs, float eps,
                  float* d_m_out, void* d_w_out, void* d_workspace, size_t workspace_bytes, void* stream) {
  int st = check_matrices(B, M, N, dtype);
  if (st != MOE_OK) return st;
  Steps s;
  if (steps < 1 || steps > kMaxSteps || !(eps > 0.f) || isinf(eps) || !make_steps(s, steps, coefs, std::min(M, N), std::max(M, N), dtype == MOE_F32))
    return MOE_ERR_INVALID_ARG;
  if (!isfinite(mu) || !isfinite(lr) || !isfinite(weight_decay) || !isfinite(scale) || (nesterov != 0 && nesterov != 1))
    return MOE_ERR_INVALID_ARG;
  if (B == 0) return MOE_OK;
  if (!good(d_g) || !good(d_m) || !good(d_m_out) || !good(d_w_out) || !aligned(d_master) || !aligned(d_w) || (!d_w && !d_master))
    return MOE_ERR_INVALID_ARG;
  const Plan L = make_plan(B, M, N, dtype);
  if ((st = check_call(L, d_workspace, workspace_bytes)) != MOE_OK) return st;
  const size_t n = (size_t)B * M * N, nw = n * (dtype == MOE_BF16 ? 2 : 4);
  // in place or apart: a group's outputs are written before the next group's inputs are read
  if ((d_m_out != d_m && overlap(d_m_out, n * 4, d_m, n * 4)) || overlap(d_m_out, n * 4, d_g, nw) || overlap(d_m_out, n * 4, d_w_out, nw) ||
      overlap(d_m_out, n * 4, d_w, nw) || overlap(d_m_out, n * 4, d_master, n * 4) || overlap(d_w_out, nw, d_master, n * 4) ||
      (d_w_out != d_w && !d_master && overlap(d_w_out, nw, d_w, nw)) || overlap(d_w_out, nw, d_g, nw) || overlap(d_w_out, nw, d_m, n * 4) ||
      overlap(d_master, n * 4, d_g, nw) || overlap(d_master, n * 4, d_m, n * 4))
    return MOE_ERR_INVALID_ARG;
  Update u{};
  u.g = d_g; u.m = d_m; u.m_out = d_m_out; u.w = d_w; u.master = d_master; u.out = d_w_out;
  u.mu = mu; u.nesterov = nesterov; u.eps = eps;
  u.w_keep = (float)(1.0 - (double)lr * weight_decay);
  u.w_step = (float)((double)lr * scale);
  return run(L, dtype, s, u, d_workspace, stream);
}

}  // extern "C"
