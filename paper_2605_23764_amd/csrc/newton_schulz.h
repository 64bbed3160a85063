// An update made orthogonal by Newton-Schulz products, and the optimiser's step around it.
//
//   X0 = u / (|u| + eps) (Frobenius norm), turned so that it has S <= L rows;  per step with its coefficients a, b, c
//   A = X X^T;  B = a I + b A + c A^2;  X <- B X          every singular value s of X becomes a s + b s^3 + c s^5
//
// Per step 3 S^2 L + S^3 multiply-adds' flops, as A and B are symmetric and half of their tiles are computed: bound by the matrix cores.
//
// All products are of one form, C[i,j] = sum over k of P[i,k] Q[j,k] with both operands k-contiguous, which the copies to LDS and the
// operand reads like best: A = X X^T, A^2 = A A^T, and B X = B (X^T)^T, for which X is kept together with its transpose.  A tile's
// epilogue writes both: straight, and transposed by way of LDS.  For a symmetric product the transposed write is the mirrored tile.
// The matrices in between are padded with zeros to multiples of 64, so that products know no borders.
//
// Types.  Operands are fp16, sums fp32.  Singular values never exceed the bound S_max that the host takes from the coefficients (1.2 with
// the usual ones), so fp16's range suffices and its 11 bits are worth eight times bf16's 8: the error of a step's roundings is
// multiplied by up to a per later step (3.4^4 = 140 for the first).  Every matrix is stored times a power of two that brings its
// entries near 1 where they are typical, clear of both ends of the range: X by about sqrt(L), A and B by about S.
// fp32 storage: operands are pairs of fp16 (hi, and the rest times 2^11), products hi hi + hi lo + lo hi, so 22 bits.
#pragma once
#include "gemm_bf16.h"

namespace moe {

constexpr float kNsLoScale = 2048.0f;      // what the second half of a pair is stored times
constexpr int kNsMaxParts = 256;           // partial sums of squares per matrix
constexpr int kNsPad = 64;

struct NsMat {                             // fp16 [rows][ld] of each matrix
  char* hi;
  char* lo;                                // null: single
};

enum NsEpilogue { kNsGram = 0, kNsPoly = 1, kNsNext = 2, kNsOut = 3 };

struct NsGemmParams {
  NsMat P, Q, C, CT;                       // C straight, CT transposed (gram, poly: the same array)
  NsMat A;                                 // poly: the matrix that b is for
  long p_stride, q_stride, c_stride, a_stride;   // bytes between matrices (of CT: c_stride as well)
  int rows, cols, K;                       // multiples of 64
  int ld_c, ld_ct;
  int n;                                   // matrices
  float s_acc, s_a, diag;                  // result = s_acc * sum + s_a * A + diag * I
  // out: o = s_acc * sum, M x N of them, weights w [M,N]
  const void* w;                           // null: out = o
  float* master;                           // fp32 weights, updated in place, instead of w
  void* out;
  float w_keep, w_step;                    // out = w_keep * w - w_step * o
  int M, N;
};

// Values of four columns of this lane's row, fp16.
__device__ __forceinline__ u32x2 pack_f16x4(const float (&v)[4]) {
  typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
  return __builtin_bit_cast(u32x2, (f16x4){(_Float16)v[0], (_Float16)v[1], (_Float16)v[2], (_Float16)v[3]});
}
__device__ __forceinline__ void unpack_f16x4(u32x2 p, float (&v)[4]) {
  typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
  const f16x4 h = __builtin_bit_cast(f16x4, p);
#pragma unroll
  for (int x = 0; x < 4; ++x) v[x] = (float)h[x];
}

// A block of 32 rows x 128 columns through the wave's LDS region: rows to C, 256 bytes of each; columns to CT, 64 bytes of each, by
// transposing reads.  Either may be null.
__device__ __forceinline__ void ns_store_block(char* region, const u32x2 (&pk)[4][4], char* C, int ld_c, char* CT, int ld_ct, int cols_valid) {
  typedef __attribute__((address_space(3))) char* lds_ptr;
  typedef __attribute__((address_space(3))) u32x2* lds_u32x2_ptr;
  typedef __attribute__((address_space(3))) const u32x4* lds_u32x4_cptr;
  int lane = lane_id();
  asm volatile("" : "+v"(lane));
  const int l32 = lane & 31, lh = lane >> 5;
  const lds_ptr base = (lds_ptr)region;
#pragma unroll
  for (int nt = 0; nt < 4; ++nt)
#pragma unroll
    for (int q = 0; q < 4; ++q) *(lds_u32x2_ptr)(base + l32 * kEpiRowBytes + (nt * 32 + q * 8 + lh * 4) * 2) = pk[nt][q];
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  if (C) {
    const int r4 = lane >> 4, ch = lane & 15;
    u32x4 v[8];
#pragma unroll
    for (int it = 0; it < 8; ++it) v[it] = *(lds_u32x4_cptr)(base + (it * 4 + r4) * kEpiRowBytes + ch * 16);
    char* dst = C + ((size_t)r4 * ld_c + ch * 8) * 2;
    if (ch * 8 < cols_valid)
#pragma unroll
      for (int it = 0; it < 8; ++it) *reinterpret_cast<u32x4*>(dst + (size_t)(it * 4) * ld_c * 2) = v[it];
  }
  if (CT) {
    // 16 lanes read 4 rows x 16 columns and get a column's 4 rows each; lane (g, i): rows 8 g .. 8 g + 7 of column i
    const int g = lane >> 4, i = lane & 15;
    const lds_ptr at = base + (8 * g + (i >> 2)) * kEpiRowBytes + (i & 3) * 8;
    u32x4 v[8];
#pragma unroll
    for (int cg = 0; cg < 8; ++cg) {
      const u32x2 a = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_ptr)(at + cg * 32)));
      const u32x2 b = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_ptr)(at + cg * 32 + 4 * kEpiRowBytes)));
      v[cg] = u32x4{a.x, a.y, b.x, b.y};
    }
    char* dst = CT + ((size_t)i * ld_ct + 8 * g) * 2;
#pragma unroll
    for (int cg = 0; cg < 8; ++cg)
      if (cg * 16 < cols_valid) *reinterpret_cast<u32x4*>(dst + (size_t)(cg * 16) * ld_ct * 2) = v[cg];
  }
  wait_lgkmcnt0();                         // see store_block_via_lds
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// Weights of four columns n .. n + 3 of row m from the update o.  T: storage.
template <typename T> __device__ __forceinline__ void ns_store_out(const NsGemmParams& p, int e, int m, int n, const float (&o)[4]) {
  const size_t at = ((size_t)e * p.M + m) * p.N + n;
#pragma unroll
  for (int x = 0; x < 4; ++x) {
    if (n + x >= p.N) break;
    float v = o[x];
    if (p.master) {
      v = p.w_keep * p.master[at + x] - p.w_step * v;
      p.master[at + x] = v;
    } else if (p.w) {
      v = p.w_keep * (float)static_cast<const T*>(p.w)[at + x] - p.w_step * v;
    }
    static_cast<T*>(p.out)[at + x] = (T)v;
  }
}

// One tile of 256 x 256: rows from i0, columns from j0 of matrix e.
template <int EPI, bool SPLIT, typename T>
__device__ __forceinline__ void ns_tile(const NsGemmParams& p, int e, int i0, int j0, char* smem) {
  int lane = lane_id();
  asm volatile("" : "+v"(lane));
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave >> 1, wn = wave & 1;
  const int l32 = lane & 31, lh = lane >> 5;
  const int n_steps = p.K / kBK;
  GemmTileCtx t;
  t.wave = wave;
  t.nA = 8;
  t.lda_bytes = t.ldb_bytes = p.K * 2;
  const int kc_r = lane >> 3;
  const int kc_c = (lane & 7) ^ ((4 * (wave & 1) + (kc_r >> 1)) & 7);
#pragma unroll
  for (int i = 0; i < 8; ++i) {            // rows past the end read the last one again; they are not stored
    const int r = (wave + 4 * i) * 8 + kc_r;
    t.a_off[i] = (uint32_t)min(i0 + r, p.rows - 1) * (uint32_t)(p.K * 2) + (uint32_t)(kc_c * 16);
    t.b_off[i] = (uint32_t)min(j0 + r, p.cols - 1) * (uint32_t)(p.K * 2) + (uint32_t)(kc_c * 16);
  }
  t.lds0 = lds_addr_of(smem);
  {
    const int f = (l32 >> 1) & 7;
    const uint32_t a0 = (uint32_t)((wm * 128 >> 3) * kLine + (l32 >> 3) * kLine + (l32 & 7) * 128);
    const uint32_t w0 = (uint32_t)((wn * 128 >> 3) * kLine + (l32 >> 3) * kLine + (l32 & 7) * 128);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      t.a_rd[q] = a0 + (uint32_t)((((q * 2 + lh) ^ f) & 7) << 4);
      t.b_rd[q] = w0 + (uint32_t)((((q * 2 + lh) ^ f) & 7) << 4);
    }
  }
  f32x16 acc[kMaxMT][4], accx[4];
#pragma unroll
  for (int i = 0; i < kMaxMT; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
  auto product = [&](const char* P, const char* Q) __attribute__((always_inline)) {
    t.a_base = uniform_ptr(P + (size_t)e * p.p_stride);
    t.b_base = uniform_ptr(Q + (size_t)e * p.q_stride);
    gemm_k_loop<kLayNT, kMaxMT, false, 0, false, true>(acc, accx, t, smem, n_steps);
  };
  if constexpr (SPLIT) {                   // the small products first, in units of 2^-11
    product(p.P.lo, p.Q.hi);
    product(p.P.hi, p.Q.lo);
#pragma unroll
    for (int i = 0; i < kMaxMT; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[i][j][r] *= 1.0f / kNsLoScale;
  }
  product(p.P.hi, p.Q.hi);

  // lane: row l32 of each block of 32 x 32, per q the columns q * 8 + lh * 4 .. + 3
  char* region = epilogue_region(smem, wave);
  const int c0 = j0 + wn * 128;
  if (c0 >= p.cols) return;
  const int cols_valid = min(128, p.cols - c0);
#pragma unroll
  for (int mt = 0; mt < kMaxMT; ++mt) {
    const int r0 = i0 + wm * 128 + mt * 32;
    if (r0 >= p.rows) return;
    if constexpr (EPI == kNsOut) {
      const int m = r0 + l32;
#pragma unroll
      for (int nt = 0; nt < 4; ++nt)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int n = c0 + nt * 32 + q * 8 + lh * 4;
          const float o[4] = {acc[mt][nt][q * 4] * p.s_acc, acc[mt][nt][q * 4 + 1] * p.s_acc, acc[mt][nt][q * 4 + 2] * p.s_acc,
                              acc[mt][nt][q * 4 + 3] * p.s_acc};
          if (m < p.M && n < p.N) ns_store_out<T>(p, e, m, n, o);
        }
    } else {
      u32x2 hi[4][4], lo[4][4];
#pragma unroll
      for (int nt = 0; nt < 4; ++nt)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int col = nt * 32 + q * 8 + lh * 4;
          float v[4] = {acc[mt][nt][q * 4] * p.s_acc, acc[mt][nt][q * 4 + 1] * p.s_acc, acc[mt][nt][q * 4 + 2] * p.s_acc,
                        acc[mt][nt][q * 4 + 3] * p.s_acc};
          if constexpr (EPI == kNsPoly) {
            if (col < cols_valid) {
              const size_t at = (size_t)e * p.a_stride + ((size_t)(r0 + l32) * p.ld_c + c0 + col) * 2;
              float a[4];
              unpack_f16x4(*reinterpret_cast<const u32x2*>(p.A.hi + at), a);
              if constexpr (SPLIT) {
                float b[4];
                unpack_f16x4(*reinterpret_cast<const u32x2*>(p.A.lo + at), b);
#pragma unroll
                for (int x = 0; x < 4; ++x) a[x] += b[x] * (1.0f / kNsLoScale);
              }
#pragma unroll
              for (int x = 0; x < 4; ++x) v[x] += p.s_a * a[x] + (r0 + l32 == c0 + col + x ? p.diag : 0.f);
            }
          }
          hi[nt][q] = pack_f16x4(v);
          if constexpr (SPLIT) {
            float h[4];
            unpack_f16x4(hi[nt][q], h);
#pragma unroll
            for (int x = 0; x < 4; ++x) h[x] = (v[x] - h[x]) * kNsLoScale;
            lo[nt][q] = pack_f16x4(h);
          }
        }
      const size_t at = (size_t)e * p.c_stride + ((size_t)r0 * p.ld_c + c0) * 2, att = (size_t)e * p.c_stride + ((size_t)c0 * p.ld_ct + r0) * 2;
      const bool mirror = EPI == kNsNext || i0 != j0;            // a tile on the diagonal is its own mirror
      ns_store_block(region, hi, p.C.hi + at, p.ld_c, mirror ? p.CT.hi + att : nullptr, p.ld_ct, cols_valid);
      if constexpr (SPLIT) ns_store_block(region, lo, p.C.lo + at, p.ld_c, mirror ? p.CT.lo + att : nullptr, p.ld_ct, cols_valid);
    }
  }
}

// Tiles of all matrices, by workgroups that walk on in strides; gram and poly: those on and above the diagonal.
template <int EPI, bool SPLIT, typename T>
__global__ __launch_bounds__(kGemmThreads) __attribute__((amdgpu_waves_per_eu(1, 1))) void ns_gemm_kernel(NsGemmParams p) {
  __shared__ __attribute__((aligned(1024))) char smem[kGemmLdsBytes];
  constexpr bool SYM = EPI == kNsGram || EPI == kNsPoly;
  const int ti = (p.rows + kBM - 1) / kBM, tj = (p.cols + kBN - 1) / kBN;
  const int per = SYM ? ti * (ti + 1) / 2 : ti * tj, total = per * p.n;
  const int G = gridDim.x;
  for (int it = 0; it * G < total; ++it) {
    const int tile = xcd_spread_tile(it, blockIdx.x, G, total);
    if (tile < 0) continue;
    const int e = __builtin_amdgcn_readfirstlane(tile / per);
    int r = tile - e * per, i, j;
    if (SYM) {
      i = 0;
      while (r >= ti - i) r -= ti - i++;
      j = i + r;
    } else {                               // strips of four tile rows, column by column
      const int strip = __builtin_amdgcn_readfirstlane(r / (4 * tj)), h = min(4, ti - 4 * strip);
      r -= strip * 4 * tj;
      j = __builtin_amdgcn_readfirstlane(r / h);
      i = strip * 4 + r - j * h;
    }
    ns_tile<EPI, SPLIT, T>(p, e, i * kBM, j * kBN, smem);
  }
}

// ---- momentum, norm, and the first X ----

struct NsPrepParams {
  const void* g;                           // gradient, or the update itself (momentum null)
  const float* m;                          // momentum
  float* m_out;
  float mu;
  int nesterov;
  double* part;                            // [n][parts] sums of squares
  int parts;
  float scale;                             // 2^x
  float eps;
  NsMat X, XT;                             // [M padded][N padded] and its transpose
  long stride;                             // bytes between matrices
  int M, N, Mp, Np, n;
};

template <typename T> __device__ __forceinline__ float ns_update(const NsPrepParams& p, size_t at) {
  const float g = (float)static_cast<const T*>(p.g)[at];
  if (!p.m) return g;
  const float m = p.m_out[at];
  return p.nesterov ? g + p.mu * m : m;
}

// Sums of squares in 64 bits, so that no update is too large or small; momentum on the way.  In 64 bits they also have no order to speak
// of in the rounded result, and it is fixed all the same.
template <typename T> __global__ __launch_bounds__(256) void ns_norm_kernel(NsPrepParams p) {
  __shared__ double s_sum[4];
  const int e = blockIdx.x / p.parts, part = blockIdx.x % p.parts;
  const size_t n = (size_t)p.M * p.N, base = (size_t)e * n;
  double sum = 0.0;
  for (size_t i = (size_t)part * 256 + threadIdx.x; i < n; i += (size_t)p.parts * 256) {
    float u = (float)static_cast<const T*>(p.g)[base + i];
    if (p.m) {
      const float m = p.mu * p.m[base + i] + u;
      p.m_out[base + i] = m;
      u = p.nesterov ? u + p.mu * m : m;
    }
    sum += (double)u * (double)u;
  }
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) sum += __shfl_xor(sum, o);
  if (lane_id() == 0) s_sum[threadIdx.x / kWave] = sum;
  __syncthreads();
  if (threadIdx.x == 0) p.part[(size_t)e * p.parts + part] = s_sum[0] + s_sum[1] + s_sum[2] + s_sum[3];
}

// Tiles of 64 x 64 of the padded matrix: fp16 straight and transposed.
template <typename T, bool SPLIT> __global__ __launch_bounds__(256) void ns_first_kernel(NsPrepParams p) {
  __shared__ float s[64][65];
  __shared__ double s_norm[4];
  const int tj = p.Np / 64, per = (p.Mp / 64) * tj;
  const int e = blockIdx.x / per, r = blockIdx.x % per, i0 = (r / tj) * 64, j0 = (r % tj) * 64;
  double sum = threadIdx.x < (unsigned)p.parts ? p.part[(size_t)e * p.parts + threadIdx.x] : 0.0;
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) sum += __shfl_xor(sum, o);
  if (lane_id() == 0) s_norm[threadIdx.x / kWave] = sum;
  __syncthreads();
  sum = s_norm[0] + s_norm[1] + s_norm[2] + s_norm[3];
  const double f = (double)p.scale / (sqrt(sum) + (double)p.eps);   // beyond fp32 for a tiny norm
  const int l = threadIdx.x & 63, w = threadIdx.x / 64;
  for (int k = w; k < 64; k += 4) {
    const int i = i0 + k, j = j0 + l;
    s[k][l] = i < p.M && j < p.N ? (float)((double)ns_update<T>(p, ((size_t)e * p.M + i) * p.N + j) * f) : 0.f;
  }
  __syncthreads();
  auto store = [&](const NsMat& m, size_t at, float v) __attribute__((always_inline)) {
    const _Float16 h = (_Float16)v;
    *reinterpret_cast<_Float16*>(m.hi + at) = h;
    if constexpr (SPLIT) *reinterpret_cast<_Float16*>(m.lo + at) = (_Float16)((v - (float)h) * kNsLoScale);
  };
  for (int k = w; k < 64; k += 4) {
    store(p.X, (size_t)e * p.stride + ((size_t)(i0 + k) * p.Np + j0 + l) * 2, s[k][l]);
    store(p.XT, (size_t)e * p.stride + ((size_t)(j0 + k) * p.Mp + i0 + l) * 2, s[l][k]);
  }
}

}  // namespace moe
