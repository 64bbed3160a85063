// An update made orthogonal by Newton-Schulz products, and the optimiser's step around it.
//
//   X0 = u / (|u| + eps) (Frobenius norm), turned so that it has S <= L rows;  per step with its coefficients a, b, c
//   A = X X^T;  B = a I + b A + c A^2;  X <- B X          every singular value s of X becomes a s + b s^3 + c s^5
//
// Per step 3 S^2 L + S^3 multiply-adds' flops, as A and B are symmetric and half of their tiles are computed: bound by the matrix cores where
// matrices are large (bf16 storage, the next X of 4 x 4096 x 7168: 822 us = 1.17 PFLOP/s with the cores busy for 73 % of the clocks, which the
// power limit holds at 1.5 GHz; library products of that size reach 1.09 to 1.29), by the latency of a chain of 2 + 3 steps launches where they
// are small (200 x 330: 4.1 to 5.6 us each).
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
// fp32 storage: operands are pairs of fp16, hi and the rest, products hi hi + hi lo + lo hi in one sum, so 22 bits.  Their scale brings the
// bound of the entries, not the entries, to the top of the range, 2^14: a rest is then off by 2^-25 at most, below 2^-32 of a typical entry.
#pragma once
#include "rows.h"
#include "tile128.h"

namespace moe {

constexpr int kNsMaxParts = 256;           // partial sums of squares per matrix
constexpr int kNsPad = 64;

enum NsEpilogue { kNsGram = 0, kNsPoly = 1, kNsNext = 2, kNsOut = 3 };
constexpr bool ns_symmetric(int epi) { return epi == kNsGram || epi == kNsPoly; }

// Matrices in between: fp16 [rows][k]; as pairs [rows][k / 32][hi 32 | lo 32], so that a line of 128 bytes has both.
struct NsGemmParams {
  const char *P, *Q;                       // C[i,j] = sum over k of P[i,k] Q[j,k]
  char *C, *CT;                            // straight and transposed (gram, poly: the same array)
  const char* A;                           // poly: the matrix that b is for
  long p_stride, q_stride, c_stride, a_stride;   // bytes between matrices (of CT: c_stride)
  int rows, cols, K;                       // multiples of 64
  int ld_c, ld_ct;                         // elements
  int n;                                   // matrices
  int first, tiles;                        // those of all tiles that this launch does
  float* part;                             // sums along a share of k: [tile of the launch][splits][128 x 128 in the waves' order]
  int splits;
  float s_acc, s_a, diag;                  // result = s_acc * sum + s_a * A + diag * I
  // out: o = s_acc * sum, M x N of them, weights w [M,N]
  const void* w;                           // null: out = o
  float* master;                           // fp32 weights, updated in place, instead of w
  void* out;
  float w_keep, w_step;                    // out = w_keep * w - w_step * o
  int M, N;
};

typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) char* lds_ptr;
typedef __attribute__((address_space(3))) u32x2* lds_u32x2_ptr;
typedef __attribute__((address_space(3))) u32x4* lds_u32x4_ptr;
typedef __attribute__((address_space(3))) f32x4* lds_f32x4_ptr;

__device__ __forceinline__ u32x2 pack_f16x4(const float (&v)[4]) {
  return __builtin_bit_cast(u32x2, (f16x4){(_Float16)v[0], (_Float16)v[1], (_Float16)v[2], (_Float16)v[3]});
}
__device__ __forceinline__ void unpack_f16x4(u32x2 p, float (&v)[4]) {
  const f16x4 h = __builtin_bit_cast(f16x4, p);
#pragma unroll
  for (int x = 0; x < 4; ++x) v[x] = (float)h[x];
}
__device__ __forceinline__ void lds_settled() {            // a wave's own LDS accesses, which complete in order
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// Four columns n .. n + 3 of a row.  VEC: all four are there, and aligned; else those below N.
template <typename T, bool VEC> __device__ __forceinline__ f32x4 ns_get(const T* src, size_t at, int n, int N) {
  typedef T T4 __attribute__((ext_vector_type(4)));
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
  if constexpr (VEC) {
    const T4 a = *reinterpret_cast<const T4*>(src + at);
#pragma unroll
    for (int x = 0; x < 4; ++x) v[x] = (float)a[x];
  } else {
#pragma unroll
    for (int x = 0; x < 4; ++x)
      if (n + x < N) v[x] = (float)src[at + x];
  }
  return v;
}
template <typename T, bool VEC> __device__ __forceinline__ void ns_put(T* dst, size_t at, int n, int N, f32x4 v) {
  typedef T T4 __attribute__((ext_vector_type(4)));
  if constexpr (VEC) {
    T4 o;
#pragma unroll
    for (int x = 0; x < 4; ++x) o[x] = (T)v[x];
    *reinterpret_cast<T4*>(dst + at) = o;
  } else {
#pragma unroll
    for (int x = 0; x < 4; ++x)
      if (n + x < N) dst[at + x] = (T)v[x];
  }
}
// Eight rows, every fourth from m on, of the result: weights, or the update itself.  All weights are read ahead of the first store: they may be
// the output, so no load passes a store by itself.
template <typename T, bool VEC> __device__ __forceinline__ void ns_put_rows(const NsGemmParams& p, int e, int m, int n, f32x4 (&o)[8]) {
  const size_t at = ((size_t)e * p.M + m) * p.N + n, step = (size_t)4 * p.N;
  const int rows = n < p.N ? (p.M - m + 3) / 4 : 0;
  if (p.master || p.w) {
    f32x4 w[8];
#pragma unroll
    for (int it = 0; it < 8; ++it)
      if (it < rows) w[it] = p.master ? ns_get<float, VEC>(p.master, at + it * step, n, p.N) : ns_get<T, VEC>(static_cast<const T*>(p.w), at + it * step, n, p.N);
#pragma unroll
    for (int it = 0; it < 8; ++it) {
#pragma unroll
      for (int x = 0; x < 4; ++x) o[it][x] = __builtin_fmaf(p.w_keep, w[it][x], -(p.w_step * o[it][x]));
      if (p.master && it < rows) ns_put<float, VEC>(p.master, at + it * step, n, p.N, o[it]);
    }
  }
#pragma unroll
  for (int it = 0; it < 8; ++it)
    if (it < rows) ns_put<T, VEC>(static_cast<T*>(p.out), at + it * step, n, p.N, o[it]);
}

// A wave's 32 rows x 32 NB columns of a result from (r0, c0) on, by way of its LDS region (kNsRegion bytes).
// acc[nt]: lane (l32, lh) holds row l32 and, per q, columns 32 nt + 8 q + 4 lh .. + 3.
constexpr int kNsRegion = 16384;
template <int EPI, bool SPLIT, typename T, int NB>
__device__ __forceinline__ void ns_block(const NsGemmParams& p, const f32x16 (&acc)[NB], char* region, int e, int r0, int c0) {
  int lane = lane_id();
  asm volatile("" : "+v"(lane));           // see store_block_via_lds
  const int l32 = lane & 31, lh = lane >> 5;
  const lds_ptr base = (lds_ptr)region;
  // Fused by hand, here and below, so that a matrix's result is the same bits whichever tiles it goes through (shares of a tile's sum, which depend
  // on the matrices beside it, add up in another order).
  auto value = [&](int nt, int q, int x) __attribute__((always_inline)) {
    return acc[nt][q * 4 + x];
  };
  if constexpr (EPI == kNsOut) {           // rows of fp32, 64 columns at a time
    constexpr int kRow = 64 * 4 + 16;
    static_assert(32 * kRow <= kNsRegion, "region");
#pragma unroll
    for (int h = 0; h < NB / 2; ++h) {
#pragma unroll
      for (int nt = 0; nt < 2; ++nt)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          *(lds_f32x4_ptr)(base + l32 * kRow + (nt * 32 + q * 8 + lh * 4) * 4) =
              f32x4{value(2 * h + nt, q, 0), value(2 * h + nt, q, 1), value(2 * h + nt, q, 2), value(2 * h + nt, q, 3)} * p.s_acc;
      lds_settled();
      const int ch = lane & 15, r4 = lane >> 4, n = c0 + h * 64 + ch * 4;
      f32x4 o[8];
#pragma unroll
      for (int it = 0; it < 8; ++it) o[it] = *(lds_f32x4_ptr)(base + (it * 4 + r4) * kRow + ch * 16);
      if (p.N % 4 == 0) ns_put_rows<T, true>(p, e, r0 + r4, n, o);
      else ns_put_rows<T, false>(p, e, r0 + r4, n, o);
      wait_lgkmcnt0();
      lds_settled();
    }
  } else {
    constexpr int kRow = 32 * NB * 2 + 16, kHalf = 32 * kRow, kLanes = NB * 4, kRows = kWave / kLanes, kIts = 32 / kRows;
    static_assert((SPLIT ? 2 : 1) * kHalf <= kNsRegion, "region");
    const int cols_valid = p.cols - c0;    // a multiple of 64
    const int r = lane / kLanes, ch = lane % kLanes;
    // Of a symmetric matrix: the blocks of 64 x 64 on the diagonal and above it, the latter also as those below (sums with the operands exchanged
    // differ by a last bit now and then: that way the matrix is symmetric, and the same whichever tiles it is made of, but for shares).
    constexpr bool SYM = ns_symmetric(EPI);
    const bool col_ok = ch * 8 < cols_valid && (!SYM || (c0 + ch * 8) >> 6 >= r0 >> 6);
    // bytes from a matrix's first to element (row, col) of 8-column chunk `col`, col a multiple of 8
    auto offset = [&](int row, int col, int ld) __attribute__((always_inline)) {
      return SPLIT ? (size_t)row * ld * 4 + (size_t)(col >> 5) * 128 + (col & 31) * 2 : ((size_t)row * ld + col) * 2;
    };
    if constexpr (EPI == kNsPoly) {        // A's block comes in whole lines as well
      const char* A = p.A + (size_t)e * p.a_stride;
#pragma unroll
      for (int h = 0; h < (SPLIT ? 2 : 1); ++h) {
        u32x4 v[kIts];
#pragma unroll
        for (int it = 0; it < kIts; ++it)
          v[it] = *reinterpret_cast<const u32x4*>(A + offset(r0 + it * kRows + r, ch * 8 < cols_valid ? c0 + ch * 8 : c0, p.ld_c) + h * 64);
#pragma unroll
        for (int it = 0; it < kIts; ++it) *(lds_u32x4_ptr)(base + h * kHalf + (it * kRows + r) * kRow + ch * 16) = v[it];
      }
      lds_settled();
    }
    const lds_ptr mine = base + l32 * kRow + lh * 8;
#pragma unroll
    for (int nt = 0; nt < NB; ++nt)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const lds_ptr at = mine + (nt * 32 + q * 8) * 2;
        float v[4] = {value(nt, q, 0), value(nt, q, 1), value(nt, q, 2), value(nt, q, 3)};
        if constexpr (EPI == kNsPoly) {
          float a[4], b[4] = {0.f, 0.f, 0.f, 0.f};
          unpack_f16x4(*(lds_u32x2_ptr)at, a);
          if constexpr (SPLIT) unpack_f16x4(*(lds_u32x2_ptr)(at + kHalf), b);
          const int d = r0 + l32 - (c0 + nt * 32 + q * 8 + lh * 4);      // the column of the diagonal
#pragma unroll
          for (int x = 0; x < 4; ++x)
            v[x] = __builtin_fmaf(v[x], p.s_acc, __builtin_fmaf(p.s_a, SPLIT ? a[x] + b[x] : a[x], d == x ? p.diag : 0.f));
        } else {
#pragma unroll
          for (int x = 0; x < 4; ++x) v[x] *= p.s_acc;
        }
        const u32x2 hi = pack_f16x4(v);
        *(lds_u32x2_ptr)at = hi;
        if constexpr (SPLIT) {
          float h[4];
          unpack_f16x4(hi, h);
#pragma unroll
          for (int x = 0; x < 4; ++x) h[x] = v[x] - h[x];
          *(lds_u32x2_ptr)(at + kHalf) = pack_f16x4(h);
        }
      }
    lds_settled();
    char* C = p.C + (size_t)e * p.c_stride;
    char* CT = p.CT + (size_t)e * p.c_stride;
#pragma unroll
    for (int h = 0; h < (SPLIT ? 2 : 1); ++h) {
      u32x4 v[kIts];
#pragma unroll
      for (int it = 0; it < kIts; ++it) v[it] = *(lds_u32x4_ptr)(base + h * kHalf + (it * kRows + r) * kRow + ch * 16);
#pragma unroll
      for (int it = 0; it < kIts; ++it)
        if (col_ok) *reinterpret_cast<u32x4*>(C + offset(r0 + it * kRows + r, c0 + ch * 8, p.ld_c) + h * 64) = v[it];
      if (!SYM || (c0 + NB * 32 - 1) >> 6 > r0 >> 6) {
        // 16 lanes read 4 rows x 16 columns and get a column's 4 rows each; lane (g, i): rows 8 g .. 8 g + 7 of column i
        const int g = lane >> 4, i = lane & 15;
        const lds_ptr at = base + h * kHalf + (8 * g + (i >> 2)) * kRow + (i & 3) * 8;
        u32x4 t[NB * 2];
#pragma unroll
        for (int cg = 0; cg < NB * 2; ++cg) {
          const u32x2 a = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_ptr)(at + cg * 32)));
          const u32x2 b = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_ptr)(at + cg * 32 + 4 * kRow)));
          t[cg] = u32x4{a.x, a.y, b.x, b.y};
        }
#pragma unroll
        for (int cg = 0; cg < NB * 2; ++cg)
          if (cg * 16 < cols_valid && (!SYM || (c0 + cg * 16) >> 6 > r0 >> 6))
            *reinterpret_cast<u32x4*>(CT + offset(c0 + cg * 16 + i, r0 + 8 * g, p.ld_ct) + h * 64) = t[cg];
      }
    }
    wait_lgkmcnt0();                       // the region is free again
    lds_settled();
  }
}

// The update's 128 x 128 of a wave from (r0, c0) on, by 32 rows x 64 columns.  W: type of the weights that are read (float: the master, else p.w), or
// void.  Their blocks are fetched eight, or of four bytes three, ahead: a block's way from HBM each time took 34 us per tile (4 x 7168 x 4096: 1062 us,
// so 864).
template <typename T, typename W, bool VEC>
__device__ __forceinline__ void ns_out128(const NsGemmParams& p, f32x16 (&acc)[kMaxMT][4], char* region, int e, int r0, int c0) {
  constexpr bool kWeights = !std::is_void<W>::value, kMaster = std::is_same<W, float>::value;
  constexpr int kRow = 64 * 4 + 16, kBlocks = 2 * kMaxMT, kAhead = kMaster ? 3 : VEC ? kBlocks : kBlocks / 2;
  typedef typename std::conditional<kWeights, W, float>::type WS;
  typedef WS W4 __attribute__((ext_vector_type(4)));
  int lane = lane_id();
  asm volatile("" : "+v"(lane));
  const int l32 = lane & 31, lh = lane >> 5, ch = lane & 15, r4 = lane >> 4;
  const lds_ptr base = (lds_ptr)region;
  const WS* src = kMaster ? reinterpret_cast<const WS*>(p.master) : static_cast<const WS*>(p.w);
  W4 w[kAhead][8];
  auto place = [&](int b, int it, int& n) __attribute__((always_inline)) {
    const int m = r0 + (b >> 1) * 32 + r4 + it * 4;
    n = c0 + (b & 1) * 64 + ch * 4;
    return m < p.M && n < p.N ? ((size_t)e * p.M + m) * p.N + n : ~(size_t)0;
  };
  auto fetch = [&](auto bc) __attribute__((always_inline)) {
    constexpr int b = decltype(bc)::value;
    if constexpr (kWeights && b < kBlocks) {
#pragma unroll
      for (int it = 0; it < 8; ++it) {
        int n;
        const size_t at = place(b, it, n);
        W4 v = {};
        if (at != ~(size_t)0) {
          if constexpr (VEC) {
            v = *reinterpret_cast<const W4*>(src + at);
          } else {
#pragma unroll
            for (int x = 0; x < 4; ++x)
              if (n + x < p.N) v[x] = src[at + x];
          }
        }
        w[b % kAhead][it] = v;
      }
    }
  };
  static_for<0, kAhead>([&](auto bc) __attribute__((always_inline)) { fetch(bc); });
  __builtin_amdgcn_s_barrier();            // every wave has read its last operands, its copies have landed
  static_for<0, kBlocks>([&](auto bc) __attribute__((always_inline)) {
    constexpr int b = decltype(bc)::value, mt = b >> 1, h = b & 1;
#pragma unroll
    for (int nt = 0; nt < 2; ++nt) {
      asm volatile("" : "+a"(acc[mt][2 * h + nt]));          // until here they stay in the accumulators
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const f32x16& a = acc[mt][2 * h + nt];
        *(lds_f32x4_ptr)(base + l32 * kRow + (nt * 32 + q * 8 + lh * 4) * 4) = f32x4{a[q * 4], a[q * 4 + 1], a[q * 4 + 2], a[q * 4 + 3]} * p.s_acc;
      }
    }
    lds_settled();
    f32x4 o[8];
#pragma unroll
    for (int it = 0; it < 8; ++it) o[it] = *(lds_f32x4_ptr)(base + (it * 4 + r4) * kRow + ch * 16);
#pragma unroll
    for (int it = 0; it < 8; ++it) {
      int n;
      const size_t at = place(b, it, n);
      if constexpr (kWeights) {
#pragma unroll
        for (int x = 0; x < 4; ++x) o[it][x] = __builtin_fmaf(p.w_keep, (float)w[b % kAhead][it][x], -(p.w_step * o[it][x]));
      }
      if (at != ~(size_t)0) {
        if constexpr (kMaster) ns_put<float, VEC>(p.master, at, n, p.N, o[it]);
        ns_put<T, VEC>(static_cast<T*>(p.out), at, n, p.N, o[it]);
      }
    }
    wait_lgkmcnt0();
    lds_settled();
    fetch(std::integral_constant<int, b + kAhead>{});
  });
}

// One tile of 256 x 256 by four waves of 128 x 128 (the K loop of the grouped products): rows from i0, columns from j0 of matrix e.
template <int EPI, typename T, typename W, bool VEC>
__device__ __forceinline__ void ns_tile256(const NsGemmParams& p, int e, int i0, int j0, char* smem) {
  int lane = lane_id();
  asm volatile("" : "+v"(lane));
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave >> 1, wn = wave & 1;
  const int l32 = lane & 31, lh = lane >> 5;
  GemmTileCtx t;
  t.wave = wave;
  t.nA = 8;
  t.lda_bytes = t.ldb_bytes = p.K * 2;
  const int kc_r = lane >> 3;
  const int kc_c = (lane & 7) ^ ((4 * (wave & 1) + (kc_r >> 1)) & 7);
#pragma unroll
  for (int i = 0; i < 8; ++i) {            // rows past the end read the last one again; they are not stored
    const int r = (wave + 4 * i) * 8 + kc_r;
    t.a_off[i] = (uint32_t)min(i0 + r, p.rows - 1) * (uint32_t)t.lda_bytes + (uint32_t)(kc_c * 16);
    t.b_off[i] = (uint32_t)min(j0 + r, p.cols - 1) * (uint32_t)t.ldb_bytes + (uint32_t)(kc_c * 16);
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
  t.a_base = uniform_ptr(p.P + (size_t)e * p.p_stride);
  t.b_base = uniform_ptr(p.Q + (size_t)e * p.q_stride);
  int n_steps = p.K / kBK;
  asm volatile("" : "+s"(n_steps));        // else what follows from it is kept over the tiles, beyond the registers
  gemm_k_loop<kLayNT, kMaxMT, false, 0, false, true>(acc, accx, t, smem, n_steps);
  const int c0 = j0 + wn * 128;
  if constexpr (EPI == kNsOut) {
    ns_out128<T, W, VEC>(p, acc, smem + wave * kNsRegion, e, i0 + wm * 128, c0);
    __builtin_amdgcn_s_barrier();                            // the next tile's copies go to the same places
  } else {
    // The regions of epilogue_region lie clear of the next tile's first copies, so waves go on to it one by one; rows of fp32 need more.
    char* region = epilogue_region(smem, wave);
#pragma unroll
    for (int mt = 0; mt < kMaxMT; ++mt) {
      const int r0 = i0 + wm * 128 + mt * 32;
      if (r0 >= p.rows || c0 >= p.cols) continue;
#pragma unroll
      for (int nt = 0; nt < 4; ++nt) asm volatile("" : "+a"(acc[mt][nt]));   // until here they stay in the accumulators
      ns_block<EPI, false, T, 4>(p, acc[mt], region, e, r0, c0);
    }
  }
}

// A wave's blocks of 32 x 64 of a result, from row r0 of its BI blocks on.
template <int EPI, bool SPLIT, typename T, int BI>
__device__ __forceinline__ void ns_blocks(const NsGemmParams& p, const f32x16 (&acc)[BI][2], char* region, int e, int r0, int c0) {
#pragma unroll
  for (int mt = 0; mt < BI; ++mt)
    if (r0 + mt * 32 < p.rows && c0 < p.cols) ns_block<EPI, SPLIT, T, 2>(p, acc[mt], region, e, r0 + mt * 32, c0);
}

// One tile of SIDE x SIDE (tile128.h).  share, item: with splits > 1 the tile's k's are dealt to that many workgroups, of which this is number
// `share`; its sums go to place `item`.
template <int SIDE, int EPI, bool SPLIT, typename T, int STAGES, bool SHARES>
__device__ __forceinline__ void ns_tile(const NsGemmParams& p, int e, int i0, int j0, int share, int item, char* smem) {
  constexpr int BI = SIDE / 64;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = lane_id();
  const int row_bytes = p.K * (SPLIT ? 4 : 2), all_steps = row_bytes / 128;
  const int first_step = SHARES ? all_steps * share / p.splits : 0;
  const int n_steps = SHARES ? all_steps * (share + 1) / p.splits - first_step : all_steps;
  f32x16 acc[BI][2];
  tile_multiply<SIDE, SPLIT, STAGES>(p.P + (size_t)e * p.p_stride + (size_t)first_step * 128, p.Q + (size_t)e * p.q_stride + (size_t)first_step * 128,
                                     row_bytes, p.rows, p.cols, i0, j0, n_steps, smem, acc);
  if constexpr (SHARES) {
    static_assert(SIDE == 128, "shares");
    float* dst = p.part + ((size_t)item * 4 + wave) * 4096 + lane;
#pragma unroll
    for (int i = 0; i < BI; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) dst[((i * 2 + j) * 16 + r) * 64] = acc[i][j][r];
  } else {
    ns_blocks<EPI, SPLIT, T, BI>(p, acc, smem + wave * kNsRegion, e, i0 + (SIDE == 128 ? (wave >> 1) * 64 : wave * 32),
                                        j0 + (SIDE == 128 ? (wave & 1) * 64 : 0));
  }
}

// Tile r of a matrix of ti x tj tiles.  SYM: those on and above the diagonal, row by row; else strips of four tile rows, column by column,
// so that tiles under way together share operands.
template <bool SYM> __device__ __forceinline__ void ns_tile_at(int r, int ti, int tj, int& i, int& j) {
  if (SYM) {
    i = 0;
    while (r >= ti - i) r -= ti - i++;
    j = i + r;
  } else {
    const int strip = __builtin_amdgcn_readfirstlane(r / (4 * tj)), h = min(4, ti - 4 * strip);
    r -= strip * 4 * tj;
    j = __builtin_amdgcn_readfirstlane(r / h);
    i = strip * 4 + r - j * h;
  }
}

// Whole tiles of 256 x 256, by workgroups that walk on in strides.
template <int EPI, typename T, typename W, bool VEC>
__global__ __launch_bounds__(kGemmThreads) __attribute__((amdgpu_waves_per_eu(1, 1))) void ns_gemm256_kernel(NsGemmParams p) {
  __shared__ __attribute__((aligned(1024))) char smem[kGemmLdsBytes];
  constexpr bool SYM = ns_symmetric(EPI);
  const int ti = (p.rows + kBM - 1) / kBM, tj = (p.cols + kBN - 1) / kBN;
  const int per = SYM ? ti * (ti + 1) / 2 : ti * tj, G = gridDim.x;
  for (int it = 0; it * G < p.tiles; ++it) {
    const int tile = xcd_spread_tile(it, blockIdx.x, G, p.tiles);
    if (tile < 0) continue;
    const int at = p.first + tile, e = __builtin_amdgcn_readfirstlane(at / per);
    int i, j;
    ns_tile_at<SYM>(at - e * per, ti, tj, i, j);
    ns_tile256<EPI, T, W, VEC>(p, e, i * kBM, j * kBN, smem);
  }
}

// Tile `at` of 128 x 128.  QUARTERS: at / 4 counts tiles of 256 x 256.  Returns false where there is none.
template <bool SYM, bool QUARTERS> __device__ __forceinline__ bool ns_tile128_at(const NsGemmParams& p, int at, int& e, int& i, int& j) {
  constexpr int kSide = QUARTERS ? 256 : 128;
  const int ti = (p.rows + kSide - 1) / kSide, tj = (p.cols + kSide - 1) / kSide;
  const int per = SYM ? ti * (ti + 1) / 2 : ti * tj, big = QUARTERS ? at >> 2 : at;
  e = __builtin_amdgcn_readfirstlane(big / per);
  ns_tile_at<SYM>(big - e * per, ti, tj, i, j);
  if (!QUARTERS) return true;
  i = 2 * i + ((at >> 1) & 1);
  j = 2 * j + (at & 1);
  return i * 128 < p.rows && j * 128 < p.cols && !(SYM && i > j);
}

// Tiles of 128 x 128 (p.first .. p.first + p.tiles - 1), one to a workgroup, or p.splits workgroups to each.
template <int EPI, bool SPLIT, typename T, bool QUARTERS, int STAGES, bool SHARES>
__global__ __launch_bounds__(256, STAGES == 2 ? 2 : 1) void ns_gemm128_kernel(NsGemmParams p) {
  static_assert(STAGES == 2 || STAGES == 4, "stages");
  __shared__ __attribute__((aligned(1024))) char smem[STAGES * tile_stage(128)];
  // workgroups are dealt to the dies in turn: a die's take a contiguous eighth
  const int item = xcd_spread_tile(0, blockIdx.x, gridDim.x, SHARES ? p.tiles * p.splits : p.tiles);
  if (item < 0) return;
  const int tile = SHARES ? __builtin_amdgcn_readfirstlane(item / p.splits) : item;
  int e, i, j;
  if (!ns_tile128_at<ns_symmetric(EPI), QUARTERS>(p, p.first + tile, e, i, j)) return;
  ns_tile<128, EPI, SPLIT, T, STAGES, SHARES>(p, e, i * 128, j * 128, SHARES ? item - tile * p.splits : 0, item, smem);
}

// Tiles of 256 x 256 of pairs, one to a workgroup: 4 x 4096 x 4096, the next X 1273 us, 1.30 PFLOP/s of its three products.
template <int EPI, typename T>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(1, 1))) void ns_gemm256_pairs_kernel(NsGemmParams p) {
  __shared__ __attribute__((aligned(1024))) char smem[2 * tile_stage(256)];
  constexpr bool SYM = ns_symmetric(EPI);
  const int tile = xcd_spread_tile(0, blockIdx.x, gridDim.x, p.tiles);
  if (tile < 0) return;
  const int ti = (p.rows + 255) / 256, tj = (p.cols + 255) / 256, per = SYM ? ti * (ti + 1) / 2 : ti * tj;
  const int at = p.first + tile, e = __builtin_amdgcn_readfirstlane(at / per);
  int i, j;
  ns_tile_at<SYM>(at - e * per, ti, tj, i, j);
  f32x16 acc[4][4];
  tile_multiply<256, true, 2>(p.P + (size_t)e * p.p_stride, p.Q + (size_t)e * p.q_stride, p.K * 4, p.rows, p.cols, i * 256, j * 256, p.K / 32, smem, acc);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
  for (int mt = 0; mt < 4; ++mt)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int r0 = i * 256 + (wave >> 1) * 128 + mt * 32, c0 = j * 256 + (wave & 1) * 128 + h * 64;
      if (r0 >= p.rows || c0 >= p.cols) continue;
#pragma unroll
      for (int nt = 0; nt < 2; ++nt) asm volatile("" : "+a"(acc[mt][2 * h + nt]));   // until here they stay in the accumulators
      const f32x16 block[2] = {acc[mt][2 * h], acc[mt][2 * h + 1]};
      ns_block<EPI, true, T, 2>(p, block, smem + wave * kNsRegion, e, r0, c0);
    }
}

// Tiles of 64 x 64, one to a workgroup.
template <int EPI, bool SPLIT, typename T>
__global__ __launch_bounds__(128, 2) void ns_gemm64_kernel(NsGemmParams p) {
  __shared__ __attribute__((aligned(1024))) char smem[4 * tile_stage(64)];
  const int tile = xcd_spread_tile(0, blockIdx.x, gridDim.x, p.tiles);
  if (tile < 0) return;
  constexpr bool SYM = ns_symmetric(EPI);
  const int ti = p.rows / 64, tj = p.cols / 64, per = SYM ? ti * (ti + 1) / 2 : ti * tj;
  const int e = __builtin_amdgcn_readfirstlane(tile / per);
  int i, j;
  ns_tile_at<SYM>(tile - e * per, ti, tj, i, j);
  ns_tile<64, EPI, SPLIT, T, 4, false>(p, e, i * 64, j * 64, 0, 0, smem);
}

// The shares of a tile joined, in their order: a workgroup of one wave for each of the tile's eight blocks of 32 x 64, as few tiles are left over and
// a CU pulls in only some 50 bytes a nanosecond, four shares' loads ahead of the first sum (four waves in one workgroup, a share at a time, 16 shares:
// 16 us).
template <int EPI, bool SPLIT, typename T, bool QUARTERS>
__global__ __launch_bounds__(64) void ns_join_kernel(NsGemmParams p) {
  __shared__ __attribute__((aligned(1024))) char smem[kNsRegion];
  const int tile = blockIdx.x >> 3, wave = (blockIdx.x >> 1) & 3, mt = blockIdx.x & 1;
  int e, i, j;
  if (!ns_tile128_at<ns_symmetric(EPI), QUARTERS>(p, p.first + tile, e, i, j)) return;
  const float* src = p.part + ((size_t)tile * p.splits * 4 + wave) * 4096 + mt * 2048 + lane_id();
  f32x16 acc[1][2];
#pragma unroll
  for (int x = 0; x < 32; ++x) acc[0][x >> 4][x & 15] = 0.f;
  for (int s = 0; s < p.splits; s += 4) {
    float v[4][32];
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int x = 0; x < 32; ++x) v[u][x] = src[(size_t)min(s + u, p.splits - 1) * 4 * 4096 + x * 64];
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int x = 0; x < 32; ++x) acc[0][x >> 4][x & 15] += s + u < p.splits ? v[u][x] : 0.f;
  }
  ns_blocks<EPI, SPLIT, T, 1>(p, acc, smem, e, i * 128 + (wave >> 1) * 64 + mt * 32, j * 128 + (wave & 1) * 64);
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
  char *X, *XT;                            // [M padded][N padded] and its transpose
  long stride;                             // bytes between matrices
  int M, N, Mp, Np, n;
};

// Sums of squares in 64 bits, so that no update is too large or too small for them; momentum on the way.  A workgroup takes every
// parts-th piece of 2048 values, a thread eight of them.  Bound by HBM: 4 x 4096 x 7168 in bf16 with momentum 203 us, 5.8 TB/s.
template <typename T> __global__ __launch_bounds__(256) void ns_norm_kernel(NsPrepParams p) {
  __shared__ double s_sum[4];
  const int e = blockIdx.x / p.parts, part = blockIdx.x % p.parts;
  const size_t n = (size_t)p.M * p.N, base = (size_t)e * n;
  const T* g = static_cast<const T*>(p.g) + base;
  double sum = 0.0;
  for (size_t i = ((size_t)part * 256 + threadIdx.x) * 8; i < n; i += (size_t)p.parts * 2048) {
    float u[8];
    if (i + 8 <= n) {
      const Raw8<T> a = raw_load<T, false>(g + i, 0, 8);
#pragma unroll
      for (int x = 0; x < 8; ++x) u[x] = raw_get<T>(a, x);
      if (p.m) {
        const Raw8<float> b = raw_load<float, false>(p.m + base + i, 0, 8);
        float m[8];
#pragma unroll
        for (int x = 0; x < 8; ++x) {
          m[x] = p.mu * raw_get<float>(b, x) + u[x];
          u[x] = p.nesterov ? u[x] + p.mu * m[x] : m[x];
        }
        raw_store<float, false>(p.m_out + base + i, 0, 8, raw_pack<float>(m));
      }
    } else {
#pragma unroll
      for (int x = 0; x < 8; ++x) {
        u[x] = 0.f;
        if (i + x >= n) continue;
        u[x] = (float)g[i + x];
        if (p.m) {
          const float m = p.mu * p.m[base + i + x] + u[x];
          p.m_out[base + i + x] = m;
          u[x] = p.nesterov ? u[x] + p.mu * m : m;
        }
      }
    }
#pragma unroll
    for (int x = 0; x < 8; ++x) sum += (double)u[x] * (double)u[x];
  }
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) sum += __shfl_xor(sum, o);
  if (lane_id() == 0) s_sum[threadIdx.x / kWave] = sum;
  __syncthreads();
  if (threadIdx.x == 0) p.part[(size_t)e * p.parts + part] = s_sum[0] + s_sum[1] + s_sum[2] + s_sum[3];
}

// Tiles of 64 x 64 of the padded matrix: fp16 straight, and transposed by way of LDS; a thread has eight columns of two rows, then
// eight rows of two columns.  Bound by HBM: 4 x 4096 x 7168 in bf16 with momentum 255 us, 4.6 TB/s.
template <typename T, bool SPLIT> __global__ __launch_bounds__(256) void ns_first_kernel(NsPrepParams p) {
  __shared__ float s[64][65];
  __shared__ double s_norm[4];
  const int tj = p.Np / 64, per = (p.Mp / 64) * tj;
  const int e = blockIdx.x / per, r = blockIdx.x % per, i0 = (r / tj) * 64, j0 = (r % tj) * 64;
  const int ch = threadIdx.x & 7, row = threadIdx.x >> 3;
  float u[2][8];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int i = i0 + row + 32 * h, j = j0 + ch * 8;
    const size_t at = ((size_t)e * p.M + i) * p.N + j;
    const T* g = static_cast<const T*>(p.g) + at;
    if (i < p.M && j + 8 <= p.N) {
      const Raw8<T> a = raw_load<T, false>(g, 0, 8);
#pragma unroll
      for (int x = 0; x < 8; ++x) u[h][x] = raw_get<T>(a, x);
      if (p.m) {
        const Raw8<float> b = raw_load<float, false>(p.m_out + at, 0, 8);
#pragma unroll
        for (int x = 0; x < 8; ++x) u[h][x] = p.nesterov ? u[h][x] + p.mu * raw_get<float>(b, x) : raw_get<float>(b, x);
      }
    } else {
#pragma unroll
      for (int x = 0; x < 8; ++x) {
        u[h][x] = 0.f;
        if (i >= p.M || j + x >= p.N) continue;
        u[h][x] = (float)g[x];
        if (p.m) u[h][x] = p.nesterov ? u[h][x] + p.mu * p.m_out[at + x] : p.m_out[at + x];
      }
    }
  }
  double sum = threadIdx.x < (unsigned)p.parts ? p.part[(size_t)e * p.parts + threadIdx.x] : 0.0;
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) sum += __shfl_xor(sum, o);
  if (lane_id() == 0) s_norm[threadIdx.x / kWave] = sum;
  __syncthreads();
  sum = s_norm[0] + s_norm[1] + s_norm[2] + s_norm[3];
  const double f = (double)p.scale / (sqrt(sum) + (double)p.eps);   // beyond fp32 for a tiny norm
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int x = 0; x < 8; ++x) {
      u[h][x] = (float)((double)u[h][x] * f);
      s[row + 32 * h][ch * 8 + x] = u[h][x];
    }
  auto store = [&](char* m, int i, int j, int ld, const float (&v)[8]) __attribute__((always_inline)) {
    float a[4], b[4];
#pragma unroll
    for (int x = 0; x < 4; ++x) { a[x] = v[x]; b[x] = v[4 + x]; }
    const u32x2 h0 = pack_f16x4(a), h1 = pack_f16x4(b);
    char* at = m + (size_t)e * p.stride + (SPLIT ? (size_t)i * ld * 4 + (size_t)(j >> 5) * 128 + (j & 31) * 2 : ((size_t)i * ld + j) * 2);
    *reinterpret_cast<u32x4*>(at) = u32x4{h0.x, h0.y, h1.x, h1.y};
    if constexpr (SPLIT) {
      float c[4], d[4];
      unpack_f16x4(h0, c);
      unpack_f16x4(h1, d);
#pragma unroll
      for (int x = 0; x < 4; ++x) { c[x] = a[x] - c[x]; d[x] = b[x] - d[x]; }
      const u32x2 l0 = pack_f16x4(c), l1 = pack_f16x4(d);
      *reinterpret_cast<u32x4*>(at + 64) = u32x4{l0.x, l0.y, l1.x, l1.y};
    }
  };
#pragma unroll
  for (int h = 0; h < 2; ++h) store(p.X, i0 + row + 32 * h, j0 + ch * 8, p.Np, u[h]);
  __syncthreads();
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    float v[8];
#pragma unroll
    for (int x = 0; x < 8; ++x) v[x] = s[ch * 8 + x][row + 32 * h];
    store(p.XT, j0 + row + 32 * h, i0 + ch * 8, p.Mp, v);
  }
}

}  // namespace moe
