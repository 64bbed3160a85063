// The router's projection: logits = x W, and its backward dx = dres + dlogits W^T, dW = x^T dlogits, to fp32 accuracy on bf16 MFMA.
//
// An fp32 value is the exact sum of three bf16 pieces: its upper 16 bits (8 of significand), those of what is left (below 2^-7 of it),
// and the rest (below 2^-15).  A product of two sums is the sum of the pieces' products: three MFMAs where x is bf16 (one piece against
// three, nothing left out), six where both sides are fp32 (left out: below 2 * 2^-7 * 2^-15 of the product); dx in bf16 takes two pieces
// of each side, three products (left out: below 2^-14 + 2 * 2^-15), in front of a rounding of 2^-8.  At 16 times the rate of fp32 MFMA
// that is 5 and 2.7 times as fast.  (An infinity has NaN pieces.  The last bit of a piece is 2^-133 at least, so of values below 2^-109 bits are lost.)
//
// One form, C[i,j] = sum over k of P(i,k) Q(j,k), with either operand k-contiguous or row-contiguous in memory.  Tiles of 128 x 128 by
// four waves of 64 x 64, of 128 x 64 by four of 32 x 64, of 128 x 32 by four of 32 x 32; k steps of 64: a step's values are fetched into
// registers while the step before is multiplied, split there, and stand in LDS k-contiguous by rows of 128 bytes, whose eight 16-byte chunks
// are swizzled so that operand reads and the writes of row-contiguous operands spread over the banks.  logits (long H) and dW (long T)
// split k over workgroups, as they have few tiles; a second launch joins the partial sums in a fixed order.
//
// Large calls are bound by MFMA and the splitting's VALU work together, which the two or three waves of a SIMD overlap by half, and by waits at
// a step's two barriers: 8192 x 7168 x 256 in bf16, logits 100 us (matrix cores 44 % of the clocks, VALU 30 %), dW 120, dx 158 (28 and 39 %);
// each product's three MFMA products take 67 us at a library product's rate, the 117 MB of x 23, the 235 of dres and dx 45.  Small ones by
// their launches, 5 to 9 us.
#pragma once
#include <type_traits>

#include "rows.h"

namespace moe {

constexpr int kProjTile = 128, kProjK = 64, kProjThreads = 256, kLdsBytes = 160 * 1024;

struct ProjParams {
  const void *P, *Q;             // P(i,k): k-contiguous P[i ld_p + k], else P[k ld_p + i]
  int ld_p, ld_q;
  int rows, cols, K;             // C is rows x cols
  int k_split, splits;           // k's of a workgroup (a multiple of kProjK), workgroups along k
  int tj;                        // tiles along the columns
  float* part;                   // [splits][rows][cols]; the result itself with one
  const void* add;               // out: added, [rows][cols] of the storage type, or null
  void* out;
};

__device__ __forceinline__ uint32_t high_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302); }   // a's low

// Eight consecutive k of one row, as they come: fp32, or bf16 pairs.
template <typename T> struct ProjChunk;
template <> struct ProjChunk<float> { float v[8]; };
template <> struct ProjChunk<__bf16> { uint32_t w[4]; };

// Their pieces, 16 bytes each.
template <int N> __device__ __forceinline__ void proj_pieces(const ProjChunk<float>& c, u32x4 (&out)[N]) {
  float r[8];
#pragma unroll
  for (int x = 0; x < 8; ++x) r[x] = c.v[x];
#pragma unroll
  for (int n = 0; n < N; ++n)
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const uint32_t a = __builtin_bit_cast(uint32_t, r[2 * x]), b = __builtin_bit_cast(uint32_t, r[2 * x + 1]);
      out[n][x] = high_halves(a, b);
      r[2 * x] -= __builtin_bit_cast(float, a & 0xFFFF0000u);
      r[2 * x + 1] -= __builtin_bit_cast(float, b & 0xFFFF0000u);
    }
}
template <int N> __device__ __forceinline__ void proj_pieces(const ProjChunk<__bf16>& c, u32x4 (&out)[N]) {
  static_assert(N == 1, "a bf16 value is its own piece");
  out[0] = u32x4{c.w[0], c.w[1], c.w[2], c.w[3]};
}

typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
typedef float f32x2_any __attribute__((ext_vector_type(2), aligned(4)));
typedef uint32_t u32x4_half __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32_half __attribute__((aligned(2)));

// 16-byte chunk c of row r in its row of a stage.
__device__ __forceinline__ int proj_chunk(int r, int c) { return r * 128 + ((c ^ (r >> 1) ^ (r >> 4)) & 7) * 16; }

// One side's step of R rows: R / 32 chunks per thread.  k-contiguous: rows tid / 8 and every 32nd behind it, k's 8 (tid % 8) on.
// Row-contiguous: R / 32 neighbouring rows from R / 32 (tid % 32) on, k's 8 (tid / 32) on: eight loads of those rows' values.
template <typename T, bool KC, int R> struct ProjSide {
  static constexpr int kN = R / 32;
  typedef float fvec __attribute__((ext_vector_type(kN), aligned(4)));
  typedef uint16_t hvec __attribute__((ext_vector_type(kN), aligned(2)));
  ProjChunk<T> c[kN];
  __device__ __forceinline__ static int row(int n) { return KC ? (threadIdx.x >> 3) + 32 * n : kN * (threadIdx.x & 31) + n; }
  __device__ __forceinline__ static int chunk() { return KC ? threadIdx.x & 7 : threadIdx.x >> 5; }

  __device__ __forceinline__ void fetch(const T* base, int ld, int rows, int i0, int k0, int k_end) {
    const int k = k0 + chunk() * 8;
    if constexpr (KC) {
#pragma unroll
      for (int n = 0; n < kN; ++n) {
        const int i = i0 + row(n);
        const T* src = base + (size_t)i * ld + k;
        c[n] = ProjChunk<T>{};
        if (i < rows && k + 8 <= k_end) {
          if constexpr (sizeof(T) == 4) {
            const f32x4_any a = reinterpret_cast<const f32x4_any*>(src)[0], b = reinterpret_cast<const f32x4_any*>(src)[1];
#pragma unroll
            for (int x = 0; x < 4; ++x) { c[n].v[x] = a[x]; c[n].v[4 + x] = b[x]; }
          } else {
            const u32x4_half a = *reinterpret_cast<const u32x4_half*>(src);
#pragma unroll
            for (int x = 0; x < 4; ++x) c[n].w[x] = a[x];
          }
        } else if (i < rows) {
#pragma unroll
          for (int x = 0; x < 8; ++x)
            if (k + x < k_end) put(n, x, src[x]);
        }
      }
    } else {
#pragma unroll
      for (int n = 0; n < kN; ++n) c[n] = ProjChunk<T>{};
      const int i = i0 + row(0);
      if (i + kN <= rows && k + 8 <= k_end) {
        const T* src = base + (size_t)k * ld + i;
        if constexpr (sizeof(T) == 4) {
          fvec v[8];
#pragma unroll
          for (int x = 0; x < 8; ++x) v[x] = *reinterpret_cast<const fvec*>(src + (size_t)x * ld);
#pragma unroll
          for (int n = 0; n < kN; ++n)
#pragma unroll
            for (int x = 0; x < 8; ++x) c[n].v[x] = v[x][n];
        } else {
          hvec v[8];
#pragma unroll
          for (int x = 0; x < 8; ++x) v[x] = *reinterpret_cast<const hvec*>(src + (size_t)x * ld);
#pragma unroll
          for (int n = 0; n < kN; ++n)
#pragma unroll
            for (int x = 0; x < 4; ++x) c[n].w[x] = (uint32_t)v[2 * x][n] | (uint32_t)v[2 * x + 1][n] << 16;
        }
      } else {
#pragma unroll
        for (int n = 0; n < kN; ++n)
#pragma unroll
          for (int x = 0; x < 8; ++x)
            if (i + n < rows && k + x < k_end) put(n, x, base[(size_t)(k + x) * ld + i + n]);
      }
    }
  }
  __device__ __forceinline__ void put(int n, int x, T v) {
    if constexpr (sizeof(T) == 4) c[n].v[x] = v;
    else c[n].w[x >> 1] |= (uint32_t)__builtin_bit_cast(uint16_t, v) << (16 * (x & 1));
  }
  template <int N> __device__ __forceinline__ void store(char* lds) const {
#pragma unroll
    for (int n = 0; n < kN; ++n) {
      u32x4 piece[N];
      proj_pieces<N>(c[n], piece);
#pragma unroll
      for (int i = 0; i < N; ++i) *reinterpret_cast<u32x4*>(lds + i * R * 128 + proj_chunk(row(n), chunk())) = piece[i];
    }
  }
};

// Four columns from `at` on, n of them there: one access where all four are, at any element's address.
template <typename T> using ProjVec __attribute__((aligned(sizeof(T)))) = T __attribute__((ext_vector_type(4)));
template <typename T> __device__ __forceinline__ ProjVec<T> proj_get(const T* src, size_t at, int n) {
  ProjVec<T> v = {};
  if (n >= 4) {
    v = *reinterpret_cast<const ProjVec<T>*>(src + at);
  } else {
#pragma unroll
    for (int x = 0; x < 3; ++x)
      if (x < n) v[x] = src[at + x];
  }
  return v;
}
template <typename T> __device__ __forceinline__ void proj_put(T* dst, size_t at, int n, f32x4 v) {
  if (n >= 4) {
    ProjVec<T> o;
#pragma unroll
    for (int x = 0; x < 4; ++x) o[x] = (T)v[x];
    *reinterpret_cast<ProjVec<T>*>(dst + at) = o;
  } else {
#pragma unroll
    for (int x = 0; x < 3; ++x)
      if (x < n) dst[at + x] = (T)v[x];
  }
}

// A wave's 32 rows x 64 columns of a result, whole lines, by way of the wave's place in LDS (kProjRegion bytes).  What is added comes ahead of
// the sums: its way from HBM is longer than they take (dx of 8192 x 7168 x 256 with dres in HBM: 160 us, with it behind them 184).
constexpr int kProjRow = 64 * 4 + 16, kProjRegion = 32 * kProjRow;
template <typename OUT> struct ProjRows {
  ProjVec<OUT> add[8];
  __device__ __forceinline__ void fetch(const ProjParams& p, int r0, int c0) {
    const OUT* src = static_cast<const OUT*>(p.add);
    const int c = c0 + (lane_id() & 15) * 4, r = r0 + (lane_id() >> 4), left = p.cols - c;
    const size_t at = (size_t)r * p.cols + c, step = (size_t)4 * p.cols;
#pragma unroll
    for (int it = 0; it < 8; ++it) {
      add[it] = ProjVec<OUT>{};
      if (src && r + it * 4 < p.rows && left > 0) add[it] = proj_get(src, at + it * step, left);
    }
  }
  __device__ __forceinline__ void store(const ProjParams& p, const f32x16 (&acc)[2], int r0, int c0, char* region) const {
    const int lane = lane_id(), l32 = lane & 31, lh = lane >> 5;
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *reinterpret_cast<f32x4*>(region + l32 * kProjRow + (j * 32 + q * 8 + lh * 4) * 4) =
            f32x4{acc[j][q * 4], acc[j][q * 4 + 1], acc[j][q * 4 + 2], acc[j][q * 4 + 3]};
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    const int c = c0 + (lane & 15) * 4, r = r0 + (lane >> 4), left = p.cols - c;
    const size_t at = (size_t)r * p.cols + c, step = (size_t)4 * p.cols;
#pragma unroll
    for (int it = 0; it < 8; ++it) {
      f32x4 v = *reinterpret_cast<const f32x4*>(region + (it * 4 + (lane >> 4)) * kProjRow + (lane & 15) * 16);
#pragma unroll
      for (int x = 0; x < 4; ++x) v[x] += (float)add[it][x];
      if (r + it * 4 < p.rows && left > 0) proj_put(static_cast<OUT*>(p.out), at + it * step, left, v);
    }
  }
};
struct ProjNoRows {};

// NP, NQ: pieces of a value of each side.  TN: columns of a tile, 128, 64 or 32 (with OUT 64).  OUT: storage of the result of dx, void: partial sums in fp32.
// Two workgroups to a CU where their LDS allows it (all but fp32's pairs of three pieces): they cover each other's waits (dx, 8192 x 7168 x 256, 260
// registers and one workgroup: 312 us).
template <typename TP, bool KCP, int NP, typename TQ, bool KCQ, int NQ, int TN, typename OUT>
__global__ __launch_bounds__(kProjThreads, (NP * kProjTile + NQ * TN) * 256 <= kLdsBytes ? 2 : 1) void project_kernel(ProjParams p) {
  constexpr int kOrder = NP > NQ ? NP : NQ, kPieceP = kProjTile * 128, kPieceQ = TN * 128;
  constexpr int BI = TN == 128 ? 2 : 1, BJ = TN == 32 ? 1 : 2;   // blocks of 32 x 32 of a wave
  constexpr int kStage = NP * kPieceP + NQ * kPieceQ;
  constexpr int kLds = !std::is_void<OUT>::value && kStage < 4 * kProjRegion ? 4 * kProjRegion : kStage;
  __shared__ __attribute__((aligned(1024))) char smem[kLds];
  // the splits of a tile go to different dies, a split's tiles to the same ones: there its part of W stays in the L2
  int b = blockIdx.x;
  const int split = b % p.splits;
  b /= p.splits;
  const int j0 = (b % p.tj) * TN, i0 = (b / p.tj) * kProjTile;
  const int k0 = split * p.k_split, k_end = k0 + min(p.K - k0, p.k_split);   // of up to 2^31 tokens
  const int lane = lane_id(), wave = threadIdx.x / kWave, l32 = lane & 31, lh = lane >> 5;
  const int pr = TN == 128 ? (wave >> 1) * 64 : wave * 32, qr = TN == 128 ? (wave & 1) * 64 : 0;   // the wave's first row of each side
  const TP* P = static_cast<const TP*>(p.P);
  const TQ* Q = static_cast<const TQ*>(p.Q);
  f32x16 acc[BI][BJ];
#pragma unroll
  for (int i = 0; i < BI; ++i)
#pragma unroll
    for (int j = 0; j < BJ; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
  typename std::conditional<std::is_void<OUT>::value, ProjNoRows, ProjRows<OUT>>::type rows;
  if constexpr (!std::is_void<OUT>::value) rows.fetch(p, i0 + pr, j0 + qr);
  ProjSide<TP, KCP, kProjTile> sp;
  ProjSide<TQ, KCQ, TN> sq;
  sp.fetch(P, p.ld_p, p.rows, i0, k0, k_end);
  sq.fetch(Q, p.ld_q, p.cols, j0, k0, k_end);
  for (int k = k0; k < k_end; k += kProjK) {
    sp.template store<NP>(smem);
    sq.template store<NQ>(smem + NP * kPieceP);
    __syncthreads();
    if (k + kProjK < k_end) {
      sp.fetch(P, p.ld_p, p.rows, i0, k + kProjK, k_end);
      sq.fetch(Q, p.ld_q, p.cols, j0, k + kProjK, k_end);
    }
#pragma unroll
    for (int ks = 0; ks < kProjK / 16; ++ks) {
      if (ks * 16 >= k_end - k) break;       // the rest of the step is zeros
      bf16x8 fp[BI][NP], fq[BJ][NQ];
#pragma unroll
      for (int x = 0; x < BI; ++x)
#pragma unroll
        for (int n = 0; n < NP; ++n)
          fp[x][n] = *reinterpret_cast<const bf16x8*>(smem + n * kPieceP + proj_chunk(pr + x * 32 + l32, ks * 2 + lh));
#pragma unroll
      for (int x = 0; x < BJ; ++x)
#pragma unroll
        for (int n = 0; n < NQ; ++n)
          fq[x][n] = *reinterpret_cast<const bf16x8*>(smem + NP * kPieceP + n * kPieceQ + proj_chunk(qr + x * 32 + l32, ks * 2 + lh));
      // smallest products first
#pragma unroll
      for (int o = kOrder - 1; o >= 0; --o)
#pragma unroll
        for (int n = 0; n < NP; ++n)
          if (o - n >= 0 && o - n < NQ)
#pragma unroll
            for (int i = 0; i < BI; ++i)
#pragma unroll
              for (int j = 0; j < BJ; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fq[j][o - n], fp[i][n], acc[i][j], 0, 0, 0);
    }
    __syncthreads();                       // every wave has read the stage
  }
  // lane: row l32 of each block, per q the columns 8 q + 4 lh .. + 3
#pragma unroll
  for (int i = 0; i < BI; ++i) {
    const int r0 = i0 + pr + i * 32;
    if constexpr (std::is_void<OUT>::value) {
      const int r = r0 + l32;
      if (r >= p.rows) continue;
      float* dst = p.part + ((size_t)split * p.rows + r) * p.cols;
#pragma unroll
      for (int j = 0; j < BJ; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int c = j0 + qr + j * 32 + q * 8 + lh * 4;
          if (c + 4 <= p.cols)
            *reinterpret_cast<f32x4_any*>(dst + c) =
                f32x4_any{acc[i][j][q * 4], acc[i][j][q * 4 + 1], acc[i][j][q * 4 + 2], acc[i][j][q * 4 + 3]};
          else
#pragma unroll
            for (int x = 0; x < 3; ++x)
              if (c + x < p.cols) dst[c + x] = acc[i][j][q * 4 + x];
        }
    } else {
      static_assert(BI == 1 && BJ == 2, "32 rows and 64 columns of a wave");
      rows.store(p, acc[i], r0, j0 + qr, smem + wave * kProjRegion);
    }
  }
}

// out[i] = sum over the splits of part[split][i], n of them: 256 / PARTS values per workgroup, whose PARTS shares take every PARTS-th split
// (eight loads at a time) and are added up in their order.
template <int PARTS> __global__ __launch_bounds__(256) void project_join_kernel(const float* part, int splits, size_t n, float* out) {
  constexpr int kValues = 256 / PARTS;
  __shared__ float s[PARTS][kValues];
  const int value = threadIdx.x % kValues, share = threadIdx.x / kValues;
  const size_t i = (size_t)blockIdx.x * kValues + value;
  float v = 0.f;
  if (i < n)
    for (int w = share; w < splits; w += 8 * PARTS) {
      float x[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) x[u] = part[(size_t)min(w + u * PARTS, splits - 1) * n + i];
#pragma unroll
      for (int u = 0; u < 8; ++u) v += w + u * PARTS < splits ? x[u] : 0.f;
    }
  s[share][value] = v;
  __syncthreads();
  if (share == 0 && i < n) {
    float t = s[0][value];
#pragma unroll
    for (int w = 1; w < PARTS; ++w) t += s[w][value];
    out[i] = t;
  }
}

// Few splits of many values: four at a time.
__global__ __launch_bounds__(256) void project_join4_kernel(const float* part, int splits, size_t n4, float* out) {
  const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= n4) return;
  f32x4 v = reinterpret_cast<const f32x4*>(part)[i];
  for (int w = 1; w < splits; ++w) v += reinterpret_cast<const f32x4*>(part)[(size_t)w * n4 + i];
  reinterpret_cast<f32x4*>(out)[i] = v;
}

}  // namespace moe
