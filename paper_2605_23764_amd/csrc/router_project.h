// The router's projection: logits = x W, and its backward dx = dres + dlogits W^T, dW = x^T dlogits, to fp32 accuracy on bf16 MFMA.
//
// An fp32 value is the exact sum of three bf16 pieces: its upper 16 bits (8 of significand), those of what is left (below 2^-7 of it),
// and the rest (below 2^-15).  A product of two sums is the sum of the pieces' products: three MFMAs where x is bf16 (one piece against
// three, nothing left out), six where both sides are fp32 (left out: below 2 * 2^-7 * 2^-15 of the product); dx in bf16 takes two pieces
// of each side, three products (left out: below 2^-14 + 2 * 2^-15), in front of a rounding of 2^-8.  At 16 times the rate of fp32 MFMA
// that is 5 and 2.7 times as fast.  (An infinity has NaN pieces.)
//
// One form, C[i,j] = sum over k of P(i,k) Q(j,k), with either operand k-contiguous or row-contiguous in memory.  Tiles of 128 x 128 by
// four waves of 64 x 64, k steps of 32: a step's values are fetched into registers while the step before is multiplied, split there,
// and stand in LDS k-contiguous by rows of 64 bytes, whose four 16-byte chunks are swizzled so that operand reads spread over the
// banks.  logits (long H) and dW (long T) split k over workgroups, as they have few tiles; a second launch joins the partial sums in a
// fixed order.
#pragma once
#include <type_traits>

#include "common.h"

namespace moe {

constexpr int kProjTile = 128, kProjK = 32, kProjThreads = 256;
constexpr int kProjPiece = kProjTile * kProjK * 2;   // bytes of a piece of a side's step

struct ProjParams {
  const void *P, *Q;             // P(i,k): k-contiguous P[i ld_p + k], else P[k ld_p + i]
  int ld_p, ld_q;
  int rows, cols, K;             // C is rows x cols
  int k_split, splits;           // k's of a workgroup (a multiple of kProjK), workgroups along k
  int ti, tj;                    // tiles
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

// One side's step: two chunks per thread.  k-contiguous: rows tid / 4 and 64 more, k's 8 (tid % 4) on.  Row-contiguous: rows 2 (tid % 64)
// and the next, k's 8 (tid / 64) on: eight loads of two neighbouring rows' values.
template <typename T, bool KC> struct ProjSide {
  ProjChunk<T> c[2];
  __device__ __forceinline__ static int row(int n) { return KC ? (threadIdx.x >> 2) + 64 * n : 2 * (threadIdx.x & 63) + n; }
  __device__ __forceinline__ static int chunk() { return KC ? threadIdx.x & 3 : threadIdx.x >> 6; }

  __device__ __forceinline__ void fetch(const T* base, int ld, int rows, int i0, int k0, int k_end) {
    const int k = k0 + chunk() * 8;
    if constexpr (KC) {
#pragma unroll
      for (int n = 0; n < 2; ++n) {
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
      c[0] = ProjChunk<T>{};
      c[1] = ProjChunk<T>{};
      const int i = i0 + row(0);
      if (i + 1 < rows && k + 8 <= k_end) {
        if constexpr (sizeof(T) == 4) {
          f32x2_any v[8];
#pragma unroll
          for (int x = 0; x < 8; ++x) v[x] = *reinterpret_cast<const f32x2_any*>(base + (size_t)(k + x) * ld + i);
#pragma unroll
          for (int x = 0; x < 8; ++x) { c[0].v[x] = v[x][0]; c[1].v[x] = v[x][1]; }
        } else {
          uint32_t v[8];
#pragma unroll
          for (int x = 0; x < 8; ++x) v[x] = *reinterpret_cast<const u32_half*>(base + (size_t)(k + x) * ld + i);
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            c[0].w[x] = __builtin_amdgcn_perm(v[2 * x + 1], v[2 * x], 0x05040100);
            c[1].w[x] = high_halves(v[2 * x], v[2 * x + 1]);
          }
        }
      } else {
#pragma unroll
        for (int n = 0; n < 2; ++n)
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
    for (int n = 0; n < 2; ++n) {
      u32x4 piece[N];
      proj_pieces<N>(c[n], piece);
      const int r = row(n);
#pragma unroll
      for (int i = 0; i < N; ++i) *reinterpret_cast<u32x4*>(lds + i * kProjPiece + r * 64 + ((chunk() ^ (r >> 1)) & 3) * 16) = piece[i];
    }
  }
};

// NP, NQ: pieces of a value of each side.  OUT: storage of the result of dx, void: partial sums in fp32.
template <typename TP, bool KCP, int NP, typename TQ, bool KCQ, int NQ, typename OUT>
__global__ __launch_bounds__(kProjThreads) void project_kernel(ProjParams p) {
  constexpr int kStage = (NP + NQ) * kProjPiece, kOrder = NP > NQ ? NP : NQ;
  __shared__ __attribute__((aligned(1024))) char smem[2 * kStage];
  // the splits of a tile go to different dies, a split's tiles to the same ones: there its part of W stays in the L2
  int b = blockIdx.x;
  const int split = b % p.splits;
  b /= p.splits;
  const int j0 = (b % p.tj) * kProjTile, i0 = (b / p.tj) * kProjTile;
  const int k0 = split * p.k_split, k_end = min(p.K, k0 + p.k_split);
  const int lane = lane_id(), wave = threadIdx.x / kWave, wm = wave >> 1, wn = wave & 1, l32 = lane & 31, lh = lane >> 5;
  const TP* P = static_cast<const TP*>(p.P);
  const TQ* Q = static_cast<const TQ*>(p.Q);
  f32x16 acc[2][2];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
  ProjSide<TP, KCP> sp;
  ProjSide<TQ, KCQ> sq;
  sp.fetch(P, p.ld_p, p.rows, i0, k0, k_end);
  sq.fetch(Q, p.ld_q, p.cols, j0, k0, k_end);
  int stage = 0;
  for (int k = k0; k < k_end; k += kProjK) {
    char* lds = smem + stage * kStage;
    sp.template store<NP>(lds);
    sq.template store<NQ>(lds + NP * kProjPiece);
    __syncthreads();                       // a wave is here only once it has read the stage of the step before
    if (k + kProjK < k_end) {
      sp.fetch(P, p.ld_p, p.rows, i0, k + kProjK, k_end);
      sq.fetch(Q, p.ld_q, p.cols, j0, k + kProjK, k_end);
    }
    auto at = [&](int piece, int r, int ks) __attribute__((always_inline)) {
      return *reinterpret_cast<const bf16x8*>(lds + piece * kProjPiece + r * 64 + (((ks * 2 + lh) ^ (r >> 1)) & 3) * 16);
    };
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      bf16x8 fp[2][NP], fq[2][NQ];
#pragma unroll
      for (int x = 0; x < 2; ++x) {
#pragma unroll
        for (int n = 0; n < NP; ++n) fp[x][n] = at(n, wm * 64 + x * 32 + l32, ks);
#pragma unroll
        for (int n = 0; n < NQ; ++n) fq[x][n] = at(NP + n, wn * 64 + x * 32 + l32, ks);
      }
      // smallest products first
#pragma unroll
      for (int o = kOrder - 1; o >= 0; --o)
#pragma unroll
        for (int n = 0; n < NP; ++n)
          if (o - n >= 0 && o - n < NQ)
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
              for (int j = 0; j < 2; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fq[j][o - n], fp[i][n], acc[i][j], 0, 0, 0);
    }
    stage ^= 1;
  }
  // lane: row l32 of each block, per q the columns 8 q + 4 lh .. + 3
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int r = i0 + wm * 64 + i * 32 + l32;
    if (r >= p.rows) continue;
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int c = j0 + wn * 64 + j * 32 + q * 8 + lh * 4;
        const size_t at = (size_t)r * p.cols + c;
        float v[4];
#pragma unroll
        for (int x = 0; x < 4; ++x) v[x] = acc[i][j][q * 4 + x];
        if constexpr (std::is_void<OUT>::value) {
          float* dst = p.part + (size_t)split * p.rows * p.cols + at;
          if (c + 4 <= p.cols) *reinterpret_cast<f32x4_any*>(dst) = f32x4_any{v[0], v[1], v[2], v[3]};
          else
#pragma unroll
            for (int x = 0; x < 4; ++x)
              if (c + x < p.cols) dst[x] = v[x];
        } else {
          const OUT* add = static_cast<const OUT*>(p.add);
          OUT* dst = static_cast<OUT*>(p.out);
#pragma unroll
          for (int x = 0; x < 4; ++x)
            if (c + x < p.cols) dst[at + x] = (OUT)(add ? (float)add[at + x] + v[x] : v[x]);
        }
      }
  }
}

// out[i] = sum over the splits of part[split][i]: 64 values per workgroup, whose waves take every fourth split.
__global__ __launch_bounds__(256) void project_join_kernel(const float* part, int splits, size_t n, float* out) {
  __shared__ float s[4][kWave];
  const int lane = lane_id(), wave = threadIdx.x / kWave;
  const size_t i = (size_t)blockIdx.x * kWave + lane;
  float v = 0.f;
  if (i < n)
    for (int w = wave; w < splits; w += 4) v += part[(size_t)w * n + i];
  s[wave][lane] = v;
  __syncthreads();
  if (wave == 0 && i < n) out[i] = (s[0][lane] + s[1][lane]) + (s[2][lane] + s[3][lane]);
}

}  // namespace moe
