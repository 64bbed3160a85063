// Grouped products of few rows with 4-bit expert weights: the layer's two GEMMs in a serving step.
//
// Weights are 4-bit floats (sign, 2 bits of exponent, 1 of mantissa: +-{0, .5, 1, 1.5, 2, 3, 4, 6}) with a power-of-two scale per 32
// consecutive k of a column, the block format of the OCP MX specification: w = code * 2^(scale - 127).  A block is 16 bytes, low nibble the
// even k; blocks lie [expert][k / 32][column], their scales (a byte each) alike.
//
// Few rows per expert make the launch a read of 17/32 byte per weight, so what counts is that enough of it is under way:
//   * a lane loads a whole block, 16 bytes; 16 neighbouring lanes take neighbouring columns (256 bytes in a row), the four lane rows of
//     a wave four consecutive blocks: 1 KB per load and wave, each byte once.
//   * A block feeds four MFMAs 16x16x32: the hardware conversion makes eight bf16 of a 32-bit word, scale included and exact; which
//     eight of the 128 k a lane's word holds is the same for the activations, which come from the L2 in the same order (64
//     contiguous bytes per lane), so that neither side is ever shuffled.
//   * The waves of a workgroup split K, so that an item is narrow (16 gate + 16 up columns, or 32 columns) and even one token's few
//     experts give several items per CU; their sums meet in LDS, in wave order.
// Products are exact in fp32 (bf16 x 2 bits), sums fp32.  GEMM-1's results are rounded to bf16 (they are an MFMA's operand next), GEMM-2's
// stay fp32 until Combine has added them up, which rounds the layer's output once: 8 bytes of traffic per value of few rows.
#pragma once
#include "common.h"

namespace moe {

constexpr int kW4Waves = 4;                // waves of a workgroup, each with a share of K
constexpr int kW4Rows = 64;                // rows in hand at a time, at most
constexpr int kW4Blocks = 2;               // 16-column blocks of an item

struct W4Params {
  const __bf16* x;               // activations, rows of K
  const int32_t* gather;         // row r of the experts' rows is row gather[r] of x; null: r
  const uint8_t* q;              // [E_local][K / 32][cols][16]
  const uint8_t* scale;          // [E_local][K / 32][cols]
  const int32_t* offsets;        // [E_local + 1]
  void* out;                     // rows of N: bf16 (SwiGLU) or fp32
  int K, N, cols, n_items;       // N: output columns (cols = 2 N with the gate and up halves)
};

__device__ __forceinline__ bf16x8 w4_bf16(uint32_t w, float scale) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// Rows row0 + m0 .. (up to 16 RT) of an expert with rows n_rows, times the item's columns.
template <int RT, bool SWIGLU>
__device__ __forceinline__ void w4_rows(const W4Params& p, const uint8_t* q, const uint8_t* scale, int item, int row0, int m0, int n_rows,
                                        float* s_acc) {
  constexpr int NB = kW4Blocks;
  const int lane = lane_id(), l16 = lane & 15, lq = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int groups = p.K / 32;
  // a lane's column of each block: 16 gate and the matching up columns, or 32 in a row
  size_t at[NB];
  const __bf16* xr[RT];
  bool live[RT];
#pragma unroll
  for (int b = 0; b < NB; ++b) at[b] = (SWIGLU ? b * p.N + item * 16 : item * 32 + b * 16) + l16;
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    const int m = m0 + r * 16 + l16;
    live[r] = m < n_rows;
    const int row = live[r] ? (p.gather ? p.gather[row0 + m] : row0 + m) : 0;
    xr[r] = p.x + (size_t)row * p.K;
  }
  f32x4 acc[RT][NB];
#pragma unroll
  for (int r = 0; r < RT; ++r)
#pragma unroll
    for (int b = 0; b < NB; ++b) acc[r][b] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int steps = (groups + 3) / 4;
  const int s0 = steps * wave / kW4Waves, s1 = steps * (wave + 1) / kW4Waves;
  for (int s = s0; s < s1; ++s) {
    const int g = s * 4 + lq;
    const bool in = g < groups;                                  // the last step may hold two groups
    u32x4 w[NB];
    float sc[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      w[b] = u32x4{0, 0, 0, 0};
      sc[b] = 1.f;
      if (in) {
        const size_t blk = (size_t)g * p.cols + at[b];
        w[b] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(q + blk * 16));
        sc[b] = __builtin_bit_cast(float, (uint32_t)scale[blk] << 23);
      }
    }
    bf16x8 x[RT][4];
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        u32x4 v = {0, 0, 0, 0};
        if (live[r] && in) v = *reinterpret_cast<const u32x4*>(xr[r] + g * 32 + i * 8);
        x[r][i] = __builtin_bit_cast(bf16x8, v);
      }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        const bf16x8 wf = w4_bf16(w[b][i], sc[b]);
#pragma unroll
        for (int r = 0; r < RT; ++r) acc[r][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wf, x[r][i], acc[r][b], 0, 0, 0);
      }
  }
  // the waves' shares of K meet: row block r is joined by wave r
#pragma unroll
  for (int r = 0; r < RT; ++r)
#pragma unroll
    for (int b = 0; b < NB; ++b) *reinterpret_cast<f32x4*>(s_acc + (((wave * RT + r) * NB + b) * kWave + lane) * 4) = acc[r][b];
  __syncthreads();
  if (wave < RT) {
    f32x4 t[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      t[b] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < kW4Waves; ++w) t[b] += *reinterpret_cast<const f32x4*>(s_acc + (((w * RT + wave) * NB + b) * kWave + lane) * 4);
    }
    // lane: row l16 of the block, columns 4 lq .. 4 lq + 3 of each 16
    const int m = m0 + wave * 16 + l16;
    if (m < n_rows) {
      const size_t row = (size_t)(row0 + m) * p.N;
      if constexpr (SWIGLU) {
        float a[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) a[c] = t[0][c] * sigmoid_bf16_(t[0][c]) * t[NB - 1][c];
        *reinterpret_cast<u32x2*>(static_cast<__bf16*>(p.out) + row + item * 16 + lq * 4) = u32x2{pack_bf16(a[0], a[1]), pack_bf16(a[2], a[3])};
      } else {
#pragma unroll
        for (int b = 0; b < NB; ++b) *reinterpret_cast<f32x4*>(static_cast<float*>(p.out) + row + item * 32 + b * 16 + lq * 4) = t[b];
      }
    }
  }
}

// An item per workgroup: blockIdx.x = expert * n_items + item.
template <bool SWIGLU>
__global__ __launch_bounds__(kW4Waves* kWave) void experts_w4_kernel(W4Params p) {
  __shared__ __align__(16) float s_acc[kW4Waves * (kW4Rows / 16) * kW4Blocks * kWave * 4];
  const int e = blockIdx.x / p.n_items, item = blockIdx.x - e * p.n_items;
  const int row0 = p.offsets[e], rows = p.offsets[e + 1] - row0;
  if (rows <= 0) return;
  const size_t blocks = (size_t)e * (p.K / 32) * p.cols;
  const uint8_t *q = p.q + blocks * 16, *scale = p.scale + blocks;
  for (int m0 = 0; m0 < rows; m0 += kW4Rows) {
    if (m0) __syncthreads();                                     // s_acc has been read
    if (rows - m0 <= 16) w4_rows<1, SWIGLU>(p, q, scale, item, row0, m0, rows, s_acc);
    else if (rows - m0 <= 32) w4_rows<2, SWIGLU>(p, q, scale, item, row0, m0, rows, s_acc);
    else w4_rows<4, SWIGLU>(p, q, scale, item, row0, m0, rows, s_acc);
  }
}

// out[t,:] = sum over the local slots j of topk_w[t,j] * y[row_of[t,j],:], in slot order: a lane per eight columns of a token.
__global__ __launch_bounds__(256) void combine_w4_kernel(const float* y, const int32_t* row_of, const float* topk_w, __bf16* out, int T, int H,
                                                         int k) {
  const int per = H / 8;
  const long n = (long)T * per;
  for (long i = (long)blockIdx.x * 256 + threadIdx.x; i < n; i += (long)gridDim.x * 256) {
    const long t = i / per;
    const int c = (int)(i - t * per) * 8;
    f32x4 lo = {0.f, 0.f, 0.f, 0.f}, hi = lo;
    for (int j = 0; j < k; ++j) {
      const int r = row_of[t * k + j];
      if (r < 0) continue;
      const float w = topk_w[t * k + j];
      const f32x4* src = reinterpret_cast<const f32x4*>(y + (size_t)r * H + c);
      lo += w * src[0];
      hi += w * src[1];
    }
    *reinterpret_cast<u32x4*>(out + (size_t)t * H + c) =
        u32x4{pack_bf16(lo[0], lo[1]), pack_bf16(lo[2], lo[3]), pack_bf16(hi[0], hi[1]), pack_bf16(hi[2], hi[3])};
  }
}

// Weights to blocks: a lane per block.  The scale brings the largest magnitude of the 32 into [4, 8), values are rounded to the nearest
// code (ties to the even one), those above 6 to 6.  A block of zeros has scale 1.  Non-finite values have no code: the block's
// scale is 255.
template <typename T>
__global__ __launch_bounds__(256) void quantize_w4_kernel(const T* w, uint8_t* q, uint8_t* scale, long blocks, int groups, int N) {
  const long stride = (long)gridDim.x * 256;
  for (long i = (long)blockIdx.x * 256 + threadIdx.x; i < blocks; i += stride) {
    const long eg = i / N;                                       // expert * groups + group
    const int n = (int)(i - eg * N);
    const T* src = w + (size_t)eg * 32 * N + n;
    float v[32], top = 0.f;
    uint32_t bits = 0;
#pragma unroll
    for (int k = 0; k < 32; ++k) {
      v[k] = (float)src[(size_t)k * N];
      bits = max(bits, __builtin_bit_cast(uint32_t, v[k]) & 0x7FFFFFFFu);   // ordered like the magnitudes, NaN on top
    }
    top = __builtin_bit_cast(float, bits);
    int s = bits == 0 ? 127 : max((int)(bits >> 23) - 2, 1);
    const float unit = __builtin_bit_cast(float, (uint32_t)(254 - s) << 23);   // 1 / 2^(s - 127)
    u32x4 o = {0, 0, 0, 0};
#pragma unroll
    for (int k = 0; k < 32; ++k) {
      const float m = __builtin_fabsf(v[k]) * unit;
      // codes up to m: the borders lie half way, a border itself goes to the even code
      const uint32_t c = (m > 0.25f) + (m >= 0.75f) + (m > 1.25f) + (m >= 1.75f) + (m > 2.5f) + (m >= 3.5f) + (m > 5.0f);
      o[k >> 3] |= (c | (__builtin_bit_cast(uint32_t, v[k]) >> 31) << 3) << (4 * (k & 7));
    }
    if (bits >= 0x7F800000u) { s = 255; o = u32x4{0, 0, 0, 0}; }
    *reinterpret_cast<u32x4*>(q + i * 16) = o;
    scale[i] = (uint8_t)s;
  }
}

}  // namespace moe
