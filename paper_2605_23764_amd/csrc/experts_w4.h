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
// Bound by that read: 32 tokens, H = 7168, I = 2048, 32 of 256 experts, k = 8 (about 20 with rows, 482 MB): GEMM-1 57 us, GEMM-2 30, 5.5 TB/s
// where a loop that only loads pieces of 256 bytes reaches 6.2; with few weights (one token, H = 2048, I = 1408: 18 MB, 7.4 + 5.7 us) by
// the latency of a workgroup's start, four steps and a join; with many rows by the activations' fetches.
// Products are exact in fp32 (bf16 x 2 bits), sums fp32.  GEMM-1's results are rounded to bf16, as the layer's are with bf16 weights: they are
// an MFMA's operand next, and keeping more of them would take two operands, twice the MFMAs and the activations' fetches.  That rounding
// costs 1.6e-3 of the output (2-norm) beside the 1.7e-3 of its own rounding, 2.3e-3 together.  GEMM-2's results stay fp32 until Combine has
// added them up, which rounds the layer's output once: 8 bytes of traffic per value of few rows.
#pragma once
#include "experts_w4_launch.h"
#include "route_select.h"

namespace moe {

// Waves of a workgroup, each with a share of K.  2, 4 or 8 of them, us: H = 2048, I = 1408, 16 experts, k = 4, T = 1 17.4, 15.4, 18.2, T = 64
// 33.2, 34.5, 35.7, T = 128 56.9, 55.5, 58.9; H = 7168, I = 2048, 32 of 256, k = 8, T = 1 22.7, 21.5, 27.9, T = 8 55.5, 55.2, 51.9, T = 32 101.7,
// 91.8, 93.9.
constexpr int kW4Waves = 4;
// Waves per SIMD that the registers have to leave room for.  A wave has one step of its share in registers and no more (a ring of two or
// three steps: 2 to 30 % slower), so the bytes under way come from the number of waves.
constexpr int w4_occupancy(int row_blocks, int blocks) { return row_blocks == 2 ? 3 : blocks == 4 ? 4 : 5; }
// Output columns of an item of `blocks` 16-column blocks; SwiGLU: half of them gate, half the matching up columns.
constexpr int w4_columns(int blocks, bool swiglu) { return swiglu ? 8 * blocks : 16 * blocks; }

struct W4Params {
  const __bf16* x;               // activations: rows of K (gather), or the experts' rows in tiles (w4_tile_at)
  const int32_t* gather;         // row r of the experts' rows is row gather[r] of x; null: tiles
  const uint8_t* q;              // [E_local][K / 32][cols][16]
  const uint8_t* scale;          // [E_local][K / 32][cols]
  const int32_t* offsets;        // [E_local + 1]
  void* out;                     // bf16 in tiles (SwiGLU), or rows of N fp32
  int K, N, cols, n_items;       // N: output columns (cols = 2 N with the gate and up halves)
  RouteParams route;             // up to kW4RoutedT tokens: see experts_w4_kernel
};

// Rows of an expert, for the routed form: where each comes from and goes to.
constexpr int kW4RoutedT = kW4MaxRoutedT;
struct W4Rows { int32_t in[kW4RoutedT], out[kW4RoutedT]; };

__device__ __forceinline__ bf16x8 w4_bf16(uint32_t w, float scale) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// Activations in tiles: up to 16 rows of an expert (n of them) as [K / 8][n][8], so that what the 64 lanes of a load want, eight k of 16 rows
// from four blocks, lies in four runs of 256 bytes; in rows it lies in 32 pieces of 64 bytes, and the L1 takes a load line by line.
// Tiles follow each other like the rows in them.  Element of (row r of the tile, k):
__device__ __forceinline__ uint32_t w4_tile_at(int r, int k, int n) { return (uint32_t)(((k >> 3) * n + r) * 8 + (k & 7)); }

// A buffer descriptor over `bytes` from p (the same in all lanes): what a lane asks for beyond is 0 and costs no memory access.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t w4_buffer(const void* p, uint32_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, (int)bytes, 0x00027000);
}
constexpr uint32_t kW4Beyond = 0x80000000u;   // an offset past every buffer here
constexpr int kW4Nt = 2;                      // non-temporal: a block is read once

// Rows row0 + m0 .. (up to 16 RT) of an expert with n_rows rows, times the NB column blocks of an item.
template <int RT, int NB, bool SWIGLU, bool ROUTED>
__device__ __forceinline__ void w4_rows(const W4Params& p, const uint8_t* q, const uint8_t* scale, int item, int row0, int m0, int n_rows,
                                        const W4Rows* s_rows, float* s_acc) {
  constexpr int kCols = w4_columns(NB, SWIGLU);
  const int lane = lane_id(), l16 = lane & 15, lq = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int groups = p.K / 32, steps = (groups + 3) / 4;         // a step: 128 k, four blocks of every column
  const int s0 = steps * wave / kW4Waves, n = steps * (wave + 1) / kW4Waves - s0;
  // this wave's blocks: from its first step to its last, no further than the matrix (the last step may hold two blocks)
  const int g0 = s0 * 4, n_groups = min((s0 + n) * 4, groups) - g0;
  const __amdgpu_buffer_rsrc_t bq = w4_buffer(q + (size_t)g0 * p.cols * 16, (uint32_t)n_groups * p.cols * 16);
  const __amdgpu_buffer_rsrc_t bs = w4_buffer(scale + (size_t)g0 * p.cols, (uint32_t)n_groups * p.cols);
  uint32_t at[NB];                                               // block of this lane in step 0
#pragma unroll
  for (int b = 0; b < NB; ++b) at[b] = lq * p.cols + item * kCols + (SWIGLU ? (b >= NB / 2 ? p.N : 0) + b % (NB / 2) * 16 : b * 16) + l16;
  u32x4 w[NB];
  uint32_t sc[NB];
  bf16x8 x[RT][4];
  auto request_w = [&](int b, int s) __attribute__((always_inline)) {   // past the wave's share: nothing
    const uint32_t blk = at[b] + (uint32_t)s * 4 * p.cols;
    w[b] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(bq, blk * 16, 0, kW4Nt));
    sc[b] = __builtin_amdgcn_raw_buffer_load_b8(bs, blk, 0, 0);
  };
#pragma unroll
  for (int b = 0; b < NB; ++b) request_w(b, 0);                  // ahead of the permutation's lookup
  // activations: rows past the expert's last one, and k past the wave's share, read zeros
  const bool by_row = ROUTED || p.gather;
  const __amdgpu_buffer_rsrc_t bx = w4_buffer(by_row ? p.x : p.x + (size_t)(row0 + m0) * p.K, 0x7FFFFFFFu);
  uint32_t xo[RT];                                               // byte of this lane's block in step 0
  int n_tile[RT];
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    n_tile[r] = min(max(n_rows - m0 - r * 16, 0), 16);
    xo[r] = kW4Beyond;
    if (l16 < n_tile[r]) {
      const int m = m0 + r * 16 + l16;
      if (by_row) xo[r] = (uint32_t)(ROUTED ? s_rows->in[m] : p.gather[row0 + m]) * (uint32_t)(p.K * 2) + (uint32_t)(g0 + lq) * 64;
      else xo[r] = (uint32_t)(r * 16) * (uint32_t)(p.K * 2) + 2 * w4_tile_at(l16, (g0 + lq) * 32, n_tile[r]);
    }
  }
  auto request_x = [&](int s) __attribute__((always_inline)) {
    const bool in = s * 4 + lq < n_groups;
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      const uint32_t eight = by_row ? 16 : n_tile[r] * 16;      // bytes from eight k to the next
      const uint32_t o = in ? xo[r] + (uint32_t)s * 16 * eight : kW4Beyond;
#pragma unroll
      for (int i = 0; i < 4; ++i) x[r][i] = __builtin_bit_cast(bf16x8, __builtin_amdgcn_raw_buffer_load_b128(bx, o + i * eight, 0, 0));
    }
  };
  request_x(0);
  f32x4 acc[RT][NB];
#pragma unroll
  for (int r = 0; r < RT; ++r)
#pragma unroll
    for (int b = 0; b < NB; ++b) acc[r][b] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int s = 0; s < n; ++s) {
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      bf16x8 wf[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) wf[i] = w4_bf16(w[b][i], __builtin_bit_cast(float, sc[b] << 23));
      request_w(b, s + 1);                                       // as soon as the registers are free
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int r = 0; r < RT; ++r) acc[r][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wf[i], x[r][i], acc[r][b], 0, 0, 0);
    }
    request_x(s + 1);
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
      const size_t to = (size_t)(ROUTED ? s_rows->out[m] : row0 + m) * p.N;
      if constexpr (SWIGLU) {
        const int n = min(n_rows - m0 - wave * 16, 16);
        __bf16* tile = static_cast<__bf16*>(p.out) + (ROUTED ? to : to - (size_t)l16 * p.N);
#pragma unroll
        for (int b = 0; b < NB / 2; ++b) {
          float a[4];
#pragma unroll
          for (int c = 0; c < 4; ++c) a[c] = t[b][c] * sigmoid_bf16_(t[b][c]) * t[b + NB / 2][c];
          const int c = item * kCols + b * 16 + lq * 4;
          *reinterpret_cast<u32x2*>(tile + (ROUTED ? c : w4_tile_at(l16, c, n))) = u32x2{pack_bf16(a[0], a[1]), pack_bf16(a[2], a[3])};
        }
      } else {
        float* row = static_cast<float*>(p.out) + to;
#pragma unroll
        for (int b = 0; b < NB; ++b) *reinterpret_cast<f32x4*>(row + item * kCols + b * 16 + lq * 4) = t[b];
      }
    }
  }
}

// The routed form, for up to kW4RoutedT tokens: no routing launch ahead.  Every workgroup of GEMM-1 finds its expert's tokens itself, one
// more workgroup routes all tokens for what follows, and the row of (token, slot) is token * k + slot, which nobody has to add up.
//
// GEMM-1: the expert's slot in a token's selection is the number of experts ahead of it: larger logit, or equal and lower id (the router's
// order); a slot if that is less than k.  Returns the number of rows.
__device__ __forceinline__ int w4_select(const RouteParams& p, int e, W4Rows* s_rows, int32_t* s_slot) {
  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), id = p.expert_base + e;
  constexpr int kTokens = kW4RoutedT / kW4Waves, kPieces = kMaxE / kWave;
  float mine[kTokens], other[kTokens][kPieces];
#pragma unroll
  for (int q = 0; q < kTokens; ++q) {                            // all requested together
    if (wave + q * kW4Waves >= p.T) break;
    const float* row = p.logits + (size_t)(wave + q * kW4Waves) * p.E;
    mine[q] = row[id];
#pragma unroll
    for (int i = 0; i < kPieces; ++i)
      if (i * kWave < p.E) other[q][i] = row[min(i * kWave + lane, p.E - 1)];
  }
#pragma unroll
  for (int q = 0; q < kTokens; ++q) {
    if (wave + q * kW4Waves >= p.T) break;
    const uint32_t key = float_order_key(mine[q]);
    int ahead = 0;
#pragma unroll
    for (int i = 0; i < kPieces; ++i)
      if (i * kWave < p.E) {
        const int e2 = i * kWave + lane;
        const uint32_t key2 = float_order_key(other[q][i]);
        ahead += __popcll(__ballot(e2 < p.E && (key2 > key || (key2 == key && e2 < id))));
      }
    if (lane == 0) s_slot[wave + q * kW4Waves] = ahead < p.k ? ahead : -1;
  }
  __syncthreads();
  const int slot = lane < p.T ? s_slot[lane] : -1;
  const uint64_t members = __ballot(slot >= 0);
  if (wave == 0 && slot >= 0) {
    const int m = __popcll(members & ((1ull << lane) - 1));
    s_rows->in[m] = lane;
    s_rows->out[m] = lane * p.k + slot;
  }
  __syncthreads();
  return __popcll(members);
}
// GEMM-2: from the selections that GEMM-1's launch has left.
__device__ __forceinline__ int w4_selected(const RouteParams& p, int e, W4Rows* s_rows) {
  const int lane = lane_id(), id = p.expert_base + e;
  int slot = -1;
  if (lane < p.T)
    for (int j = 0; j < p.k; ++j)
      if (p.topk_idx[lane * p.k + j] == id) slot = j;
  const uint64_t members = __ballot(slot >= 0);
  if (threadIdx.x < kWave && slot >= 0) {
    const int m = __popcll(members & ((1ull << lane) - 1));
    s_rows->in[m] = s_rows->out[m] = lane * p.k + slot;
  }
  __syncthreads();
  return __popcll(members);
}
// topk_idx, topk_w and row_of of all tokens by one workgroup, and the workspace's status, which a routing launch would clear.
__device__ __forceinline__ void w4_route(const RouteParams& p, int32_t* s_idx, float* s_val) {
  const int lane = lane_id(), wave = threadIdx.x / kWave;
  if (threadIdx.x == 0) p.tiles.meta[kMetaStatus] = 0;
  s_idx += wave * kRouteTokensPerWave * kMaxK;
  s_val += wave * kRouteTokensPerWave * kMaxK;
  for (int t0 = wave * kRouteTokensPerWave; t0 < p.T; t0 += kW4Waves * kRouteTokensPerWave) {
    with_route_keys(p.E, [&](auto kp) __attribute__((always_inline)) {
      uint32_t key[decltype(kp)::value];
      route_load(p, t0, lane, key);
      route_select(p, t0, lane, key, s_idx, s_val);
    });
    const int r = lane >> 4, j = lane & 15, t = t0 + r;
    if (t < p.T && j < p.k) {
      const int local = s_idx[r * kMaxK + j] - p.expert_base;
      p.row_of[t * p.k + j] = local >= 0 && local < p.E_local ? t * p.k + j : -1;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");        // read before the next tokens' selection is filed
  }
}

// An item per workgroup.  The dispatcher deals consecutive workgroups to the eight dies in turn; consecutive items, whose blocks and above
// all scales share lines, go to one die instead, eight at a time.
template <int RT, int NB, bool SWIGLU, bool ROUTED>
__global__ __launch_bounds__(kW4Waves* kWave, w4_occupancy(RT, NB)) void experts_w4_kernel(W4Params p) {
  constexpr int kRouting = ROUTED && SWIGLU;                     // workgroup 0 routes
  __shared__ __align__(16) float s_acc[kW4Waves * RT * NB * kWave * 4];
  __shared__ W4Rows s_rows[1];                                   // the routed form alone
  static_assert(!kRouting || sizeof(s_acc) >= 2 * kW4Waves * kRouteTokensPerWave * kMaxK * 4, "the selection's words");
  int id = (int)blockIdx.x - kRouting;
  if (kRouting && id < 0) {
    w4_route(p.route, reinterpret_cast<int32_t*>(s_acc), s_acc + kW4Waves * kRouteTokensPerWave * kMaxK);
    return;
  }
  if ((id | 63) < (int)gridDim.x - kRouting) id = (id & ~63) | (id & 7) << 3 | (id >> 3 & 7);
  const int e = id / p.n_items, item = id - e * p.n_items;
  int row0 = 0, rows;
  if constexpr (!ROUTED) {
    row0 = p.offsets[e];
    rows = p.offsets[e + 1] - row0;
  } else if constexpr (SWIGLU) {
    rows = w4_select(p.route, e, s_rows, reinterpret_cast<int32_t*>(s_acc));
  } else {
    rows = w4_selected(p.route, e, s_rows);
  }
  const size_t blocks = (size_t)e * (p.K / 32) * p.cols;
#pragma unroll 1
  for (int m0 = 0; m0 < rows; m0 += RT * 16) {                   // no rows: the weights are not touched
    if (m0) __syncthreads();                                     // s_acc has been read
    w4_rows<RT, NB, SWIGLU, ROUTED>(p, p.q + blocks * 16, p.scale + blocks, item, row0, m0, rows, s_rows, s_acc);
  }
}

// Token rows into tiles: blockIdx.x an expert, blockIdx.y a share of its tiles' 16-byte pieces.
__global__ __launch_bounds__(256) void tiles_w4_kernel(const __bf16* x, const int32_t* token_of, const int32_t* offsets, __bf16* tiles, int K) {
  const int row0 = offsets[blockIdx.x], rows = offsets[blockIdx.x + 1] - row0;
  for (int m0 = 0; m0 < rows; m0 += 16) {
    const int n = min(rows - m0, 16);
    __bf16* tile = tiles + (size_t)(row0 + m0) * K;
    for (int i = blockIdx.y * 256 + threadIdx.x; i < K / 8 * n; i += gridDim.y * 256) {
      const int k8 = i / n, r = i - k8 * n;
      reinterpret_cast<u32x4*>(tile)[i] = *reinterpret_cast<const u32x4*>(x + (size_t)token_of[row0 + m0 + r] * K + k8 * 8);
    }
  }
}

// Combine: out[t,:] = sum over the local slots j of topk_w[t,j] * y[row_of[t,j],:], in slot order: a workgroup per 2048 columns of a token, a
// lane per eight.  The token's local slots are listed first, so that the rows of four of them are under way together.
__global__ __launch_bounds__(256) void combine_w4_kernel(const float* y, const int32_t* row_of, const float* topk_w, __bf16* out, int T, int H,
                                                         int k) {
  __shared__ int32_t s_row[kMaxK];
  __shared__ float s_w[kMaxK];
  const int chunks = (H + 2047) / 2048, lane = lane_id();
  for (long task = blockIdx.x; task < (long)T * chunks; task += gridDim.x) {
    const long t = task / chunks;
    const int c = ((int)(task - t * chunks) * 256 + threadIdx.x) * 8;
    const int r = lane < k ? row_of[t * k + lane] : -1;
    const float w = lane < k ? topk_w[t * k + lane] : 0.f;
    const uint64_t local = __ballot(r >= 0);
    const int n = __popcll(local);
    __syncthreads();                                             // the list of the task before has been read
    if (threadIdx.x < kWave && r >= 0) {
      const int m = __popcll(local & ((1ull << lane) - 1));
      s_row[m] = r;
      s_w[m] = w;
    }
    __syncthreads();
    if (c >= H) continue;
    f32x4 lo = {0.f, 0.f, 0.f, 0.f}, hi = lo;
    for (int j = 0; j < n; j += 4) {
      f32x4 a[4], b[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const f32x4* src = reinterpret_cast<const f32x4*>(y + (size_t)s_row[min(j + q, n - 1)] * H + c);
        a[q] = src[0];
        b[q] = src[1];
      }
#pragma unroll
      for (int q = 0; q < 4; ++q)
        if (j + q < n) {
          lo += s_w[j + q] * a[q];
          hi += s_w[j + q] * b[q];
        }
    }
    *reinterpret_cast<u32x4*>(out + (size_t)t * H + c) =
        u32x4{pack_bf16(lo[0], lo[1]), pack_bf16(lo[2], lo[3]), pack_bf16(hi[0], hi[1]), pack_bf16(hi[2], hi[3])};
  }
}

// Weights to blocks: a lane per block.  The scale brings the largest magnitude of the 32 into [4, 8), values are rounded to the nearest
// code (ties to the even one), those above 6 to 6.  A block of zeros has scale 1.  Non-finite values have no code: the block's
// scale is 255.  Bound by the weights' read, once: 32 x 7168 x 4096 bf16 (2.4 GB with the blocks) 531 us, 4.5 TB/s where a large copy takes
// 436; fp32 759 us, 5.6 TB/s.
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
