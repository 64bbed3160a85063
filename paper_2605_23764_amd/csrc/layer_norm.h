// Layer norm, dropout with residual, and the two in one pass, forward and backward.
//
//   z = residual + drop(v)                 (layer norm alone: z is the input)
//   y = (z - mean) * rstd * gamma + beta   mean, rstd = 1 / sqrt(var + eps) of the row of z as it is stored
//   backward: t = dy * gamma, xh = (z - mean) * rstd,
//     dz = rstd * (t - mean(t) - xh * mean(t * xh)) + dres;  dv = drop'(dz);  dgamma = sum dy * xh, dbeta = sum dy over rows
//
// A handful of flops per element: what bounds them is the bytes, each array once.  So a row stays in the registers of the lanes that
// read it (a vector of eight per lane, up to 16 waves a row; longer rows are read again), mean and variance are taken one after the other from
// there (no cancellation), and the dropout bits are made again from the counter instead of stored.
// All sums are fp32, in a fixed order.
#pragma once
#include "rows.h"

namespace moe {

constexpr int kRowMaxH = kRowMaxWaves * kWave * 8;               // longest row that stays in registers
constexpr int kNormMaxParts = 256;                               // partial sums of dgamma / dbeta, at most: workgroups of the backward
// norm_backward_few_kernel takes up to so many rows, in arrays of up to so many bytes, in workgroups of up to so many lanes
constexpr int kNormFewRows = 1024;
constexpr size_t kNormFewBytes = 6u << 20;
constexpr int kNormFewLanes = 1024;

// Arrays are [T, H], vectors [H]; what may be null is looked at once per launch.
struct NormForwardParams {
  const void *v, *x;              // v: dropped and added to x (fused form only); x may be null there
  const void *gamma, *beta;       // null: 1, 0
  void *z, *y;                    // z: fused form only
  float *mean, *rstd;             // [T], may be null
  DropParams drop;
  float eps;
  int T, H, group;
};

struct NormBackwardParams {
  const void *dy, *x, *gamma, *dres;   // gamma, dres may be null
  const float *mean, *rstd;
  void *dx, *dv;                       // dv: fused form only
  float* part;                         // [parts][2][H] sums of dy * xh and dy, null: not wanted (here)
  void *dgamma, *dbeta;                // the launch of few rows alone: either may be null
  int row_groups;                      // its workgroups for rows; those behind them have columns
  DropParams drop;
  float inv_h;
  int T, H, group, groups;             // lanes per row; rows that a workgroup has in hand at a time
};

template <typename T> __device__ __forceinline__ const T* row_of(const void* p, int t, int H) {
  return static_cast<const T*>(p) + (size_t)t * H;
}
template <typename T> __device__ __forceinline__ T* row_of(void* p, int t, int H) { return static_cast<T*>(p) + (size_t)t * H; }

// NT (these kernels and drop_add; arrays above kNormNtBytes): what is read or written once in the training step (y, v and the residual, dy,
// dres, dx, dv) passes the caches by, which leaves them to x or z, read again by the backward.  T = 8192, H = 7168 bf16 (117 MB an array): forward + backward
// 147 -> 140 us, with dropout and residual 209 -> 200, and 184 -> 182 with the residual; where everything fits into the caches it costs up to a fifth.
constexpr size_t kNormNtBytes = 64u << 20;

// A group of lanes per row, ITEMS vectors per lane; groups of up to a wave share a workgroup.  Workgroups walk rows in strides, the next
// row's loads under way while this one is reduced, with gamma and beta in registers (a workgroup per row instead, 14 waves: 100 us for 43).
// T = 8192, H = 7168 bf16: 43 us, 5.5 TB/s; with dropout and residual 86 us, 5.5 TB/s (a large copy: 5.46).
template <typename T, int ITEMS, bool TAIL, bool FUSED, bool NT>
__global__ __launch_bounds__(512) void norm_forward_kernel(NormForwardParams p) {
  __shared__ float s_sum[2][kRowMaxWaves];
  const int G = p.group, H = p.H;
  const int g = G > kWave ? (int)threadIdx.x : (int)threadIdx.x & (G - 1);
  const int rows = G > kWave ? 1 : blockDim.x / G, r = G > kWave ? 0 : threadIdx.x / G;
  const DropKey key = FUSED ? drop_key(p.drop) : DropKey{};
  Raw8<T> gamma[ITEMS], beta[ITEMS];
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    const int at = (i * G + g) * 8;
    gamma[i] = p.gamma && at < H ? raw_load<T, TAIL>(static_cast<const T*>(p.gamma), at, H) : raw_zero<T>();
    beta[i] = p.beta && at < H ? raw_load<T, TAIL>(static_cast<const T*>(p.beta), at, H) : raw_zero<T>();
  }
  struct Row { Raw8<T> x[ITEMS], v[FUSED ? ITEMS : 1]; };
  auto load = [&](Row& q, long t) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      const int at = (i * G + g) * 8;
      q.x[i] = raw_zero<T>();
      if (FUSED) q.v[i] = raw_zero<T>();
      if (t < p.T && at < H) {
        if (p.x) q.x[i] = raw_request<T, TAIL, NT && FUSED>(row_of<T>(p.x, (int)t, H), at, H);
        if (FUSED) q.v[i] = raw_request<T, TAIL, NT>(row_of<T>(p.v, (int)t, H), at, H);
      }
    }
  };
  const long stride = (long)gridDim.x * rows;
  Row cur;
  load(cur, (long)blockIdx.x * rows + r);
  for (long t0 = (long)blockIdx.x * rows; t0 < p.T; t0 += stride) {
    const int t = (int)min(t0 + r, (long)p.T);
    Row next;
    load(next, t0 + r + stride);
    float sum[1] = {0.f}, sq[1] = {0.f};
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      const int vec = i * G + g, at = vec * 8;
      raw_trim<T, TAIL>(cur.x[i], at, H);
      if (FUSED) raw_trim<T, TAIL>(cur.v[i], at, H);
      if (FUSED && t < p.T && at < H) {
        float v[8];
#pragma unroll
        for (int x = 0; x < 8; ++x) v[x] = raw_get<T>(cur.v[i], x);
        drop8(v, p.drop, key, (uint32_t)t, (uint32_t)vec);
#pragma unroll
        for (int x = 0; x < 8; ++x) v[x] += raw_get<T>(cur.x[i], x);
        cur.x[i] = raw_pack<T>(v);                               // z is an output, and y the norm of it as it is stored
        raw_store<T, TAIL>(row_of<T>(p.z, t, H), at, H, cur.x[i]);
      }
#pragma unroll
      for (int x = 0; x < 8; ++x) sum[0] += raw_get<T>(cur.x[i], x);                    // 0 outside the row
    }
    group_sum<1>(sum, G, s_sum[0]);
    const float mean = sum[0] / (float)H;                        // not * (1 / H): a constant row then has mean x, variance 0
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      const int at = (i * G + g) * 8;
#pragma unroll
      for (int x = 0; x < 8; ++x) {
        const float d = raw_get<T>(cur.x[i], x) - mean;
        if (TAIL ? at + x < H : at < H) sq[0] += d * d;
      }
    }
    group_sum<1>(sq, G, s_sum[1]);
    const float rstd = 1.0f / sqrtf(sq[0] / (float)H + p.eps);
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      raw_settle<T>(next.x[i]);
      if (FUSED) raw_settle<T>(next.v[i]);
    }
    if (t < p.T) {
      if (g == 0) {
        if (p.mean) p.mean[t] = mean;
        if (p.rstd) p.rstd[t] = rstd;
      }
#pragma unroll
      for (int i = 0; i < ITEMS; ++i) {
        const int at = (i * G + g) * 8;
        if (at >= H) continue;
        float o[8];
#pragma unroll
        for (int x = 0; x < 8; ++x) {
          o[x] = (raw_get<T>(cur.x[i], x) - mean) * rstd;
          if (p.gamma) o[x] *= raw_get<T>(gamma[i], x);
          if (p.beta) o[x] += raw_get<T>(beta[i], x);
        }
        raw_store<T, TAIL, NT>(row_of<T>(p.y, t, H), at, H, raw_pack<T>(o));
      }
    }
    cur = next;
  }
}

// A workgroup walks rows in strides with `groups` of them in hand, the next ones' loads under way while these are reduced, and keeps
// its rows' sums of dy * xh and dy in registers: one partial per workgroup at the end, a row per CU and 15 MB in all at H = 7168 (two
// workgroups per CU with twice the partials: +1 .. +3 us).  T = 8192, H = 7168 bf16: 76 us, 6.4 TB/s (x still comes from the
// memory-side cache in part); with dropout 101 us, 5.8 TB/s.
// block: this workgroup among n_blocks.  s_part, for several groups' sums: [groups][4][G][4].
template <typename T, bool TAIL, bool FUSED, bool NT>
__device__ __forceinline__ void norm_backward_rows(const NormBackwardParams& p, int block, int n_blocks, float* s_part) {
  __shared__ float s_sum[2][2][kRowMaxWaves];
  const int G = p.group, H = p.H;
  const int rg = threadIdx.x / G, g = threadIdx.x - rg * G, at = g * 8;
  const DropKey key = FUSED ? drop_key(p.drop) : DropKey{};
  float acc_g[8], acc_b[8];
#pragma unroll
  for (int x = 0; x < 8; ++x) acc_g[x] = acc_b[x] = 0.f;
  const Raw8<T> gamma = p.gamma && at < H ? raw_load<T, TAIL>(static_cast<const T*>(p.gamma), at, H) : raw_zero<T>();
  struct Row { Raw8<T> dy, x, dres; float mean, rstd; };
  auto load = [&](Row& r, int t) __attribute__((always_inline)) {
    const bool live = t < p.T;
    r.mean = live ? p.mean[t] : 0.f;
    r.rstd = live ? p.rstd[t] : 0.f;
    r.dy = r.x = r.dres = raw_zero<T>();
    if (live && at < H) {
      r.dy = raw_request<T, TAIL, NT>(row_of<T>(p.dy, t, H), at, H);
      r.x = raw_request<T, TAIL>(row_of<T>(p.x, t, H), at, H);
      if (p.dres) r.dres = raw_request<T, TAIL, NT>(row_of<T>(p.dres, t, H), at, H);
    }
  };
  const int stride = n_blocks * p.groups;
  Row cur;
  load(cur, block * p.groups + rg);
  // as many turns for every group of the workgroup: the barrier of a turn is reached by all.  (64 bits: t0 + stride may pass 2^31.)
  int turn = 0;
  for (long t0 = (long)block * p.groups; t0 < p.T; t0 += stride, turn ^= 1) {
    const int t = (int)min(t0 + rg, (long)p.T);
    Row next;
    load(next, (int)min(t0 + rg + stride, (long)p.T));
    raw_trim<T, TAIL>(cur.dy, at, H);
    raw_trim<T, TAIL>(cur.x, at, H);
    raw_trim<T, TAIL>(cur.dres, at, H);
    float dxh[8], xh[8], sum[2] = {0.f, 0.f};
#pragma unroll
    for (int x = 0; x < 8; ++x) {
      const float d = raw_get<T>(cur.dy, x);                     // 0 outside the row
      xh[x] = (raw_get<T>(cur.x, x) - cur.mean) * cur.rstd;
      if (TAIL ? at + x >= H : at >= H) xh[x] = 0.f;             // there x is not, and 0 * rstd may be no number
      dxh[x] = p.gamma ? d * raw_get<T>(gamma, x) : d;
      acc_g[x] += d * xh[x];
      acc_b[x] += d;
      sum[0] += dxh[x];
      sum[1] += dxh[x] * xh[x];
    }
    group_sum<2>(sum, G, &s_sum[turn][0][0]);
    const float m1 = sum[0] * p.inv_h, m2 = sum[1] * p.inv_h;
    float o[8];
#pragma unroll
    for (int x = 0; x < 8; ++x) o[x] = cur.rstd * (dxh[x] - m1 - xh[x] * m2) + raw_get<T>(cur.dres, x);
    raw_settle<T>(next.dy);
    raw_settle<T>(next.x);
    raw_settle<T>(next.dres);
    if (t < p.T && at < H) {
      raw_store<T, TAIL, NT>(row_of<T>(p.dx, t, H), at, H, raw_pack<T>(o));
      if (FUSED) {
        drop8(o, p.drop, key, (uint32_t)t, (uint32_t)g);
        raw_store<T, TAIL, NT>(row_of<T>(p.dv, t, H), at, H, raw_pack<T>(o));
      }
    }
    cur = next;
  }
  if (!p.part) return;
  float* out = p.part + (size_t)block * 2 * H;
  if (p.groups == 1) {
    if (at >= H) return;
    raw_store<float, TAIL>(out, at, H, raw_pack<float>(acc_g));
    raw_store<float, TAIL>(out + H, at, H, raw_pack<float>(acc_b));
    return;
  }
  // the groups' sums of a column meet, a quarter of a lane's 16 sums (four columns of dgamma or dbeta) to a group at a time
  f32x4* s = reinterpret_cast<f32x4*>(s_part);
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    s[(rg * 4 + h) * G + g] = f32x4{acc_g[4 * h], acc_g[4 * h + 1], acc_g[4 * h + 2], acc_g[4 * h + 3]};
    s[(rg * 4 + 2 + h) * G + g] = f32x4{acc_b[4 * h], acc_b[4 * h + 1], acc_b[4 * h + 2], acc_b[4 * h + 3]};
  }
  __syncthreads();
  for (int q = rg; q < 4; q += p.groups) {
    f32x4 t = {0.f, 0.f, 0.f, 0.f};
    for (int r = 0; r < p.groups; ++r) t += s[(r * 4 + q) * G + g];
    float* to = out + (q >> 1) * H;
    const int c = at + (q & 1) * 4;
    if (c + 4 <= H) {
      *reinterpret_cast<u32x4_any*>(to + c) = __builtin_bit_cast(u32x4_any, t);
    } else if (TAIL) {
#pragma unroll
      for (int x = 0; x < 3; ++x)
        if (c + x < H) to[c + x] = t[x];
    }
  }
}

template <typename T, bool TAIL, bool FUSED, bool NT>
__global__ __launch_bounds__(1024) void norm_backward_kernel(NormBackwardParams p) {
  extern __shared__ __align__(16) float s_part[];
  norm_backward_rows<T, TAIL, FUSED, NT>(p, blockIdx.x, gridDim.x, s_part);
}

// Few rows in one launch: workgroups behind those of the rows take 64 columns each and go down all rows of dy and x for
// them, mostly out of the L2s, so nothing has to meet across workgroups and the launch that adds up partial sums goes
// away.  dx and dv may not lie over dy or x while both kinds run: then the columns have a launch of their own first, in the
// same order.  Forward and backward of a step, two launches for the backward -> one, us: 64 x 2048 bf16 20.2 -> 14.9, 600 x
// 4096 19.2 -> 17.0, 800 x 1408 fp32 19.0 -> 16.2; with dropout 600 x 1408 fp32 20.8 -> 16.7, 700 x 4096 bf16 23.2 -> 22.0.
// Past the limits the columns' workgroups are too few for their bytes and too long for their rows: 512 x 7168 (7 MB) 20.8
// -> 20.9, 1000 x 4096 (8 MB) 19.8 -> 24.4, 1500 x 512 18.4 -> 19.2, 3000 x 256 17.5 -> 30.8.  512 lanes in place of 1024:
// 3 us more at 1000 x 512, level at few rows.
template <typename T, bool TAIL, bool FUSED>
__global__ __launch_bounds__(1024) void norm_backward_few_kernel(NormBackwardParams p) {
  __shared__ float s_col[2][kRowMaxWaves][kWave];
  if ((int)blockIdx.x < p.row_groups) {
    norm_backward_rows<T, TAIL, FUSED, false>(p, blockIdx.x, p.row_groups, nullptr);
    return;
  }
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), waves = blockDim.x / kWave, lane = lane_id();
  const int col = ((int)blockIdx.x - p.row_groups) * kWave + lane, at = min(col, p.H - 1);
  float g = 0.f, b = 0.f;
#pragma unroll 8
  for (int t = wave; t < p.T; t += waves) {
    const float d = (float)row_of<T>(p.dy, t, p.H)[at], x = (float)row_of<T>(p.x, t, p.H)[at];
    g += d * ((x - p.mean[t]) * p.rstd[t]);
    b += d;
  }
  s_col[0][wave][lane] = g;
  s_col[1][wave][lane] = b;
  __syncthreads();
  T* out = static_cast<T*>(wave ? p.dbeta : p.dgamma);           // one wave dgamma, one dbeta
  if (wave < 2 && col < p.H && out) {
    float t = 0.f;
    for (int w = 0; w < waves; ++w) t += s_col[wave][w][lane];
    out[col] = (T)t;
  }
}

// ---- rows longer than kRowMaxH: a workgroup of 16 waves goes over its row again instead of keeping it (from the L2) ----
// T = 2048, H = 16384 bf16: forward 32 us, backward 54, column sums 22 + 5; reading everything once would take 25, 49 and nothing.
template <typename T, bool TAIL, bool FUSED>
__global__ __launch_bounds__(1024) void norm_forward_long_kernel(NormForwardParams p) {
  __shared__ float s_sum[2][kRowMaxWaves];
  const int H = p.H, step = blockDim.x * 8;
  for (long tl = blockIdx.x; tl < p.T; tl += gridDim.x) {
    const int t = (int)tl;
    const T* in = row_of<T>(FUSED ? (const void*)p.z : p.x, t, H);
    const DropKey key = FUSED ? drop_key(p.drop) : DropKey{};
    float sum[1] = {0.f}, sq[1] = {0.f};
    for (int at = threadIdx.x * 8; at < H; at += step) {
      Raw8<T> r = raw_zero<T>();
      if (p.x) r = raw_load<T, TAIL>(row_of<T>(p.x, t, H), at, H);
      if (FUSED) {
        const Raw8<T> rv = raw_load<T, TAIL>(row_of<T>(p.v, t, H), at, H);
        float v[8];
#pragma unroll
        for (int x = 0; x < 8; ++x) v[x] = raw_get<T>(rv, x);
        drop8(v, p.drop, key, (uint32_t)t, (uint32_t)(at / 8));
#pragma unroll
        for (int x = 0; x < 8; ++x) v[x] += raw_get<T>(r, x);
        r = raw_pack<T>(v);
        raw_store<T, TAIL>(row_of<T>(p.z, t, H), at, H, r);        // read again below by the same lane
      }
#pragma unroll
      for (int x = 0; x < 8; ++x) sum[0] += raw_get<T>(r, x);
    }
    group_sum<1>(sum, blockDim.x, s_sum[0]);
    const float mean = sum[0] / (float)H;                          // not * (1 / H): a constant row then has mean x, variance 0
    for (int at = threadIdx.x * 8; at < H; at += step) {
      const Raw8<T> r = raw_load<T, TAIL>(in, at, H);
#pragma unroll
      for (int x = 0; x < 8; ++x) {
        const float d = raw_get<T>(r, x) - mean;
        if (!TAIL || at + x < H) sq[0] += d * d;
      }
    }
    group_sum<1>(sq, blockDim.x, s_sum[1]);
    const float rstd = 1.0f / sqrtf(sq[0] / (float)H + p.eps);
    if (threadIdx.x == 0) {
      if (p.mean) p.mean[t] = mean;
      if (p.rstd) p.rstd[t] = rstd;
    }
    for (int at = threadIdx.x * 8; at < H; at += step) {
      const Raw8<T> r = raw_load<T, TAIL>(in, at, H);
      Raw8<T> rg, rb;
      if (p.gamma) rg = raw_load<T, TAIL>(static_cast<const T*>(p.gamma), at, H);
      if (p.beta) rb = raw_load<T, TAIL>(static_cast<const T*>(p.beta), at, H);
      float o[8];
#pragma unroll
      for (int x = 0; x < 8; ++x) {
        o[x] = (raw_get<T>(r, x) - mean) * rstd;
        if (p.gamma) o[x] *= raw_get<T>(rg, x);
        if (p.beta) o[x] += raw_get<T>(rb, x);
      }
      raw_store<T, TAIL>(row_of<T>(p.y, t, H), at, H, raw_pack<T>(o));
    }
  }
}

template <typename T, bool TAIL, bool FUSED>
__global__ __launch_bounds__(1024) void norm_backward_long_kernel(NormBackwardParams p) {
  __shared__ float s_sum[2][2][kRowMaxWaves];
  const int H = p.H, step = blockDim.x * 8;
  const DropKey key = FUSED ? drop_key(p.drop) : DropKey{};
  int turn = 0;
  for (long tl = blockIdx.x; tl < p.T; tl += gridDim.x, turn ^= 1) {
    const int t = (int)tl;
    const float mean = p.mean[t], rstd = p.rstd[t];
    float sum[2] = {0.f, 0.f};
    auto terms = [&](int at, float (&dxh)[8], float (&xh)[8]) __attribute__((always_inline)) {
      const Raw8<T> rd = raw_load<T, TAIL>(row_of<T>(p.dy, t, H), at, H), rx = raw_load<T, TAIL>(row_of<T>(p.x, t, H), at, H);
      Raw8<T> rg;
      if (p.gamma) rg = raw_load<T, TAIL>(static_cast<const T*>(p.gamma), at, H);
#pragma unroll
      for (int x = 0; x < 8; ++x) {
        xh[x] = TAIL && at + x >= H ? 0.f : (raw_get<T>(rx, x) - mean) * rstd;
        dxh[x] = raw_get<T>(rd, x);
        if (p.gamma) dxh[x] *= raw_get<T>(rg, x);
      }
    };
    for (int at = threadIdx.x * 8; at < H; at += step) {
      float dxh[8], xh[8];
      terms(at, dxh, xh);
#pragma unroll
      for (int x = 0; x < 8; ++x) {
        sum[0] += dxh[x];
        sum[1] += dxh[x] * xh[x];
      }
    }
    group_sum<2>(sum, blockDim.x, &s_sum[turn][0][0]);
    const float m1 = sum[0] * p.inv_h, m2 = sum[1] * p.inv_h;
    for (int at = threadIdx.x * 8; at < H; at += step) {
      float dxh[8], xh[8], o[8];
      terms(at, dxh, xh);
      Raw8<T> rr = raw_zero<T>();
      if (p.dres) rr = raw_load<T, TAIL>(row_of<T>(p.dres, t, H), at, H);
#pragma unroll
      for (int x = 0; x < 8; ++x) o[x] = rstd * (dxh[x] - m1 - xh[x] * m2) + raw_get<T>(rr, x);
      raw_store<T, TAIL>(row_of<T>(p.dx, t, H), at, H, raw_pack<T>(o));
      if (FUSED) {
        drop8(o, p.drop, key, (uint32_t)t, (uint32_t)(at / 8));
        raw_store<T, TAIL>(row_of<T>(p.dv, t, H), at, H, raw_pack<T>(o));
      }
    }
  }
}

// Column sums of the long rows: a lane has eight columns, a workgroup column (blockIdx.y) a share of the rows.
template <typename T, bool TAIL>
__global__ __launch_bounds__(256) void norm_columns_long_kernel(NormBackwardParams p) {
  const int H = p.H, at = (blockIdx.x * 256 + threadIdx.x) * 8;
  if (at >= H) return;
  float acc_g[8], acc_b[8];
#pragma unroll
  for (int x = 0; x < 8; ++x) acc_g[x] = acc_b[x] = 0.f;
  for (long tl = blockIdx.y; tl < p.T; tl += gridDim.y) {
    const int t = (int)tl;
    const Raw8<T> rd = raw_load<T, TAIL>(row_of<T>(p.dy, t, H), at, H), rx = raw_load<T, TAIL>(row_of<T>(p.x, t, H), at, H);
    const float mean = p.mean[t], rstd = p.rstd[t];
#pragma unroll
    for (int x = 0; x < 8; ++x) {
      const float d = raw_get<T>(rd, x);
      acc_g[x] += d * ((raw_get<T>(rx, x) - mean) * rstd);
      acc_b[x] += d;
    }
  }
  float* out = p.part + (size_t)blockIdx.y * 2 * H;
  raw_store<float, TAIL>(out, at, H, raw_pack<float>(acc_g));
  raw_store<float, TAIL>(out + H, at, H, raw_pack<float>(acc_b));
}

// dgamma, dbeta from the partial sums (256 of them at H = 7168: 15 MB, 4.7 us): a workgroup adds 64 columns of one of the two, 16 waves a sixteenth of the partials each.
template <typename T>
__global__ __launch_bounds__(1024) void norm_columns_kernel(const float* part, int parts, int H, void* dgamma, void* dbeta) {
  __shared__ float s[kRowMaxWaves][kWave];
  const int wave = threadIdx.x / kWave, lane = lane_id();
  const int col = blockIdx.x * kWave + lane;
  T* out = static_cast<T*>(blockIdx.y ? dbeta : dgamma);
  if (!out) return;
  float a = 0.f;
  if (col < H) {
    const float* src = part + (size_t)blockIdx.y * H + col;
#pragma unroll 8
    for (int i = wave; i < parts; i += kRowMaxWaves) a += src[(size_t)i * 2 * H];
  }
  s[wave][lane] = a;
  __syncthreads();
  if (wave == 0 && col < H) {
    float t = 0.f;
#pragma unroll
    for (int w = 0; w < kRowMaxWaves; ++w) t += s[w][lane];
    out[col] = (T)t;
  }
}

// ---- dropout + residual alone (and its backward: no residual): two vectors per lane, requested together ----
// The generator takes 20 products of 32 x 32 bits per vector, some 150 instructions, which hide behind the three arrays: T = 8192, H = 7168
// bf16, both directions, 100 us (5.9 TB/s; one vector per lane 105, four 104, by way of the caches 116); T = 4096, H = 2048 18.2 (19.7, 21.2).
struct DropAddParams {
  const void *v, *res;            // res may be null
  void* out;
  DropParams drop;
  int T, H, group;                // lanes per row: a power of two up to kDropGroup
};
constexpr int kDropItems = 2, kDropGroup = 128;

template <typename T, bool TAIL, bool NT>
__global__ __launch_bounds__(256) void drop_add_kernel(DropAddParams p) {
  constexpr int kItems = kDropItems;
  const int H = p.H, rows = 256 / p.group, wide = p.group * 8 * kItems, chunks = (H + wide - 1) / wide;
  const int r = threadIdx.x / p.group, g = threadIdx.x & (p.group - 1);
  const DropKey key = drop_key(p.drop);
  const long tasks = (long)(((uint32_t)p.T + (uint32_t)rows - 1) / (uint32_t)rows) * chunks;   // T may be all that 31 bits hold
  for (long task = blockIdx.x; task < tasks; task += gridDim.x) {
    const long rb = task / chunks;
    const int first = (int)(task - rb * chunks) * p.group * kItems + g;
    const long t = rb * rows + r;
    if (t >= p.T) continue;
    Raw8<T> rv[kItems], rr[kItems];
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      const int at = (first + i * p.group) * 8;
      rr[i] = raw_zero<T>();
      if (at < H) {
        rv[i] = raw_request<T, TAIL, NT>(row_of<T>(p.v, (int)t, H), at, H);
        if (p.res) rr[i] = raw_request<T, TAIL, NT>(row_of<T>(p.res, (int)t, H), at, H);
      }
    }
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      const int vec = first + i * p.group, at = vec * 8;
      if (at >= H) continue;
      raw_trim<T, TAIL>(rv[i], at, H);
      raw_trim<T, TAIL>(rr[i], at, H);
      float v[8];
#pragma unroll
      for (int x = 0; x < 8; ++x) v[x] = raw_get<T>(rv[i], x);
      drop8(v, p.drop, key, (uint32_t)t, (uint32_t)vec);
      if (p.res)
#pragma unroll
        for (int x = 0; x < 8; ++x) v[x] += raw_get<T>(rr[i], x);
      raw_store<T, TAIL, NT>(row_of<T>(p.out, (int)t, H), at, H, raw_pack<T>(v));
    }
  }
}

}  // namespace moe
