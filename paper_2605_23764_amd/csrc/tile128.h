// A tile of 128 x 128 of C[i,j] = sum over k of P[i,k] Q[j,k], both operands of 16 bits and k-contiguous, by four waves of 64 x 64: the K loop
// that the orthogonal updates and the gradient of the router's rows share.
//
// STAGES of 64 halves per row and side in LDS: two, and two workgroups to a CU, or four and one, whose copies are then three steps under
// way.  Lines and their swizzle are those of the grouped products (gemm_bf16.h).  Pairs: a row is [k / 32][hi 32 | lo 32], so that a line of
// 128 bytes has both halves of 32 k, and every fragment read serves three products: hi hi into acc, lo hi and hi lo into mix.
#pragma once
#include "gemm_bf16.h"

namespace moe {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
template <>                                // 16 bits of any kind travel as bf16x8
__device__ __forceinline__ f32x16 mfma_16bit<true>(const bf16x8& a, const bf16x8& b, const f32x16& c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

constexpr int kTile128 = 128, kTile128Stage = 2 * kTile128 * 128;

// P, Q: the matrices from the first step's columns on, row_bytes (below 2^32 / rows) from row to row; F16: fp16, else bf16.
template <bool PAIRS, bool F16, int STAGES>
__device__ __forceinline__ void tile128_multiply(const char* Pv, const char* Qv, int row_bytes, int rows, int cols, int i0, int j0, int n_steps, char* smem,
                                                 f32x16 (&acc)[2][2], f32x16 (&mix)[2][2]) {
  int lane = lane_id();
  asm volatile("" : "+v"(lane));           // see gemm_tile_bf16
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave >> 1, wn = wave & 1;
  const int l32 = lane & 31, lh = lane >> 5;
  const int kc_r = lane >> 3;
  const int kc_c = (lane & 7) ^ ((4 * (wave & 1) + (kc_r >> 1)) & 7);
  uint32_t off[8];                         // of the lines that this wave copies: four of P, four of Q
#pragma unroll
  for (int i = 0; i < 4; ++i) {            // rows past the end read the last one again; they are not stored
    const int r = (wave + 4 * i) * 8 + kc_r;
    off[i] = (uint32_t)min(i0 + r, rows - 1) * (uint32_t)row_bytes + (uint32_t)(kc_c * 16);
    off[4 + i] = (uint32_t)min(j0 + r, cols - 1) * (uint32_t)row_bytes + (uint32_t)(kc_c * 16);
  }
  const char *P = uniform_ptr(Pv), *Q = uniform_ptr(Qv);
  const uint32_t lds0 = uniform_u32(lds_addr_of(smem) + (uint32_t)(wave * kLine));
  // copy i of a step into its stage
  auto copy = [&](auto ic, const char* ps, const char* qs, uint32_t stage) __attribute__((always_inline)) {
    constexpr int i = decltype(ic)::value;
    if constexpr (i < 4) lds_dma16_at<4 * i * kLine>(ps, off[i], stage);
    else lds_dma16_at<kTile128 * 128 + 4 * (i - 4) * kLine>(qs, off[i], stage);
  };
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = mix[i][j][r] = 0.f;

  // A part of a step: a slice of 16 k, or of pairs 16 k's both halves; per side kFrags fragments: block x % 2 of 32 rows, half x / 2.
  constexpr int kParts = PAIRS ? 2 : 4, kFrags = PAIRS ? 4 : 2, kMfma = PAIRS ? 12 : 4;
  uint32_t at_p[4], at_q[4];               // a lane's place in a stage, per slice
  {
    const uint32_t f = (uint32_t)((l32 >> 1) & 7), lane_at = lds_addr_of(smem) + (uint32_t)((l32 >> 3) * kLine + (l32 & 7) * 128);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      at_p[q] = lane_at + (uint32_t)(wm * 8 * kLine) + ((((uint32_t)(q * 2 + lh)) ^ f) & 7) * 16;
      at_q[q] = lane_at + (uint32_t)(kTile128 * 128 + wn * 8 * kLine) + ((((uint32_t)(q * 2 + lh)) ^ f) & 7) * 16;
    }
  }
  struct Frags { bf16x8 p[kFrags], q[kFrags]; };
  auto read = [&](Frags& f, auto rc, int part, uint32_t stage) __attribute__((always_inline)) {     // read r of 2 kFrags
    constexpr int r = decltype(rc)::value, x = r >> 1;
    const uint32_t at = (r & 1 ? at_q : at_p)[part + (x >> 1) * 2] + stage;
    (r & 1 ? f.q : f.p)[x] = *(lds_bf16x8_cptr)((lds_cptr)(uintptr_t)at + (x & 1) * 4 * kLine);
  };
  // The part's MFMAs with the next part's operand reads between them, and behind those CFROM .. CTO - 1 of the copies: a wave is alone on its
  // SIMD, or with one other, and what it issues in a row leaves the matrix core idle.
  auto multiply = [&](const Frags& f, Frags& next, bool reads, int part, uint32_t stage, auto from, auto to, const char* ps, const char* qs,
                      uint32_t dst) __attribute__((always_inline)) {
    constexpr int kFrom = decltype(from)::value, kReads = 2 * kFrags, kActs = kReads + decltype(to)::value - kFrom;
    static_for<0, kMfma>([&](auto mc) __attribute__((always_inline)) {
      constexpr int m = decltype(mc)::value, i = (m >> 1) & 1, j = m & 1, kind = m >> 2;     // kind: hi hi, lo hi, hi lo
      if constexpr (kind == 0) acc[i][j] = mfma_16bit<F16>(f.q[j], f.p[i], acc[i][j]);
      else if constexpr (kind == 1) mix[i][j] = mfma_16bit<F16>(f.q[j], f.p[kFrags - 2 + i], mix[i][j]);
      else mix[i][j] = mfma_16bit<F16>(f.q[kFrags - 2 + j], f.p[i], mix[i][j]);
      static_for<0, kActs>([&](auto ac) __attribute__((always_inline)) {
        constexpr int a = decltype(ac)::value;
        if constexpr (a * kMfma / kActs == m) {
          if constexpr (a < kReads) {
            if (reads) read(next, ac, part, stage);
          } else {
            copy(std::integral_constant<int, a - kReads + kFrom>{}, ps, qs, dst);
          }
        }
      });
      __builtin_amdgcn_sched_barrier(0);
    });
  };
  typedef std::integral_constant<int, 0> C0;
  typedef std::integral_constant<int, 8> C8;
  // Behind it the copies of a step have landed in every wave, but for those of `ahead` later steps, and all have read what they had asked for.
  auto settle = [&](int ahead) __attribute__((always_inline)) {
    if (STAGES == 4 && ahead >= 2) asm volatile("s_waitcnt vmcnt(16) lgkmcnt(0)" ::: "memory");
    else if (STAGES == 4 && ahead == 1) asm volatile("s_waitcnt vmcnt(8) lgkmcnt(0)" ::: "memory");
    else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  Frags fa, fb;
  static_for<0, STAGES>([&](auto sc) __attribute__((always_inline)) {
    constexpr int s = decltype(sc)::value;
    if (s < n_steps)
      static_for<0, 8>([&](auto ic) __attribute__((always_inline)) { copy(ic, P + s * 128, Q + s * 128, lds0 + s * kTile128Stage); });
  });
  if (STAGES == 4 && n_steps >= 4) asm volatile("s_waitcnt vmcnt(24)" ::: "memory");
  else if (STAGES == 4 && n_steps == 3) asm volatile("s_waitcnt vmcnt(16)" ::: "memory");
  else if (n_steps >= 2) asm volatile("s_waitcnt vmcnt(8)" ::: "memory");
  else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  static_for<0, 2 * kFrags>([&](auto rc) __attribute__((always_inline)) { read(fa, rc, 0, 0); });
  const char *ps = P + STAGES * 128, *qs = Q + STAGES * 128;   // of the copies that come next
  uint32_t stage = 0;                                          // bytes from the first stage
  // A step; MORE: with the copies of the step STAGES later, into this one's stage.  The barrier is ahead of the last part, whose operands are
  // in registers then.
  auto step = [&](auto more, bool last, int ahead) __attribute__((always_inline)) {
    constexpr bool MORE = decltype(more)::value;
#pragma unroll
    for (int part = 0; part + 2 < kParts; part += 2) {
      multiply(fa, fb, true, part + 1, stage, C0{}, C0{}, nullptr, nullptr, 0);
      multiply(fb, fa, true, part + 2, stage, C0{}, C0{}, nullptr, nullptr, 0);
    }
    multiply(fa, fb, true, kParts - 1, stage, C0{}, C0{}, nullptr, nullptr, 0);
    const uint32_t old = stage;
    stage = stage == (STAGES - 1) * kTile128Stage ? 0 : stage + kTile128Stage;
    if (!last) settle(ahead);
    if constexpr (MORE) {
      multiply(fb, fa, true, 0, stage, C0{}, C8{}, ps, qs, lds0 + old);
      ps += 128;
      qs += 128;
    } else {
      multiply(fb, fa, !last, 0, stage, C0{}, C0{}, nullptr, nullptr, 0);
    }
  };
  int s = 0;
  for (; s + STAGES < n_steps; ++s) step(std::true_type{}, false, STAGES - 2);
  for (; s < n_steps; ++s) step(std::false_type{}, s + 1 == n_steps, n_steps - 2 - s);
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();            // every wave has read its last operands
  asm volatile("" ::: "memory");
}

}  // namespace moe
