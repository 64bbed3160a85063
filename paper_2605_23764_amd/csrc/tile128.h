// A tile of 256 x 256, 128 x 128 or 64 x 64 of C[i,j] = sum over k of P[i,k] Q[j,k], both operands fp16 or pairs of it and k-contiguous: the K loop of the
// orthogonal updates beside that of the grouped products (gemm_bf16.h), which multiplies tiles of 256 x 256 without pairs.
//
// STAGES of 64 halves per row and side in LDS: two, and two workgroups to a CU, or four and one (64 x 64: two), whose copies are then three
// steps under way.  Lines and their swizzle are those of the grouped products.  Pairs: a row is [k / 32][hi 32 | lo 32], so that a line of
// 128 bytes has both halves of 32 k, and the fragments serve three products, hi hi, lo hi and hi lo, all into one sum (into two, for half the
// roundings, they would leave tiles of 256 x 256 no registers: 4 of 1408 x 2048 off by 2.4e-6 so, 1.3e-6 with two, fp32 products 3.4e-6).
//
// With pairs, 256 tiles of 128 x 128 of 64 steps in 53 us: the MFMAs alone would take 25, with launch and epilogue 35, the copies alone 30,
// without copies 42, without operand reads 41.  A step's 64 KB of operand reads and 32 KB of copies keep LDS busy for as many clocks as its MFMAs
// last, and one wave on a SIMD does not cover what the barrier costs it.
#pragma once
#include "gemm_bf16.h"

namespace moe {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
template <>                                // 16 bits of any kind travel as bf16x8
__device__ __forceinline__ f32x16 mfma_16bit<true>(const bf16x8& a, const bf16x8& b, const f32x16& c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

constexpr int tile_stage(int side) { return 2 * side * 128; }    // bytes

// SIDE 256: by four waves of 128 x 128; 128: by four of 64 x 64; 64: by two of 32 x 64.  P, Q: the matrices from the first step's columns on,
// row_bytes (below 2^32 / rows) from row to row.
template <int SIDE, bool PAIRS, int STAGES>
__device__ __forceinline__ void tile_multiply(const char* Pv, const char* Qv, int row_bytes, int rows, int cols, int i0, int j0, int n_steps, char* smem,
                                              f32x16 (&acc)[SIDE / 64][SIDE == 256 ? 4 : 2]) {
  constexpr int BI = SIDE / 64, BJ = SIDE == 256 ? 4 : 2, kWaves = SIDE == 64 ? 2 : 4, kStage = tile_stage(SIDE);
  constexpr int kLines = SIDE / 8 / kWaves, kCopies = 2 * kLines;   // of eight rows that a wave copies, per side and of both
  int lane = lane_id();
  asm volatile("" : "+v"(lane));           // see gemm_tile_bf16
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = SIDE == 64 ? wave : wave >> 1, wn = SIDE == 64 ? 0 : wave & 1;
  const int l32 = lane & 31, lh = lane >> 5;
  const int kc_r = lane >> 3;
  const int kc_c = (lane & 7) ^ ((4 * (wave & 1) + (kc_r >> 1)) & 7);
  uint32_t off[kCopies];                   // of the lines that this wave copies: P's, then Q's
#pragma unroll
  for (int i = 0; i < kLines; ++i) {       // rows past the end read the last one again; they are not stored
    const int r = (wave + kWaves * i) * 8 + kc_r;
    off[i] = (uint32_t)min(i0 + r, rows - 1) * (uint32_t)row_bytes + (uint32_t)(kc_c * 16);
    off[kLines + i] = (uint32_t)min(j0 + r, cols - 1) * (uint32_t)row_bytes + (uint32_t)(kc_c * 16);
  }
  const char *P = uniform_ptr(Pv), *Q = uniform_ptr(Qv);
  const uint32_t lds0 = uniform_u32(lds_addr_of(smem) + (uint32_t)(wave * kLine));
  // copy i of a step into its stage
  auto copy = [&](auto ic, const char* ps, const char* qs, uint32_t stage) __attribute__((always_inline)) {
    constexpr int i = decltype(ic)::value;
    if constexpr (i < kLines) lds_dma16_at<kWaves * i * kLine>(ps, off[i], stage);
    else lds_dma16_at<SIDE * 128 + kWaves * (i - kLines) * kLine>(qs, off[i], stage);
  };
#pragma unroll
  for (int i = 0; i < BI; ++i)
#pragma unroll
    for (int j = 0; j < BJ; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;

  // A part of a step: a slice of 16 k, or of pairs 16 k's both halves; a side's fragments: those of its blocks of 32 rows, of
  // pairs first all hi, then all lo.
  constexpr int kParts = PAIRS ? 2 : 4, kP = BI * (PAIRS ? 2 : 1), kQ = BJ * (PAIRS ? 2 : 1), kMfma = BI * BJ * (PAIRS ? 3 : 1);
  uint32_t at_p[4], at_q[4];               // a lane's place in a stage, per slice
  {
    const uint32_t f = (uint32_t)((l32 >> 1) & 7), lane_at = lds_addr_of(smem) + (uint32_t)((l32 >> 3) * kLine + (l32 & 7) * 128);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      at_p[q] = lane_at + (uint32_t)(wm * BI * 4 * kLine) + ((((uint32_t)(q * 2 + lh)) ^ f) & 7) * 16;
      at_q[q] = lane_at + (uint32_t)(SIDE * 128 + wn * BJ * 4 * kLine) + ((((uint32_t)(q * 2 + lh)) ^ f) & 7) * 16;
    }
  }
  struct Frags { bf16x8 p[kP], q[kQ]; };
  auto read = [&](Frags& f, auto rc, int part, uint32_t stage) __attribute__((always_inline)) {     // read r of kP + kQ
    constexpr int r = decltype(rc)::value, x = r < kP ? r : r - kP, B = r < kP ? BI : BJ;
    const uint32_t at = (r < kP ? at_p : at_q)[part + (x / B) * 2] + stage;
    const bf16x8 v = *(lds_bf16x8_cptr)((lds_cptr)(uintptr_t)at + (x % B) * 4 * kLine);
    if constexpr (r < kP) f.p[x] = v;
    else f.q[x] = v;
  };
  // The part's MFMAs with the next part's operand reads between them, and copies FROM .. TO - 1 of a step: a wave is alone on its
  // SIMD, or with one other, and what it issues in a row leaves the matrix core idle.  Reads come first, as they are needed first.
  auto multiply = [&](const Frags& f, Frags& next, bool reads, int part, uint32_t stage, auto from, auto to, const char* ps, const char* qs,
                      uint32_t dst) __attribute__((always_inline)) {
    constexpr int kFrom = decltype(from)::value, kNow = decltype(to)::value - kFrom, kReads = kP + kQ;
    constexpr int kPer = PAIRS ? 2 : 1, kBusy = PAIRS ? (kReads + kPer - 1) / kPer : 0;   // reads behind an MFMA; MFMAs that have them
    static_for<0, kMfma>([&](auto mc) __attribute__((always_inline)) {
      constexpr int m = decltype(mc)::value, i = m / BJ % BI, j = m % BJ, kind = m / (BI * BJ);     // kind: hi hi, lo hi, hi lo
      acc[i][j] = mfma_16bit<true>(f.q[kind == 2 ? kQ - BJ + j : j], f.p[kind == 1 ? kP - BI + i : i], acc[i][j]);
      static_for<0, kReads>([&](auto rc) __attribute__((always_inline)) {
        constexpr int at = decltype(rc)::value / kPer;
        if constexpr ((at < kMfma ? at : kMfma - 1) == m) {
          if (reads) read(next, rc, part, stage);
        }
      });
      static_for<0, kNow>([&](auto cc) __attribute__((always_inline)) {
        constexpr int c = decltype(cc)::value;
        if constexpr (kBusy + c * (kMfma - kBusy) / kNow == m) copy(std::integral_constant<int, c + kFrom>{}, ps, qs, dst);
      });
      __builtin_amdgcn_sched_barrier(0);
    });
  };
  typedef std::integral_constant<int, 0> C0;
  // Copies of a step: with two stages all between the last part's MFMAs, as their place is free behind the barrier ahead of it and they are
  // needed a step later; with four a part's share in each from there on: the waves' 32 in a row keep the CU's address unit busy for longer than
  // the MFMAs beside them last (all steps of one 2048 x 2048 in bf16 314 us, spread 284).
  constexpr bool kSpread = STAGES == 4;
  constexpr int kShare = kSpread ? kCopies / kParts : kCopies;
  static_assert(STAGES == 2 || kCopies == 8, "counts of copies under way");
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
      static_for<0, (kSpread && s == STAGES - 1 ? kShare : kCopies)>(
          [&](auto ic) __attribute__((always_inline)) { copy(ic, P + s * 128, Q + s * 128, lds0 + s * kStage); });
  });
  if (STAGES == 4 && n_steps >= 4) wait_vmcnt<16 + kShare>();
  else if (STAGES == 4 && n_steps == 3) wait_vmcnt<16>();
  else if (n_steps >= 2) wait_vmcnt<kCopies>();
  else wait_vmcnt<0>();
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  static_for<0, kP + kQ>([&](auto rc) __attribute__((always_inline)) { read(fa, rc, 0, 0); });
  // where the copies that come next are from: those of step s + STAGES - 1 until the barrier of step s, of the step behind it from there on
  const char *ps = P + (kSpread ? STAGES - 1 : STAGES) * 128, *qs = Q + (kSpread ? STAGES - 1 : STAGES) * 128;
  uint32_t stage = 0;                                          // bytes from the first stage
  // A step.  FIRST: with the rest of the copies of the step STAGES - 1 later, into the stage of the step before (SPREAD); MORE: with those that
  // come first of the step STAGES later, into this one's.  The barrier is ahead of the last part, whose operands are in registers then.
  auto step = [&](auto first, auto more, bool last, int ahead) __attribute__((always_inline)) {
    constexpr bool FIRST = decltype(first)::value, MORE = decltype(more)::value;
    const uint32_t before = lds0 + (stage == 0 ? (STAGES - 1) * kStage : stage - kStage);
    static_for<0, kParts - 1>([&](auto pc) __attribute__((always_inline)) {
      constexpr int part = decltype(pc)::value, kFrom = FIRST ? kShare * (part + 1) : 0, kTo = FIRST ? kFrom + kShare : 0;
      multiply(part & 1 ? fb : fa, part & 1 ? fa : fb, true, part + 1, stage, std::integral_constant<int, kFrom>{}, std::integral_constant<int, kTo>{}, ps, qs,
               before);
    });
    static_assert(kParts % 2 == 0, "parts");
    if (kSpread) {
      ps += 128;
      qs += 128;
    }
    const uint32_t old = stage;
    stage = stage == (STAGES - 1) * kStage ? 0 : stage + kStage;
    if (!last) settle(ahead);
    if constexpr (MORE) {
      multiply(fb, fa, true, 0, stage, C0{}, std::integral_constant<int, kShare>{}, ps, qs, lds0 + old);
      if (!kSpread) {
        ps += 128;
        qs += 128;
      }
    } else {
      multiply(fb, fa, !last, 0, stage, C0{}, C0{}, nullptr, nullptr, 0);
    }
  };
  typedef std::integral_constant<bool, kSpread> Spread;
  int s = 0;
  for (; s + STAGES < n_steps; ++s) step(Spread{}, std::true_type{}, false, STAGES - 2);
  if (kSpread && s + STAGES == n_steps) {
    step(Spread{}, std::false_type{}, false, STAGES - 2);
    ++s;
  }
  for (; s < n_steps; ++s) step(std::false_type{}, std::false_type{}, s + 1 == n_steps, n_steps - 2 - s);
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();            // every wave has read its last operands
  asm volatile("" ::: "memory");
}

}  // namespace moe
