// Rows of eight-element vectors: what the row operators (layer_norm.h) share.
//
// A row of H elements is ceil(H / 8) vectors.  Every vector is one 16-byte load (fp32: two), also in rows of odd H that start at no
// multiple of 16 bytes: global memory takes vector accesses at any element's address.  Only a row's last vector may be short
// (TAIL: H % 8 != 0): it is loaded as the row's last eight elements and moved down, and stored element by element.
#pragma once
#include "common.h"
#include "philox.h"

namespace moe {

// Eight elements as they lie in memory.
template <typename T> struct Raw8;
template <> struct Raw8<__bf16> { uint32_t w[4]; };
template <> struct Raw8<float> { uint32_t w[8]; };

template <typename T> __device__ __forceinline__ float raw_get(const Raw8<T>& r, int x) {
  if constexpr (sizeof(T) == 2) return (x & 1) ? bf16_hi(r.w[x >> 1]) : bf16_lo(r.w[x >> 1]);
  else return __builtin_bit_cast(float, r.w[x]);
}

template <typename T> __device__ __forceinline__ Raw8<T> raw_zero() {
  Raw8<T> r;
#pragma unroll
  for (int i = 0; i < (int)(sizeof(r.w) / 4); ++i) r.w[i] = 0;
  return r;
}

typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));   // 16 bytes at any element's address

// Elements i .. i + 7 of a row of H; those past the end are zero.  A short last vector is the row's last eight elements moved down: one
// load like the others' (in rows of fewer than eight, element by element).  The load alone, whose result nothing waits for yet, and the
// rest of it.  NT: non-temporal, for what is read once and larger than the caches.
template <typename T, bool TAIL, bool NT = false> __device__ __forceinline__ Raw8<T> raw_request(const T* row, int i, int H) {
  Raw8<T> r;
  if (TAIL && H < 8) {
    r = raw_zero<T>();
#pragma unroll
    for (int x = 0; x < 7; ++x)
      if (x < H) {
        if constexpr (sizeof(T) == 2) r.w[x >> 1] |= (uint32_t)__builtin_bit_cast(uint16_t, row[x]) << (16 * (x & 1));
        else r.w[x] = __builtin_bit_cast(uint32_t, row[x]);
      }
    return r;
  }
  const u32x4_any* src = reinterpret_cast<const u32x4_any*>(row + (TAIL ? min(i, H - 8) : i));
#pragma unroll
  for (int v = 0; v < (int)sizeof(r) / 16; ++v) {
    const u32x4_any a = NT ? __builtin_nontemporal_load(src + v) : src[v];
#pragma unroll
    for (int w = 0; w < 4; ++w) r.w[4 * v + w] = a[w];
  }
  return r;
}
template <typename T, bool TAIL> __device__ __forceinline__ void raw_trim(Raw8<T>& r, int i, int H) {
  constexpr int kWords = sizeof(r) / 4;
  if (!TAIL || H < 8) return;
  const int down = max(i + 8 - H, 0);                            // elements, 0 .. 7 in lanes with a part of the row
#pragma unroll
  for (int bit = 4; bit >= 1; bit >>= 1) {
    const bool on = (down & bit) != 0;
    if (sizeof(T) == 2 && bit == 1) {
#pragma unroll
      for (int w = 0; w < kWords; ++w) {
        const uint32_t up = w + 1 < kWords ? r.w[w + 1] : 0;
        r.w[w] = on ? r.w[w] >> 16 | up << 16 : r.w[w];
      }
    } else {
      const int step = sizeof(T) == 2 ? bit / 2 : bit;
#pragma unroll
      for (int w = 0; w < kWords; ++w) {
        const uint32_t up = w + step < kWords ? r.w[w + step] : 0;
        r.w[w] = on ? up : r.w[w];
      }
    }
  }
}
template <typename T, bool TAIL, bool NT = false> __device__ __forceinline__ Raw8<T> raw_load(const T* row, int i, int H) {
  Raw8<T> r = raw_request<T, TAIL, NT>(row, i, H);
  raw_trim<T, TAIL>(r, i, H);
  return r;
}

// Waits for a load here.  Placed ahead of a turn's stores: waiting behind them would be for them as well, as loads and stores are counted
// together and the compiler cannot tell how many of these (lanes past the row have none) follow the load.
template <typename T> __device__ __forceinline__ void raw_settle(Raw8<T>& r) {
#pragma unroll
  for (int i = 0; i < (int)(sizeof(r.w) / 4); ++i) asm volatile("" : "+v"(r.w[i]));
}

// Rounded to T, once.
template <typename T> __device__ __forceinline__ Raw8<T> raw_pack(const float (&v)[8]) {
  Raw8<T> r;
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int x = 0; x < 4; ++x) r.w[x] = pack_bf16(v[2 * x], v[2 * x + 1]);
  } else {
#pragma unroll
    for (int x = 0; x < 8; ++x) r.w[x] = __builtin_bit_cast(uint32_t, v[x]);
  }
  return r;
}

template <typename T, bool TAIL, bool NT = false> __device__ __forceinline__ void raw_store(T* row, int i, int H, const Raw8<T>& r) {
  if (!TAIL || i + 8 <= H) {
    u32x4_any* dst = reinterpret_cast<u32x4_any*>(row + i);
#pragma unroll
    for (int v = 0; v < (int)sizeof(r) / 16; ++v) {
      const u32x4_any a = {r.w[4 * v], r.w[4 * v + 1], r.w[4 * v + 2], r.w[4 * v + 3]};
      if (NT) __builtin_nontemporal_store(a, dst + v);
      else dst[v] = a;
    }
  } else {
#pragma unroll
    for (int x = 0; x < 7; ++x)
      if (i + x < H) {
        if constexpr (sizeof(T) == 2) row[i + x] = __builtin_bit_cast(T, (uint16_t)(r.w[x >> 1] >> (16 * (x & 1))));
        else row[i + x] = __builtin_bit_cast(T, r.w[x]);
      }
  }
}

// Dropout: the element's 16 random bits are kept if at least `thr` (= 65536 p), and kept values are scaled by `scale`.
struct DropParams {
  const uint64_t* rng;   // device {seed, offset}; read only if thr > 0
  uint32_t thr;          // 0 (nothing is dropped) .. 65536 (everything is)
  float scale;           // 65536 / (65536 - thr); 0 if everything is dropped
};
struct DropKey { uint32_t k0, k1, o0, o1; };

__device__ __forceinline__ DropKey drop_key(const DropParams& d) {
  DropKey k = {0, 0, 0, 0};
  if (d.thr) {
    const uint64_t seed = d.rng[0], offset = d.rng[1];
    k = DropKey{(uint32_t)seed, (uint32_t)(seed >> 32), (uint32_t)offset, (uint32_t)(offset >> 32)};
  }
  return k;
}

// v[x] = kept ? scale * v[x] : 0 for the vector `vec` of row t.  A select, not a product: what is dropped may hold anything.
__device__ __forceinline__ void drop8(float (&v)[8], const DropParams& d, const DropKey& k, uint32_t t, uint32_t vec) {
  if (d.thr == 0) return;
  const Philox4 r = philox4x32_10(vec, t, k.o0, k.o1, k.k0, k.k1);
#pragma unroll
  for (int x = 0; x < 8; ++x) {
    const uint32_t u = (x & 1) ? r.w[x >> 1] >> 16 : r.w[x >> 1] & 0xFFFFu;
    v[x] = u >= d.thr ? v[x] * d.scale : 0.f;
  }
}

// Sum over the G lanes that hold one row (G: 8, 16, 32, 64, or whole waves), the same in all of them.  A wave: DPP exchanges inside
// 16 lanes, then the two lane-row swaps; several waves meet in `s` (kMaxWaves words per value, this call's alone until the next
// barrier but one) behind one barrier, which every wave of the workgroup has to reach.  The order is fixed.
constexpr int kRowMaxWaves = 16;
template <int N> __device__ __forceinline__ void group_sum(float (&v)[N], int G, float* s) {
#pragma unroll
  for (int n = 0; n < N; ++n) {
#define MOE_ADD(ctrl) v[n] += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v[n]), ctrl, 0xf, 0xf, false))
    MOE_ADD(0xB1);                                               // neighbour, other pair of four, half of eight
    MOE_ADD(0x4E);
    MOE_ADD(0x141);
    if (G >= 16) MOE_ADD(0x140);
#undef MOE_ADD
    if (G >= 32) {
      const auto r = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, v[n]), __builtin_bit_cast(uint32_t, v[n]), false, false);
      v[n] = __builtin_bit_cast(float, (uint32_t)r[0]) + __builtin_bit_cast(float, (uint32_t)r[1]);
    }
    if (G >= 64) {
      const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, v[n]), __builtin_bit_cast(uint32_t, v[n]), false, false);
      v[n] = __builtin_bit_cast(float, (uint32_t)r[0]) + __builtin_bit_cast(float, (uint32_t)r[1]);
    }
  }
  if (G <= kWave) return;
  const int wave = threadIdx.x / kWave, W = G / kWave, first = wave / W * W;
  if (lane_id() == 0)
#pragma unroll
    for (int n = 0; n < N; ++n) s[n * kRowMaxWaves + wave] = v[n];
  __syncthreads();
#pragma unroll
  for (int n = 0; n < N; ++n) {
    float t = 0.f;
    for (int w = 0; w < W; ++w) t += s[n * kRowMaxWaves + first + w];
    v[n] = t;
  }
}

}  // namespace moe
