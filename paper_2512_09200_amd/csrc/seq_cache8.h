// Blocks of 16 slots of an 8-bit ring cache: e4m3 codes under one power-of-two
// scale.
//
// Why a power of two: an event that raises or lowers its block's scale has the
// block's other codes written anew, and dividing e4m3 values by a power of two is
// exact until they become subnormal (2^-6 of a value range of 2^8: 14 halvings
// below the block's largest), so the many rewrites of a block's life lose nothing that a
// single one would not.  Why e4m3: its relative step does not grow when a
// large neighbour sets the scale.
#pragma once
#include "e4m3.h"
#include "lanes.h"
#include "seq_fill8.h"
#include "seq_tile.h"

namespace lat {

// The smallest power of two s >= 2^-117 with top <= 448 s (448 = 1.75 2^8); 1 for 0.
__host__ __device__ inline float cache8_scale(float top) {
  union { float f; uint32_t u; } v;
  v.f = top;
  if (!(top > 0.f)) return 1.f;
  int e = (int)(v.u >> 23) - 8 + ((v.u & 0x7fffffu) > 0x600000u);      // exponents with their bias
  e = e < 10 ? 10 : e;
  v.u = (uint32_t)e << 23;
  return v.f;
}
__host__ __device__ inline float pow2_inv(float s) {                   // 1 / s, s a power of two of 2^-126 .. 2^126
  union { float f; uint32_t u; } v;
  v.f = s;
  v.u = (254u << 23) - v.u;
  return v.f;
}

// Four codes of scaled values; one that is not finite becomes NaN (0x7f).  Codes times
// the scale stay finite: 256 * 2^120 would not (values next to fp32's largest).
__device__ inline uint32_t cache8_codes(const float* x, float s) {
  const float inv = pow2_inv(s), lim = s >= 0x1p120f ? 240.f : E4M3_MAX;
  float v[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = __builtin_amdgcn_fmed3f(x[e] * inv, -lim, lim);
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(v[0], v[1], 0, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(v[2], v[3], w, true);
  uint32_t u = (uint32_t)w;
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (nonfinite(x[e])) u = (u & ~(0xffu << (8 * e))) | 0x7fu << (8 * e);
  return u;
}

// A wave's view of a block: lane l holds slot l / 4, of its row (padded to DP) the
// elements 16 (l % 4) .. + 15 of every 64 (8 (l % 4) .. + 7 where DP is 32) in chunks
// of eight, as the memory words of a fresh row (of T) or of old codes.  Four lanes'
// codes are 64 neighbouring bytes.
// Values are decoded where they are used, eight at a time: once for the scale,
// once for the codes.
template <typename T, int DP> struct Block8 {
  static constexpr int C = DP / 32;                  // chunks of a lane
  Frag<T> row[C];
  u32x2 code[C];
  bool fresh, old;
  float s0;

  __device__ static inline int slot() { return (threadIdx.x & 63) >> 2; }
  __device__ static inline int at(int i) {           // the chunk's first element
    const int l = threadIdx.x & 3;
    return DP == 32 ? 8 * l : 16 * (l + 4 * (i >> 1)) + 8 * (i & 1);
  }

  // p: the row's first element, valid memory in any case
  __device__ inline void load_row(const T* p, int dim, bool on) {
    fresh = on;
#pragma unroll
    for (int i = 0; i < C; ++i) {
      const int d = at(i);
      load_frag(p + (d < dim ? d : 0), on && d < dim, row[i]);
    }
  }
  // p: a row of ld bytes, valid memory in any case
  __device__ inline void load_codes(const uint8_t* p, int ld) {
#pragma unroll
    for (int i = 0; i < C; ++i) {
      const int d = at(i);
      code[i] = *reinterpret_cast<const u32x2*>(p + (d < ld ? d : 0));
    }
  }
  __device__ inline void chunk(int i, int dim, float (&x)[8]) const {
    if constexpr (sizeof(T) == 2) {
      Vec16<bf16_t>::unpack(__builtin_bit_cast(u32x4, row[i].v), x);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = row[i].v[e];
    }
    const bool on = old && at(i) < dim;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const f32x2_t a = j & 1 ? __builtin_amdgcn_cvt_pk_f32_fp8((int)code[i][j >> 1], true)
                              : __builtin_amdgcn_cvt_pk_f32_fp8((int)code[i][j >> 1], false);
#pragma unroll
      for (int e = 0; e < 2; ++e) x[2 * j + e] = fresh ? x[2 * j + e] : on ? a[e] * s0 : 0.f;
    }
  }
  // The scale of a block of fresh rows alone, all finite (else false: the general
  // way).  The largest magnitude is that of the bits, two bf16 an operation; the general
  // way's 25 operations an element would be above the fill's memory time.
  __device__ inline bool fresh_scale(float* s) const {
    uint32_t top = 0;
    if constexpr (sizeof(T) == 2) {
      typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
      u16x2 m{0, 0};
#pragma unroll
      for (int i = 0; i < C; ++i) {
        const u32x4 w = __builtin_bit_cast(u32x4, row[i].v);
#pragma unroll
        for (int j = 0; j < 4; ++j) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, w[j] & 0x7fff7fffu));
      }
      top = (uint32_t)max(m[0], m[1]) << 16;
    } else {
#pragma unroll
      for (int i = 0; i < C; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(row[i].v[e]) & 0x7fffffffu);
    }
    top = __builtin_amdgcn_readfirstlane(lanes_join<64>(top, Max()));
    *s = cache8_scale(__uint_as_float(top));
    return top < 0x7f800000u && *s < 0x1p120f;
  }
  // Their codes: |x| <= 448 s, nothing to clamp
  __device__ inline void encode_fresh(float s, uint8_t* p, int ld) const {
    constexpr int N = DP == 32 ? 1 : 2;
    typedef typename std::conditional<N == 1, u32x2, u32x4>::type V;
    const float inv = pow2_inv(s);
#pragma unroll
    for (int i = 0; i < C; i += N) {
      V w;
#pragma unroll
      for (int j = 0; j < N; ++j) {
        float x[8];
        if constexpr (sizeof(T) == 2) {
          Vec16<bf16_t>::unpack(__builtin_bit_cast(u32x4, row[i + j].v), x);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] = row[i + j].v[e];
        }
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          int c = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * y] * inv, x[4 * y + 1] * inv, 0, false);
          c = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * y + 2] * inv, x[4 * y + 3] * inv, c, true);
          w[2 * j + y] = (uint32_t)c;
        }
      }
      if (fresh && at(i) < ld) *reinterpret_cast<V*>(p + at(i)) = w;
    }
  }
  // the wave's scale
  __device__ inline float scale(int dim) const {
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < C; ++i) {
      float x[8];
      chunk(i, dim, x);
#pragma unroll
      for (int e = 0; e < 8; ++e) top = fmaxf(top, nonfinite(x[e]) ? 0.f : fabsf(x[e]));
    }
    return cache8_scale(lanes_join<64>(top, Max()));
  }
  // Codes under scale s to p (a row of ld bytes) where `write`, and to q (DP bytes)
  // where it is not null.
  __device__ inline void encode(float s, int dim, uint8_t* p, int ld, bool write, uint8_t* q) const {
    constexpr int N = DP == 32 ? 1 : 2;               // chunks of a store
    typedef typename std::conditional<N == 1, u32x2, u32x4>::type V;
#pragma unroll
    for (int i = 0; i < C; i += N) {
      V w;
#pragma unroll
      for (int j = 0; j < N; ++j) {
        float x[8];
        chunk(i + j, dim, x);
        w[2 * j] = cache8_codes(x, s);
        w[2 * j + 1] = cache8_codes(x + 4, s);
      }
      const int d = at(i);                            // (ld is a multiple of 16)
      if (write && d < ld) *reinterpret_cast<V*>(p + d) = w;
      if (q) *reinterpret_cast<V*>(q + d) = w;
    }
  }
};

}  // namespace lat
