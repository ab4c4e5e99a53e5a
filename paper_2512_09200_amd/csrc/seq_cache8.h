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
#include "seq_tile.h"

namespace lat {

constexpr int CACHE8_BLOCK = 16;

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

// A wave's view of a block: lane l holds slot l / 4, elements (l % 4) E .. + E - 1
// of a row padded to DP.
template <int DP> struct Block8 {
  static constexpr int E = DP / 4, W = E / 4;        // elements, code words
  float x[E];
  __device__ static inline int slot() { return (threadIdx.x & 63) >> 2; }
  __device__ static inline int first() { return (threadIdx.x & 3) * E; }

  // rows of the storage type; p: the row's first element (valid memory whether `on` or not)
  template <typename T>
  __device__ inline void from_row(const T* p, int dim, bool on) {
#pragma unroll
    for (int i = 0; i < E; i += 8) {
      const int d = first() + i;
      const bool ok = on && d < dim;
      Frag<T> f;
      load_frag(p + (d < dim ? d : 0), ok, f);
      float y[8];
      if constexpr (sizeof(T) == 2) {
        Vec16<bf16_t>::unpack(__builtin_bit_cast(u32x4, f.v), y);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = f.v[e];
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) x[i + e] = y[e];
    }
  }
  // codes of a row (ld bytes); adds to x where `on`, which the caller cleared
  __device__ inline void from_codes(const uint8_t* p, float s, int dim, int ld, bool on) {
#pragma unroll
    for (int i = 0; i < E; i += 8) {
      const int d = first() + i;
      const u32x2 w = *reinterpret_cast<const u32x2*>(p + (d < ld ? d : 0));
      const bool ok = on && d < dim;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const f32x2_t a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[j], false);
        const f32x2_t b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[j], true);
        const float y[4] = {a[0] * s, a[1] * s, b[0] * s, b[1] * s};
#pragma unroll
        for (int e = 0; e < 4; ++e) x[i + 4 * j + e] = ok ? y[e] : x[i + 4 * j + e];
      }
    }
  }
  // the wave's scale
  __device__ inline float scale() const {
    float top = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) top = fmaxf(top, nonfinite(x[e]) ? 0.f : fabsf(x[e]));
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
    return cache8_scale(top);
  }
  __device__ inline void codes(float s, uint32_t (&w)[W]) const {
#pragma unroll
    for (int i = 0; i < W; ++i) w[i] = cache8_codes(x + 4 * i, s);
  }
  // a row's codes to memory, `ld` bytes of it
  __device__ static inline void store(uint8_t* p, int ld, const uint32_t (&w)[W]) {
#pragma unroll
    for (int i = 0; i < W; i += 2)
      if (first() + 4 * i < ld) *reinterpret_cast<u32x2*>(p + first() + 4 * i) = u32x2{w[i], w[i + 1]};
  }
};

}  // namespace lat
