// Eight neighbouring elements of a row: the unit of the row kernels, at any
// alignment (gfx950 takes 16-byte accesses at any address of the element's own
// alignment).
#pragma once
#include "common.h"

namespace lat {

typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));

template <typename T> struct Row8 {
  static constexpr int W = (int)sizeof(T) / 2;      // 16-byte words: bf16 1, fp32 2
  u32x4 w[W];
  __device__ inline void get(float (&o)[8]) const {
#pragma unroll
    for (int i = 0; i < W; ++i) Vec16<T>::unpack(w[i], o + i * Vec16<T>::N);
  }
  __device__ inline void put(const float (&o)[8]) {
#pragma unroll
    for (int i = 0; i < W; ++i) w[i] = Vec16<T>::pack(o + i * Vec16<T>::N);
  }
  __device__ inline void clear() {
#pragma unroll
    for (int i = 0; i < W; ++i) w[i] = u32x4{0u, 0u, 0u, 0u};
  }
};

// Elements n .. of r move to 0 .., zeros behind them (0 <= n < 8, the same for
// every lane that uses the result).
__device__ inline void shift8(Row8<bf16_t>& r, int n) {
  u32x4 v = r.w[0];
  if (n & 4) v = u32x4{v[2], v[3], 0u, 0u};
  if (n & 2) v = u32x4{v[1], v[2], v[3], 0u};
  if (n & 1) v = u32x4{v[0] >> 16 | v[1] << 16, v[1] >> 16 | v[2] << 16, v[2] >> 16 | v[3] << 16, v[3] >> 16};
  r.w[0] = v;
}
__device__ inline void shift8(Row8<float>& r, int n) {
  const u32x4 z{0u, 0u, 0u, 0u};
  u32x4 a = r.w[0], b = r.w[1];
  if (n & 4) { a = b; b = z; }
  if (n & 2) { a = u32x4{a[2], a[3], b[0], b[1]}; b = u32x4{b[2], b[3], 0u, 0u}; }
  if (n & 1) { a = u32x4{a[1], a[2], a[3], b[0]}; b = u32x4{b[1], b[2], b[3], 0u}; }
  r.w[0] = a;
  r.w[1] = b;
}

// Group g (columns 8 g .. 8 g + 7) of a row of `cols` elements, as memory words that
// fix8 makes the group's values of, where they are used: a load whose value is
// selected or branched on at once is waited for there.  TAIL: cols is no multiple of
// 8; the last group is read as the row's last eight elements, so that no load
// leaves the row.  NT: past the caches (data that is larger than they are).
template <typename T, bool TAIL, bool NT = false>
__device__ inline Row8<T> load8(const T* row, int g, int cols) {
  Row8<T> r;
  if (TAIL && cols < 8) {
    uint32_t x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const T v = row[e < cols ? e : 0];
      if constexpr (sizeof(T) == 2) x[e] = v; else x[e] = __float_as_uint(v);
    }
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int i = 0; i < 4; ++i) r.w[0][i] = x[2 * i] | x[2 * i + 1] << 16;
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) r.w[e >> 2][e & 3] = x[e];
    }
    return r;
  }
  const int c = 8 * g < cols - 8 ? 8 * g : cols - 8;
  const char* p = reinterpret_cast<const char*>(row + c);
#pragma unroll
  for (int i = 0; i < Row8<T>::W; ++i) {
    const u32x4_any* q = reinterpret_cast<const u32x4_any*>(p + 16 * i);
    r.w[i] = NT ? __builtin_nontemporal_load(q) : *q;
  }
  return r;
}

// The group's values; columns past the row are zeros.
template <typename T, bool TAIL>
__device__ inline void fix8(Row8<T>& r, int g, int cols) {
  if (TAIL && 8 * g > cols - 8) {
    if (cols < 8) {                                   // (read in their own places)
      Row8<T> m = r;
      r.clear();
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e < cols) {
          if constexpr (sizeof(T) == 2) r.w[0][e >> 1] |= m.w[0][e >> 1] & (e & 1 ? 0xffff0000u : 0xffffu);
          else r.w[e >> 2][e & 3] = m.w[e >> 2][e & 3];
        }
    } else {
      shift8(r, 8 - (cols & 7));
    }
  }
  if (8 * g >= cols) r.clear();
}

template <typename T, bool TAIL, bool NT = false>
__device__ inline void store8(T* row, int g, int cols, const Row8<T>& r) {
  if (8 * g >= cols) return;
  char* p = reinterpret_cast<char*>(row + 8 * g);
  if (TAIL && 8 * g > cols - 8) {
    // four, two and one elements, as cols has them
    Row8<T> s = r;
    typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(2)));
    typedef uint32_t u32_any __attribute__((aligned(2)));
    constexpr int B = sizeof(T);
    if (cols & 4) {
      if constexpr (B == 2) *reinterpret_cast<u32x2_any*>(p) = u32x2_any{s.w[0][0], s.w[0][1]};
      else *reinterpret_cast<u32x4_any*>(p) = s.w[0];
      p += 4 * B;
      shift8(s, 4);
    }
    if (cols & 2) {
      if constexpr (B == 2) *reinterpret_cast<u32_any*>(p) = s.w[0][0];
      else *reinterpret_cast<u32x2_any*>(p) = u32x2_any{s.w[0][0], s.w[0][1]};
      p += 2 * B;
      shift8(s, 2);
    }
    if (cols & 1) {
      if constexpr (B == 2) *reinterpret_cast<bf16_t*>(p) = (bf16_t)s.w[0][0];
      else *reinterpret_cast<float*>(p) = __uint_as_float(s.w[0][0]);
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < Row8<T>::W; ++i) {
    u32x4_any* q = reinterpret_cast<u32x4_any*>(p + 16 * i);
    if (NT) __builtin_nontemporal_store((u32x4_any)r.w[i], q); else *q = r.w[i];
  }
}

}  // namespace lat
