// Tiles of the attention kernels: rows of a [rows, heads, dim] tensor in LDS,
// brought there by direct loads, and the matrix-instruction fragments read
// from them, for both storage types.
#pragma once
#include "common.h"
#include "seq.h"

namespace lat {

// Eight consecutive values along a contraction, one lane's share of a 32 x 16
// operand (lane: row lane % 32, contraction index 8 (lane / 32) + e).
template <typename T> struct Frag;
template <> struct Frag<bf16_t> { bf16x8 v; };
template <> struct Frag<float> { float v[8]; };

// c += A B^T over 16 contraction indices, 32 x 32.  Element r of c: row
// 8 (r / 4) + 4 (lane / 32) + r % 4 of A, row lane % 32 of B.  fp32 takes
// eight 32x32x2 products, product e over index e of both lane halves: the
// order of a contraction is free as long as both operands agree.
__device__ inline void mma32(const Frag<bf16_t>& a, const Frag<bf16_t>& b, f32x16& c) {
  c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.v, b.v, c, 0, 0, 0);
}
__device__ inline void mma32(const Frag<float>& a, const Frag<float>& b, f32x16& c) {
#pragma unroll
  for (int e = 0; e < 8; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a.v[e], b.v[e], c, 0, 0, 0);
}

// Elements 8 half .. 8 half + 7 of a product c as the B operand of the next one:
// contraction slot e of lane half h is then row 16 half + 8 (e / 4) + 4 h + e % 4,
// which Tile::colfrag follows, so a product's result feeds the next product
// from its own registers.
__device__ inline void pack_frag(const f32x16& c, int half, Frag<bf16_t>& f) {
  u32x4 w;
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = pack_bf2(c[8 * half + 2 * i], c[8 * half + 2 * i + 1]);
  f.v = __builtin_bit_cast(bf16x8, w);
}
__device__ inline void pack_frag(const f32x16& c, int half, Frag<float>& f) {
#pragma unroll
  for (int e = 0; e < 8; ++e) f.v[e] = c[8 * half + e];
}

// 8 consecutive elements from memory, zeros where !ok
__device__ inline void load_frag(const bf16_t* p, bool ok, Frag<bf16_t>& f) {
  u32x4 w = ldg16(p);
  f.v = __builtin_bit_cast(bf16x8, ok ? w : u32x4{0u, 0u, 0u, 0u});
}
__device__ inline void load_frag(const float* p, bool ok, Frag<float>& f) {
  const f32x4 a = *reinterpret_cast<const f32x4*>(p), b = *reinterpret_cast<const f32x4*>(p + 4);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    f.v[e] = ok ? a[e] : 0.f;
    f.v[4 + e] = ok ? b[e] : 0.f;
  }
}
__device__ inline float dot_frag(const Frag<bf16_t>& a, const Frag<bf16_t>& b) {
  const u32x4 x = __builtin_bit_cast(u32x4, a.v), y = __builtin_bit_cast(u32x4, b.v);
  float u[8], w[8], s = 0.f;
  Vec16<bf16_t>::unpack(x, u);
  Vec16<bf16_t>::unpack(y, w);
#pragma unroll
  for (int e = 0; e < 8; ++e) s += u[e] * w[e];
  return s;
}
__device__ inline float dot_frag(const Frag<float>& a, const Frag<float>& b) {
  float s = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) s += a.v[e] * b.v[e];
  return s;
}

__device__ inline bool nonfinite(float x) { return (__float_as_uint(x) & 0x7f800000u) == 0x7f800000u; }
// A fragment's finite values, zeros elsewhere (drop 0); or ones where it is
// neither finite nor the infinity whose 32 bits are `drop`.
__device__ inline Frag<float> finite_or_count(const Frag<float>& f, uint32_t drop) {
  Frag<float> o;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const uint32_t x = __float_as_uint(f.v[e]);
    const bool nf = nonfinite(f.v[e]);
    o.v[e] = __uint_as_float(drop ? (nf && x != drop ? 0x3f800000u : 0u) : nf ? 0u : x);
  }
  return o;
}
__device__ inline Frag<bf16_t> finite_or_count(const Frag<bf16_t>& f, uint32_t drop) {
  u32x4 w = __builtin_bit_cast(u32x4, f.v);
  auto half = [&](uint32_t x) __attribute__((always_inline)) {     // a bf16 in the upper half of x
    const bool nf = (x & 0x7f800000u) == 0x7f800000u;
    return drop ? (nf && x != drop ? 0x3f800000u : 0u) : nf ? 0u : x;
  };
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = half(w[i] & 0xffff0000u) | (half(w[i] << 16) >> 16);
  return {__builtin_bit_cast(bf16x8, w)};
}

typedef __attribute__((address_space(3))) void seq_lds_void;
typedef short seq_i16x4 __attribute__((ext_vector_type(4)));

// Rows of DP elements (dim padded to 32, 64 or 128) in LDS, unpadded, in
// 16-byte units; unit c of row r lies at c ^ swz(r).  swz is linear over the
// bits of r and puts, for row fragments (32 rows, one unit each), eight
// consecutive rows on distinct banks, and, for column fragments by transposed
// reads (four consecutive rows, 64 bytes each), those four rows on distinct
// quarters of the banks.
template <typename T, int DP>
struct Tile {
  static constexpr int RB = DP * (int)sizeof(T);   // bytes of a row
  static constexpr int UPR = RB / 16;              // units of a row
  static constexpr int KS = DP / 16;               // contraction steps over a row
  static constexpr int DB = DP / 32;               // 32-wide blocks of a row
  __host__ __device__ static constexpr int swz(int r) {
    return RB == 64 ? (r >> 2) & 3
         : RB == 128 ? (((r >> 1) & 1) << 2) | ((r >> 2) & 3)
         : RB == 256 ? ((r & 3) << 2) | ((r >> 2) & 3)
                     : r & 15;
  }
  // Lane's address parts (bytes); a constant row (bits apart from the
  // lane's) and unit are added by at().
  __device__ static inline uint32_t row_lane() {
    const int lane = threadIdx.x & 63, r = lane & 31, u = (lane >> 5) * (sizeof(T) == 2 ? 1 : 2);
    return (uint32_t)(r * RB + ((u ^ swz(r)) << 4));
  }
  __device__ static inline uint32_t col_lane() {
    const int lane = threadIdx.x & 63, h = lane >> 5;
    if constexpr (sizeof(T) == 2) {
      const int g = lane >> 4, j = lane & 15;
      const int r = 4 * h + (j >> 2), col = 16 * (g & 1) + 4 * (j & 3);
      return (uint32_t)(r * RB + (((col >> 3) ^ swz(r)) << 4) + (col & 7) * 2);
    } else {
      const int r = 4 * h, col = lane & 31;
      return (uint32_t)(r * RB + (((col >> 2) ^ swz(r)) << 4) + (col & 3) * 4);
    }
  }
  __device__ static inline uint32_t at(uint32_t lane, int row, int unit) {
    return (lane ^ (uint32_t)((unit ^ swz(row)) << 4)) + (uint32_t)(row * RB);
  }
  // rows row0 .. row0+31 (a multiple of 32), elements 16 s + 8 (lane / 32) + e
  __device__ static inline Frag<T> rowfrag(const char* S, uint32_t rl, int row0, int s) {
    Frag<T> f;
    if constexpr (sizeof(T) == 2) {
      f.v = *reinterpret_cast<const bf16x8*>(S + at(rl, row0, 2 * s));
    } else {
      const f32x4 a = *reinterpret_cast<const f32x4*>(S + at(rl, row0, 4 * s));
      const f32x4 b = *reinterpret_cast<const f32x4*>(S + at(rl, row0, 4 * s + 1));
#pragma unroll
      for (int e = 0; e < 4; ++e) { f.v[e] = a[e]; f.v[4 + e] = b[e]; }
    }
    return f;
  }
  // Transposed: lane's row is element 32 db + lane % 32, contraction slot e is
  // row row0 + 8 (e / 4) + 4 (lane / 32) + e % 4 (row0 a multiple of 16).
  // bf16: ds_read_b64_tr_b16 returns to lane j of a 16-lane group, as element
  // e, element j % 4 of the 8 bytes addressed by lane 4 e + j / 4.
  __device__ static inline Frag<T> colfrag(const char* S, uint32_t cl, int row0, int db) {
    Frag<T> f;
    if constexpr (sizeof(T) == 2) {
      typedef __attribute__((address_space(3))) seq_i16x4 lds_v4;
      const seq_i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4*)(S + at(cl, row0, 4 * db)));
      const seq_i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4*)(S + at(cl, row0 + 8, 4 * db)));
      f.v = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        f.v[e] = *reinterpret_cast<const float*>(S + at(cl, row0 + 8 * (e >> 2) + (e & 3), 8 * db));
    }
    return f;
  }
};

// Direct loads of R rows of a tensor into a Tile by NW waves: R * UPR units,
// 64 consecutive ones a wave load.  Rows from `rows` on (or whose bit of
// `keep` is 0), and units past dim, become zeros: their offset lies past the
// buffer.
template <typename T, int DP, int R, int NW>
struct TileLoad {
  using TL = Tile<T, DP>;
  static constexpr int PER = R * TL::UPR / 64 / NW;
  static_assert(PER * 64 * NW == R * TL::UPR, "whole wave loads");
  uint32_t off[PER];
  int row[PER];
  __device__ inline void init(int wave, int dim, int64_t ld) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int u = 0; u < PER; ++u) {
      const int unit = (u * NW + wave) * 64 + lane, r = unit / TL::UPR, c = (unit % TL::UPR) ^ TL::swz(r);
      row[u] = r;
      off[u] = c * 16 < dim * (int)sizeof(T) ? (uint32_t)(r * (ld * (int)sizeof(T)) + c * 16) : 0x80000000u;
    }
  }
  __device__ inline void issue(char* S, int wave, const T* p, int rows, uint64_t keep) const {
    const __amdgpu_buffer_rsrc_t rs =
        __builtin_amdgcn_make_buffer_rsrc(const_cast<T*>(p), (short)0, (int)0x7fffffff, BUF_RSRC_WORD3);
#pragma unroll
    for (int u = 0; u < PER; ++u) {
      const bool ok = row[u] < rows && ((keep >> (row[u] & 63)) & 1);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (seq_lds_void*)(S + (u * NW + wave) * 1024), 16,
                                               (int)(ok ? off[u] : 0x80000000u), 0, 0, 0);
    }
  }
};

// A value of the lane and of lane +- 32 joined, in registers.
__device__ inline float max32(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ inline float add32(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ inline bool wave_all(bool b) { return __ballot(!b) == 0; }
__device__ inline bool wave_any(bool b) { return __ballot(b) != 0; }

}  // namespace lat
