// Root-mean-square norm of a residual sum, and dropout.
//
// Forward:  h = round(drop(x) + r),  rho = 1 / sqrt(mean(h^2) + eps),  y = gain h rho,
// as the storage type, as e4m3 codes with the row's scale, or both.
// Backward, from h alone:  n = h rho,  dn = dy gain,
//   dr = rho (dn - n mean(dn n)) + dh,  dx = drop(dr),  dgain = sum over rows of dy n.
// mean(dn n) = rho sum(dn h) / cols, so one sweep takes both sums of a row, and
// the backward needs no statistic of the forward.
//
// Bound by memory: every tensor is read or written once.  131072 rows of 1024, bf16,
// residual and dropout: forward 193 us at best and 200 on average, backward 245 and 251
// (5.4 and 5.3 TB/s of what they cannot do without; a copy of 0.5 GB reaches 5.3); 8192
// rows to codes 14 us (4.2); dropout alone 83 and 91 us (5.9).  A row's elements stay in registers between the sums
// and the results.  Narrow rows share a wave (2 to 32 lanes each), a row of up to
// 1024 columns has a wave, longer ones a block.  Lanes hold groups of eight
// neighbouring columns (the generator's and the codes' unit); waves walk the rows in
// steps of the grid with the gains (and the gains' gradient) in registers, and the
// next row's loads go out before a row's sums.
//
// Sums are fp32; the residual sum is rounded to the storage type before the norm,
// so that the backward differentiates what the forward computed.
#include "e4m3.h"
#include "kernels.h"
#include "lanes.h"
#include "norm.h"
#include "row8.h"

namespace lat {

// Lanes a row, groups a lane, waves a row
template <int LPR_, int CH_, int WPR_> struct RowCfg {
  static constexpr int LPR = LPR_, CH = CH_, WPR = WPR_;
  static constexpr int THREADS = WPR > 1 ? 64 * WPR : 256;
  static constexpr int RPW = 64 / LPR;                       // rows of a wave
  static constexpr int RPB = WPR > 1 ? 1 : 4 * RPW;          // rows of a block
  static constexpr int STEP = LPR * WPR;                     // groups between a lane's own
  static constexpr int COLS = 8 * CH * STEP;
  static constexpr bool AHEAD = CH <= 2;                     // the next row's loads before a row's sums (registers)
};

struct NormK {
  int64_t rows;
  int cols;
  float eps, inv_cols;
  const float* gain;
  DropArgs drop;
  RowTensor x, r, h, y, dy, dh, dr, dx;
  uint8_t* q;
  int64_t ldq;
  float *scales, *part;
};

// A value of every lane joined over the row's lanes.  Two places of LDS in turn:
// a barrier lies between a place's reads and its next writes.
template <typename C, typename V, int N, typename F>
__device__ inline void row_join(V (&v)[N], F f, V* red, int& turn) {
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = lanes_join<C::LPR>(v[i], f);
  if constexpr (C::WPR > 1) {
    V* p = red + turn * N * C::WPR;
    turn ^= 1;
    if ((threadIdx.x & 63) == 0)
#pragma unroll
      for (int i = 0; i < N; ++i) p[i * C::WPR + (threadIdx.x >> 6)] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      v[i] = p[i * C::WPR];
#pragma unroll
      for (int w = 1; w < C::WPR; ++w) v[i] = f(v[i], p[i * C::WPR + w]);
    }
  }
}

// Where a thread works: its row in the block's, its first group.
template <typename C> struct RowAt {
  int lane, sub;
  int64_t first;                                  // the wave's first row of all (the block's, WPR > 1)
  __device__ inline RowAt() {
    const int l = threadIdx.x & 63, w = threadIdx.x >> 6;
    lane = C::WPR > 1 ? (int)threadIdx.x : l % C::LPR;
    sub = C::WPR > 1 ? 0 : l / C::LPR;
    first = (int64_t)blockIdx.x * C::RPB + (C::WPR > 1 ? 0 : w * C::RPW);
  }
};

template <typename C, bool TAIL>
__device__ inline void load_gain(const NormK& A, int lane, float (&g)[C::CH][8]) {
  Row8<float> r[C::CH];
#pragma unroll
  for (int i = 0; i < C::CH; ++i) {
    if (A.gain) {
      r[i] = load8<float, TAIL>(A.gain, lane + i * C::STEP, A.cols);
      fix8<float, TAIL>(r[i], lane + i * C::STEP, A.cols);
    } else r[i].w[0] = r[i].w[1] = u32x4{0x3f800000u, 0x3f800000u, 0x3f800000u, 0x3f800000u};
    r[i].get(g[i]);
  }
}

template <typename T>
__device__ inline const T* row_of(const RowTensor& t, int64_t row) { return (const T*)t.p + row * t.ld; }

template <typename T, bool TAIL, typename C>
__global__ __launch_bounds__(C::THREADS) void add_rmsnorm_fwd_kernel(NormK A) {
#pragma clang fp contract(off)
  static_assert(C::AHEAD, "the forward's configurations");
  __shared__ float red[2 * C::WPR];
  __shared__ uint32_t red_top[2 * C::WPR];
  int turn = 0, turn_top = 0;
  const RowAt<C> at;
  const DropKey key = drop_key(A.drop);
  float gain[C::CH][8];
  load_gain<C, TAIL>(A, at.lane, gain);
  const int64_t step = (int64_t)gridDim.x * C::RPB;
  Row8<T> xr[C::CH], rr[C::CH];
  auto fetch = [&](int64_t base) {
    int64_t row = base + at.sub;
    row = row < A.rows ? row : A.rows - 1;
#pragma unroll
    for (int i = 0; i < C::CH; ++i) xr[i] = load8<T, TAIL>(row_of<T>(A.x, row), at.lane + i * C::STEP, A.cols);
    if (A.r.p)
#pragma unroll
      for (int i = 0; i < C::CH; ++i) rr[i] = load8<T, TAIL>(row_of<T>(A.r, row), at.lane + i * C::STEP, A.cols);
  };
  if (at.first < A.rows) fetch(at.first);
  for (int64_t base = at.first; base < A.rows; base += step) {
    const int64_t row = base + at.sub;
    const bool live = row < A.rows;
    float h[C::CH][8], s[1] = {0.f};
#pragma unroll
    for (int i = 0; i < C::CH; ++i) {
      fix8<T, TAIL>(xr[i], at.lane + i * C::STEP, A.cols);
      xr[i].get(h[i]);
      if (A.drop.t) drop8(A.drop, key, at.lane + i * C::STEP, (uint32_t)row, h[i]);
      if (A.r.p) {
        float r[8];
        fix8<T, TAIL>(rr[i], at.lane + i * C::STEP, A.cols);
        rr[i].get(r);
#pragma unroll
        for (int e = 0; e < 8; ++e) h[i][e] += r[e];
      }
      Row8<T> o;                                   // the sum as it is kept
      o.put(h[i]);
      if (A.h.p && live) store8<T, TAIL>((T*)A.h.p + row * A.h.ld, at.lane + i * C::STEP, A.cols, o);
      o.get(h[i]);
    }
    if (base + step < A.rows) fetch(base + step);
#pragma unroll
    for (int i = 0; i < C::CH; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) s[0] += h[i][e] * h[i][e];
    row_join<C>(s, Add(), red, turn);
    const float rho = 1.f / sqrtf(s[0] * A.inv_cols + A.eps);
    uint32_t top[1] = {0u};                        // of |y|, in its bits: NaN is above all
#pragma unroll
    for (int i = 0; i < C::CH; ++i) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        h[i][e] = h[i][e] * rho * gain[i][e];
        top[0] = max(top[0], __float_as_uint(h[i][e]) & 0x7fffffffu);
      }
      if (A.y.p && live) {
        Row8<T> o;
        o.put(h[i]);
        store8<T, TAIL>((T*)A.y.p + row * A.y.ld, at.lane + i * C::STEP, A.cols, o);
      }
    }
    if (!A.q) continue;
    row_join<C>(top, Max(), red_top, turn_top);
    // a row that is not finite says so: NaN scale and codes.  A scale is a normal number, as
    // the reciprocal of a smaller one is infinite
    const float amax = __uint_as_float(top[0]);
    const bool bad = !(s[0] < INFINITY) || !(amax < INFINITY);
    const float sc = bad ? NAN : amax > 0.f ? fmaxf(amax / E4M3_MAX, 0x1p-126f) : 1.f, inv = 1.f / sc;
    if (!live) continue;
    if (at.lane == 0) A.scales[row] = sc;
    uint8_t* const q = A.q + row * A.ldq;
#pragma unroll
    for (int i = 0; i < C::CH; ++i) {
      const int c = 8 * (at.lane + i * C::STEP);
      if (c >= A.ldq) continue;
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = c + e < A.cols ? h[i][e] * inv : 0.f;
      u32x2 w{e4m3x4(v[0], v[1], v[2], v[3]), e4m3x4(v[4], v[5], v[6], v[7])};
      if (bad) {
        const int k = A.cols - c;                        // columns of the group (bytes behind them stay 0)
        const uint64_t n = k >= 8 ? ~0ull : k > 0 ? (1ull << (8 * k)) - 1 : 0ull;
        w = __builtin_bit_cast(u32x2, n & 0x7f7f7f7f7f7f7f7full);
      }
      *reinterpret_cast<u32x2*>(q + c) = w;
    }
    for (int64_t c = C::COLS + 8 * at.lane; c < A.ldq; c += 8 * C::STEP) *reinterpret_cast<u32x2*>(q + c) = u32x2{0u, 0u};
  }
}

template <typename T, bool TAIL, bool NT, typename C>
__global__ __launch_bounds__(C::THREADS) void add_rmsnorm_bwd_kernel(NormK A) {
  constexpr int PARTS = C::WPR > 1 ? 1 : 4;
  __shared__ float red[4 * C::WPR];
  __shared__ float sum[PARTS > 1 ? PARTS * C::COLS : 1];
  int turn = 0;
  const RowAt<C> at;
  const DropKey key = drop_key(A.drop);
  float gain[C::CH][8], dg[C::CH][8];
  load_gain<C, TAIL>(A, at.lane, gain);
#pragma unroll
  for (int i = 0; i < C::CH; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) dg[i][e] = 0.f;
  const int64_t step = (int64_t)gridDim.x * C::RPB;
  Row8<T> hr[C::CH], yr[C::CH], rr[C::CH];
  auto fetch = [&](int64_t base) {
    int64_t row = base + at.sub;
    row = row < A.rows ? row : A.rows - 1;
#pragma unroll
    for (int i = 0; i < C::CH; ++i) {
      hr[i] = load8<T, TAIL, NT>(row_of<T>(A.h, row), at.lane + i * C::STEP, A.cols);
      yr[i] = load8<T, TAIL, NT>(row_of<T>(A.dy, row), at.lane + i * C::STEP, A.cols);
    }
    if (A.dh.p)
#pragma unroll
      for (int i = 0; i < C::CH; ++i) rr[i] = load8<T, TAIL, NT>(row_of<T>(A.dh, row), at.lane + i * C::STEP, A.cols);
  };
  if (C::AHEAD && at.first < A.rows) fetch(at.first);
  for (int64_t base = at.first; base < A.rows; base += step) {
    if (!C::AHEAD) fetch(base);
    const int64_t row = base + at.sub;
    const bool live = row < A.rows;
    float h[C::CH][8], dn[C::CH][8], s[2] = {0.f, 0.f};
    Row8<T> add[C::CH];
#pragma unroll
    for (int i = 0; i < C::CH; ++i) {
      fix8<T, TAIL>(hr[i], at.lane + i * C::STEP, A.cols);
      fix8<T, TAIL>(yr[i], at.lane + i * C::STEP, A.cols);
      hr[i].get(h[i]);
      yr[i].get(dn[i]);
      add[i] = rr[i];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        s[0] += h[i][e] * h[i][e];
        s[1] += dn[i][e] * gain[i][e] * h[i][e];
      }
    }
    if (C::AHEAD && base + step < A.rows) fetch(base + step);
    row_join<C>(s, Add(), red, turn);
    const float rho = 1.f / sqrtf(s[0] * A.inv_cols + A.eps);
    // mean(dn n) rho; not from rho^2, which is infinite where a row's root mean square is
    // below 2^-64 (eps 0)
    const float c = rho * (rho * s[1] * A.inv_cols);
#pragma unroll
    for (int i = 0; i < C::CH; ++i) {
      float r[8];
      fix8<T, TAIL>(add[i], at.lane + i * C::STEP, A.cols);
      add[i].get(r);
      float g[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float n = h[i][e] * rho;
        dg[i][e] += live ? dn[i][e] * n : 0.f;
        g[e] = rho * (dn[i][e] * gain[i][e]) - n * c;
        if (A.dh.p) g[e] += r[e];
      }
      if (!live) continue;
      Row8<T> o;
      if (A.dr.p) {
        o.put(g);
        store8<T, TAIL, NT>((T*)A.dr.p + row * A.dr.ld, at.lane + i * C::STEP, A.cols, o);
      }
      if (A.dx.p) {
        if (A.drop.t) drop8(A.drop, key, at.lane + i * C::STEP, (uint32_t)row, g);
        o.put(g);
        store8<T, TAIL, NT>((T*)A.dx.p + row * A.dx.ld, at.lane + i * C::STEP, A.cols, o);
      }
    }
  }
  if (!A.part) return;
  // the block's sum: over a wave's rows, then over its waves in order
  float* const out = A.part + (int64_t)blockIdx.x * A.cols;
#pragma unroll
  for (int o = C::LPR; o < 64; o <<= 1)
#pragma unroll
    for (int i = 0; i < C::CH; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) dg[i][e] += __shfl_xor(dg[i][e], o, 64);
  if constexpr (PARTS > 1) {
    const int w = threadIdx.x >> 6;
    if (at.sub == 0)
#pragma unroll
      for (int i = 0; i < C::CH; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[w * C::COLS + 8 * (at.lane + i * C::STEP) + e] = dg[i][e];
    __syncthreads();
    for (int c = threadIdx.x; c < A.cols; c += C::THREADS)
      out[c] = (sum[c] + sum[C::COLS + c]) + (sum[2 * C::COLS + c] + sum[3 * C::COLS + c]);
  } else {
#pragma unroll
    for (int i = 0; i < C::CH; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int c = 8 * (at.lane + i * C::STEP) + e;
        if (c < A.cols) out[c] = dg[i][e];
      }
  }
}

// dgain from the blocks' sums: 16 columns a block, 64 strands of rows of `part`,
// joined in a fixed order.  512 rows of 1024 columns: 4.5 us, of which a launch that
// has nothing to do would take 2.
__global__ __launch_bounds__(1024) void norm_dgain_kernel(const float* __restrict__ part, int n, int cols,
                                                          float* __restrict__ dgain) {
  __shared__ float sum[64][17];
  const int x = threadIdx.x & 15, y = threadIdx.x >> 4, c = blockIdx.x * 16 + x;
  float v = 0.f;
  if (c < cols)
#pragma unroll 8
    for (int i = y; i < n; i += 64) v += part[(int64_t)i * cols + c];
  sum[y][x] = v;
  __syncthreads();
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    if (y < o) sum[y][x] += sum[y + o][x];
    __syncthreads();
  }
  if (y == 0 && c < cols) dgain[c] = sum[0][x];
}

// Calls f(RowCfg) with the narrowest configuration that holds `cols`: lanes a row as
// few as its groups fill (1M rows of 16, bf16: forward 22 us with two, 112 with 16), two
// groups a lane and more waves a row from there on (four groups left two waves a
// SIMD: 2048 rows of 8192, bf16, backward 68 us, so 32).  The longest rows' backward, with four
// sets of values a group, does not fit the 128 registers of a block of 16 waves: 2048
// rows of 16384, bf16 / fp32, 72 / 126 us so, 132 / 373 with 16 waves, whose
// forward is the faster one (53 and 55).
template <bool BWD, typename F>
static auto with_cfg(int cols, F f) {
  const int g = cdiv(cols, 8);
  if (g <= 2) return f(RowCfg<2, 1, 1>());
  if (g <= 4) return f(RowCfg<4, 1, 1>());
  if (g <= 8) return f(RowCfg<8, 1, 1>());
  if (g <= 16) return f(RowCfg<16, 1, 1>());
  if (g <= 32) return f(RowCfg<32, 1, 1>());
  if (g <= 64) return f(RowCfg<64, 1, 1>());
  if (g <= 128) return f(RowCfg<64, 2, 1>());
  if (g <= 256) return f(RowCfg<64, 2, 2>());
  if (g <= 512) return f(RowCfg<64, 2, 4>());
  if (g <= 1024) return f(RowCfg<64, 2, 8>());
  return f(std::conditional_t<BWD, RowCfg<64, 4, 8>, RowCfg<64, 2, 16>>());
}

// Blocks of a launch: rows in steps of the grid, at most `most` waves in all: few
// enough that a wave's gains serve several rows and its next loads are out before a
// row's sums.  131072 / 8192 rows of 1024, bf16: forward 194 / 13.6 us with 4096 waves, 195 /
// 14.0 with 8192; backward (and 2048 rows of 8192) 257 / 32 us with 2048, 263 / 38 with 4096,
// 259 / 43 with 1024.
template <typename C>
static int norm_blocks(int64_t rows, int most) {
  const int64_t n = cdiv(rows, C::RPB), cap = most / (C::THREADS / 64);
  return (int)(n < cap ? n : cap);
}
// Data of more bytes than the 256 MB that memory's own cache holds goes past the
// caches, where that was found to pay: bf16, and for the backward, which also writes so,
// whole 128-byte lines at once (a part of a line costs a read of the rest).  us past the
// caches / through them:
//   backward with dropout, 131072 rows of 1024, bf16 243 / 257, 16 bytes off a line 273 / 273,
//   of 1001 289 / 271, 400000 of 520 472 / 428, 4M of 16 106 / 122; fp32, whose lanes' two
//   words of 16 bytes are 32 apart, 131072 of 1024 534 / 499, 16384 of 8192 505 / 528
//   dropout alone, 131072 rows of 1024, bf16 83 / 96, of 1001 85 / 95, in its input's place
//   82 / 79 and 95 / 81; fp32 203 / 192
//   forward the same either way (193, 195)
// Below 256 MB, what the operator before has just written is still there: 8192 rows of 1024,
// forward 13.5 us, past the caches 15.4.
constexpr double CACHED_BYTES = 256 << 20;
constexpr int NORM_FWD_WAVES = 4096, NORM_BWD_WAVES = 2048;

static NormK norm_k(const NormArgs& a) {
  NormK A{};
  A.rows = a.rows;
  A.cols = a.cols;
  A.eps = a.eps;
  A.inv_cols = 1.f / (float)a.cols;
  A.gain = a.gain;
  A.drop = a.drop;
  A.x = a.x; A.r = a.r; A.h = a.h; A.y = a.y;
  A.dy = a.dy; A.dh = a.dh; A.dr = a.dr; A.dx = a.dx;
  A.q = a.q;
  A.ldq = a.ldq;
  A.scales = a.scales;
  return A;
}

hipError_t add_rmsnorm_fwd(const NormArgs& a, hipStream_t s) {
  if (a.rows == 0) return hipSuccess;
  const NormK A = norm_k(a);
  with_cfg<false>(a.cols, [&](auto cfg) {
    using C = decltype(cfg);
    const int n = norm_blocks<C>(a.rows, NORM_FWD_WAVES);
    const bool tail = a.cols % 8 != 0;
    if (a.dt == DT_BF16) {
      if (tail) add_rmsnorm_fwd_kernel<bf16_t, true, C><<<n, C::THREADS, 0, s>>>(A);
      else add_rmsnorm_fwd_kernel<bf16_t, false, C><<<n, C::THREADS, 0, s>>>(A);
    } else {
      if (tail) add_rmsnorm_fwd_kernel<float, true, C><<<n, C::THREADS, 0, s>>>(A);
      else add_rmsnorm_fwd_kernel<float, false, C><<<n, C::THREADS, 0, s>>>(A);
    }
    return 0;
  });
  LAT_LAUNCH_CHECK();
  return hipSuccess;
}

static int norm_bwd_blocks(int64_t rows, int cols) {
  return with_cfg<true>(cols, [&](auto cfg) { return norm_blocks<decltype(cfg)>(rows, NORM_BWD_WAVES); });
}

size_t add_rmsnorm_bwd_workspace(int64_t rows, int cols) {
  return (size_t)norm_bwd_blocks(rows, cols) * cols * sizeof(float);
}

// Whether what a wave reads or writes at once is whole 128-byte lines (bf16): rows of
// whole lines, or rows that follow each other.
template <typename C>
static bool whole_lines(const NormArgs& a) {
  for (const RowTensor& t : {a.h, a.dy, a.dh, a.dr, a.dx}) {
    if (!t.p) continue;
    if ((uintptr_t)t.p % 128) return false;
    if (!(a.cols % 64 == 0 && t.ld % 64 == 0) && !(t.ld == a.cols && C::RPW * a.cols % 64 == 0)) return false;
  }
  return true;
}

hipError_t add_rmsnorm_bwd(const NormArgs& a, void* ws, hipStream_t s) {
  NormK A = norm_k(a);
  A.part = a.dgain ? (float*)ws : nullptr;
  const int n = a.rows > 0 ? norm_bwd_blocks(a.rows, a.cols) : 0;
  const int tensors = 2 + !!a.dh.p + !!a.dr.p + !!a.dx.p;
  if (n > 0) {
    with_cfg<true>(a.cols, [&](auto cfg) {
      using C = decltype(cfg);
      auto launch = [&](auto kern) { kern<<<n, C::THREADS, 0, s>>>(A); };
      const bool tail = a.cols % 8 != 0;
      const bool nt = (double)a.rows * a.cols * 2 * tensors > CACHED_BYTES && whole_lines<C>(a);
      if (a.dt == DT_BF16) {
        if (tail) launch(add_rmsnorm_bwd_kernel<bf16_t, true, false, C>);
        else if (nt) launch(add_rmsnorm_bwd_kernel<bf16_t, false, true, C>);
        else launch(add_rmsnorm_bwd_kernel<bf16_t, false, false, C>);
      } else {
        if (tail) launch(add_rmsnorm_bwd_kernel<float, true, false, C>);
        else launch(add_rmsnorm_bwd_kernel<float, false, false, C>);
      }
      return 0;
    });
    LAT_LAUNCH_CHECK();
  }
  if (a.dgain) {
    norm_dgain_kernel<<<cdiv(a.cols, 16), 1024, 0, s>>>(A.part, n, a.cols, a.dgain);
    LAT_LAUNCH_CHECK();
  }
  return hipSuccess;
}

// ---------------------------------------------------------------------------
// Dropout alone.  A block takes DROP_GROUPS neighbouring groups of eight columns
// of the whole matrix, each thread every 256th.  One read and one write of memory:
// 131072 x 1024, bf16, 83 to 93 us (6.5 to 5.8 TB/s), the generator's ten rounds and the
// selection issuing in 73% of the cycles.
constexpr int DROP_PER = 4, DROP_GROUPS = 256 * DROP_PER;

template <typename T, bool TAIL, bool NT>
__global__ __launch_bounds__(256) void dropout_kernel(int64_t total, int cols, uint32_t groups, FastDiv div, DropArgs d,
                                                      RowTensor x, RowTensor out) {
  const DropKey key = drop_key(d);
  const int64_t g0 = (int64_t)blockIdx.x * DROP_GROUPS, row0 = g0 / groups;
  const uint32_t c0 = (uint32_t)(g0 - row0 * groups);
  const int left = (int)min(total - g0, (int64_t)DROP_GROUPS);
  Row8<T> v[DROP_PER];
  int64_t row[DROP_PER];
  uint32_t g[DROP_PER];
#pragma unroll
  for (int i = 0; i < DROP_PER; ++i) {
    const uint32_t n = c0 + (uint32_t)min((int)threadIdx.x + 256 * i, left - 1), down = div(n);
    row[i] = row0 + down;
    g[i] = n - down * groups;
    v[i] = load8<T, TAIL, NT>(row_of<T>(x, row[i]), (int)g[i], cols);
  }
#pragma unroll
  for (int i = 0; i < DROP_PER; ++i) {
    float f[8];
    fix8<T, TAIL>(v[i], (int)g[i], cols);
    v[i].get(f);
    if (d.t) drop8(d, key, g[i], (uint32_t)row[i], f);
    v[i].put(f);
    if ((int)threadIdx.x + 256 * i < left) store8<T, TAIL>((T*)out.p + row[i] * out.ld, (int)g[i], cols, v[i]);
  }
}

hipError_t dropout(DType dt, int64_t rows, int cols, const DropArgs& d, RowTensor x, RowTensor out, hipStream_t s) {
  if (rows == 0) return hipSuccess;
  const uint32_t groups = (uint32_t)cdiv(cols, 8);
  const int64_t total = rows * groups;
  const FastDiv div(groups);
  const int n = cdiv(total, DROP_GROUPS);
  auto launch = [&](auto kern) { kern<<<n, 256, 0, s>>>(total, cols, groups, div, d, x, out); };
  const bool tail = cols % 8 != 0, nt = (double)rows * cols * 2 * 2 > CACHED_BYTES && x.p != out.p;
  if (dt == DT_BF16) {
    if (tail) nt ? launch(dropout_kernel<bf16_t, true, true>) : launch(dropout_kernel<bf16_t, true, false>);
    else nt ? launch(dropout_kernel<bf16_t, false, true>) : launch(dropout_kernel<bf16_t, false, false>);
  } else {
    tail ? launch(dropout_kernel<float, true, false>) : launch(dropout_kernel<float, false, false>);
  }
  LAT_LAUNCH_CHECK();
  return hipSuccess;
}

}  // namespace lat
