// Per-head RMSNorm of queries and keys with the rotary position rotation, in
// one pass (Section 3.3.4: QK-norm; Section 3.3.2: rotary positions of the
// sequence path), its backward, and the plan of a packed batch.
//
//   z = g x r, r = 1 / sqrt(mean(x^2) + eps);  (u, v) of pair m at position p:
//   y_u = z_u cos a - z_v sin a, y_v = z_u sin a + z_v cos a.
// Backward: dz = the rotation by -a of dy; dg = sum dz x r; h = g dz;
//   dx = r h - x r^3 mean(h x).
//
// Memory bound: forward reads and writes each element once, backward reads
// two and writes one.  A lane holds both elements of its pairs (2 E elements:
// two runs of E, one from each half of the rotated part, or 2 E neighbours),
// so the rotation needs no other lane and a head takes dim / (2 E) lanes, whose
// sums of squares are added by shuffles inside the group.  Angles are
// computed once per row and pair for all heads (64-bit reduction and sincos
// are the expensive part) and shared through LDS: a block takes `tb` rows,
// its threads make tb * rotary / 2 angles, then its lane groups go over the
// tb * (heads + kv_heads) head vectors, the first one's loads made before the
// angles.  Gains are read from LDS, not kept in registers, for the sake of
// waves: 131072 rows, 10 heads of 128, bf16, forward: 164 -> 131 us, 5.1 TB/s
// (a plain copy of that size reaches 4.85).  Loading every next head vector
// ahead as well took registers from the waves and was slower (175 us).
#include "kernels.h"
#include "seq_rope.h"

#include <cmath>

namespace lat {

// One thread per row: the last sequence that starts at or before it.
__global__ __launch_bounds__(256) void seq_plan_kernel(const int32_t* __restrict__ off, int S, int rows,
                                                       SeqSpan* __restrict__ span) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i >= rows) return;
  int lo = 0, hi = S;                       // off[lo] <= i (lo = 0: assumed), off[hi] > i or hi = S
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (off[mid] <= i) lo = mid; else hi = mid;
  }
  SeqSpan r{SEQ_NO_ROW, 0};
  if (S > 0) {
    const int a = off[lo], e = min(off[lo + 1], rows);
    if (a >= 0 && a <= i && i < e) r = {a, e};
  }
  span[i] = r;
}

hipError_t seq_plan(const int32_t* offsets, int num_seqs, int64_t rows, SeqSpan* span, hipStream_t s) {
  if (rows == 0) return hipSuccess;
  seq_plan_kernel<<<cdiv(rows, 256), 256, 0, s>>>(offsets, num_seqs, (int)rows, span);
  LAT_LAUNCH_CHECK();
  return hipSuccess;
}

void rope_turns(double theta, int rotary, RopeTurns* t) {
  // a geometric row in extended precision: its error stays below a double's
  const long double r = rotary > 0 ? std::pow((long double)theta, -2.0L / rotary) : 0.0L;
  long double f = 0.159154943091895335768883763372514362L;           // 1 / (2 pi)
  for (int m = 0; m < ROPE_MAX_PAIRS; ++m, f *= r) t->f[m] = m < rotary / 2 ? (double)f : 0.0;
}

struct RopeK {                               // kernel arguments
  int rows, heads, hk, dim, rotary, tb, lp, chunks, groups;   // hk = heads + kv_heads
  float eps, inv_dim;
  const SeqSpan* span;
  const int32_t* pos;
  const float *gq, *gk;
  SeqTensor xq, xk, dyq, dyk, oq, ok;
  float* partial;                            // backward: [blocks][2][dim]
};

// E consecutive elements as fp32, 16- or 8-byte accesses
template <typename T, int E> __device__ inline void ldE(const T* p, float* o) {
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < E; i += 4) {
      const f32x4 v = *reinterpret_cast<const f32x4*>(p + i);
#pragma unroll
      for (int e = 0; e < 4; ++e) o[i + e] = v[e];
    }
  } else if constexpr (E == 8) {
    Vec16<bf16_t>::unpack(ldg16(p), o);
  } else {
    const u32x2 v = *reinterpret_cast<const u32x2*>(p);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      o[2 * i] = __uint_as_float(v[i] << 16);
      o[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u);
    }
  }
}
template <typename T, int E> __device__ inline void stE(T* p, const float* o) {
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < E; i += 4) *reinterpret_cast<f32x4*>(p + i) = f32x4{o[i], o[i + 1], o[i + 2], o[i + 3]};
  } else if constexpr (E == 8) {
    stg16(p, Vec16<bf16_t>::pack(o));
  } else {
    *reinterpret_cast<u32x2*>(p) = u32x2{pack_bf2(o[0], o[1]), pack_bf2(o[2], o[3])};
  }
}

__device__ inline float group_sum(float v, int lp) {
  for (int o = lp >> 1; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}

// T storage type, E elements of a run, INTER pairs of neighbours; blocks go
// over groups of tb rows.
template <typename T, int E, bool BWD, bool INTER>
__global__ __launch_bounds__(256) void rope_kernel(RopeK A, RopeTurns turns) {
  extern __shared__ __attribute__((aligned(16))) float2 cs[];   // [tb][rotary / 2]; backward's end: dgain partials
  const int tid = threadIdx.x, np = A.rotary >> 1;
  const int group = tid / A.lp, c = tid % A.lp;
  const bool lane_on = c < A.chunks;
  // where this lane's two runs lie in a head, and its first pair
  int lo, hi;
  bool rot;
  const int m0 = c * E;
  if (INTER) {
    lo = c * 2 * E;
    hi = lo + E;
    rot = lo < A.rotary;
  } else {
    rot = m0 < np;
    lo = rot ? m0 : A.rotary + (c - np / E) * 2 * E;
    hi = rot ? np + m0 : lo + E;
  }
  if (!lane_on) { lo = 0; hi = 0; rot = false; }
  // gains of q, then k, in the lane's order, behind the angles
  float* const gains = reinterpret_cast<float*>(cs) + 2 * A.tb * np;
  for (int j = tid; j < 2 * A.dim; j += 256) {
    const float* g = j < A.dim ? A.gq : A.gk;
    gains[j] = g ? g[j < A.dim ? j : j - A.dim] : 1.f;
  }
  float dg[2][2 * E];
  if constexpr (BWD)
#pragma unroll
    for (int e = 0; e < 2 * E; ++e) dg[0][e] = dg[1][e] = 0.f;

  // an item's loads: head h of row t0 + t
  auto fetch = [&](int64_t t0, int it, float (&v)[2 * E], float (&d)[2 * E], int& start) __attribute__((always_inline)) {
    const int t = it / A.hk, h = it - t * A.hk;
    const int64_t row = t0 + t;
    const bool isk = h >= A.heads;
    const int hh = isk ? h - A.heads : h;
    const SeqTensor X = isk ? A.xk : A.xq;
    const T* x = (const T*)X.p + row * X.ld + hh * A.dim;
    ldE<T, E>(x + lo, v);
    ldE<T, E>(x + hi, v + E);
    if constexpr (BWD) {
      const SeqTensor Y = isk ? A.dyk : A.dyq;
      const T* y = (const T*)Y.p + row * Y.ld + hh * A.dim;
      ldE<T, E>(y + lo, d);
      ldE<T, E>(y + hi, d + E);
    }
    start = A.span ? A.span[row].start : 0;
  };
  const int64_t step = (int64_t)gridDim.x * A.tb;
  for (int64_t t0 = (int64_t)blockIdx.x * A.tb; t0 < A.rows; t0 += step) {
    const int tn = (int)min((int64_t)A.tb, A.rows - t0), items = tn * A.hk;
    // the first item's loads are in flight while the angles are made
    float v[2 * E], d[2 * E];
    int start = SEQ_NO_ROW;
    if (group < items) fetch(t0, group, v, d, start);
    if (t0 != (int64_t)blockIdx.x * A.tb) __syncthreads();           // the rows before read cs
    for (int u = tid; u < tn * np; u += 256) {
      const int t = u / np, m = u - t * np;
      int p;
      if (A.pos) p = A.pos[t0 + t];
      else p = (int)(t0 + t) - A.span[t0 + t].start;                 // rows of no sequence: not used
      cs[u] = rope_cs(p, turns.f[m]);
    }
    __syncthreads();
    for (int it = group; it < items; it += A.groups) {
      if (it != group) fetch(t0, it, v, d, start);
      if (start != SEQ_NO_ROW) {                                     // uniform over the head's lanes
        const int t = it / A.hk, h = it - t * A.hk;
        const bool isk = h >= A.heads;
        const SeqTensor O = isk ? A.ok : A.oq;
        T* o = (T*)O.p + (t0 + t) * O.ld + (isk ? h - A.heads : h) * A.dim;
        float ss = 0.f;
#pragma unroll
        for (int e = 0; e < 2 * E; ++e) ss += v[e] * v[e];
        if (!lane_on) ss = 0.f;
        ss = group_sum(ss, A.lp);
        const float r = 1.f / sqrtf(ss * A.inv_dim + A.eps);
        const float2* w = cs + t * np + m0;
        const float* gn = gains + (isk ? A.dim : 0);
        float gain[2 * E];
#pragma unroll
        for (int e = 0; e < E; e += 4) {
          const f32x4 a = *reinterpret_cast<const f32x4*>(gn + lo + e), b = *reinterpret_cast<const f32x4*>(gn + hi + e);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            gain[e + i] = a[i];
            gain[E + e + i] = b[i];
          }
        }
        if constexpr (!BWD) {
          float z[2 * E];
#pragma unroll
          for (int e = 0; e < 2 * E; ++e) z[e] = v[e] * r * gain[e];
          if (rot) {
#pragma unroll
            for (int m = 0; m < E; ++m) {
              const int a = INTER ? 2 * m : m, b = INTER ? 2 * m + 1 : E + m;
              const float za = z[a], zb = z[b];
              z[a] = za * w[m].x - zb * w[m].y;
              z[b] = za * w[m].y + zb * w[m].x;
            }
          }
          if (lane_on) {
            stE<T, E>(o + lo, z);
            stE<T, E>(o + hi, z + E);
          }
        } else {
          if (rot) {
#pragma unroll
            for (int m = 0; m < E; ++m) {
              const int a = INTER ? 2 * m : m, b = INTER ? 2 * m + 1 : E + m;
              const float da = d[a], db = d[b];
              d[a] = da * w[m].x + db * w[m].y;
              d[b] = db * w[m].x - da * w[m].y;
            }
          }
          float hx = 0.f;
#pragma unroll
          for (int e = 0; e < 2 * E; ++e) {
            const float n = v[e] * r;
            dg[0][e] += isk ? 0.f : d[e] * n;
            dg[1][e] += isk ? d[e] * n : 0.f;
            d[e] *= gain[e];
            hx += d[e] * n;
          }
          if (!lane_on) hx = 0.f;
          hx = group_sum(hx, A.lp) * A.inv_dim;
#pragma unroll
          for (int e = 0; e < 2 * E; ++e) d[e] = r * (d[e] - v[e] * r * hx);
          if (lane_on) {
            stE<T, E>(o + lo, d);
            stE<T, E>(o + hi, d + E);
          }
        }
      }
    }
  }
  if constexpr (BWD) {
    if (!A.partial) return;
    // the block's sum over its groups, in group order
    float* sum = reinterpret_cast<float*>(cs);                       // [groups][dim]
    auto put = [&](const float (&x)[2 * E], int g) __attribute__((always_inline)) {
      __syncthreads();
      if (lane_on)
#pragma unroll
        for (int e = 0; e < E; ++e) {
          sum[group * A.dim + lo + e] = x[e];
          sum[group * A.dim + hi + e] = x[E + e];
        }
      __syncthreads();
      for (int j = tid; j < A.dim; j += 256) {
        float a = 0.f;
        for (int u = 0; u < A.groups; ++u) a += sum[u * A.dim + j];
        A.partial[((int64_t)blockIdx.x * 2 + g) * A.dim + j] = a;
      }
    };
    put(dg[0], 0);
    put(dg[1], 1);
  }
}

// dgain[j] = sum over blocks (fp32, as a lane's sum over its head vectors and the
// block's over its lane groups before it: three short sums, not one long one), 16 columns and 64 strands of blocks a workgroup
// of 1024; the strands' sums are added in a fixed tree.
__global__ __launch_bounds__(1024) void rope_dgain_kernel(const float* __restrict__ partial, int blocks, int dim,
                                                          float* __restrict__ dgq, float* __restrict__ dgk) {
  __shared__ float s[64][17];
  const int c = threadIdx.x & 15, strand = threadIdx.x >> 4;
  const int col = blockIdx.x * 16 + c;
  float a = 0.f;
  if (col < 2 * dim)
#pragma unroll 8
    for (int b = strand; b < blocks; b += 64) a += partial[(int64_t)b * 2 * dim + col];
  s[strand][c] = a;
  __syncthreads();
  for (int o = 32; o > 0; o >>= 1) {
    if (strand < o) s[strand][c] += s[strand + o][c];
    __syncthreads();
  }
  if (strand == 0 && col < 2 * dim) {
    float* out = col < dim ? dgq : dgk;
    if (out) out[col < dim ? col : col - dim] = s[0][c];
  }
}

// Rows a block takes at a time.  Many share the lanes better between angles
// and heads, few give a small batch more blocks and shorter chains.  Measured at
// these two sizes; that rows x heads fill whole rounds of a block's lane groups is
// not looked at.  131072
// rows, 10 heads of 128, bf16: 131 us with 16 rows, 148 with 4, 318 with 1; 5021
// rows, 9 heads of 96, fp32, forward: 14.6, 13.1, 14.7, backward: 21.4, 24.9, 32.8.
static int rope_tb(int64_t rows, bool bwd) {
  return rows >= 32768 || (bwd && rows >= 4096) ? 16 : rows >= 4096 ? 4 : 1;
}
constexpr int ROPE_BWD_BLOCKS = 1024;        // partial gain sums: bounds the second launch's work

static int rope_blocks(int64_t rows, bool bwd) {
  const int n = cdiv(rows, rope_tb(rows, bwd)), most = bwd ? ROPE_BWD_BLOCKS : 1 << 20;
  return n > most ? most : n;
}

static bool rope_wide(int dim, int rotary) { return dim % 16 == 0 && rotary % 16 == 0; }

size_t rope_bwd_workspace(int64_t rows, int dim) {
  return rows == 0 ? 0 : (size_t)rope_blocks(rows, true) * 2 * dim * sizeof(float);
}

template <bool BWD>
static hipError_t rope_launch(const RopeArgs& a, const RopeTurns& t, float* partial, hipStream_t s) {
  const int E = rope_wide(a.dim, a.rotary) ? 8 : 4;
  RopeK A;
  A.rows = (int)a.rows;
  A.heads = a.heads;
  A.hk = a.heads + a.kv_heads;
  A.dim = a.dim;
  A.rotary = a.rotary;
  A.tb = rope_tb(a.rows, BWD);
  A.chunks = a.dim / (2 * E);
  A.lp = 1;
  while (A.lp < A.chunks) A.lp *= 2;
  A.groups = 256 / A.lp;
  A.eps = a.eps;
  A.inv_dim = 1.f / a.dim;
  A.span = a.span;
  A.pos = a.positions;
  A.gq = a.gain_q;
  A.gk = a.gain_k;
  A.xq = a.q; A.xk = a.k; A.dyq = a.gq; A.dyk = a.gk; A.oq = a.oq; A.ok = a.ok;
  A.partial = partial;
  size_t lds = (size_t)A.tb * (a.rotary / 2) * sizeof(float2) + 2 * a.dim * sizeof(float);
  if (BWD) {
    const size_t need = (size_t)A.groups * a.dim * sizeof(float);    // at most 16 KB
    lds = lds > need ? lds : need;
  }
  const int grid = rope_blocks(a.rows, BWD);
  auto launch = [&](auto kern) { kern<<<grid, 256, lds, s>>>(A, t); };
#define ROPE_PICK(T, E_) \
  (a.interleaved ? launch(rope_kernel<T, E_, BWD, true>) : launch(rope_kernel<T, E_, BWD, false>))
  if (a.dt == DT_BF16) {
    if (E == 8) ROPE_PICK(bf16_t, 8); else ROPE_PICK(bf16_t, 4);
  } else {
    if (E == 8) ROPE_PICK(float, 8); else ROPE_PICK(float, 4);
  }
#undef ROPE_PICK
  LAT_LAUNCH_CHECK();
  return hipSuccess;
}

hipError_t rope_fwd(const RopeArgs& a, const RopeTurns& t, hipStream_t s) {
  return a.rows == 0 ? hipSuccess : rope_launch<false>(a, t, nullptr, s);
}

hipError_t rope_bwd(const RopeArgs& a, const RopeTurns& t, void* ws, hipStream_t s) {
  const bool gains = a.dgain_q || a.dgain_k;
  const int grid = rope_blocks(a.rows, true);
  if (a.rows > 0) {
    hipError_t e = rope_launch<true>(a, t, gains ? (float*)ws : nullptr, s);
    if (e != hipSuccess) return e;
  }
  if (!gains) return hipSuccess;
  rope_dgain_kernel<<<cdiv(2 * a.dim, 16), 1024, 0, s>>>((const float*)ws, grid, a.dim, a.dgain_q, a.dgain_k);
  LAT_LAUNCH_CHECK();
  return hipSuccess;
}

// ---------------------------------------------------------------------------
// Ring cache fill: a block takes 256 / (16-byte units of a row) rows; a row's
// kv_heads * dim elements of k and of v go to its slot, 16 bytes a lane.
// Rows whose slot a later row of the call takes are not written, so no two
// rows write one slot.  Copy bound: reads and writes the kept rows once.
template <typename T>
__global__ __launch_bounds__(256) void seq_fill_kernel(SeqCacheArgs C, int rows, const int32_t* __restrict__ off,
                                                       int S, const int32_t* __restrict__ first, SeqTensor k,
                                                       SeqTensor v, int units, int per_block) {
  const int u = threadIdx.x % units, rr = threadIdx.x / units;
  if (rr >= per_block) return;
  const int cap = C.sinks + C.window;
  constexpr int N = 16 / sizeof(T);
  // blockIdx.y: sequence; blockIdx.x: rows of it
  for (int s = blockIdx.y; s < S; s += gridDim.y) {
    const int ci = C.index ? C.index[s] : s;
    if (ci < 0 || ci >= C.num_caches) continue;
    const int a = max(off[s], 0), e = min(off[s + 1], rows), n = e - a;
    const int f = first ? first[s] : 0;
    if (n <= 0 || f < 0) continue;
    // rows kept: positions below sinks, and the last `window`
    const int64_t total = (int64_t)f + n;
    const int64_t from = total - C.window;   // first position of the window
    const int head = (int)min((int64_t)n, max((int64_t)0, C.sinks - (int64_t)f));   // rows in sinks
    const int tail0 = (int)max((int64_t)head, from - f);                            // first kept row after them
    const int kept = head + max(0, n - tail0);
    for (int i = blockIdx.x * per_block + rr; i < kept; i += gridDim.x * per_block) {
      const int local = i < head ? i : tail0 + (i - head);
      const int slot = (int)((int64_t)f + local < C.sinks ? (int64_t)f + local
                                                          : C.sinks + ((int64_t)f + local - C.sinks) % C.window);
      const int64_t row = (int64_t)a + local;
      for (int x = u; x < C.kv_heads * C.dim / N; x += units) {
        const int h = x * N / C.dim, d = x * N - h * C.dim;
        const int64_t dst = (((int64_t)ci * C.kv_heads + h) * cap + slot) * C.dim + d;
        const u32x4 kv = ldg16((const T*)k.p + row * k.ld + x * N), vv = ldg16((const T*)v.p + row * v.ld + x * N);
        stg16((T*)C.kc + dst, kv);
        stg16((T*)C.vc + dst, vv);
      }
    }
  }
}

hipError_t seq_cache_fill(const SeqCacheArgs& c, int64_t rows, const int32_t* offsets, int num_seqs,
                          const int32_t* first, SeqTensor k, SeqTensor v, hipStream_t s) {
  if (rows == 0 || num_seqs == 0) return hipSuccess;
  const int N = c.dt == DT_BF16 ? 8 : 4;
  int units = c.kv_heads * c.dim / N;
  if (units > 256) units = 256;
  const int per_block = 256 / units;
  // enough blocks a sequence for its mean number of kept rows, four rows a lane
  const int64_t mean = cdiv(rows, num_seqs), cap = (int64_t)c.sinks + c.window;
  int bx = cdiv(mean < cap ? mean : cap, (int64_t)per_block * 4);
  if (bx > 1024) bx = 1024;
  const int by = num_seqs < 65535 ? num_seqs : 65535;
  if (c.dt == DT_BF16)
    seq_fill_kernel<bf16_t><<<dim3(bx, by), 256, 0, s>>>(c, (int)rows, offsets, num_seqs, first, k, v, units, per_block);
  else
    seq_fill_kernel<float><<<dim3(bx, by), 256, 0, s>>>(c, (int)rows, offsets, num_seqs, first, k, v, units, per_block);
  LAT_LAUNCH_CHECK();
  return hipSuccess;
}

}  // namespace lat
