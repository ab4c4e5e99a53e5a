// One event for each user of a serving batch: the query's and key's norm and
// rotation, the append to the user's ring cache, and the query's attention over
// the cache's visible slots, in one launch (two where the slots are split).
//
// Memory bound: every visible slot's k and v are read once.  A block is a
// user, a key head (up to 16 of its query heads at a time) and a split of the
// slots; its four waves take tiles of 32 slots in turn and keep their own
// running maximum, sum and output, joined at the end.  Scores are S^T = K Q^T on
// 16x16x32 matrix instructions, the keys' fragments straight from memory (a
// lane's 16 bytes of one slot), 16 head columns whether used or not: the
// matrix cores are far from the bound.  A lane then holds one head's
// probabilities of 8 slots, which are the next product's operand
// (O^T = V^T P^T); only V passes through LDS, to be read transposed.  The next
// tile's loads go out before a tile's scores; before the tile's first transposed
// read of V the compiler waits for all of them (bf16), as it cannot tell that
// they write elsewhere.
//
// The new event's own k and v replace their slot's row where the tile is
// used (registers for k, the LDS row for v), so nothing waits for the cache's
// update; the split that holds the slot writes it.
//
// 1024 users, windows of 1024 slots of 128, 2 key heads, bf16: 183 us, 5.1 TB/s
// of the bytes it cannot do without (a plain copy reaches 4.85).
#include "kernels.h"
#include "seq_rope.h"
#include "seq_step.h"
#include "seq_tile.h"

namespace lat {

constexpr int STEP_TILE = 32;                // slots of a wave's tile

struct StepK {
  SeqCacheArgs c;
  int heads, group, hg, ns, cap;             // hg: blocks of 16 heads of a group
  float scale, eps, inv_dim;
  int rope, rotary, inter;
  SeqTensor q, k, v, out;
  const int32_t *lens, *pos;
  const float *gq, *gk;
  float* part;                               // [batch][heads][ns][dim + 2]: o, m, l
  StepJoin join;
};

__device__ inline void mma16(const Frag<float>& a, const Frag<float>& b, f32x4& c) {
#pragma unroll
  for (int e = 0; e < 8; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.v[e], b.v[e], c, 0, 0, 0);
}
// Operands that the step itself computes (the rotated query, probabilities) go
// into the matrix instructions as two bf16 parts, value and remainder: the
// matrix cores have the time, and the result is then rounded once, at the
// end.  fp32 operands are taken as they are.
template <typename T> struct Parts { static constexpr int N = sizeof(T) == 2 ? 2 : 1; Frag<T> p[N]; };
__device__ inline void split(const float* x, Parts<bf16_t>& f) {
  float r[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) r[e] = x[e] - bf2f(f2bf(x[e]));
  f.p[0].v = __builtin_bit_cast(bf16x8, Vec16<bf16_t>::pack(x));
  f.p[1].v = __builtin_bit_cast(bf16x8, Vec16<bf16_t>::pack(r));
}
__device__ inline void split(const float* x, Parts<float>& f) {
#pragma unroll
  for (int e = 0; e < 8; ++e) f.p[0].v[e] = x[e];
}
template <typename T, int DP> struct StepCfg {
  using TL = Tile<T, DP>;
  static constexpr int VT = STEP_TILE * TL::RB;                       // a wave's V stage
  static constexpr int NEW = STEP_HEADS * DP * 4 + 2 * DP * (int)sizeof(T);   // q rows (fp32), new k, new v
  static constexpr size_t LOOP = (size_t)8 * VT + NEW;
  static constexpr size_t JOIN = (size_t)4 * STEP_HEADS * (DP + 4) * sizeof(float);
  static constexpr size_t LDS = LOOP > JOIN ? LOOP : JOIN;
};

template <typename T, int DP>
__global__ __launch_bounds__(256, sizeof(T) == 4 && DP == 128 ? 1 : 2) void seq_step_kernel(StepK A, RopeTurns turns) {
  using TL = Tile<T, DP>;
  using Cfg = StepCfg<T, DP>;
  constexpr int KS = DP / 32, OB = DP / 16;
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g16 = lane >> 4, l16 = lane & 15, D = A.c.dim;
  int blk = blockIdx.x;
  const int u = blk % A.ns; blk /= A.ns;
  const int hg = blk % A.hg; blk /= A.hg;
  const int kv = blk % A.c.kv_heads, b = blk / A.c.kv_heads;
  const int p = A.lens[b], ci = A.c.index ? A.c.index[b] : b;
  if (p < 0 || ci < 0 || ci >= A.c.num_caches) return;
  const int n = min(p, A.cap - 1) + 1, slot = seq_slot(p, A.c.sinks, A.c.window);
  // the split's slots, whole rounds of the four waves
  const int chunk = ((n + A.ns - 1) / A.ns + 4 * STEP_TILE - 1) & ~(4 * STEP_TILE - 1);
  const int a0 = (int)min((int64_t)u * chunk, (int64_t)n), a1 = (int)min((int64_t)a0 + chunk, (int64_t)n);
  const int nh = min(STEP_HEADS, A.group - hg * STEP_HEADS), h0 = kv * A.group + hg * STEP_HEADS;
  const int64_t base = ((int64_t)ci * A.c.kv_heads + kv) * A.cap;
  T* const kc = (T*)A.c.kc + base * D;
  T* const vc = (T*)A.c.vc + base * D;
  float* const qn = reinterpret_cast<float*>(smem + 8 * Cfg::VT);     // [16][DP]
  T* const kn = reinterpret_cast<T*>(qn + STEP_HEADS * DP);
  T* const vn = kn + DP;

  TileLoad<T, DP, STEP_TILE, 1> lv;
  lv.init(0, D, D);
  char* const VS = smem + w * 2 * Cfg::VT;
  Frag<T> kf[2][2 * KS];
  const int tiles = a1 > a0 ? (a1 - a0 + STEP_TILE - 1) / STEP_TILE : 0;
  auto issue = [&](int t, Frag<T>* f) {
    const int j0 = a0 + t * STEP_TILE, nk = min(STEP_TILE, a1 - j0);
    lv.issue(VS + ((t >> 2) & 1) * Cfg::VT, 0, vc + (int64_t)j0 * D, nk, ~0ull);
#pragma unroll
    for (int r = 0; r < 2; ++r)
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        const int row = min(16 * r + l16, nk - 1), d = 32 * s + 8 * g16;
        load_frag(kc + (int64_t)(j0 + row) * D + (d < D ? d : 0), d < D, f[r * KS + s]);
      }
  };
  if (w < tiles) issue(w, kf[0]);

  // the event's own vectors: rows of qn (zeros past the heads), kn, vn
  {
    const int np = A.rotary >> 1;
    const bool rot = lane < np;
    int x, y;
    if (A.inter || !rot) { x = 2 * lane; y = x + 1; } else { x = lane; y = np + lane; }
    const bool on = x < D;
    float2 cs{1.f, 0.f};
    if (A.rope && rot) cs = rope_cs(A.pos ? A.pos[b] : p, turns.f[lane]);
    for (int r = w; r < STEP_HEADS + 2; r += 4) {
      const bool isq = r < STEP_HEADS, live = !isq || r < nh;
      const T* src = isq ? (const T*)A.q.p + (int64_t)b * A.q.ld + (h0 + min(r, nh - 1)) * D
                   : r == STEP_HEADS ? (const T*)A.k.p + (int64_t)b * A.k.ld + kv * D
                                     : (const T*)A.v.p + (int64_t)b * A.v.ld + kv * D;
      float zx = on ? ld(src + x) : 0.f, zy = on ? ld(src + y) : 0.f;
      if (A.rope && r <= STEP_HEADS) {
        const float rr = 1.f / sqrtf(wave_sum(zx * zx + zy * zy) * A.inv_dim + A.eps);
        const float* g = isq ? A.gq : A.gk;
        zx *= rr * (g && on ? g[x] : 1.f);
        zy *= rr * (g && on ? g[y] : 1.f);
        const float tx = zx * cs.x - zy * cs.y, ty = zx * cs.y + zy * cs.x;
        zx = tx;
        zy = ty;
      }
      zx = live && on ? zx : 0.f;
      zy = live && on ? zy : 0.f;
      if (x < DP) {
        if (isq) {
          qn[r * DP + x] = zx;
          qn[r * DP + y] = zy;
        } else {
          T* dst = kn + (r - STEP_HEADS) * DP;
          st(dst + x, zx);
          st(dst + y, zy);
        }
      }
    }
  }
  __syncthreads();
  const bool owner = slot >= a0 && slot < a1;
  if (owner && hg == 0) {
    constexpr int N = 16 / sizeof(T);
    for (int x = threadIdx.x; x < 2 * D / N; x += 256) {
      const int m = x >= D / N, d = (x - m * (D / N)) * N;
      *reinterpret_cast<u32x4*>((m ? vc : kc) + (int64_t)slot * D + d) =
          *reinterpret_cast<const u32x4*>((m ? vn : kn) + d);
    }
  }
  Parts<T> qf[KS];
#pragma unroll
  for (int s = 0; s < KS; ++s) {
    Frag<float> f;
    load_frag(qn + l16 * DP + 32 * s + 8 * g16, true, f);
    split(f.v, qf[s]);
  }

  const float c = A.scale * STEP_LOG2E;
  f32x4 o[OB];
#pragma unroll
  for (int i = 0; i < OB; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;
  // column fragments of a 32-slot tile: slot 16 (e / 4) + 4 g16 + e % 4
  uint32_t cl;
  if constexpr (sizeof(T) == 2) {
    const int r = 4 * g16 + (l16 >> 2), col = 4 * (l16 & 3);
    cl = (uint32_t)(r * TL::RB + (((col >> 3) ^ TL::swz(r)) << 4) + (col & 7) * 2);
  } else {
    const int r = 4 * g16;
    cl = (uint32_t)(r * TL::RB + (((l16 >> 2) ^ TL::swz(r)) << 4) + (l16 & 3) * 4);
  }
  auto vfrag = [&](const char* S, int ob) {
    Frag<T> f;
    if constexpr (sizeof(T) == 2) {
      typedef __attribute__((address_space(3))) seq_i16x4 lds_v4;
      const seq_i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4*)(S + TL::at(cl, 0, 2 * ob)));
      const seq_i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4*)(S + TL::at(cl, 16, 2 * ob)));
      f.v = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        f.v[e] = *reinterpret_cast<const float*>(S + TL::at(cl, 16 * (e >> 2) + (e & 3), 4 * ob));
    }
    return f;
  };
  auto tile = [&](int t, const Frag<T>* kt) {
    const int j0 = a0 + t * STEP_TILE, nk = min(STEP_TILE, a1 - j0);
    char* S = VS + ((t >> 2) & 1) * Cfg::VT;
    const int at = slot - j0;
    const bool here = at >= 0 && at < STEP_TILE && owner;
    if (here) {                                          // the new event's v over its slot's row
      constexpr int N = 16 / sizeof(T);
      if (lane < TL::UPR && lane * N < D)
        *reinterpret_cast<u32x4*>(S + at * TL::RB + ((lane ^ TL::swz(at)) << 4)) =
            *reinterpret_cast<const u32x4*>(vn + lane * N);
    }
    f32x4 s[2];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      s[r] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < KS; ++i) {
        Frag<T> f = kt[r * KS + i];
        if (here) {
          Frag<T> fn;
          load_frag(kn + 32 * i + 8 * g16, true, fn);
          if (at == 16 * r + l16) f = fn;
        }
#pragma unroll
        for (int x = Parts<T>::N - 1; x >= 0; --x) mma16(f, qf[i].p[x], s[r]);
      }
    }
    float x[8], tm = -INFINITY;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      x[e] = 16 * (e >> 2) + 4 * g16 + (e & 3) < nk ? s[e >> 2][e & 3] : -INFINITY;
      tm = fmaxf(tm, x[e]);
    }
    tm = fmaxf(tm, __shfl_xor(tm, 16, 64));
    tm = fmaxf(tm, __shfl_xor(tm, 32, 64));
    const bool up = (tm - m) * c > 8.f;                  // as in the batch's forward
    if (wave_any(up)) {
      const float mn = up ? tm : m, f = up ? __builtin_amdgcn_exp2f((m - mn) * c) : 1.f;
      l *= f;
#pragma unroll
      for (int i = 0; i < OB; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) o[i][r] *= f;
      m = mn;
    }
    const float mc = m == -INFINITY ? 0.f : m * c;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      x[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[e], c, -mc));
      l += x[e];
    }
    Parts<T> pf;
    split(x, pf);
#pragma unroll
    for (int i = 0; i < OB; ++i) {
      const Frag<T> f = vfrag(S, i);
#pragma unroll
      for (int y = Parts<T>::N - 1; y >= 0; --y) mma16(f, pf.p[y], o[i]);
    }
  };
#pragma unroll 1
  for (int t = w; t < tiles; t += 8) {
    // the wave's own stages: its loads of tile t have landed, its reads of
    // the tile before returned
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    if (t + 4 < tiles) issue(t + 4, kf[1]);
    tile(t, kf[0]);
    if (t + 4 >= tiles) break;
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    if (t + 8 < tiles) issue(t + 8, kf[0]);
    tile(t + 4, kf[1]);
  }
  l += __shfl_xor(l, 16, 64);
  l += __shfl_xor(l, 32, 64);
  // join of the waves: O[w][head][DP], then m and l
  float* const J = reinterpret_cast<float*>(smem);
  __syncthreads();
  float* const Jw = J + (w * STEP_HEADS + l16) * (DP + 4);
#pragma unroll
  for (int i = 0; i < OB; ++i) *reinterpret_cast<f32x4*>(Jw + 16 * i + 4 * g16) = o[i];
  if (g16 == 0) {
    Jw[DP] = m;
    Jw[DP + 1] = l;
  }
  __syncthreads();
  for (int x = threadIdx.x; x < nh * D; x += 256) {
    const int h = x / D, d = x - h * D;
    float mm[4], M = -INFINITY;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      mm[i] = J[(i * STEP_HEADS + h) * (DP + 4) + DP];
      M = fmaxf(M, mm[i]);
    }
    float L = 0.f, O = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float* P = J + (i * STEP_HEADS + h) * (DP + 4);
      const float f = mm[i] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((mm[i] - M) * c);
      L += P[DP + 1] * f;
      O += P[d] * f;
    }
    if (A.ns == 1) {
      st((T*)A.out.p + (int64_t)b * A.out.ld + (h0 + h) * D + d, O / L);
    } else {
      float* P = A.part + (((int64_t)b * A.heads + h0 + h) * A.ns + u) * (D + 2);
      P[d] = O;
      if (d == 0) {
        P[D] = M;
        P[D + 1] = L;
      }
    }
  }
}

size_t seq_step_workspace(int batch, int heads, int kv_heads, int dim, int cap) {
  if (batch == 0) return 0;
  const int ns = step_splits(batch, heads, kv_heads, cap);
  return ns > 1 ? (size_t)batch * heads * ns * (dim + 2) * sizeof(float) : 0;
}

template <typename T, int DP>
static hipError_t step_launch(const StepK& A, const RopeTurns& t, int batch, hipStream_t s) {
  static LdsLimit lim;
  LAT_HIP_CHECK(lds_limit(seq_step_kernel<T, DP>, StepCfg<T, DP>::LDS, lim));
  seq_step_kernel<T, DP><<<batch * A.c.kv_heads * A.hg * A.ns, 256, StepCfg<T, DP>::LDS, s>>>(A, t);
  LAT_LAUNCH_CHECK();
  if (A.ns > 1) {
    seq_step_join_kernel<T, DP><<<batch * A.heads, 256, 0, s>>>(A.join);
    LAT_LAUNCH_CHECK();
  }
  return hipSuccess;
}

hipError_t seq_step(const SeqStepArgs& a, const RopeTurns& t, void* ws, hipStream_t s) {
  if (a.batch == 0) return hipSuccess;
  StepK A{};
  A.c = a.c;
  A.heads = a.heads;
  A.group = a.heads / a.c.kv_heads;
  A.hg = cdiv(A.group, STEP_HEADS);
  A.cap = a.c.sinks + a.c.window;
  A.ns = step_splits(a.batch, a.heads, a.c.kv_heads, A.cap);
  A.scale = a.scale;
  A.eps = a.eps;
  A.inv_dim = 1.f / a.c.dim;
  A.rope = a.rope;
  A.rotary = a.rope ? a.rotary : 0;
  A.inter = a.interleaved;
  A.q = a.q; A.k = a.k; A.v = a.v; A.out = a.out;
  A.lens = a.lens;
  A.pos = a.positions;
  A.gq = a.gain_q;
  A.gk = a.gain_k;
  A.part = (float*)ws;
  A.join = {a.lens, a.c.index, a.c.num_caches, a.heads, a.c.dim, A.ns, a.scale, A.part, a.out};
  const int D = a.c.dim;
  if (a.c.dt == DT_BF16)
    return D <= 32 ? step_launch<bf16_t, 32>(A, t, a.batch, s) : D <= 64 ? step_launch<bf16_t, 64>(A, t, a.batch, s)
                                                                        : step_launch<bf16_t, 128>(A, t, a.batch, s);
  return D <= 32 ? step_launch<float, 32>(A, t, a.batch, s) : D <= 64 ? step_launch<float, 64>(A, t, a.batch, s)
                                                                     : step_launch<float, 128>(A, t, a.batch, s);
}

}  // namespace lat
