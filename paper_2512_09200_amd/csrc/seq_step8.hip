// The single-event step over ring caches of e4m3 codes, and their fill.
//
//   s_j = scale ks(j / 16) <q, kc_j>,  P = softmax(s),  out = sum_j P_j vs(j / 16) vc_j
//
// Memory bound: every visible slot's two rows of codes are read once, half the
// bytes of bf16.  Work is split as in the bf16 step: a block is a user, a key head
// and a split of the slots, its four waves take tiles of 64 slots in turn with
// their own running maximum, sum and output.  Codes become bf16 in registers
// (exactly: three bits of fraction) and go to 16x16x32 matrix instructions; a
// block's scale multiplies the 16 scores of its slots and their probabilities.
// What the step computes itself (query, probabilities) enters as two bf16 parts,
// three where the storage type is fp32, so that out is rounded once.
//
// Keys are fragments straight from memory.  Values are loaded to registers, go
// through the wave's own LDS rows and come back transposed, eight codes of one
// dimension a lane: a direct load to LDS would have the compiler wait for the
// next tile's loads before the first transposed read.
//
// The new event may change its block's scale, and with it the codes of the block's
// other slots.  The split that holds the slot makes the block anew before its
// tiles (one wave for k, one for v), writes it, and puts a copy into LDS that
// replaces what the tiles load of it; no other block of the launch reads these
// slots.  More than 16 query heads on a key head are taken in turn by the same
// block for the same reason.
#include "kernels.h"
#include "seq_cache8.h"
#include "seq_rope.h"
#include "seq_step.h"

namespace lat {

constexpr int STEP8_TILE = 64;               // slots of a wave's tile

struct Step8K {
  SeqCache8Args c;
  int heads, group, cap, ld, nb;             // bytes of a slot, blocks of a cache and head
  float eps, inv_dim;
  int rope, rotary, inter;
  SeqTensor q, k, v;
  const int32_t* pos;
  const float *gq, *gk;
  float* part;
  StepJoin j;
};

// x as the sum of N bf16 values, the largest first
template <int N> struct Bf16Parts { Frag<bf16_t> p[N]; };
template <int N>
__device__ inline void split(const float* x, Bf16Parts<N>& f) {
  float r[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) r[e] = x[e];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    f.p[i].v = __builtin_bit_cast(bf16x8, Vec16<bf16_t>::pack(r));
#pragma unroll
    for (int e = 0; e < 8; ++e) r[e] -= bf2f(f2bf(r[e]));
  }
}

// Eight codes as bf16 (v_cvt_scalef32_pk_bf16_fp8, scale 1)
__device__ inline Frag<bf16_t> decode(u32x2 w) {
  typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
  u32x4 o;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    o[2 * i] = __builtin_bit_cast(uint32_t, (bf2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], 1.f, false));
    o[2 * i + 1] = __builtin_bit_cast(uint32_t, (bf2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], 1.f, true));
  }
  return {__builtin_bit_cast(bf16x8, o)};
}

// A wave's tile of value codes in LDS: rows of DP bytes, 16-byte unit c of row r at
// c ^ swz(r), so that the 16 rows that half a wave reads at a time (0 .. 7 and 16 ..
// 23 of each 32) lie on distinct banks.
template <int DP> struct Tile8 {
  static constexpr int UPR = DP / 16;
  static constexpr int BYTES = STEP8_TILE * DP;
  __device__ static constexpr int swz(int r) {
    return DP == 128 ? ((r >> 1) & 3) | (((r >> 4) & 1) << 2) : DP == 64 ? ((r >> 2) & 1) | (((r >> 4) & 1) << 1)
                                                                         : (r >> 4) & 1;
  }
  __device__ static inline int at(int row, int unit) { return row * DP + ((unit ^ swz(row)) << 4); }
};

template <typename T, int DP> struct Step8Cfg {
  static constexpr int PARTS = sizeof(T) == 2 ? 2 : 3;
  static constexpr int JOIN = 4 * STEP_HEADS * (DP + 4) * 4, VT = 4 * Tile8<DP>::BYTES;
  static constexpr int WORK = JOIN > VT ? JOIN : VT;                  // tiles, then the join of the waves
  static constexpr int QN = WORK, KN = QN + STEP_HEADS * DP * 4;      // q rows; new k, v; all fp32
  static constexpr int COPY = KN + 2 * DP * 4;                        // the block's codes, k then v
  static constexpr int SC = COPY + 2 * CACHE8_BLOCK * DP;             // its scales
  static constexpr size_t LDS = SC + 16;
};

template <typename T, int DP>
__global__ __launch_bounds__(256, 2) void seq_step8_kernel(Step8K A, RopeTurns turns) {
  using Cfg = Step8Cfg<T, DP>;
  using TL = Tile8<DP>;
  using B8 = Block8<DP>;
  constexpr int NP = Cfg::PARTS, KS = DP / 32, OB = DP / 16, KV = DP == 128 ? 2 : 1, UPR = TL::UPR;
  typedef typename std::conditional<DP == 32, u32x2, u32x4>::type KVec;
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g16 = lane >> 4, l16 = lane & 15, D = A.c.dim, ns = A.j.ns;
  int blk = blockIdx.x;
  const int u = blk % ns; blk /= ns;
  const int kv = blk % A.c.kv_heads, b = blk / A.c.kv_heads;
  const int p = A.j.lens[b], ci = A.c.index ? A.c.index[b] : b;
  if (p < 0 || ci < 0 || ci >= A.c.num_caches) return;
  const int n = min(p, A.cap - 1) + 1, slot = seq_slot(p, A.c.sinks, A.c.window);
  // the split's slots, whole rounds of the four waves
  constexpr int ROUND = 4 * STEP8_TILE;
  const int chunk = ((n + ns - 1) / ns + ROUND - 1) & ~(ROUND - 1);
  const int a0 = (int)min((int64_t)u * chunk, (int64_t)n), a1 = (int)min((int64_t)a0 + chunk, (int64_t)n);
  const int64_t head = (int64_t)ci * A.c.kv_heads + kv;
  uint8_t* const kc = A.c.kc + head * A.cap * A.ld;
  uint8_t* const vc = A.c.vc + head * A.cap * A.ld;
  float* const ks = A.c.ks + head * A.nb;
  float* const vs = A.c.vs + head * A.nb;
  float* const qn = reinterpret_cast<float*>(smem + Cfg::QN);         // [16][DP]
  float* const kn = reinterpret_cast<float*>(smem + Cfg::KN);         // k, v
  char* const copy = smem + Cfg::COPY;
  float* const sc = reinterpret_cast<float*>(smem + Cfg::SC);
  char* const VS = smem + w * TL::BYTES;

  // a lane's share of a tile: keys (slot 16 r + l16), values, the blocks' scales
  struct Load { KVec k[4 * KV]; u32x4 v[UPR]; float ks, vs; };
  Load L;
  const int tiles = a1 > a0 ? (a1 - a0 + STEP8_TILE - 1) / STEP8_TILE : 0;
  auto issue = [&](int t) {
    const int j0 = a0 + t * STEP8_TILE, nk = min(STEP8_TILE, a1 - j0);
    const uint8_t* kp = kc + (int64_t)j0 * A.ld;
    const uint8_t* vp = vc + (int64_t)j0 * A.ld;
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int i = 0; i < KV; ++i) {
        const int row = min(16 * r + l16, nk - 1), d = DP == 32 ? 8 * g16 : 64 * i + 16 * g16;
        L.k[r * KV + i] = *reinterpret_cast<const KVec*>(kp + row * A.ld + (d < A.ld ? d : 0));
      }
#pragma unroll
    for (int i = 0; i < UPR; ++i) {
      const int x = i * 64 + lane, row = min(x / UPR, nk - 1), c = 16 * (x % UPR);
      L.v[i] = *reinterpret_cast<const u32x4*>(vp + row * A.ld + (c < A.ld ? c : 0));
    }
    const int at = min(j0 / CACHE8_BLOCK + (lane & 3), (n - 1) / CACHE8_BLOCK);
    L.ks = ks[at];
    L.vs = vs[at];
  };

  const bool owner = slot >= a0 && slot < a1;
  const int sb = slot & ~(CACHE8_BLOCK - 1);         // the first slot of the event's block
  const int hgs = (A.group + STEP_HEADS - 1) / STEP_HEADS;
#pragma unroll 1
  for (int hg = 0; hg < hgs; ++hg) {
    const int nh = min(STEP_HEADS, A.group - hg * STEP_HEADS), h0 = kv * A.group + hg * STEP_HEADS;
    if (hg > 0) __syncthreads();                     // the join's reads of LDS
    if (w < tiles) issue(w);

    // the event's own vectors: rows of qn (zeros past the heads), kn, vn
    {
      const int np = A.rotary >> 1;
      const bool rot = lane < np;
      int x, y;
      if (A.inter || !rot) { x = 2 * lane; y = x + 1; } else { x = lane; y = np + lane; }
      const bool on = x < D;
      const int pos = A.pos ? A.pos[b] : p;
      float2 cs{1.f, 0.f};
      if (A.rope && rot) cs = rope_cs(pos, turns.f[lane]);
      for (int r = w; r < (hg == 0 ? STEP_HEADS + 2 : STEP_HEADS); r += 4) {
        const bool isq = r < STEP_HEADS, live = !isq || r < nh;
        const T* src = isq ? (const T*)A.q.p + (int64_t)b * A.q.ld + (h0 + min(r, nh - 1)) * D
                     : r == STEP_HEADS ? (const T*)A.k.p + (int64_t)b * A.k.ld + kv * D
                                       : (const T*)A.v.p + (int64_t)b * A.v.ld + kv * D;
        float zx = on ? ld(src + x) : 0.f, zy = on ? ld(src + y) : 0.f;
        if (sizeof(T) == 4 && A.rope && r == STEP_HEADS) {
          // An fp32 key is rounded to eight bits next; its norm and rotation are
          // taken in 64, so that which code it gets does not hang on the order of
          // a sum (one row a user: no time is seen).
          const double dx = zx, dy = zy;
          const double rr = 1.0 / sqrt(wave_sum(dx * dx + dy * dy) / D + (double)A.eps);
          const double ux = dx * rr * (A.gk && on ? A.gk[x] : 1.f), uy = dy * rr * (A.gk && on ? A.gk[y] : 1.f);
          double c = 1.0, s = 0.0;
          if (rot) {
            const double t = (double)pos * turns.f[lane];
            sincospi(2.0 * (t - rint(t)), &s, &c);
          }
          zx = (float)(ux * c - uy * s);
          zy = (float)(ux * s + uy * c);
        } else if (A.rope && r <= STEP_HEADS) {
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
          float* dst = isq ? qn + r * DP : kn + (r - STEP_HEADS) * DP;
          dst[x] = isq ? zx : ld_round<T>(zx);
          dst[y] = isq ? zy : ld_round<T>(zy);
        }
      }
    }
    __syncthreads();
    if (hg == 0 && owner && w < 2) {
      // the event's block anew: wave 0 its keys, wave 1 its values
      uint8_t* const c = w == 0 ? kc : vc;
      float* const s = (w == 0 ? ks : vs) + sb / CACHE8_BLOCK;
      const int row = sb + B8::slot();
      const bool mine = row == slot, old = !mine && row < n;
      const float s0 = *s;
      B8 x;
      x.from_row(kn + w * DP, DP, mine);
      x.from_codes(c + (int64_t)min(row, n - 1) * A.ld, s0, D, A.ld, old);
      const float s1 = x.scale();
      uint32_t code[B8::W];
      x.codes(s1, code);
      if (mine || (old && s1 != s0)) B8::store(c + (int64_t)row * A.ld, A.ld, code);
      if (lane == 0) {
        *s = s1;
        sc[w] = s1;
      }
      B8::store(reinterpret_cast<uint8_t*>(copy) + (w * CACHE8_BLOCK + B8::slot()) * DP, DP, code);
    }
    __syncthreads();
    Bf16Parts<NP> qf[KS];
#pragma unroll
    for (int i = 0; i < KS; ++i) {
      Frag<float> f;
      load_frag(qn + l16 * DP + (DP == 32 ? 8 * g16 : 64 * (i >> 1) + 16 * g16 + 8 * (i & 1)), true, f);
      split(f.v, qf[i]);
    }

    const float c = A.j.scale * STEP_LOG2E;
    f32x4 o[OB];
#pragma unroll
    for (int i = 0; i < OB; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f;
    auto tile = [&](int t) {
      const int j0 = a0 + t * STEP8_TILE, nk = min(STEP8_TILE, a1 - j0);
      const int nr = owner && sb >= j0 && sb < j0 + STEP8_TILE ? (sb - j0) / CACHE8_BLOCK : -1;   // the event's block here
      // values to the wave's LDS rows; slots that are not there are zeros
#pragma unroll
      for (int i = 0; i < UPR; ++i) {
        const int x = i * 64 + lane, row = x / UPR;
        u32x4 v = L.v[i];
        if (row >= nk) v = u32x4{0u, 0u, 0u, 0u};
        *reinterpret_cast<u32x4*>(VS + TL::at(row, x % UPR)) = v;
      }
      if (nr >= 0)
        for (int x = lane; x < CACHE8_BLOCK * UPR; x += 64)
          *reinterpret_cast<u32x4*>(VS + TL::at(CACHE8_BLOCK * nr + x / UPR, x % UPR)) =
              *reinterpret_cast<const u32x4*>(copy + CACHE8_BLOCK * DP + 16 * x);
      float x[16], pv[4], tm = -INFINITY;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        f32x4 s{0.f, 0.f, 0.f, 0.f};
        float kscale = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(L.ks), r));
        // (behind the last slot: weights 0 under a scale that may be anything)
        pv[r] = 16 * r < nk ? __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(L.vs), r)) : 0.f;
        if (r == nr) {
          kscale = sc[0];
          pv[r] = sc[1];
        }
#pragma unroll
        for (int i = 0; i < KV; ++i) {
          KVec kw = L.k[r * KV + i];
          const int d = DP == 32 ? 8 * g16 : 64 * i + 16 * g16;
          if (r == nr) kw = *reinterpret_cast<const KVec*>(copy + l16 * DP + d);
#pragma unroll
          for (int h = 0; h < (DP == 32 ? 1 : 2); ++h) {
            u32x2 w8{kw[2 * h], kw[2 * h + 1]};
            if (d + 8 * h >= D) w8 = u32x2{0u, 0u};
            const Frag<bf16_t> f = decode(w8);
            const Bf16Parts<NP>& q = qf[DP == 32 ? 0 : 2 * i + h];
#pragma unroll
            for (int y = NP - 1; y >= 0; --y) mma16(f, q.p[y], s);
          }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          x[4 * r + i] = 16 * r + 4 * g16 + i < nk ? s[i] * kscale : -INFINITY;
          tm = fmaxf(tm, x[4 * r + i]);
        }
      }
      if (t + 4 < tiles) issue(t + 4);                     // into the registers that are free now
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
      for (int e = 0; e < 16; ++e) {
        x[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[e], c, -mc));
        l += x[e];
        x[e] *= pv[e >> 2];
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        Bf16Parts<NP> pf;
        split(x + 8 * h, pf);
        // lane's piece of the transposed read: row 32 h + 16 (e / 4) + 4 g16 + e % 4, e = l16 / 2
        const int e = l16 >> 1, row = 32 * h + 16 * (e >> 2) + 4 * g16 + (e & 3);
#pragma unroll
        for (int i = 0; i < OB; ++i) {
          typedef int i32x2 __attribute__((ext_vector_type(2)));
          typedef __attribute__((address_space(3))) i32x2 lds_v2;
          const i32x2 w8 = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_v2*)(VS + TL::at(row, i) + 8 * (l16 & 1)));
          const Frag<bf16_t> f = decode(u32x2{(uint32_t)w8[0], (uint32_t)w8[1]});
#pragma unroll
          for (int y = NP - 1; y >= 0; --y) mma16(f, pf.p[y], o[i]);
        }
      }
    };
#pragma unroll 1
    for (int t = w; t < tiles; t += 4) tile(t);
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
      float S = 0.f, O = 0.f;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float* P = J + (i * STEP_HEADS + h) * (DP + 4);
        const float f = mm[i] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((mm[i] - M) * c);
        S += P[DP + 1] * f;
        O += P[d] * f;
      }
      if (ns == 1) {
        st((T*)A.j.out.p + (int64_t)b * A.j.out.ld + (h0 + h) * D + d, O / S);
      } else {
        float* P = A.part + (((int64_t)b * A.heads + h0 + h) * ns + u) * (D + 2);
        P[d] = O;
        if (d == 0) {
          P[D] = M;
          P[D + 1] = S;
        }
      }
    }
  }
}

// Blocks of one launch do not go by 16 query heads here: those share a block.
static int step8_splits(int batch, int kv_heads, int cap) { return step_splits(batch, kv_heads, kv_heads, cap); }

size_t seq_step8_workspace(int batch, int heads, int kv_heads, int dim, int cap) {
  if (batch == 0) return 0;
  const int ns = step8_splits(batch, kv_heads, cap);
  return ns > 1 ? (size_t)batch * heads * ns * (dim + 2) * sizeof(float) : 0;
}

template <typename T, int DP>
static hipError_t step8_launch(const Step8K& A, const RopeTurns& t, int batch, hipStream_t s) {
  constexpr size_t lds = Step8Cfg<T, DP>::LDS;
  static LdsLimit lim;
  LAT_HIP_CHECK(lds_limit(seq_step8_kernel<T, DP>, lds, lim));
  seq_step8_kernel<T, DP><<<batch * A.c.kv_heads * A.j.ns, 256, lds, s>>>(A, t);
  LAT_LAUNCH_CHECK();
  if (A.j.ns > 1) {
    seq_step_join_kernel<T, DP><<<batch * A.heads, 256, 0, s>>>(A.j);
    LAT_LAUNCH_CHECK();
  }
  return hipSuccess;
}

hipError_t seq_step8(const SeqStepArgs& a, const SeqCache8Args& c, const RopeTurns& t, void* ws, hipStream_t s) {
  if (a.batch == 0) return hipSuccess;
  Step8K A{};
  A.c = c;
  A.heads = a.heads;
  A.group = a.heads / c.kv_heads;
  A.cap = c.sinks + c.window;
  A.ld = cache8_ld(c.dim);
  A.nb = cdiv(A.cap, CACHE8_BLOCK);
  A.eps = a.eps;
  A.inv_dim = 1.f / c.dim;
  A.rope = a.rope;
  A.rotary = a.rope ? a.rotary : 0;
  A.inter = a.interleaved;
  A.q = a.q; A.k = a.k; A.v = a.v;
  A.pos = a.positions;
  A.gq = a.gain_q;
  A.gk = a.gain_k;
  A.part = (float*)ws;
  A.j = {a.lens, c.index, c.num_caches, a.heads, c.dim, step8_splits(a.batch, c.kv_heads, A.cap), a.scale, A.part, a.out};
  const int D = c.dim;
  if (c.dt == DT_BF16)
    return D <= 32 ? step8_launch<bf16_t, 32>(A, t, a.batch, s) : D <= 64 ? step8_launch<bf16_t, 64>(A, t, a.batch, s)
                                                                         : step8_launch<bf16_t, 128>(A, t, a.batch, s);
  return D <= 32 ? step8_launch<float, 32>(A, t, a.batch, s) : D <= 64 ? step8_launch<float, 64>(A, t, a.batch, s)
                                                                      : step8_launch<float, 128>(A, t, a.batch, s);
}

// ---------------------------------------------------------------------------
// Fill.  A wave takes a block of 16 slots of k or v of a key head.  The slots that
// a sequence's rows go to are at most three ranges (sinks, and the window's, which
// may wrap); their blocks are numbered through, each once.  Reads and writes the
// kept rows once.
struct SlotRanges {
  int lo[3], hi[3];                          // blocks, ascending, no block twice
  int count;
  __device__ inline SlotRanges(uint32_t f, uint32_t total, int sinks, int window) {
    count = 0;
    int last = -1;
    auto add = [&](int i, int a, int b) {    // slots a .. b
      lo[i] = max(a / CACHE8_BLOCK, last + 1);
      hi[i] = b / CACHE8_BLOCK;
      last = max(last, hi[i]);
      count += max(0, hi[i] - lo[i] + 1);
    };
    auto none = [&](int i) { lo[i] = 0; hi[i] = -1; };
    if (f < (uint32_t)sinks) add(0, (int)f, (int)min(total, (uint32_t)sinks) - 1); else none(0);
    const uint32_t pa = max(max(f, (uint32_t)sinks), total > (uint32_t)window ? total - window : 0u);
    if (pa < total) {
      const int a = sinks + (int)((pa - sinks) % window), b = sinks + (int)((total - 1 - sinks) % window);
      if (a <= b) { add(1, a, b); none(2); } else { add(1, sinks, b); add(2, a, sinks + window - 1); }
    } else {
      none(1);
      none(2);
    }
  }
  __device__ inline int block(int i) const {
    int b = 0;
#pragma unroll
    for (int r = 0; r < 3; ++r) {
      const int c = max(0, hi[r] - lo[r] + 1);
      if (i >= 0 && i < c) b = lo[r] + i;
      i -= c;
    }
    return b;
  }
};

template <typename T, int DP>
__global__ __launch_bounds__(256) void seq_fill8_kernel(SeqCache8Args C, int rows, const int32_t* __restrict__ off, int S,
                                                        const int32_t* __restrict__ first, SeqTensor k, SeqTensor v,
                                                        int ld, int nb) {
  using B8 = Block8<DP>;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), cap = C.sinks + C.window;
  for (int s = blockIdx.y; s < S; s += gridDim.y) {
    const int ci = C.index ? C.index[s] : s;
    if (ci < 0 || ci >= C.num_caches) continue;
    const int a = max(off[s], 0), e = min(off[s + 1], rows), f = first ? first[s] : 0;
    if (e <= a || f < 0) continue;
    const uint32_t total = (uint32_t)f + (uint32_t)(e - a);
    const SlotRanges R((uint32_t)f, total, C.sinks, C.window);
    const int64_t items = (int64_t)R.count * C.kv_heads * 2;
    for (int64_t it = blockIdx.x * 4 + w; it < items; it += (int64_t)gridDim.x * 4) {
      const int vside = (int)(it & 1), h = (int)((it >> 1) % C.kv_heads), blk = R.block((int)((it >> 1) / C.kv_heads));
      const SeqTensor& t = vside ? v : k;
      const int64_t head = (int64_t)ci * C.kv_heads + h;
      uint8_t* const codes = (vside ? C.vc : C.kc) + head * cap * ld;
      float* const sp = (vside ? C.vs : C.ks) + head * nb + blk;
      // the last position that is in the lane's slot, and whether this call brings it
      const int slot = blk * CACHE8_BLOCK + B8::slot();
      const bool reached = slot < cap && (uint32_t)slot < total;
      uint32_t p = (uint32_t)slot;
      if (reached && slot >= C.sinks) p = total - 1 - (total - 1 - (uint32_t)slot) % (uint32_t)C.window;
      const bool fresh = reached && p >= (uint32_t)f, old = reached && !fresh;
      const float s0 = *sp;
      B8 x;
      x.from_row((const T*)t.p + (a + (int64_t)(fresh ? p - (uint32_t)f : 0u)) * t.ld + h * C.dim, C.dim, fresh);
      const bool any_old = wave_any(old);
      if (any_old) x.from_codes(codes + (int64_t)(old ? slot : blk * CACHE8_BLOCK) * ld, s0, C.dim, ld, old);
      const float s1 = x.scale();
      uint32_t code[B8::W];
      x.codes(s1, code);
      if (fresh || (old && s1 != s0)) B8::store(codes + (int64_t)slot * ld, ld, code);
      if ((threadIdx.x & 63) == 0) *sp = s1;
    }
  }
}

hipError_t seq_cache8_fill(const SeqCache8Args& c, int64_t rows, const int32_t* offsets, int num_seqs,
                           const int32_t* first, SeqTensor k, SeqTensor v, hipStream_t s) {
  if (rows == 0 || num_seqs == 0) return hipSuccess;
  // a wave an item where the sequences have the mean length
  const int64_t mean = cdiv(rows, num_seqs), cap = (int64_t)c.sinks + c.window;
  const int64_t blocks = (mean < cap ? mean : cap) / CACHE8_BLOCK + 1;
  int bx = cdiv(blocks * c.kv_heads * 2, 4);
  if (bx > 1024) bx = 1024;
  const int by = num_seqs < 65535 ? num_seqs : 65535;
  const int ld = cache8_ld(c.dim), nb = cdiv(cap, CACHE8_BLOCK);
  auto launch = [&](auto kern) { kern<<<dim3(bx, by), 256, 0, s>>>(c, (int)rows, offsets, num_seqs, first, k, v, ld, nb); };
  const int D = c.dim;
  if (c.dt == DT_BF16) {
    if (D <= 32) launch(seq_fill8_kernel<bf16_t, 32>);
    else if (D <= 64) launch(seq_fill8_kernel<bf16_t, 64>);
    else launch(seq_fill8_kernel<bf16_t, 128>);
  } else {
    if (D <= 32) launch(seq_fill8_kernel<float, 32>);
    else if (D <= 64) launch(seq_fill8_kernel<float, 64>);
    else launch(seq_fill8_kernel<float, 128>);
  }
  LAT_LAUNCH_CHECK();
  return hipSuccess;
}

}  // namespace lat
