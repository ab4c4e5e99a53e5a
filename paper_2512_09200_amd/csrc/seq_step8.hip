// The single-event step over ring caches of e4m3 codes, and their fill.
//
//   s_j = scale ks(j / 16) <q, kc_j>,  P = softmax(s),  out = sum_j P_j vs(j / 16) vc_j
//
// Memory bound: every visible slot's two rows of codes are read once, half the
// bytes of bf16.  Work is split as in the bf16 step: a block is a user, a key head
// and a split of the slots, its four waves (one, for short windows of many users) take
// tiles of 32 slots in turn with their own running maximum, sum and output.  Codes
// become bf16 in registers (exactly: three bits of fraction) and go to 16x16x32
// matrix instructions; a block's scale multiplies the 16 scores of its slots and their
// probabilities.
// What the step computes itself (query, probabilities) enters as two bf16 parts,
// three where the storage type is fp32, so that out is rounded once.
//
// Keys are fragments straight from memory.  Values are loaded to registers, go
// through the wave's own LDS rows and come back transposed, eight codes of one
// dimension a lane: a direct load to LDS would have the compiler wait for the
// next tile's loads before the first transposed read.  The query's parts lie in LDS
// as fragments, one read of each a tile, so that twelve waves fit a compute unit.
//
// The new event may change its block's scale, and with it the codes of the block's
// other slots.  The split that holds the slot makes the block anew before its
// tiles (wave 0 its keys, wave 1 its values), writes it, and puts a copy into LDS that
// replaces what the tiles load of it; no other block of the launch reads these
// slots.  Query heads above 16 on a key head are taken by a second launch, which
// finds the block as it is now, for the same reason.
//
// 1024 users, windows of 1024 slots of 128, 2 key heads of 4 query heads, bf16: 88 us at
// best and 90 on average, 5.2 TB/s of the bytes it cannot do without (a copy of 0.5 GB
// reaches 5.3); 94 without the hint that a code is read once.  Matrix cores 15% busy, 51% of the cycles issue
// vector instructions (half of them conversions), LDS 15%.
#include "kernels.h"
#include "lanes.h"
#include "seq_cache8.h"
#include "seq_rope.h"
#include "seq_step.h"

namespace lat {

constexpr int STEP8_TILE = 32;               // slots of a wave's tile
constexpr int STEP8_ROUND = 4 * STEP8_TILE;  // of a block's four waves

struct Step8K {
  SeqCache8Args c;
  int heads, group, cap, ld, nb;             // bytes of a slot, blocks of a cache and head
  int work;                                  // bytes of LDS for tiles and join
  int hg0, hgs, append;                      // this launch's groups of 16 query heads; whether it brings the events
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

// LDS: the waves' value tiles, over them the join of the waves (`heads` of 16 head
// columns); the query's fragments; the new k and v; the block's codes, k then v,
// and its scales.
template <typename T, int DP, int WPI> struct Step8Cfg {
  static constexpr int PARTS = sizeof(T) == 2 ? 2 : 3;
  static constexpr int JROW = DP + 4, VT = WPI * Tile8<DP>::BYTES;
  static constexpr int QF = DP / 32 * PARTS * 1024;
  static constexpr int KN = QF, COPY = KN + 2 * DP * 4, SC = COPY + 2 * CACHE8_BLOCK * DP, REST = SC + 16;
  __host__ __device__ static constexpr int work(int heads) {
    return ((4 * WPI * heads * JROW > VT ? 4 * WPI * heads * JROW : VT) + 15) & ~15;
  }
};

template <typename T, int DP, int WPI>
__global__ __launch_bounds__(64 * WPI, 3) void seq_step8_kernel(Step8K A, RopeTurns turns) {
#pragma clang fp contract(off)                       // the same roundings whichever kernel a batch gets
  using Cfg = Step8Cfg<T, DP, WPI>;
  using TL = Tile8<DP>;
  using B8 = Block8<float, DP>;
  constexpr int NP = Cfg::PARTS, KS = DP / 32, OB = DP / 16, KV = DP == 128 ? 2 : 1, UPR = TL::UPR;
  constexpr int R = STEP8_TILE / CACHE8_BLOCK, VL = R * UPR / 4;     // scale blocks of a tile, value loads of a lane
  typedef typename std::conditional<DP == 32, u32x2, u32x4>::type KVec;
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g16 = lane >> 4, l16 = lane & 15, D = A.c.dim, ns = A.j.ns;
  int blk = blockIdx.x;
  const int u = blk % ns; blk /= ns;
  const int hg = A.hg0 + blk % A.hgs; blk /= A.hgs;
  const int kv = blk % A.c.kv_heads, b = blk / A.c.kv_heads;
  const int p = __builtin_amdgcn_readfirstlane(A.j.lens[b]);
  const int ci = __builtin_amdgcn_readfirstlane(A.c.index ? A.c.index[b] : b);
  if (p < 0 || ci < 0 || ci >= A.c.num_caches) return;
  const int n = min(p, A.cap - 1) + 1, slot = seq_slot(p, A.c.sinks, A.c.window);
  // the split's slots, whole rounds of the four waves
  const int chunk = ((n + ns - 1) / ns + STEP8_ROUND - 1) & ~(STEP8_ROUND - 1);
  const int a0 = (int)min((int64_t)u * chunk, (int64_t)n), a1 = (int)min((int64_t)a0 + chunk, (int64_t)n);
  const int64_t head = (int64_t)ci * A.c.kv_heads + kv;
  uint8_t* const kc = A.c.kc + head * A.cap * A.ld;
  uint8_t* const vc = A.c.vc + head * A.cap * A.ld;
  float* const ks = A.c.ks + head * A.nb;
  float* const vs = A.c.vs + head * A.nb;
  char* const rest = smem + A.work;
  float* const kn = reinterpret_cast<float*>(rest + Cfg::KN);         // k, v
  char* const copy = rest + Cfg::COPY;
  float* const sc = reinterpret_cast<float*>(rest + Cfg::SC);
  char* const VS = smem + w * TL::BYTES;             // the wave's value tile

  // The event's block: made anew by waves 0 (keys) and 1 (values; or by the only wave
  // both) of the split that holds the slot (in a launch for further query heads it
  // has been)
  const bool owner = A.append && slot >= a0 && slot < a1;
  const int sb = slot & ~(CACHE8_BLOCK - 1);
  constexpr int SIDES = WPI == 1 ? 2 : 1;
  const bool remake = owner && w < 2;
  B8 x8[SIDES];
  if (remake) {
#pragma unroll
    for (int i = 0; i < SIDES; ++i) {
      x8[i].load_codes((w + i == 0 ? kc : vc) + (int64_t)min(sb + B8::slot(), n - 1) * A.ld, A.ld);
      x8[i].s0 = (w + i == 0 ? ks : vs)[sb / CACHE8_BLOCK];
    }
  }
  // the event's own vectors, a row a wave: pairs (x0, y0) of dimensions
  const int np = A.rotary >> 1, nh = min(STEP_HEADS, A.group - hg * STEP_HEADS), h0 = kv * A.group + hg * STEP_HEADS;
  const bool rot = lane < np;
  int x0, y0;
  if (A.inter || !rot) { x0 = 2 * lane; y0 = x0 + 1; } else { x0 = lane; y0 = np + lane; }
  const bool on = x0 < D;
  const int xl = on ? x0 : 0, yl = on ? y0 : 0;      // (loads are made by every lane, in no branch)
  auto row_of = [&](const SeqTensor& t, int h, float& x, float& y) {
    const T* src = (const T*)t.p + (int64_t)b * t.ld + h * D;
    x = ld(src + xl);
    y = ld(src + yl);
  };
  const int first_q = WPI == 1 ? 0 : (w + 2) & 3;    // query rows: waves 2 and 3 first
  float qx, qy, ex[SIDES], ey[SIDES], gqx = 1.f, gqy = 1.f, gkx = 1.f, gky = 1.f;
  row_of(A.q, h0 + min(first_q, nh - 1), qx, qy);
  if (remake)
#pragma unroll
    for (int i = 0; i < SIDES; ++i) row_of(w + i == 0 ? A.k : A.v, kv, ex[i], ey[i]);
  if (A.gq) { gqx = A.gq[xl]; gqy = A.gq[yl]; }
  if (A.gk) { gkx = A.gk[xl]; gky = A.gk[yl]; }
  const int pos = A.pos ? A.pos[b] : p;

  // a lane's share of a tile: keys (slot 16 r + l16), values, the blocks' scales
  // (lanes 0 .. R - 1 of every 2 R the keys', the others the values')
  KVec lk[R * KV];
  u32x4 lv[VL];
  float ls;
  const int tiles = a1 > a0 ? (a1 - a0 + STEP8_TILE - 1) / STEP8_TILE : 0;
  auto issue_v = [&](int t) {
    const int j0 = a0 + t * STEP8_TILE, nk = min(STEP8_TILE, a1 - j0);
    const uint8_t* vp = vc + (int64_t)j0 * A.ld;
#pragma unroll
    for (int i = 0; i < VL; ++i) {
      const int x = i * 64 + lane, row = min(x / UPR, nk - 1), c = 16 * (x % UPR);
      lv[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(vp + (__umul24(row, A.ld) + (c < A.ld ? c : 0))));
    }
  };
  auto issue_k = [&](int t) {
    const int j0 = a0 + t * STEP8_TILE, nk = min(STEP8_TILE, a1 - j0);
    const uint8_t* kp = kc + (int64_t)j0 * A.ld;
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int i = 0; i < KV; ++i) {
        const int row = min(16 * r + l16, nk - 1), d = DP == 32 ? 8 * g16 : 64 * i + 16 * g16;
        lk[r * KV + i] = __builtin_nontemporal_load(
            reinterpret_cast<const KVec*>(kp + (__umul24(row, A.ld) + (d < A.ld ? d : 0))));
      }
    ls = (lane & R ? vs : ks)[min(j0 / CACHE8_BLOCK + (lane & (R - 1)), (n - 1) / CACHE8_BLOCK)];
  };

  if (w < tiles) {
    issue_v(w);
    issue_k(w);
  }

  float2 cs{1.f, 0.f};
  if (A.rope && rot) cs = rope_cs(pos, turns.f[lane]);
  auto norm_rope = [&](float& zx, float& zy, float gx, float gy) {
    const float rr = 1.f / sqrtf(lanes_join<64>(zx * zx + zy * zy, Add()) * A.inv_dim + A.eps);
    zx *= rr * gx;
    zy *= rr * gy;
    const float tx = zx * cs.x - zy * cs.y, ty = zx * cs.y + zy * cs.x;
    zx = tx;
    zy = ty;
  };
  if (remake) {
#pragma unroll
    for (int i = 0; i < SIDES; ++i) {
      const int side = w + i;                        // 0: k, 1: v
      float zx = on ? ex[i] : 0.f, zy = on ? ey[i] : 0.f;
      if (A.rope && side == 0) {
        if constexpr (sizeof(T) == 4) {
          // An fp32 key is rounded to eight bits next; its norm and rotation are
          // taken in 64, so that which code it gets does not hang on the order of
          // a sum (one row a user).
          const double dx = zx, dy = zy, rr = 1.0 / sqrt(wave_sum(dx * dx + dy * dy) / D + (double)A.eps);
          const double ux = dx * rr * gkx, uy = dy * rr * gky;
          double c = 1.0, s = 0.0;
          if (rot) {
            const double t = (double)pos * turns.f[lane];
            sincospi(2.0 * (t - rint(t)), &s, &c);
          }
          zx = (float)(ux * c - uy * s);
          zy = (float)(ux * s + uy * c);
        } else {
          norm_rope(zx, zy, gkx, gky);
        }
      }
      if (x0 < DP) {
        kn[side * DP + x0] = on ? ld_round<T>(zx) : 0.f;
        kn[side * DP + y0] = on ? ld_round<T>(zy) : 0.f;
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the wave reads what its other lanes have just written
      const int row = sb + B8::slot();
      B8& x = x8[i];
      x.load_row(kn + side * DP, DP, row == slot);
      x.old = row != slot && row < n;
      const float s1 = x.scale(D);
      x.encode(s1, D, (side == 0 ? kc : vc) + (int64_t)row * A.ld, A.ld, x.fresh || (x.old && s1 != x.s0),
               reinterpret_cast<uint8_t*>(copy) + (side * CACHE8_BLOCK + B8::slot()) * DP);
      if (lane == 0) {
        (side == 0 ? ks : vs)[sb / CACHE8_BLOCK] = s1;
        sc[side] = s1;
      }
    }
  }
  // The query's parts: those of element d of row r are element e of lane 16 g + r in
  // the fragment of step i, (i, g, e) as the keys' loads have them.
  if constexpr (WPI == 1) {                          // rows past the heads: zeros at once
#pragma unroll
    for (int i = 0; i < KS * NP; ++i) *reinterpret_cast<u32x4*>(rest + (i * 64 + lane) * 16) = u32x4{0u, 0u, 0u, 0u};
  }
  for (int r = first_q; r < (WPI == 1 ? nh : STEP_HEADS); r += WPI) {
    float zx = qx, zy = qy;
    if (r + WPI < nh) row_of(A.q, h0 + r + WPI, qx, qy);
    if (!on || r >= nh) zx = zy = 0.f;
    if (A.rope && r < nh) norm_rope(zx, zy, gqx, gqy);
    auto put = [&](int d, float z) {
      const int i = DP == 32 ? 0 : 2 * (d >> 6) + ((d >> 3) & 1), g = DP == 32 ? d >> 3 : (d >> 4) & 3, e = d & 7;
#pragma unroll
      for (int y = 0; y < NP; ++y) {
        const bf16_t h = f2bf(z);
        *reinterpret_cast<bf16_t*>(rest + ((i * NP + y) * 64 + 16 * g + r) * 16 + 2 * e) = h;
        z -= bf2f(h);
      }
    };
    if (x0 < DP) {
      put(x0, zx);
      put(y0, zy);
    }
  }
  __syncthreads();

  const float c = A.j.scale * STEP_LOG2E;
  f32x4 o[OB];
#pragma unroll
  for (int i = 0; i < OB; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;
#pragma unroll 1
  for (int t = w; t < tiles; t += WPI) {
    const int j0 = a0 + t * STEP8_TILE, nk = min(STEP8_TILE, a1 - j0);
    const int nr = owner && sb >= j0 && sb < j0 + STEP8_TILE ? (sb - j0) / CACHE8_BLOCK : -1;   // the event's block here
    // values to the wave's LDS rows; slots that are not there are zeros
#pragma unroll
    for (int i = 0; i < VL; ++i) {
      const int x = i * 64 + lane, row = x / UPR;
      u32x4 v = lv[i];
      if (row >= nk) v = u32x4{0u, 0u, 0u, 0u};
      *reinterpret_cast<u32x4*>(VS + TL::at(row, x % UPR)) = v;
    }
    if (nr >= 0) {
      for (int x = lane; x < CACHE8_BLOCK * UPR; x += 64)
        *reinterpret_cast<u32x4*>(VS + TL::at(CACHE8_BLOCK * nr + x / UPR, x % UPR)) =
            *reinterpret_cast<const u32x4*>(copy + CACHE8_BLOCK * DP + 16 * x);
#pragma unroll
      for (int r = 0; r < R; ++r)
        if (r == nr)
#pragma unroll
          for (int i = 0; i < KV; ++i)
            lk[r * KV + i] = *reinterpret_cast<const KVec*>(copy + l16 * DP + (DP == 32 ? 8 * g16 : 64 * i + 16 * g16));
    }
    if (t + WPI < tiles) issue_v(t + WPI);               // into the registers that are free now
    f32x4 s[R];
#pragma unroll
    for (int r = 0; r < R; ++r) s[r] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < KS; ++i) {
      Frag<bf16_t> q[NP];
#pragma unroll
      for (int y = 0; y < NP; ++y) q[y].v = *reinterpret_cast<const bf16x8*>(rest + ((i * NP + y) * 64 + lane) * 16);
      const int d = DP == 32 ? 8 * g16 : 64 * (i >> 1) + 16 * g16 + 8 * (i & 1);
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const KVec& kw = lk[r * KV + (i >> 1)];
        u32x2 w8{kw[2 * (i & 1)], kw[2 * (i & 1) + 1]};
        if (d >= D) w8 = u32x2{0u, 0u};
        const Frag<bf16_t> f = decode(w8);
#pragma unroll
        for (int y = NP - 1; y >= 0; --y) mma16(f, q[y], s[r]);
      }
    }
    float x[4 * R], pv[R], tm = -INFINITY;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      float kscale = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(ls), r));
      // (behind the last slot: weights 0 under a scale that may be anything)
      pv[r] = 16 * r < nk ? __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(ls), R + r)) : 0.f;
      if (r == nr) {
        kscale = sc[0];
        pv[r] = sc[1];
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[4 * r + i] = 16 * r + 4 * g16 + i < nk ? s[r][i] * kscale : -INFINITY;
        tm = fmaxf(tm, x[4 * r + i]);
      }
    }
    if (t + WPI < tiles) issue_k(t + WPI);
    tm = fmaxf(tm, __shfl_xor(tm, 16, 64));
    tm = max32(tm);
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
    for (int e = 0; e < 4 * R; ++e) {
      x[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[e], c, -mc));
      l += x[e];
      x[e] *= pv[e >> 2];
    }
    static_assert(R == 2, "one product over the tile's 32 slots");
    Bf16Parts<NP> pf;
    split(x, pf);
    // lane's piece of the transposed read: row 16 (e / 4) + 4 g16 + e % 4, e = l16 / 2
    const int e = l16 >> 1, row = 16 * (e >> 2) + 4 * g16 + (e & 3);
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
  l += __shfl_xor(l, 16, 64);
  l = add32(l);
  // join of the waves: O[w][head][DP], then m and l
  float* const J = reinterpret_cast<float*>(smem);
  __syncthreads();
  if (l16 < nh) {
    float* const Jw = J + (w * nh + l16) * Cfg::JROW;
#pragma unroll
    for (int i = 0; i < OB; ++i) *reinterpret_cast<f32x4*>(Jw + 16 * i + 4 * g16) = o[i];
    if (g16 == 0) {
      Jw[DP] = m;
      Jw[DP + 1] = l;
    }
  }
  __syncthreads();
  for (int x = threadIdx.x; x < nh * D; x += 64 * WPI) {
    const int h = x / D, d = x - h * D;
    float mm[WPI], M = -INFINITY;
#pragma unroll
    for (int i = 0; i < WPI; ++i) {
      mm[i] = J[(i * nh + h) * Cfg::JROW + DP];
      M = fmaxf(M, mm[i]);
    }
    float S = 0.f, O = 0.f;
#pragma unroll
    for (int i = 0; i < WPI; ++i) {
      const float* P = J + (i * nh + h) * Cfg::JROW;
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

// Splits of the slots: as many as leave all blocks of the launch on the chip at once
// (three a compute unit), of 128 slots (a round of a block's waves) or more, and
// no more than the join holds.  Three users, 131049 slots of 128, 2 key heads: 33 us with
// 768 blocks in all, 38 with 512, 36 with 1024 (whose join takes 8 us instead of 5).
// With hundreds of users the rounding down leaves places empty: 200 users of 2 key heads,
// 20000 slots, 392 us in 400 blocks, 402 in 800, 358 in 1200; 1020 slots 28, 33 and 35.
// One user, 1020 / 4000 / 16000 slots: 12.4 / 13.5 / 15.3 us a step, with splits of 256
// or more 13.1 / 14.4 / 16.2, of 1024 16.0 / 22.3 / 21.3.  Up to four rounds of slots
// a block alone is faster than its parts and their join: 500 slots 11.1 and 11.8 us.
constexpr int STEP8_BLOCKS = 768;
static int step8_splits(int batch, int kv_heads, int cap) {
  int64_t n = STEP8_BLOCKS / ((int64_t)batch * kv_heads);
  if (cap <= 4 * STEP8_ROUND) n = 1;
  if (n > cap / STEP8_ROUND) n = cap / STEP8_ROUND;
  if (n > STEP_MAX_SPLITS) n = STEP_MAX_SPLITS;
  return n > 1 ? (int)n : 1;
}

size_t seq_step8_workspace(int batch, int heads, int kv_heads, int dim, int cap) {
  if (batch == 0) return 0;
  const int ns = step8_splits(batch, kv_heads, cap);
  return ns > 1 ? (size_t)batch * heads * ns * (dim + 2) * sizeof(float) : 0;
}

template <typename T, int DP, int WPI>
static hipError_t step8_launch(Step8K A, const RopeTurns& t, int batch, hipStream_t s) {
  using Cfg = Step8Cfg<T, DP, WPI>;
  A.work = Cfg::work(A.group < STEP_HEADS ? A.group : STEP_HEADS);
  const size_t lds = (size_t)A.work + Cfg::REST;      // at most 64 KB: no limit to raise
  static_assert(Cfg::work(STEP_HEADS) + Cfg::REST <= 65536, "LDS");
  auto launch = [&](int hg0, int hgs, int append) -> hipError_t {
    A.hg0 = hg0;
    A.hgs = hgs;
    A.append = append;
    seq_step8_kernel<T, DP, WPI><<<batch * A.c.kv_heads * hgs * A.j.ns, 64 * WPI, lds, s>>>(A, t);
    LAT_LAUNCH_CHECK();
    return hipSuccess;
  };
  LAT_HIP_CHECK(launch(0, 1, 1));
  if (A.group > STEP_HEADS) LAT_HIP_CHECK(launch(1, cdiv(A.group, STEP_HEADS) - 1, 0));
  if (A.j.ns > 1) {
    seq_step_join_kernel<T, DP><<<batch * A.heads, 256, 0, s>>>(A.j);
    LAT_LAUNCH_CHECK();
  }
  return hipSuccess;
}

// Short windows of many users: a wave an item (a user's key head) instead of four, whose
// start and join would be most of a block's time.  The more items, the longer the windows
// it pays for.  bf16, 2 key heads of 64, 16384 items of 30 / 128 / 500 slots 102 / 118 / 226 us
// with four waves, 50 / 74 / 198 with one (16, 55 and 203 at the copy's rate); 1024 items 10.1 / 11.5 / 18.2 and 9.9 / 12.6 / 25.3.
// fp32, heads of 128, 16384 items of 30 / 500 slots: 180 / 461 and 127 / 451.
template <typename T, int DP>
static hipError_t step8_pick(const Step8K& A, const RopeTurns& t, int batch, hipStream_t s) {
  if (A.cap <= 512 && A.cap <= (int64_t)batch * A.c.kv_heads / 16) return step8_launch<T, DP, 1>(A, t, batch, s);
  return step8_launch<T, DP, 4>(A, t, batch, s);
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
    return D <= 32 ? step8_pick<bf16_t, 32>(A, t, a.batch, s) : D <= 64 ? step8_pick<bf16_t, 64>(A, t, a.batch, s)
                                                                         : step8_pick<bf16_t, 128>(A, t, a.batch, s);
  return D <= 32 ? step8_pick<float, 32>(A, t, a.batch, s) : D <= 64 ? step8_pick<float, 64>(A, t, a.batch, s)
                                                                      : step8_pick<float, 128>(A, t, a.batch, s);
}

// ---------------------------------------------------------------------------
// Fill.  A wave takes a block of 16 slots of a key head, keys and values (bf16 heads
// above 64: one of them).  The slots that
// a sequence's rows go to are at most three ranges (sinks, and the window's, which
// may wrap); their blocks are numbered through, each once.  Reads and writes the
// kept rows once: 153600 rows of 2 heads of 128, bf16, 43 us at best, 46
// on average (4.8 TB/s).
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

// Keys and values of a block by one wave, both loads out together, or by two.  Two:
// bf16 heads of 128, whose registers would leave four waves a SIMD instead of five
// (153600 kept rows, 2 heads: 44 us, by one 46).  One: 100000 histories of 5, a head of
// 32, 67 us, by two 144; fp32, 8000 of 20, 2 heads of 128, 84 and 101.
template <typename T, int DP> struct Fill8Cfg { static constexpr int SIDES = sizeof(T) == 2 && DP == 128 ? 1 : 2; };

// A sequence's items are shared out by seq_fill8.h's plan.
template <typename T, int DP>
__global__ __launch_bounds__(256) void seq_fill8_kernel(SeqCache8Args C, int rows, const int32_t* __restrict__ off, int S,
                                                        const int32_t* __restrict__ first, SeqTensor k, SeqTensor v,
                                                        int ld, int nb, Fill8Plan P) {
  using B8 = Block8<T, DP>;
  constexpr int SIDES = Fill8Cfg<T, DP>::SIDES;
  const int cap = C.sinks + C.window;
  const int wave = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
  Fill8Share w;
  if (!fill8_share(P, wave, rows, S, [&](int i) { return __builtin_amdgcn_readfirstlane(off[i]); }, &w)) return;
  for (int64_t s = w.s; s < S; s += w.ds) {
    const int ci = __builtin_amdgcn_readfirstlane(C.index ? C.index[s] : (int)s);
    const int a = max(__builtin_amdgcn_readfirstlane(off[s]), 0), e = min(__builtin_amdgcn_readfirstlane(off[s + 1]), rows);
    const int f = first ? __builtin_amdgcn_readfirstlane(first[s]) : 0;
    if (ci < 0 || ci >= C.num_caches || e <= a || f < 0 || (e - a >= P.large) != w.behind) continue;
    const uint32_t total = (uint32_t)f + (uint32_t)(e - a);
    const SlotRanges R((uint32_t)f, total, C.sinks, C.window);
    const int sides = 2 / SIDES;                 // items of a block and head
    const int64_t items = (int64_t)R.count * C.kv_heads * sides;
    for (int64_t it = w.it0; it < items; it += w.dit) {
      const int side = (int)(it % sides), h = (int)(it / sides % C.kv_heads);
      const int blk = R.block((int)(it / sides / C.kv_heads));
      const int64_t head = (int64_t)ci * C.kv_heads + h;
      // the last position that is in the lane's slot, and whether this call brings it
      const int slot = blk * CACHE8_BLOCK + B8::slot();
      const bool reached = slot < cap && (uint32_t)slot < total;
      uint32_t p = (uint32_t)slot;
      if (reached && slot >= C.sinks) p = total - 1 - (total - 1 - (uint32_t)slot) % (uint32_t)C.window;
      const bool fresh = reached && p >= (uint32_t)f, old = reached && !fresh, any_old = wave_any(old);
      const int64_t row = a + (int64_t)(fresh ? p - (uint32_t)f : 0u);
      B8 x[SIDES];                               // keys, values; or what `side` says
#pragma unroll
      for (int i = 0; i < SIDES; ++i) {
        const SeqTensor& t = side + i ? v : k;
        x[i].load_row((const T*)t.p + row * t.ld + h * C.dim, C.dim, fresh);
      }
#pragma unroll
      for (int i = 0; i < SIDES; ++i) {
        uint8_t* const base = (side + i ? C.vc : C.kc) + head * cap * ld;
        uint8_t* const codes = base + (int64_t)slot * ld;
        float* const sp = (side + i ? C.vs : C.ks) + head * nb + blk;
        x[i].old = old;
        float s1;
        if (!any_old && x[i].fresh_scale(&s1)) {
          x[i].encode_fresh(s1, codes, ld);
        } else {
          x[i].s0 = *sp;
          x[i].load_codes(old ? codes : base + (int64_t)blk * CACHE8_BLOCK * ld, ld);
          s1 = x[i].scale(C.dim);
          x[i].encode(s1, C.dim, codes, ld, fresh || (old && s1 != x[i].s0), nullptr);
        }
        if ((threadIdx.x & 63) == 0) *sp = s1;
      }
    }
  }
}

hipError_t seq_cache8_fill(const SeqCache8Args& c, int64_t rows, const int32_t* offsets, int num_seqs, int64_t max_len,
                           const int32_t* first, SeqTensor k, SeqTensor v, hipStream_t s) {
  if (rows == 0 || num_seqs == 0) return hipSuccess;
  const int D = c.dim, cap = c.sinks + c.window;
  const Fill8Plan P = fill8_plan(rows, num_seqs, max_len, cap, c.kv_heads * (c.dt == DT_BF16 && D > 64 ? 2 : 1));
  const int ld = cache8_ld(c.dim), nb = cdiv(cap, CACHE8_BLOCK);
  auto launch = [&](auto kern) {
    kern<<<cdiv(P.waves, 4), 256, 0, s>>>(c, (int)rows, offsets, num_seqs, first, k, v, ld, nb, P);
  };
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
