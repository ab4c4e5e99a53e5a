// Windowed attention over packed event sequences, forward and backward.
//
//   V(i) = { j : start(i) <= j <= i, i - j < W or j < start(i) + N, shown(j) }
//   s_ij = scale <q_i, k_j>, P_ij = exp(s_ij - lse_i), o_i = sum_j P_ij v_j
//   delta_i = <do_i, o_i>, dS_ij = P_ij (<do_i, v_j> - delta_i)
//   dq_i = scale sum_j dS_ij k_j, dk_j = scale sum_i dS_ij q_i, dv_j = sum_i P_ij do_i
//
// Tiles lie on the packed row axis, whatever the sequence boundaries: many
// short sequences fill a tile as one long sequence does, and no list of tiles
// is needed.  The keys of a tile of rows are one contiguous range (from the
// first row's window to the last row) and the sinks of the first row's
// sequence, where they lie before it: later sequences start inside the range.
// Which of them a row sees is a comparison with the row's own bounds, made
// only in key tiles that some row of the wave sees in part.
//
// Forward and dQ: a block is 4 waves of 32 rows of one head each; query heads
// that share a key head share the block (as many of 4, 2 or 1 as divide the
// group) so that a block's rows span a short range (groups of 4, window 256 of
// heads of 64, dQ: 76 us with one head a block, 69 so; window 2048 of heads of
// 128: 952 and 927).  The product is taken
// transposed, S^T = K Q^T: a lane holds one row's scores, its maximum and sum
// need one exchange between lane halves, and the probabilities are the
// next product's operand (O^T = V^T P^T) where they are.  K and V tiles go from
// memory straight to LDS; the next tile's loads go out when a tile's first
// product begins and have until its second one: the compiler cannot tell the
// places that transposed LDS reads take from those that direct loads write, and
// waits for all loads before the first such read (bf16; fp32 reads columns
// with ordinary loads and has the whole tile).
//
// dK and dV: a block takes 128 keys, a wave 32 of them, over the rows that see
// them and the group's heads, S = Q K^T.  Rows that see a
// sink after its window has passed are spread over blocks of their own
// (seq_sink_kernel: a long sequence's sinks would otherwise be one block's work),
// whose partial sums the main kernel adds in a fixed order.  No atomics.
//
// A masked pair has P = 0, but 0 * (a non-finite value) is not 0: where an
// element of a wave's result is not finite, the block sweeps again for such
// elements alone (RepairPass, below), so that they are what the rows they see make
// of them.
//
// Roundings (bf16).  P and dS are operands of one bf16 part: every term of a sum
// is off by up to 2^-8 of itself, each on its own.  In the measured cases out is off
// by 2.0e-3 of its norm and dq, dk by 2.4e-3, where one rounding of the exact
// result gives 1.5e-3 to 1.7e-3.  A second part, as the single-event step takes, would double the
// second products, which the matrix cores do not have free here.  Scores, maxima,
// sums, lse, delta and accumulators are fp32.
//
// Bound.  65536 rows in 4 histories, 8 heads of 128 over 2, window 2048, bf16 (shortest
// of six dispatches here and below; the means are 2 to 15% longer):
// forward 687 us (0.75 PFLOP/s), dQ 881, dK/dV 1191 (0.88 and 0.87 of their three
// and four products); the matrix cores are busy 42-47% of the cycles, beside
// the scores' vector work (an exponential of 16 cycles, the subtraction, sum,
// maximum and rounding for every 32 x 32 x 16 product's share) and the wait for the
// next tile before the second product, LDS 21-40%.
// 32768 rows, heads of 64, window 256, hidden keys: 58, 66 and 68 us, half of the
// cycles issuing vector instructions.  8192 histories of 20, 4 heads of 32: 63,
// 72 and 71 us for 210, 294 and 252 MB (43, 60 and 52 us of copy time).
#include <algorithm>
#include <type_traits>

#include "kernels.h"
#include "seq_tile.h"

namespace lat {

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

struct AttnK {                     // kernel arguments
  int rows, dim, heads, kv_heads, group, window, sinks;
  int hb, row_tiles;               // heads of a block (forward, dQ), its row tiles
  int chunk;                       // rows of a tile of seq_sink_kernel (0: no sequence has late rows)
  float scale;
  const SeqSpan* span;
  const uint8_t* mask;
  SeqTensor q, k, v, o, go, gq, gk, gv;
  float* lse;                      // [heads, rows]
  void* out_lo;                    // [rows, heads, dim] or null: what rounding took from o (bf16)
  float* lse2;                     // workspace [heads, rows]: lse log2 e, +inf where nothing is seen
  float* delta;                    // workspace [heads, rows]
  float* part;                     // workspace [late_slots][kv_heads][2][sinks][dim]
};

// What a lane's row sees
struct RowView {
  int i, start, lo;                // sees lo .. i (its window) and the nsk rows from start
  unsigned nsk;
  bool valid;
};

__device__ inline SeqSpan load_span(const AttnK& A, int i) {
  const SeqSpan s = A.span[min(i, A.rows - 1)];
  return i < A.rows ? s : SeqSpan{SEQ_NO_ROW, 0};
}

__device__ inline RowView row_view(const AttnK& A, int i, const SeqSpan& sp) {
  RowView v;
  v.i = i;
  v.valid = sp.start != SEQ_NO_ROW;
  v.start = sp.start;
  v.lo = v.valid ? max(sp.start, i - A.window + 1) : SEQ_NO_ROW;
  v.nsk = v.valid ? (unsigned)min(A.sinks, i - sp.start + 1) : 0u;
  return v;
}

// Key tiles of a block of rows: `ts` tiles of the sinks before its range
// [lo, hi], then the range's.
struct KeyTiles {
  int s0, nsink, ts, lo, hi, n;
  // sa, sb: the spans of rows r0 + lane and r0 + 64 + lane
  template <int BK>
  __device__ inline void init(const AttnK& A, int r0, int nrows, const SeqSpan& sa, const SeqSpan& sb) {
    const int lane = threadIdx.x & 63;
    const uint64_t ma = __ballot(lane < nrows && sa.start != SEQ_NO_ROW);
    const uint64_t mb = __ballot(lane + 64 < nrows && sb.start != SEQ_NO_ROW);
    const int last = mb ? r0 + 127 - __builtin_clzll(mb) : ma ? r0 + 63 - __builtin_clzll(ma) : -1;
    hi = last;
    n = ts = nsink = s0 = lo = 0;
    if (last < 0) return;
    // the first row that belongs to a sequence is r0 unless the offsets are malformed
    s0 = __builtin_amdgcn_readfirstlane(sa.start);
    if (s0 == SEQ_NO_ROW) s0 = r0;
    lo = max(s0, r0 - A.window + 1);
    nsink = min(A.sinks, lo - s0);
    ts = (nsink + BK - 1) / BK;
    n = ts + (hi - lo + BK) / BK;
  }
  template <int BK>
  __device__ inline void at(int t, int& kt, int& nk) const {
    kt = t < ts ? s0 + t * BK : lo + (t - ts) * BK;
    nk = min(BK, (t < ts ? s0 + nsink : hi + 1) - kt);
  }
};

// Blocks are dealt to the XCDs round-robin; this renumbers them so that an XCD
// takes runs of 32 neighbours, whose key ranges overlap in its L2, and the runs
// are still dealt in turn, so that work that grows along a sequence is spread.
// 8192 histories of 20, forward / dQ / dK and dV: 75 / 87 / 85 -> 69 / 74 / 76 us.
// (One long run an XCD: 75 / 87 / 89.)
__device__ inline int xcd_runs(int b, int n) {
  constexpr int RUN = 32, G = NUM_XCD * RUN;
  if (b >= n / G * G) return b;
  const int c = b / G, y = b - c * G;
  return c * G + y % NUM_XCD * RUN + y / NUM_XCD;
}

// Block -> (row tile, key head, heads of the group).  Rows late in a long
// sequence may see more keys, so tiles go from the last to the first; where all
// blocks run at once (two a compute unit, block b beside b + 256), the second
// half goes from the first tile on, so that heavy and light ones share a unit.
// One history of 8192, all rows before each seen, 8 heads of 128: 252 us with
// tiles from first to last, 233 from last to first, 215 so.  (Measured there
// alone: narrower heads hold more than two, fp32 heads of 128 one.)
struct BlockAt { int tile, kv, h0; };
__device__ inline BlockAt block_at(const AttnK& A) {
  const int hg = A.group / A.hb, per = A.kv_heads * hg;
  const int b = xcd_runs(blockIdx.x, gridDim.x);
  BlockAt r;
  const int x = b % per;
  const int t = b / per, n = A.row_tiles, h = (n + 1) / 2;
  r.tile = n * per <= 512 && t >= h ? t - h : n - 1 - t;
  r.kv = x / hg;
  r.h0 = r.kv * A.group + (x % hg) * A.hb;
  return r;
}

// ---------------------------------------------------------------------------
template <typename T, int DP> struct AttnCfg {
  static constexpr int BK = sizeof(T) == 4 && DP == 128 ? 32 : 64;   // keys of a tile
  static constexpr int TB = BK * DP * (int)sizeof(T);                // bytes of K or V
  static constexpr size_t LDS = (size_t)2 * 2 * TB;                  // two stages of K and V
};

// The wave's direct loads have landed and its LDS reads returned; past the
// barrier everybody's have.
__device__ __forceinline__ void landed() {
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// The K and V tiles of a block's key range, each loaded beside the first product
// of the one before (see the head of this file).  A tile's key mask is one load
// made a tile ahead of the tile's own, whose row bits depend on it.
template <typename T, int DP>
struct KeyStream {
  using Cfg = AttnCfg<T, DP>;
  static constexpr int BK = Cfg::BK, TB = Cfg::TB;
  TileLoad<T, DP, BK, 4> lk, lv;
  const KeyTiles* kt;
  const T *k, *v;
  const uint8_t* mask;
  int64_t kld, vld;
  char* smem;
  int wave, mbyte;
  uint64_t bits;

  __device__ __forceinline__ void init(const AttnK& A, const KeyTiles* tiles, int kv, char* lds, int w) {
    kt = tiles;
    k = (const T*)A.k.p + (int64_t)kv * A.dim;
    v = (const T*)A.v.p + (int64_t)kv * A.dim;
    kld = A.k.ld;
    vld = A.v.ld;
    mask = A.mask;
    smem = lds;
    wave = w;
    lk.init(w, A.dim, kld);
    lv.init(w, A.dim, vld);
  }
  __device__ __forceinline__ void fetch_mask(int t) {
    if (!mask || t >= kt->n) return;
    int at, nk;
    kt->template at<BK>(t, at, nk);
    mbyte = mask[at + min((int)(threadIdx.x & 63), nk - 1)];
  }
  __device__ __forceinline__ void issue(int t) {
    if (t >= kt->n) return;
    int at, nk;
    kt->template at<BK>(t, at, nk);
    bits = nk >= 64 ? ~0ull : (1ull << nk) - 1;          // keys that exist and are shown
    if (mask) bits &= __ballot(mbyte != 0);
    char* S = smem + (t & 1) * 2 * TB;
    lk.issue(S, wave, k + (int64_t)at * kld, nk, bits);
    lv.issue(S + TB, wave, v + (int64_t)at * vld, nk, bits);
    fetch_mask(t + 1);
  }
  __device__ __forceinline__ void start() {
    fetch_mask(0);
    issue(0);
  }
  // Tile t, in LDS for every wave; the next one goes into the place of t - 1.
  __device__ __forceinline__ const char* next(int t, uint64_t& b) {
    landed();
    b = bits;
    issue(t + 1);
    return smem + (t & 1) * 2 * TB;
  }
};

// Scores of 32 keys (row0 in the tile) against the wave's 32 rows
template <typename T, int DP>
__device__ inline f32x16 scores(const char* S, uint32_t rl, int row0, const Frag<T>* q) {
  using TL = Tile<T, DP>;
  f32x16 c;
#pragma unroll
  for (int r = 0; r < 16; ++r) c[r] = 0.f;
#pragma unroll
  for (int s = 0; s < TL::KS; ++s) mma32(TL::rowfrag(S, rl, row0, s), q[s], c);
  return c;
}

// Scores of 32 rows (row0 of the tile at S) against 32 keys (key0 of the tile
// at SK), both in LDS
template <typename T, int DP>
__device__ inline f32x16 scores_lds(const char* S, uint32_t rl, int row0, const char* SK, int key0) {
  using TL = Tile<T, DP>;
  f32x16 c;
#pragma unroll
  for (int r = 0; r < 16; ++r) c[r] = 0.f;
#pragma unroll
  for (int s = 0; s < TL::KS; ++s) mma32(TL::rowfrag(S, rl, row0, s), TL::rowfrag(SK, rl, key0, s), c);
  return c;
}

__device__ inline int frag_off(int r) { return 8 * (r >> 2) + (r & 3); }   // + 4 (lane / 32)

// Bits lo .. hi of a word (none where they miss 0 .. 31)
__device__ inline uint32_t bit_range(int lo, int hi) {
  const uint32_t m = (0xffffffffu << (max(lo, 0) & 31)) & (0xffffffffu >> ((31 - min(hi, 31)) & 31));
  return lo > 31 || hi < 0 || lo > hi ? 0u : m;
}
// Which of the keys jb .. jb+31 the lane's row sees, shifted so that element r
// of a product is bit frag_off(r): one word per 32 keys, and two operations
// an element to apply it.
__device__ inline uint32_t row_bits(const RowView& v, int jb, uint32_t keys) {
  const uint32_t m = bit_range(v.lo - jb, v.i - jb) | bit_range(v.start - jb, v.start - jb + (int)v.nsk - 1);
  return v.valid ? (m & keys) >> (4 * ((threadIdx.x & 63) >> 5)) : 0u;
}
// all ones where bit frag_off(r) of a word is set, else zero
__device__ inline uint32_t bit_mask(uint32_t w, int r) { return (uint32_t)__builtin_amdgcn_sbfe((int)w, frag_off(r), 1); }
__device__ inline float keep_or(float x, uint32_t m, uint32_t other) {
  return __uint_as_float((__float_as_uint(x) & m) | (other & ~m));
}

// whether it may see one of the keys kt .. kt + nk - 1
__device__ inline bool reaches(const RowView& v, int kt, int nk) {
  return v.valid && ((kt <= v.i && v.lo < kt + nk) || (v.start < kt + nk && v.start + (int)v.nsk > kt));
}

// Elements that came out non-finite are made again from the pairs that do see
// each other: the sum over the finite values of the second operand, and what its
// non-finite ones bring.  A term of coefficient x and value +-inf is an infinity
// of their signs' product, any other (x = 0, NaN) is NaN; which they make is
// known from whether there are terms other than +inf, and other than -inf.  Both
// are sums of ones, products of the mask and of the operand's non-finite values:
// for x not negative those that are not the infinity in question, for x not
// positive those that are not the other.  Sweeps 0 to 3 count, sweep 4 adds values.
struct RepairPass {
  static constexpr int N = 5;
  uint32_t drop;                   // sweeps 0 to 3: the infinity that is not counted
  bool neg;                        // they take coefficients that are not positive
  __device__ inline explicit RepairPass(int i)
      : drop(i == 4 ? 0u : i == 0 || i == 3 ? 0x7f800000u : 0xff800000u), neg(i & 1) {}
  // element r's coefficient, x, in this sweep
  __device__ inline float coef(float x, uint32_t see, int r) const {
    return drop == 0 ? x : bit_mask(see, r) && (neg ? !(x > 0.f) : !(x < 0.f)) ? 1.f : 0.f;
  }
};
// What sweeps 0 and 1 (2 and 3) found: bit 16 db + r for accumulator [db][r]
template <int DB> struct RepairBits {
  uint64_t not_pos = 0, not_neg = 0;
  __device__ inline void note(int pass, const f32x16 (&x)[DB]) {
    uint64_t b = 0;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int r = 0; r < 16; ++r) b |= x[db][r] > 0.f ? 1ull << (16 * db + r) : 0ull;
    if (pass < 2) not_pos |= b; else if (pass < 4) not_neg |= b;
  }
  __device__ inline void add_to(f32x16 (&x)[DB]) const {
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const bool p = (not_pos >> (16 * db + r)) & 1, n = (not_neg >> (16 * db + r)) & 1;
        x[db][r] += p && n ? NAN : n ? INFINITY : p ? -INFINITY : 0.f;
      }
  }
};
// A sweep's step of 32 pairs a lane, coefficients x, second operand in LDS
template <typename T, int DP>
__device__ __forceinline__ void repair_step(const RepairPass& P, const char* S, uint32_t cl, int row0, uint32_t see,
                                            f32x16 x, f32x16 (&c)[Tile<T, DP>::DB]) {
#pragma unroll
  for (int r = 0; r < 16; ++r) x[r] = P.coef(x[r], see, r);
#pragma unroll
  for (int hf = 0; hf < 2; ++hf) {
    Frag<T> f;
    pack_frag(x, hf, f);
#pragma unroll
    for (int db = 0; db < Tile<T, DP>::DB; ++db)
      mma32(finite_or_count(Tile<T, DP>::colfrag(S, cl, row0 + 16 * hf, db), P.drop), f, c[db]);
  }
}

// The row of a lane and its fragments of q (or d_out, ...): loads that depend
// on nothing but the row's number, made before the tile's bounds are known.
template <typename T, int DP>
__device__ __forceinline__ void load_rows(const SeqTensor& t, int i, int head, int dim, Frag<T> (&f)[Tile<T, DP>::KS]) {
  const int half = (threadIdx.x & 63) >> 5;
  const T* p = (const T*)t.p + (int64_t)i * t.ld + head * dim;
#pragma unroll
  for (int s = 0; s < Tile<T, DP>::KS; ++s) {
    const int d = 16 * s + 8 * half;
    load_frag(p + (d < dim ? d : 0), d < dim, f[s]);
  }
}

// Elements of O^T-shaped accumulators (lane: one row, element r of block db is
// column 32 db + frag_off(r) + 4 (lane / 32)) to a row of memory.  PATCH: only
// elements that are not finite in memory.  lo: what the rounding to bf16
// took, rounded to bf16: the pair is off by 2^-16 of out.
template <typename T, int DP, bool PATCH>
__device__ __forceinline__ void store_row(T* op, T* lo, int dim, f32x16 (&x)[Tile<T, DP>::DB]) {
  const int half = (threadIdx.x & 63) >> 5;
#pragma unroll
  for (int db = 0; db < Tile<T, DP>::DB; ++db)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int d = 32 * db + 8 * g + 4 * half;
      if (32 * db + 8 * g >= dim) continue;
      float y[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        y[e] = x[db][4 * g + e];
        if (PATCH && nonfinite(ld(op + d + e))) {
          st(op + d + e, y[e]);
          if (sizeof(T) == 2 && lo) st(lo + d + e, y[e] - bf2f(f2bf(y[e])));
        }
      }
      if constexpr (PATCH) {
      } else if constexpr (sizeof(T) == 2) {
        *reinterpret_cast<u32x2*>(op + d) = u32x2{pack_bf2(y[0], y[1]), pack_bf2(y[2], y[3])};
        if (lo) {
#pragma unroll
          for (int e = 0; e < 4; ++e) y[e] -= bf2f(f2bf(y[e]));
          *reinterpret_cast<u32x2*>(lo + d) = u32x2{pack_bf2(y[0], y[1]), pack_bf2(y[2], y[3])};
        }
      } else {
        *reinterpret_cast<f32x4*>(op + d) = f32x4{y[0], y[1], y[2], y[3]};
      }
    }
}

template <typename T, int DP>
__global__ __launch_bounds__(256, sizeof(T) == 4 && DP == 128 ? 1 : 2) void seq_fwd_kernel(AttnK A) {
  using TL = Tile<T, DP>;
  constexpr int BK = AttnCfg<T, DP>::BK, TB = AttnCfg<T, DP>::TB;
  // Keys taken at a time: 32 with narrow heads, whose windows are short as a
  // rule, leaving out those that no row of the wave reaches (window 256, heads
  // of 64: 73 -> 63 us); a tile with wide ones, whose maximum, exchange and test
  // are then made once.
  constexpr bool SPLIT = DP <= 64;
  constexpr int N = SPLIT ? 1 : BK / 32;
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int half = lane >> 5;
  const BlockAt B = block_at(A);
  const int brows = 128 / A.hb, r0 = B.tile * brows;
  const int head = B.h0 + w % A.hb, row = r0 + (w / A.hb) * 32 + (lane & 31);
  // loads that wait for nothing: spans first, the bounds depend on them
  const SeqSpan sa = load_span(A, r0 + lane), sb = load_span(A, r0 + 64 + lane), sr = load_span(A, row);
  Frag<T> q[TL::KS];
  load_rows<T, DP>(A.q, min(row, A.rows - 1), head, A.dim, q);
  const RowView V = row_view(A, row, sr);
  KeyTiles kt_;
  kt_.init<BK>(A, r0, brows, sa, sb);
  if (kt_.n == 0) return;
  KeyStream<T, DP> ks;
  ks.init(A, &kt_, B.kv, smem, w);
  const uint32_t rl = TL::row_lane(), cl = TL::col_lane();
  const float c = A.scale * LOG2E;
  f32x16 o[TL::DB];
  float m, l;
  uint32_t seen;                     // not 0: the row sees a key (of the half's)

  // N subtiles of 32 keys from subtile b0 of the tile at kt
  auto attend = [&](int b0, const char* SK, const char* SV, int kt, uint64_t bits) __attribute__((always_inline)) {
    const uint32_t all = 0xffffffffu;
    const bool full = (uint32_t)(bits >> (32 * b0)) == all && (N == 1 || (uint32_t)(bits >> 32) == all) &&
                      wave_all(!V.valid || (V.lo <= kt + 32 * b0 && V.i >= kt + 32 * (b0 + N) - 1));
    f32x16 s[N];
#pragma unroll
    for (int b = 0; b < N; ++b) s[b] = scores<T, DP>(SK, rl, 32 * (b0 + b), q);
    uint32_t see[N];
    if (!full) {
#pragma unroll
      for (int b = 0; b < N; ++b) {
        see[b] = row_bits(V, kt + 32 * (b0 + b), (uint32_t)(bits >> (32 * (b0 + b))));
#pragma unroll
        for (int r = 0; r < 16; ++r) s[b][r] = keep_or(s[b][r], bit_mask(see[b], r), 0xff800000u);
        seen |= see[b];
      }
    } else {
      seen = 1;
    }
    float tm = s[0][0];
#pragma unroll
    for (int b = 0; b < N; ++b)
#pragma unroll
      for (int r = 0; r < 16; ++r) tm = fmaxf(tm, s[b][r]);
    tm = max32(tm);
    // The maximum moves only when it grew by more than 8 octaves: until
    // then probabilities are up to 2^8, exact in both types' ranges, and
    // the accumulators need no rescaling.
    const bool up = (tm - m) * c > 8.f;                       // also from -inf
    if (wave_any(up)) {
      const float mn = up ? tm : m;
      const float f = up ? __builtin_amdgcn_exp2f((m - mn) * c) : 1.f;
      l *= f;
#pragma unroll
      for (int db = 0; db < TL::DB; ++db)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[db][r] *= f;
      m = mn;
    }
    const float mc = m == -INFINITY ? 0.f : m * c;
    float ls[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int b = 0; b < N; ++b)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        s[b][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][r], c, -mc));
        ls[r & 3] += s[b][r];
      }
    l += (ls[0] + ls[1]) + (ls[2] + ls[3]);
#pragma unroll
    for (int b = 0; b < N; ++b)
#pragma unroll
      for (int hf = 0; hf < 2; ++hf) {
        Frag<T> p;
        pack_frag(s[b], hf, p);
#pragma unroll
        for (int db = 0; db < TL::DB; ++db) mma32(TL::colfrag(SV, cl, 32 * (b0 + b) + 16 * hf, db), p, o[db]);
      }
  };
  auto zero = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int db = 0; db < TL::DB; ++db)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[db][r] = 0.f;
  };
  auto scale = [&](float f) __attribute__((always_inline)) {
#pragma unroll
    for (int db = 0; db < TL::DB; ++db)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[db][r] *= f;
  };
  // one pass over the block's keys
  zero();
  m = -INFINITY;
  l = 0.f;
  seen = 0;
  ks.start();
#pragma unroll 1
  for (int t = 0; t < kt_.n; ++t) {
    uint64_t bits;
    const char *SK = ks.next(t, bits), *SV = SK + TB;
    int kt, nk;
    kt_.at<BK>(t, kt, nk);
    if constexpr (SPLIT) {
#pragma unroll 1
      for (int b = 0; b < BK / 32; ++b)
        if (nk > 32 * b && wave_any(reaches(V, kt + 32 * b, min(nk - 32 * b, 32)))) attend(b, SK, SV, kt, bits);
    } else {
      if (wave_any(reaches(V, kt, nk))) attend(0, SK, SV, kt, bits);
    }
  }
  l = add32(l);
  // nothing seen: zeros; keys seen, but with scores of -inf alone: 0 / 0
  const float any = max32(seen ? 1.f : 0.f);
  if (l == 0.f && any > 0.f) l = NAN;
  const float inv = l == 0.f ? 0.f : 1.f / l;
  scale(inv);

  T* const op = (T*)A.o.p + (int64_t)V.i * A.o.ld + head * A.dim;
  T* const lo = A.out_lo ? (T*)A.out_lo + ((int64_t)V.i * A.heads + head) * A.dim : nullptr;
  if (A.lse && V.valid && half == 0)
    A.lse[(int64_t)head * A.rows + V.i] = l == 0.f ? -INFINITY : (m * c + __builtin_amdgcn_logf(l)) * LN2;
  float z = 0.f;
#pragma unroll
  for (int db = 0; db < TL::DB; ++db)
#pragma unroll
    for (int r = 0; r < 16; ++r) z = __builtin_fmaf(o[db][r], 0.f, z);
  if (V.valid) store_row<T, DP, false>(op, lo, A.dim, o);
  if (__syncthreads_or(V.valid && z != 0.f)) {
    const float mc = m == -INFINITY ? 0.f : m * c;
    RepairBits<TL::DB> R;
#pragma unroll 1
    for (int pass = 0; pass < RepairPass::N; ++pass) {
      const RepairPass P(pass);
      zero();
      ks.start();
#pragma unroll 1
      for (int t = 0; t < kt_.n; ++t) {
        uint64_t bits;
        const char *SK = ks.next(t, bits), *SV = SK + TB;
        int kt, nk;
        kt_.at<BK>(t, kt, nk);
#pragma unroll 1
        for (int b = 0; b < BK / 32; ++b) {
          f32x16 p = scores<T, DP>(SK, rl, 32 * b, q);
          const uint32_t see = row_bits(V, kt + 32 * b, (uint32_t)(bits >> (32 * b)));
#pragma unroll
          for (int r = 0; r < 16; ++r)
            p[r] = keep_or(__builtin_amdgcn_exp2f(__builtin_fmaf(p[r], c, -mc)), bit_mask(see, r), 0u);
          repair_step<T, DP>(P, SV, cl, 32 * b, see, p, o);
        }
      }
      __syncthreads();                           // the last tile is read; the next pass loads the first
      R.note(pass, o);
    }
    scale(inv);
    R.add_to(o);
    if (V.valid) store_row<T, DP, true>(op, lo, A.dim, o);
  }
}

// ---------------------------------------------------------------------------
template <typename T, int DP>
__global__ __launch_bounds__(256, sizeof(T) == 4 && DP == 128 ? 1 : 2) void seq_dq_kernel(AttnK A) {
  using TL = Tile<T, DP>;
  constexpr int BK = AttnCfg<T, DP>::BK, TB = AttnCfg<T, DP>::TB;
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int half = lane >> 5;
  const BlockAt B = block_at(A);
  const int brows = 128 / A.hb, r0 = B.tile * brows;
  const int head = B.h0 + w % A.hb, row = r0 + (w / A.hb) * 32 + (lane & 31);
  // loads that wait for nothing: spans first, the bounds depend on them
  const SeqSpan sa = load_span(A, r0 + lane), sb = load_span(A, r0 + 64 + lane), sr = load_span(A, row);
  Frag<T> q[TL::KS], go[TL::KS];
  float delta = 0.f;
  {
    const int i = min(row, A.rows - 1);
    Frag<T> ov[TL::KS];
    load_rows<T, DP>(A.go, i, head, A.dim, go);
    load_rows<T, DP>(A.o, i, head, A.dim, ov);
    load_rows<T, DP>(A.q, i, head, A.dim, q);
#pragma unroll
    for (int s = 0; s < TL::KS; ++s) delta += dot_frag(go[s], ov[s]);
    if (A.out_lo) {
      load_rows<T, DP>(SeqTensor{A.out_lo, (int64_t)A.heads * A.dim}, i, head, A.dim, ov);
#pragma unroll
      for (int s = 0; s < TL::KS; ++s) delta += dot_frag(go[s], ov[s]);
    }
  }
  const RowView V = row_view(A, row, sr);
  KeyTiles kt_;
  kt_.init<BK>(A, r0, brows, sa, sb);
  if (kt_.n == 0) return;
  KeyStream<T, DP> ks;
  ks.init(A, &kt_, B.kv, smem, w);
  delta = add32(delta);
  float lse2 = INFINITY;
  if (V.valid) {
    const float x = A.lse[(int64_t)head * A.rows + V.i];
    lse2 = x == -INFINITY ? INFINITY : x * LOG2E;
    if (x == -INFINITY) delta = 0.f;
  }
  if (V.valid && half == 0) {
    A.lse2[(int64_t)head * A.rows + V.i] = lse2;
    A.delta[(int64_t)head * A.rows + V.i] = delta;
  }
  const uint32_t rl = TL::row_lane(), cl = TL::col_lane();
  const float c = A.scale * LOG2E;
  f32x16 dq[TL::DB];

  auto zero = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int db = 0; db < TL::DB; ++db)
#pragma unroll
      for (int r = 0; r < 16; ++r) dq[db][r] = 0.f;
  };
  auto scale = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int db = 0; db < TL::DB; ++db)
#pragma unroll
      for (int r = 0; r < 16; ++r) dq[db][r] *= A.scale;
  };
  // dS of the wave's rows and 32 keys of the tile
  auto dscores = [&](const char* SK, const char* SV, int b) __attribute__((always_inline)) {
    f32x16 p = scores<T, DP>(SK, rl, 32 * b, q);
    const f32x16 dp = scores<T, DP>(SV, rl, 32 * b, go);
#pragma unroll
    for (int r = 0; r < 16; ++r)
      p[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(p[r], c, -lse2)) * (dp[r] - delta);
    return p;
  };
  auto masked = [&](f32x16& p, uint32_t see) __attribute__((always_inline)) {
#pragma unroll
    for (int r = 0; r < 16; ++r) p[r] = keep_or(p[r], bit_mask(see, r), 0u);
  };
  zero();
  ks.start();
#pragma unroll 1
  for (int t = 0; t < kt_.n; ++t) {
    uint64_t bits;
    const char *SK = ks.next(t, bits), *SV = SK + TB;
    int kt, nk;
    kt_.at<BK>(t, kt, nk);
#pragma unroll
    for (int b = 0; b < BK / 32; ++b) {
      if (nk <= 32 * b || !wave_any(reaches(V, kt + 32 * b, min(32, nk - 32 * b)))) continue;
      const bool full = (uint32_t)(bits >> (32 * b)) == 0xffffffffu &&
                        wave_all(!V.valid || (V.lo <= kt + 32 * b && V.i >= kt + 32 * b + 31));
      f32x16 p = dscores(SK, SV, b);
      if (!full) masked(p, row_bits(V, kt + 32 * b, (uint32_t)(bits >> (32 * b))));
#pragma unroll
      for (int hf = 0; hf < 2; ++hf) {
        Frag<T> f;
        pack_frag(p, hf, f);
#pragma unroll
        for (int db = 0; db < TL::DB; ++db) mma32(TL::colfrag(SK, cl, 32 * b + 16 * hf, db), f, dq[db]);
      }
    }
  }
  scale();

  T* const op = (T*)A.gq.p + (int64_t)V.i * A.gq.ld + head * A.dim;
  float z = 0.f;
#pragma unroll
  for (int db = 0; db < TL::DB; ++db)
#pragma unroll
    for (int r = 0; r < 16; ++r) z = __builtin_fmaf(dq[db][r], 0.f, z);
  if (V.valid) store_row<T, DP, false>(op, nullptr, A.dim, dq);
  if (__syncthreads_or(V.valid && z != 0.f)) {
    RepairBits<TL::DB> R;
#pragma unroll 1
    for (int pass = 0; pass < RepairPass::N; ++pass) {
      const RepairPass P(pass);
      zero();
      ks.start();
#pragma unroll 1
      for (int t = 0; t < kt_.n; ++t) {
        uint64_t bits;
        const char *SK = ks.next(t, bits), *SV = SK + TB;
        int kt, nk;
        kt_.at<BK>(t, kt, nk);
#pragma unroll 1
        for (int b = 0; b < BK / 32; ++b) {
          f32x16 p = dscores(SK, SV, b);
          const uint32_t see = row_bits(V, kt + 32 * b, (uint32_t)(bits >> (32 * b)));
          masked(p, see);
          repair_step<T, DP>(P, SK, cl, 32 * b, see, p, dq);
        }
      }
      __syncthreads();
      R.note(pass, dq);
    }
    scale();
    R.add_to(dq);
    if (V.valid) store_row<T, DP, true>(op, nullptr, A.dim, dq);
  }
}

// ---------------------------------------------------------------------------
// Late rows of a sequence: those behind the window of every sink.
__device__ inline int late_row(const AttnK& A, int start) {
  return (int)min((int64_t)start + A.sinks + A.window - 1, (int64_t)SEQ_NO_ROW);
}
// Their partial sums are taken over pieces of this many of a sequence's n late
// rows: whole subtiles, at most 64 pieces, which one block adds up, none shorter
// than a tile.
__device__ inline int late_piece(const AttnK& A, int n) { return max(A.chunk, ((n + 2047) >> 11) << 5); }
// Where those of the piece that begins at a row lie.  A sequence with late rows
// has at least sinks + window rows, so start / (sinks + window) grows from one
// such sequence to the next, and the row's tile does not fall; within a sequence
// the tile grows.  So no two pieces share a slot.
__device__ inline int late_slot(const AttnK& A, int start, int row) {
  return start / (A.sinks + A.window) + row / A.chunk;
}

// One 32-row subtile against the wave's 32 keys: accumulates dv and dk from
// the scores p and the products ds of d_out and v.  SQ / SG: the rows' q and
// d_out in LDS (row0 the subtile's first row there), L / E: their lse2 and
// delta.  d: the subtile's first row minus the lane's key; rows with
// d + offset < lim see it.
template <typename T, int DP>
__device__ __forceinline__ void dkv_subtile(f32x16 p, f32x16 ds, const char* SQ, const char* SG, const float* L,
                                            const float* E, int row0, uint32_t cl, float c, int d,
                                            unsigned lim, bool full, f32x16 (&dk)[Tile<T, DP>::DB],
                                            f32x16 (&dv)[Tile<T, DP>::DB]) {
  using TL = Tile<T, DP>;
  const int half = (threadIdx.x & 63) >> 5;
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    const f32x4 l4 = *reinterpret_cast<const f32x4*>(L + row0 + 8 * g + 4 * half);
    const f32x4 e4 = *reinterpret_cast<const f32x4*>(E + row0 + 8 * g + 4 * half);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int r = 4 * g + e;
      p[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(p[r], c, -l4[e]));
      ds[r] = p[r] * (ds[r] - e4[e]);
    }
  }
  if (!full) {
    const uint32_t see = bit_range(-d, (int)lim - 1 - d) >> (4 * half);
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      p[r] = keep_or(p[r], bit_mask(see, r), 0u);
      ds[r] = keep_or(ds[r], bit_mask(see, r), 0u);
    }
  }
#pragma unroll
  for (int hf = 0; hf < 2; ++hf) {
    Frag<T> pf, df;
    pack_frag(p, hf, pf);
    pack_frag(ds, hf, df);
#pragma unroll
    for (int db = 0; db < TL::DB; ++db) {
      const Frag<T> g = TL::colfrag(SG, cl, row0 + 16 * hf, db), q = TL::colfrag(SQ, cl, row0 + 16 * hf, db);
      mma32(g, pf, dv[db]);
      mma32(q, df, dk[db]);
    }
  }
}

// `rows` values (zeros past them) straight to LDS, one per lane
__device__ inline void issue_stats(char* S, const float* p, int rows) {
  const int lane = threadIdx.x & 63;
  const __amdgpu_buffer_rsrc_t rs =
      __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(p), (short)0, (int)0x7fffffff, BUF_RSRC_WORD3);
  __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (seq_lds_void*)S, 4, (int)(lane < rows ? lane * 4u : 0x80000000u), 0,
                                           0, 0);
}

template <typename T, int DP> struct DkvCfg {
  static constexpr int BQ = sizeof(T) == 4 && DP == 128 ? 32 : 64;    // rows of a tile
  static constexpr int STAGE = 2 * BQ * DP * (int)sizeof(T) + 512;    // q, d_out, lse2, delta (64 floats each)
  // Wide bf16 heads: the accumulators of 32 keys are half of what two waves a
  // SIMD may hold, so k and v stay in LDS and a block has eight waves, two on
  // each 32 keys that take the two subtiles of a row tile; their sums are
  // added at the end.  One wave a SIMD left its matrix cores idle while it
  // made probabilities: 1460 -> 1206 us (65536 rows, 8 heads of 128,
  // window 2048).
  static constexpr bool WIDE = sizeof(T) == 2 && DP == 128;
  static constexpr int NW = WIDE ? 8 : 4;
  static constexpr int KV = WIDE ? 2 * 128 * DP * (int)sizeof(T) : 0;   // k and v of the block's keys
  static constexpr size_t LDS = (size_t)2 * STAGE + KV;
  // waves a SIMD: narrow heads wait for memory more than they compute
  static constexpr int WAVES = sizeof(T) == 2 ? (DP == 32 ? 3 : 2) : DP == 32 ? 2 : 1;
  static constexpr int SINK_STAGE = 2 * 32 * DP * (int)sizeof(T) + 512;   // a wave's 32 rows
  static constexpr size_t SINK_LDS = (size_t)4 * SINK_STAGE;
};

template <typename T, int DP>
__global__ __launch_bounds__((64 * DkvCfg<T, DP>::NW), (DkvCfg<T, DP>::WAVES)) void seq_dkv_kernel(AttnK A) {
  using TL = Tile<T, DP>;
  using Cfg = DkvCfg<T, DP>;
  constexpr int BQ = Cfg::BQ, TB = BQ * TL::RB, NW = Cfg::NW, KB = 64 * TL::RB;
  constexpr bool WIDE = Cfg::WIDE;
  constexpr int WAVES = NW / 4;                // of a key group
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int half = lane >> 5, kg = w & 3, rh = w >> 2;   // 32 keys; of a row tile, subtile (wide heads)
  const int bid = xcd_runs(blockIdx.x, gridDim.x);
  const int kv = bid % A.kv_heads, k0 = (bid / A.kv_heads) * 128;
  // a lane's key, and how many rows from it on see it here
  const int j = k0 + 32 * kg + (lane & 31);
  const SeqSpan sp = load_span(A, j);
  // keys of no sequence or hidden are read too: their columns see no row
  Frag<T> kf[TL::KS], vf[TL::KS];
  if constexpr (!WIDE) {
    load_rows<T, DP>(A.k, min(j, A.rows - 1), kv, A.dim, kf);
    load_rows<T, DP>(A.v, min(j, A.rows - 1), kv, A.dim, vf);
  }
  const bool valid = sp.start != SEQ_NO_ROW;
  const bool shown = valid && (!A.mask || A.mask[j]);
  const bool sink = valid && j - sp.start < A.sinks;
  int end = 0;
  if (valid) end = sink ? min(sp.end, late_row(A, sp.start)) : (int)min((int64_t)sp.end, (int64_t)j + A.window);
  const unsigned lim = shown ? (unsigned)(end - j) : 0u;
  // rows [k0, bend) of the block, [.., wend) of the wave
  int wend = end;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) wend = max(wend, __shfl_xor(wend, o, 64));
  wend = __builtin_amdgcn_readfirstlane(wend);
  __shared__ int ends[4];
  if (lane == 0 && rh == 0) ends[kg] = wend;
  __syncthreads();
  const int bend = max(max(ends[0], ends[1]), max(ends[2], ends[3]));
  if (bend <= k0) return;                      // no row of a sequence here
  const int per_head = (bend - k0 + BQ - 1) / BQ, n = per_head * A.group;

  TileLoad<T, DP, BQ, NW> lq, lg;
  lq.init(w, A.dim, A.q.ld);
  lg.init(w, A.dim, A.go.ld);
  char* const KV = smem + 2 * Cfg::STAGE;       // wide heads: k (two tiles of 64 rows), v
  if constexpr (WIDE) {
    TileLoad<T, DP, 64, NW> lk;
    lk.init(w, A.dim, A.k.ld);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int at = min(k0 + 64 * h, A.rows - 1), nr = min(64, A.rows - (k0 + 64 * h));
      lk.issue(KV + h * KB, w, (const T*)A.k.p + (int64_t)at * A.k.ld + kv * A.dim, nr, ~0ull);
    }
    lk.init(w, A.dim, A.v.ld);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int at = min(k0 + 64 * h, A.rows - 1), nr = min(64, A.rows - (k0 + 64 * h));
      lk.issue(KV + (2 + h) * KB, w, (const T*)A.v.p + (int64_t)at * A.v.ld + kv * A.dim, nr, ~0ull);
    }
  }
  auto issue = [&](int t) __attribute__((always_inline)) {
    if (t >= n) return;
    const int g = t / per_head, i0 = k0 + (t - g * per_head) * BQ, h = kv * A.group + g, nr = min(BQ, bend - i0);
    char* S = smem + (t & 1) * Cfg::STAGE;
    lq.issue(S, w, (const T*)A.q.p + (int64_t)i0 * A.q.ld + h * A.dim, nr, ~0ull);
    lg.issue(S + TB, w, (const T*)A.go.p + (int64_t)i0 * A.go.ld + h * A.dim, nr, ~0ull);
    const int64_t at = (int64_t)h * A.rows + i0;
    if (w == 0) issue_stats(S + 2 * TB, A.lse2 + at, nr);
    if (w == 1) issue_stats(S + 2 * TB + 256, A.delta + at, nr);
  };
  const uint32_t rl = TL::row_lane(), cl = TL::col_lane();
  const float c = A.scale * LOG2E;
  f32x16 dk[TL::DB], dv[TL::DB];
  auto zero = [&](f32x16 (&x)[TL::DB]) __attribute__((always_inline)) {
#pragma unroll
    for (int db = 0; db < TL::DB; ++db)
#pragma unroll
      for (int r = 0; r < 16; ++r) x[db][r] = 0.f;
  };
  // f(stage, subtile of it, the subtile's first row) for those that reach the wave's keys
  auto rows = [&](auto f) __attribute__((always_inline)) {
    issue(0);
    int i0 = k0;
#pragma unroll 1
    for (int t = 0; t < n; ++t) {
      landed();
      issue(t + 1);
      const char* S = smem + (t & 1) * Cfg::STAGE;
      auto reached = [&](int b) __attribute__((always_inline)) {
        const int ib = i0 + 32 * b;
        if (ib + 31 >= k0 + 32 * kg && ib < wend) f(S, b, ib);
      };
      if constexpr (WIDE) {
        reached(rh);
      } else {
#pragma unroll
        for (int b = 0; b < BQ / 32; ++b) reached(b);
      }
      i0 = i0 + BQ >= bend ? k0 : i0 + BQ;
    }
  };
  // scores of the wave's keys (what 0) or their products with d_out (1)
  auto products = [&](const char* S, int b, int what) __attribute__((always_inline)) {
    if constexpr (WIDE)
      return scores_lds<T, DP>(S + what * TB, rl, 32 * b, KV + (kg >> 1) * KB + what * 2 * KB, 32 * (kg & 1));
    else
      return scores<T, DP>(S + what * TB, rl, 32 * b, what ? vf : kf);
  };
  // the sum of the two waves of a key group, by registers
  auto both_waves = [&](f32x16 (&x)[TL::DB]) __attribute__((always_inline)) {
    if constexpr (WIDE) {
      float* R = reinterpret_cast<float*>(smem) + kg * TL::DB * 16 * 64 + lane;
      __syncthreads();
      if (rh == 1)
#pragma unroll
        for (int i = 0; i < TL::DB * 16; ++i) R[i * 64] = x[i >> 4][i & 15];
      __syncthreads();
      if (rh == 0)
#pragma unroll
        for (int i = 0; i < TL::DB * 16; ++i) x[i >> 4][i & 15] += R[i * 64];
    }
  };
  // f(partial sums of the lane's key) for the pieces of its late rows, in their order,
  // the two waves of a key group in turn (a hidden sink has no gradient; its sums are zeros times what may not be finite)
  auto late_sums = [&](auto f) __attribute__((always_inline)) {
    if (A.chunk > 0 && sink && lim > 0 && sp.end > late_row(A, sp.start)) {
      const int l0 = late_row(A, sp.start), piece = late_piece(A, sp.end - l0);
#pragma unroll 1
      for (int i = l0 + rh * piece; i < sp.end; i += WAVES * piece)
        f(A.part + ((int64_t)late_slot(A, sp.start, i) * A.kv_heads * 2 * A.sinks +
                    (kv * 2 * A.sinks + j - sp.start)) * A.dim);
    }
  };
  // f(accumulator block, first of four elements, columns there) for the columns of dim
  auto columns = [&](auto f) __attribute__((always_inline)) {
#pragma unroll
    for (int db = 0; db < TL::DB; ++db)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        // those past dim, which are not stored, take others' sums: no branch between
        // the loads, so that they go out together; wide heads have no registers for that
        const int dd = 32 * db + 8 * g + 4 * half;
        if (DP < 128 || 32 * db + 8 * g < A.dim) f(db, 4 * g, dd < A.dim ? dd : 0);
      }
  };
  auto add4 = [&](f32x16& x, int r, const float* P) __attribute__((always_inline)) {
    const f32x4 a = *reinterpret_cast<const f32x4*>(P);
#pragma unroll
    for (int e = 0; e < 4; ++e) x[r + e] += a[e];
  };
  auto scale = [&](f32x16 (&x)[TL::DB]) __attribute__((always_inline)) {
#pragma unroll
    for (int db = 0; db < TL::DB; ++db)
#pragma unroll
      for (int r = 0; r < 16; ++r) x[db][r] *= A.scale;
  };

  zero(dk);
  zero(dv);
  rows([&](const char* S, int b, int ib) __attribute__((always_inline)) {
    const bool full = wave_all((unsigned)(ib - j) < lim && (unsigned)(ib + 31 - j) < lim);
    dkv_subtile<T, DP>(products(S, b, 0), products(S, b, 1), S, S + TB, (const float*)(S + 2 * TB),
                       (const float*)(S + 2 * TB + 256), 32 * b, cl, c, ib - j, lim, full, dk, dv);
  });
  late_sums([&](const float* P) __attribute__((always_inline)) {
    columns([&](int db, int r, int d) __attribute__((always_inline)) {
      add4(dk[db], r, P + d);
      add4(dv[db], r, P + (int64_t)A.sinks * A.dim + d);
    });
  });
  both_waves(dk);
  both_waves(dv);
  scale(dk);
  T* const kp = (T*)A.gk.p + (int64_t)j * A.gk.ld + kv * A.dim;
  T* const vp = (T*)A.gv.p + (int64_t)j * A.gv.ld + kv * A.dim;
  const bool mine = valid && rh == 0;            // the wave that stores
  float z = 0.f;
#pragma unroll
  for (int db = 0; db < TL::DB; ++db)
#pragma unroll
    for (int r = 0; r < 16; ++r) z = __builtin_fmaf(dk[db][r], 0.f, __builtin_fmaf(dv[db][r], 0.f, z));
  if (mine) {
    store_row<T, DP, false>(kp, nullptr, A.dim, dk);
    store_row<T, DP, false>(vp, nullptr, A.dim, dv);
  }
  if (!__syncthreads_or(mine && z != 0.f)) return;
  // dv, then dk, in dk's registers
#pragma unroll 1
  for (int what = 0; what < 2; ++what) {
    RepairBits<TL::DB> R;
#pragma unroll 1
    for (int pass = 0; pass < RepairPass::N; ++pass) {
      zero(dk);
      rows([&](const char* S, int b, int ib) __attribute__((always_inline)) {
        f32x16 p = products(S, b, 0);
        const float *L = (const float*)(S + 2 * TB) + 32 * b + 4 * half, *E = L + 64;
#pragma unroll
        for (int r = 0; r < 16; ++r) p[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(p[r], c, -L[frag_off(r)]));
        if (what) {
          const f32x16 d = products(S, b, 1);
#pragma unroll
          for (int r = 0; r < 16; ++r) p[r] *= d[r] - E[frag_off(r)];
        }
        const uint32_t see = bit_range(j - ib, (int)lim - 1 + j - ib) >> (4 * half);
#pragma unroll
        for (int r = 0; r < 16; ++r) p[r] = keep_or(p[r], bit_mask(see, r), 0u);
        repair_step<T, DP>(RepairPass(pass), what ? S : S + TB, cl, 32 * b, see, p, dk);
      });
      if (pass == RepairPass::N - 1)
        late_sums([&](const float* P) __attribute__((always_inline)) {
          columns([&](int db, int r, int d) __attribute__((always_inline)) {
            add4(dk[db], r, P + (what ? 0 : (int64_t)A.sinks * A.dim) + d);
          });
        });
      both_waves(dk);
      __syncthreads();                           // the next sweep loads over what this one read
      R.note(pass, dk);
    }
    if (what) scale(dk);
    R.add_to(dk);
    if (mine) store_row<T, DP, true>(what ? kp : vp, nullptr, A.dim, dk);
  }
}

// Partial dk and dv of a sequence's sinks over a piece of its late rows, every
// one of which sees every sink.  A block: 32 sinks of one key head, and the
// pieces that begin in a tile of rows; its waves take every fourth subtile of
// rows, their sums are added in wave order.  Tiles lie on the packed rows and a
// sequence has pieces by its own length, so the work is even whatever else is
// in the batch: one history of 32000 events among 3000 of 20, 8 heads of 64 over 2,
// window 256: 40 us here and 134 in the dK/dV kernel, which adds up 64 pieces in
// one block (1510 and 126 with one piece).
template <typename T, int DP>
__global__ __launch_bounds__(256, 1) void seq_sink_kernel(AttnK A, int parts) {
  using TL = Tile<T, DP>;
  using Cfg = DkvCfg<T, DP>;
  constexpr int TB = 32 * TL::RB, SCAN = 4;
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int half = lane >> 5;
  int b = blockIdx.x;
  const int part = b % parts; b /= parts;
  const int kv = b % A.kv_heads;
  const int x0 = b / A.kv_heads * A.chunk, x1 = min(x0 + A.chunk, A.rows);
  // of the rows xb + lane + 64 e: those that begin a piece
  auto pieces = [&](int xb) __attribute__((always_inline)) {
    unsigned heads = 0;
    SeqSpan sp[SCAN];                          // all loads before the first branch
#pragma unroll
    for (int e = 0; e < SCAN; ++e) sp[e] = A.span[min(xb + lane + 64 * e, x1 - 1)];
#pragma unroll
    for (int e = 0; e < SCAN; ++e) {
      const int i = xb + lane + 64 * e, l0 = late_row(A, sp[e].start), n = sp[e].end - l0;
      bool head = i == l0;
      const bool more = i > l0 && n > A.chunk;                  // may begin a later piece
      if (wave_any(more)) head |= more && (i - l0) % late_piece(A, n) == 0;
      if (head && i < x1 && n > 0) heads |= 1u << e;
    }
    return heads;
  };
  // most tiles of short sequences have none: they end before anything else is set up
  int xb = x0;
  unsigned heads = pieces(xb);
  while (!wave_any(heads != 0)) {
    if ((xb += 64 * SCAN) >= x1) return;
    heads = pieces(xb);
  }
#pragma unroll 1
  for (;;) {
    for (uint64_t found; (found = __ballot(heads != 0)) != 0;) {
      const int from = __builtin_ctzll(found), bits = __builtin_amdgcn_readlane((int)heads, from);
      if (lane == from) heads &= heads - 1;
      const int a0 = xb + from + 64 * __builtin_ctz(bits);
      const SeqSpan sp = A.span[a0];
      const int s0 = __builtin_amdgcn_readfirstlane(sp.start), end = __builtin_amdgcn_readfirstlane(sp.end);
      const int a1 = min(end, a0 + late_piece(A, end - late_row(A, s0)));   // the piece: rows a0 .. a1 - 1
      const int a = part * 32 + (lane & 31), j = s0 + a;   // late rows exist: the sequence has all its sinks
      const bool shown = a < A.sinks && (!A.mask || A.mask[j]);
      const int per_head = (a1 - a0 + 31) / 32, n = per_head * A.group;

      TileLoad<T, DP, 32, 1> lq, lg;
      lq.init(0, A.dim, A.q.ld);
      lg.init(0, A.dim, A.go.ld);
      char* S = smem + w * Cfg::SINK_STAGE;
      Frag<T> kf[TL::KS], vf[TL::KS];
      load_rows<T, DP>(A.k, a < A.sinks ? j : s0, kv, A.dim, kf);
      load_rows<T, DP>(A.v, a < A.sinks ? j : s0, kv, A.dim, vf);
      const uint32_t rl = TL::row_lane(), cl = TL::col_lane();
      const float c = A.scale * LOG2E;
      f32x16 dk[TL::DB], dv[TL::DB];
#pragma unroll
      for (int db = 0; db < TL::DB; ++db)
#pragma unroll
        for (int r = 0; r < 16; ++r) dk[db][r] = dv[db][r] = 0.f;
#pragma unroll 1
      for (int t = w; t < n; t += 4) {
        const int g = t / per_head, i0 = a0 + (t - g * per_head) * 32, h = kv * A.group + g, nr = min(32, a1 - i0);
        const int64_t at = (int64_t)h * A.rows + i0;
        // the wave's own stage: its reads of the subtile before have returned
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        lq.issue(S, 0, (const T*)A.q.p + (int64_t)i0 * A.q.ld + h * A.dim, nr, ~0ull);
        lg.issue(S + TB, 0, (const T*)A.go.p + (int64_t)i0 * A.go.ld + h * A.dim, nr, ~0ull);
        issue_stats(S + 2 * TB, A.lse2 + at, nr);
        issue_stats(S + 2 * TB + 256, A.delta + at, nr);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        dkv_subtile<T, DP>(scores<T, DP>(S, rl, 0, kf), scores<T, DP>(S + TB, rl, 0, vf), S, S + TB,
                                  (const float*)(S + 2 * TB), (const float*)(S + 2 * TB + 256), 0, cl, c, 0,
                                  shown ? (unsigned)nr : 0u, nr == 32 && wave_all(shown), dk, dv);
      }
      // waves' sums, one after the other, in LDS [2][DP][33]
      float* R = reinterpret_cast<float*>(smem);
      for (int v = 0; v < 4; ++v) {
        __syncthreads();
        if (w != v) continue;
#pragma unroll
        for (int db = 0; db < TL::DB; ++db)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int d = 32 * db + frag_off(r) + 4 * half, x = d * 33 + (lane & 31);
            R[x] = dk[db][r] + (v ? R[x] : 0.f);
            R[DP * 33 + x] = dv[db][r] + (v ? R[DP * 33 + x] : 0.f);
          }
      }
      __syncthreads();
      float* P = A.part + ((int64_t)late_slot(A, s0, a0) * A.kv_heads + kv) * 2 * A.sinks * A.dim;
      const int na = min(32, A.sinks - part * 32);
      for (int x = threadIdx.x; x < 2 * na * A.dim; x += 256) {
        const int m = x / (na * A.dim), y = x - m * na * A.dim, r = y / A.dim, d = y - r * A.dim;
        P[((int64_t)m * A.sinks + part * 32 + r) * A.dim + d] = R[m * DP * 33 + d * 33 + r];
      }
      __syncthreads();                           // R is read; the stages may be loaded again
    }
    if ((xb += 64 * SCAN) >= x1) break;
    heads = pieces(xb);
  }
}

// ---------------------------------------------------------------------------
static AttnK attn_args(const SeqAttnArgs& a) {
  AttnK A{};
  A.rows = (int)a.rows;
  A.dim = a.dim;
  A.heads = a.heads;
  A.kv_heads = a.kv_heads;
  A.group = a.heads / a.kv_heads;
  A.window = a.window < a.rows ? a.window : (int)a.rows;
  A.sinks = a.sinks;
  A.hb = A.group % 4 == 0 ? 4 : A.group % 2 == 0 ? 2 : 1;
  A.row_tiles = cdiv(a.rows, 128 / A.hb);
  A.scale = a.scale;
  A.span = a.span;
  A.mask = a.key_mask;
  A.q = a.q; A.k = a.k; A.v = a.v; A.o = a.o; A.go = a.go; A.gq = a.gq; A.gk = a.gk; A.gv = a.gv;
  A.lse = a.lse;
  A.out_lo = a.dt == DT_BF16 ? a.out_lo : nullptr;
  return A;
}

// Rows of a tile of seq_sink_kernel: 128, more where that would be more than 4096
// blocks, which fill the chip several times and bound the workspace.  0 where no
// sequence has late rows.
static int late_chunk(const SeqAttnArgs& a) {
  if (a.sinks == 0 || a.num_seqs == 0 || a.max_len < (int64_t)a.sinks + a.window) return 0;
  const int64_t n = std::max<int64_t>(128, (a.rows * a.kv_heads + 4095) / 4096);
  return (int)((n + 31) / 32 * 32);
}

// Slots that late_slot() counts.
static int64_t late_slots(const SeqAttnArgs& a, int chunk) {
  return chunk == 0 ? 0 : a.rows / ((int64_t)a.sinks + a.window) + cdiv(a.rows, chunk);
}

static size_t stats_bytes(const SeqAttnArgs& a) {
  return ((size_t)a.heads * a.rows * sizeof(float) + 255) & ~(size_t)255;
}

size_t seq_attn_bwd_workspace(const SeqAttnArgs& a) {
  return 2 * stats_bytes(a) + (size_t)late_slots(a, late_chunk(a)) * a.kv_heads * 2 * a.sinks * a.dim * sizeof(float);
}

template <typename T, int DP>
static hipError_t fwd_launch(const AttnK& A, hipStream_t s) {
  static LdsLimit lim;
  LAT_HIP_CHECK(lds_limit(seq_fwd_kernel<T, DP>, AttnCfg<T, DP>::LDS, lim));
  seq_fwd_kernel<T, DP><<<A.row_tiles * (A.heads / A.hb), 256, AttnCfg<T, DP>::LDS, s>>>(A);
  LAT_LAUNCH_CHECK();
  return hipSuccess;
}

template <typename T, int DP>
static hipError_t bwd_launch(const AttnK& A, hipStream_t s) {
  static LdsLimit l0, l1, l2;
  LAT_HIP_CHECK(lds_limit(seq_dq_kernel<T, DP>, AttnCfg<T, DP>::LDS, l0));
  LAT_HIP_CHECK(lds_limit(seq_dkv_kernel<T, DP>, DkvCfg<T, DP>::LDS, l1));
  LAT_HIP_CHECK(lds_limit(seq_sink_kernel<T, DP>, DkvCfg<T, DP>::SINK_LDS, l2));
  // dQ also writes the rows' statistics that the other two read
  seq_dq_kernel<T, DP><<<A.row_tiles * (A.heads / A.hb), 256, AttnCfg<T, DP>::LDS, s>>>(A);
  LAT_LAUNCH_CHECK();
  if (A.chunk > 0) {
    const int parts = (A.sinks + 31) / 32;
    seq_sink_kernel<T, DP><<<cdiv(A.rows, A.chunk) * A.kv_heads * parts, 256, DkvCfg<T, DP>::SINK_LDS, s>>>(A, parts);
    LAT_LAUNCH_CHECK();
  }
  seq_dkv_kernel<T, DP><<<cdiv(A.rows, 128) * A.kv_heads, 64 * DkvCfg<T, DP>::NW, DkvCfg<T, DP>::LDS, s>>>(A);
  LAT_LAUNCH_CHECK();
  return hipSuccess;
}

hipError_t seq_attn_fwd(const SeqAttnArgs& a, hipStream_t s) {
  if (a.rows == 0 || a.num_seqs == 0) return hipSuccess;
  const AttnK A = attn_args(a);
  if (a.dt == DT_BF16)
    return a.dim <= 32 ? fwd_launch<bf16_t, 32>(A, s) : a.dim <= 64 ? fwd_launch<bf16_t, 64>(A, s)
                                                                  : fwd_launch<bf16_t, 128>(A, s);
  return a.dim <= 32 ? fwd_launch<float, 32>(A, s) : a.dim <= 64 ? fwd_launch<float, 64>(A, s)
                                                               : fwd_launch<float, 128>(A, s);
}

hipError_t seq_attn_bwd(const SeqAttnArgs& a, void* ws, hipStream_t s) {
  if (a.rows == 0 || a.num_seqs == 0) return hipSuccess;
  AttnK A = attn_args(a);
  const size_t stats = stats_bytes(a);
  A.lse2 = (float*)ws;
  A.delta = (float*)((char*)ws + stats);
  A.part = (float*)((char*)ws + 2 * stats);
  A.chunk = late_chunk(a);
  if (a.dt == DT_BF16)
    return a.dim <= 32 ? bwd_launch<bf16_t, 32>(A, s) : a.dim <= 64 ? bwd_launch<bf16_t, 64>(A, s)
                                                                  : bwd_launch<bf16_t, 128>(A, s);
  return a.dim <= 32 ? bwd_launch<float, 32>(A, s) : a.dim <= 64 ? bwd_launch<float, 64>(A, s)
                                                               : bwd_launch<float, 128>(A, s);
}

}  // namespace lat
