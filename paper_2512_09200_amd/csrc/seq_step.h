// What the single-event steps over bf16 / fp32 and over 8-bit caches share: the
// split of a user's slots over blocks and the join of the splits.
#pragma once
#include "kernels.h"
#include "seq_tile.h"

namespace lat {

constexpr float STEP_LOG2E = 1.4426950408889634f;
constexpr int STEP_HEADS = 16;               // head columns of a block
constexpr int STEP_MAX_SPLITS = 512;         // of a user's slots: places of the join's LDS

__device__ inline void mma16(const Frag<bf16_t>& a, const Frag<bf16_t>& b, f32x4& c) {
  c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.v, b.v, c, 0, 0, 0);
}
template <typename F>
__device__ inline F wave_sum(F v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}

struct StepJoin {
  const int32_t *lens, *index;
  int num_caches, heads, dim, ns;
  float scale;
  const float* part;                         // [batch][heads][ns][dim + 2]: o, m, l
  SeqTensor out;
};

// out of a user's head from its splits.  A block a head: the splits' weights
// go to LDS, then 256 / DP strands of threads add every so many splits, and
// the strands' sums are added in strand order.
template <typename T, int DP>
__global__ __launch_bounds__(256) void seq_step_join_kernel(StepJoin A) {
  constexpr int ST = 256 / DP;
  __shared__ float wt[STEP_MAX_SPLITS], sum[256], red[8];
  const int bh = blockIdx.x, b = bh / A.heads, h = bh - b * A.heads, tid = threadIdx.x, D = A.dim;
  const int p = A.lens[b], ci = A.index ? A.index[b] : b;
  if (p < 0 || ci < 0 || ci >= A.num_caches) return;
  const float c = A.scale * STEP_LOG2E;
  const float* P = A.part + (int64_t)bh * A.ns * (D + 2);
  float M = -INFINITY, L = 0.f, O = 0.f;
  for (int u = tid; u < A.ns; u += 256) M = fmaxf(M, P[u * (D + 2) + D]);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor(M, o, 64));
  if ((tid & 63) == 0) red[tid >> 6] = M;
  __syncthreads();
  M = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
  for (int u = tid; u < A.ns; u += 256) {
    const float m = P[u * (D + 2) + D], f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m - M) * c);
    wt[u] = f;
    L += P[u * (D + 2) + D + 1] * f;
  }
  L = wave_sum(L);
  if ((tid & 63) == 0) red[4 + (tid >> 6)] = L;
  __syncthreads();
  L = (red[4] + red[5]) + (red[6] + red[7]);
  const int d = tid % DP, strand = tid / DP;
  if (d < D) {
#pragma unroll 8
    for (int u = strand; u < A.ns; u += ST) O += wt[u] * P[u * (D + 2) + d];
  }
  sum[tid] = O;
  __syncthreads();
  if (strand == 0 && d < D) {
#pragma unroll
    for (int i = 1; i < ST; ++i) O += sum[i * DP + d];
    st((T*)A.out.p + (int64_t)b * A.out.ld + h * D + d, O / L);
  }
}

// Splits of the slots: enough blocks for the two a compute unit holds, at
// least 256 slots (two rounds of a block's waves) each.  Three users, 65536 slots
// of 128, 2 key heads: 47 us and 6 for the join with 512 splits in all, 48 and 8.5
// with 1024, 47 and 5.5 with 256; unsplit the six blocks would take milliseconds.
inline int step_splits(int batch, int heads, int kv_heads, int cap) {
  const int hg = cdiv(heads / kv_heads, STEP_HEADS);
  const int64_t blocks = (int64_t)batch * kv_heads * hg;
  int64_t n = cdiv(STEP_MAX_SPLITS, blocks);
  if (n > cdiv(cap, 256)) n = cdiv(cap, 256);
  return (int)n;
}

}  // namespace lat
