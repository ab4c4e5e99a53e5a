// Internal interface of the event-sequence operators (namespace lat): plan,
// per-head norm with rotary positions, windowed attention, ring-cache fill
// and the single-event step.  Launchers enqueue on the given stream and return
// the first HIP error.
#pragma once
#include "common.h"

namespace lat {

// A row's sequence: first row and end row (seq_plan).  Rows of no sequence:
// start SEQ_NO_ROW, end 0.
struct SeqSpan { int start, end; };
constexpr int SEQ_NO_ROW = 0x7fffffff;

// [rows, heads, dim] with a row stride in elements
struct SeqTensor {
  void* p = nullptr;
  int64_t ld = 0;
};

hipError_t seq_plan(const int32_t* offsets, int num_seqs, int64_t rows, SeqSpan* span, hipStream_t s);

constexpr int ROPE_MAX_PAIRS = 64;
// Rotation per position of every pair, in turns (angle / 2 pi).
struct RopeTurns { double f[ROPE_MAX_PAIRS]; };
struct RopeArgs {
  DType dt = DT_BF16;
  int64_t rows = 0;
  const SeqSpan* span = nullptr;       // null: every row is taken
  const int32_t* positions = nullptr;  // null: index in the sequence
  int heads = 0, kv_heads = 0, dim = 0, rotary = 0, interleaved = 0;
  float eps = 0.f;
  const float *gain_q = nullptr, *gain_k = nullptr;
  SeqTensor q, k;                      // inputs
  SeqTensor gq, gk;                    // backward: gradients of the outputs
  SeqTensor oq, ok;                    // forward: outputs; backward: dq, dk
  float *dgain_q = nullptr, *dgain_k = nullptr;
};
void rope_turns(double theta, int rotary, RopeTurns* t);
hipError_t rope_fwd(const RopeArgs& a, const RopeTurns& t, hipStream_t s);
size_t rope_bwd_workspace(int64_t rows, int dim);
hipError_t rope_bwd(const RopeArgs& a, const RopeTurns& t, void* ws, hipStream_t s);

struct SeqAttnArgs {
  DType dt = DT_BF16;
  int64_t rows = 0;
  int num_seqs = 0;
  int64_t max_len = 0;                 // 1 .. rows
  const SeqSpan* span = nullptr;
  const uint8_t* key_mask = nullptr;
  int heads = 0, kv_heads = 0, dim = 0, window = 0, sinks = 0;
  float scale = 0.f;
  SeqTensor q, k, v, o;
  float* lse = nullptr;                // [heads, rows]
  void* out_lo = nullptr;              // [rows, heads, dim], bf16 only
  SeqTensor go, gq, gk, gv;            // backward
};
hipError_t seq_attn_fwd(const SeqAttnArgs& a, hipStream_t s);
size_t seq_attn_bwd_workspace(const SeqAttnArgs& a);
hipError_t seq_attn_bwd(const SeqAttnArgs& a, void* ws, hipStream_t s);

struct SeqCacheArgs {
  DType dt = DT_BF16;
  int kv_heads = 0, dim = 0, window = 0, sinks = 0;
  void *kc = nullptr, *vc = nullptr;
  int num_caches = 0;
  const int32_t* index = nullptr;      // null: the entry's own number
};
hipError_t seq_cache_fill(const SeqCacheArgs& c, int64_t rows, const int32_t* offsets, int num_seqs,
                          const int32_t* first, SeqTensor k, SeqTensor v, hipStream_t s);

struct SeqStepArgs {
  SeqCacheArgs c;
  int batch = 0, heads = 0;
  float scale = 0.f;
  SeqTensor q, k, v, out;
  const int32_t* lens = nullptr;
  int rope = 0;                        // 0: q and k are taken as they are
  int rotary = 0, interleaved = 0;
  float eps = 0.f;
  const float *gain_q = nullptr, *gain_k = nullptr;
  const int32_t* positions = nullptr;  // null: lens
};
size_t seq_step_workspace(int batch, int heads, int kv_heads, int dim, int cap);
hipError_t seq_step(const SeqStepArgs& a, const RopeTurns& t, void* ws, hipStream_t s);

// Slot of position p in a ring of sinks + window slots.
__host__ __device__ inline int seq_slot(int p, int sinks, int window) {
  return p < sinks ? p : sinks + (p - sinks) % window;
}

}  // namespace lat
