// C ABI of the event-sequence operators: argument checks and entry points.
#include "abi_check.h"
#include "seq.h"

#include <cmath>

using namespace lat;

// Strides reach over a tile's 64 rows in 32 bits of bytes; rows, windows and
// slots stay apart from the ends of int32.
static const int64_t MAX_STRIDE = 1 << 22, MAX_ROWS = (int64_t)1 << 30;
// blocks of 256 threads whose global thread number fits 32 bits
static const int64_t MAX_BLOCKS = ((int64_t)1 << 24) - 1;

static lattice_status check_seqs(const lattice_seqs* s) {
  REQUIRE(s, "null seqs");
  REQUIRE(s->rows >= 0 && s->num_seqs >= 0 && s->max_len >= 0, "negative sizes");
  if (s->rows >= MAX_ROWS) FAIL(LATTICE_ERR_UNSUPPORTED, "rows must be < 2^30");
  return LATTICE_OK;
}

static lattice_status check_heads(lattice_dtype dt, int heads, int kv_heads, int dim) {
  REQUIRE(dt == LATTICE_F32 || dt == LATTICE_BF16, "bad dtype");
  REQUIRE(heads >= 1 && heads <= 1024 && kv_heads >= 1 && kv_heads <= 1024, "heads outside 1..1024");
  if (dim <= 0 || dim > 128 || dim % 8) FAIL(LATTICE_ERR_UNSUPPORTED, "head_dim %d is no multiple of 8 in 8..128", dim);
  return LATTICE_OK;
}

static lattice_status check_tensor(const char* name, const void* p, int64_t stride, int heads, int dim) {
  REQUIRE(p, "null %s", name);
  REQUIRE((uintptr_t)p % 16 == 0, "%s is not 16-byte aligned", name);
  REQUIRE(stride >= (int64_t)heads * dim && stride % 8 == 0, "%s: row stride %lld is no multiple of 8 that holds a row",
          name, (long long)stride);
  REQUIRE(stride <= MAX_STRIDE, "%s: row stride above 2^22", name);
  return LATTICE_OK;
}

#define TRY(expr)                          \
  do {                                     \
    lattice_status st__ = (expr);          \
    if (st__ != LATTICE_OK) return st__;   \
  } while (0)

static lattice_status check_rope(const lattice_qk_rope_desc* d) {
  REQUIRE(d, "null rope descriptor");
  TRY(check_heads(d->dtype, d->heads, d->kv_heads, d->head_dim));
  if (d->rotary_dim < 0 || d->rotary_dim > d->head_dim || d->rotary_dim % 8)
    FAIL(LATTICE_ERR_UNSUPPORTED, "rotary_dim %d is no multiple of 8 in 0..head_dim", d->rotary_dim);
  REQUIRE(d->theta > 0 && std::isfinite(d->theta), "theta must be positive");
  REQUIRE(d->eps >= 0 && std::isfinite(d->eps), "eps must not be negative");
  return LATTICE_OK;
}

static lattice_status check_attn(const lattice_seq_attn_desc* d) {
  REQUIRE(d, "null attention descriptor");
  TRY(check_heads(d->dtype, d->heads, d->kv_heads, d->head_dim));
  REQUIRE(d->heads % d->kv_heads == 0, "heads is no multiple of kv_heads");
  REQUIRE(d->window >= 1, "window must be at least 1");
  REQUIRE(d->sinks >= 0 && d->sinks <= LATTICE_SEQ_MAX_SINKS, "sinks outside 0..%d", LATTICE_SEQ_MAX_SINKS);
  REQUIRE(d->scale > 0 && std::isfinite(d->scale), "scale must be positive and finite");
  return LATTICE_OK;
}

static lattice_status check_cache(const lattice_seq_attn_desc* d, const lattice_seq_cache* c) {
  REQUIRE(c, "null cache");
  REQUIRE(c->num_caches >= 0, "negative num_caches");
  if ((int64_t)d->window + d->sinks > MAX_ROWS) FAIL(LATTICE_ERR_UNSUPPORTED, "sinks + window above 2^30 slots");
  if (c->num_caches > 0) {
    REQUIRE(c->k && c->v, "null cache memory");
    REQUIRE((uintptr_t)c->k % 16 == 0 && (uintptr_t)c->v % 16 == 0, "cache memory is not 16-byte aligned");
  }
  return LATTICE_OK;
}

static lattice_status check_cache8(const lattice_seq_attn_desc* d, const lattice_seq_cache8* c) {
  REQUIRE(c, "null cache");
  REQUIRE(c->num_caches >= 0, "negative num_caches");
  if ((int64_t)d->window + d->sinks > MAX_ROWS) FAIL(LATTICE_ERR_UNSUPPORTED, "sinks + window above 2^30 slots");
  if (c->num_caches > 0) {
    REQUIRE(c->k && c->v && c->k_scale && c->v_scale, "null cache memory");
    REQUIRE((uintptr_t)c->k % 16 == 0 && (uintptr_t)c->v % 16 == 0, "cache memory is not 16-byte aligned");
    REQUIRE((uintptr_t)c->k_scale % 4 == 0 && (uintptr_t)c->v_scale % 4 == 0, "scales are not 4-byte aligned");
  }
  return LATTICE_OK;
}

static SeqTensor tensor(const void* p, int64_t ld) { return {const_cast<void*>(p), ld}; }

static RopeArgs rope_args(const lattice_qk_rope_desc* d, const lattice_seqs* s) {
  RopeArgs a;
  a.dt = dt_of(d->dtype);
  a.rows = s->rows;
  a.span = reinterpret_cast<const SeqSpan*>(s->span);
  a.positions = d->positions;
  a.heads = d->heads;
  a.kv_heads = d->kv_heads;
  a.dim = d->head_dim;
  a.rotary = d->rotary_dim;
  a.interleaved = d->interleaved != 0;
  a.eps = d->eps;
  a.gain_q = d->gain_q;
  a.gain_k = d->gain_k;
  return a;
}

static SeqAttnArgs attn_args(const lattice_seq_attn_desc* d, const lattice_seqs* s) {
  SeqAttnArgs a;
  a.dt = dt_of(d->dtype);
  a.rows = s->rows;
  a.num_seqs = s->num_seqs;
  a.max_len = s->max_len > 0 && s->max_len < s->rows ? s->max_len : s->rows;
  a.span = reinterpret_cast<const SeqSpan*>(s->span);
  a.key_mask = d->key_mask;
  a.heads = d->heads;
  a.kv_heads = d->kv_heads;
  a.dim = d->head_dim;
  a.window = d->window;
  a.sinks = d->sinks;
  a.scale = d->scale;
  return a;
}

static SeqCacheArgs cache_args(const lattice_seq_attn_desc* d, const lattice_seq_cache* c, const int32_t* index) {
  SeqCacheArgs a;
  a.dt = dt_of(d->dtype);
  a.kv_heads = d->kv_heads;
  a.dim = d->head_dim;
  a.window = d->window;
  a.sinks = d->sinks;
  a.kc = c->k;
  a.vc = c->v;
  a.num_caches = c->num_caches;
  a.index = index;
  return a;
}

static SeqCache8Args cache8_args(const lattice_seq_attn_desc* d, const lattice_seq_cache8* c, const int32_t* index) {
  SeqCache8Args a;
  a.dt = dt_of(d->dtype);
  a.kv_heads = d->kv_heads;
  a.dim = d->head_dim;
  a.window = d->window;
  a.sinks = d->sinks;
  a.kc = c->k;
  a.vc = c->v;
  a.ks = c->k_scale;
  a.vs = c->v_scale;
  a.num_caches = c->num_caches;
  a.index = index;
  return a;
}

static lattice_status check_step(const lattice_seq_attn_desc* d, const lattice_qk_rope_desc* rope, int32_t batch) {
  TRY(check_attn(d));
  REQUIRE(!d->key_mask, "a cache takes no key_mask");
  if (rope) {
    TRY(check_rope(rope));
    REQUIRE(rope->dtype == d->dtype && rope->heads == d->heads && rope->kv_heads == d->kv_heads &&
                rope->head_dim == d->head_dim, "rope and attention descriptors differ");
  }
  REQUIRE(batch >= 0, "negative batch");
  return LATTICE_OK;
}

// Everything of a step but its cache
static lattice_status step_args(const lattice_seq_attn_desc* d, const lattice_qk_rope_desc* rope, int32_t batch,
                                const void* q, int64_t q_stride, const void* k, int64_t k_stride, const void* v,
                                int64_t v_stride, const int32_t* lens, void* out, int64_t out_stride, SeqStepArgs* a,
                                RopeTurns* t) {
  REQUIRE(lens, "null lens");
  TRY(check_tensor("q", q, q_stride, d->heads, d->head_dim));
  TRY(check_tensor("k", k, k_stride, d->kv_heads, d->head_dim));
  TRY(check_tensor("v", v, v_stride, d->kv_heads, d->head_dim));
  TRY(check_tensor("out", out, out_stride, d->heads, d->head_dim));
  if ((int64_t)batch * d->heads > MAX_BLOCKS / 2) FAIL(LATTICE_ERR_UNSUPPORTED, "batch x heads too large for one launch");
  a->batch = batch;
  a->heads = d->heads;
  a->scale = d->scale;
  a->q = tensor(q, q_stride);
  a->k = tensor(k, k_stride);
  a->v = tensor(v, v_stride);
  a->out = tensor(out, out_stride);
  a->lens = lens;
  if (rope) {
    a->rope = 1;
    a->rotary = rope->rotary_dim;
    a->interleaved = rope->interleaved != 0;
    a->eps = rope->eps;
    a->gain_q = rope->gain_q;
    a->gain_k = rope->gain_k;
    a->positions = rope->positions;
    rope_turns(rope->theta, rope->rotary_dim, t);
  }
  return LATTICE_OK;
}

// blocks of the attention kernels: 128 rows of a head each
static lattice_status check_attn_size(const lattice_seq_attn_desc* d, const lattice_seqs* s) {
  if ((s->rows / 128 + 4) * d->heads > MAX_BLOCKS / 2)
    FAIL(LATTICE_ERR_UNSUPPORTED, "rows x heads too many for one launch");
  return LATTICE_OK;
}

extern "C" {

lattice_status lattice_seq_plan(const lattice_seqs* seqs, int32_t* span, void* stream) {
  TRY(check_seqs(seqs));
  if (seqs->rows == 0) return LATTICE_OK;
  REQUIRE(span && (uintptr_t)span % 8 == 0, "span is null or not 8-byte aligned");
  if (seqs->num_seqs > 0) REQUIRE(seqs->offsets, "null offsets");
  HIPRET(seq_plan(seqs->offsets, seqs->num_seqs, seqs->rows, reinterpret_cast<SeqSpan*>(span), strm(stream)));
  return LATTICE_OK;
}

lattice_status lattice_qk_rope_fwd(const lattice_qk_rope_desc* d, const lattice_seqs* seqs, const void* q,
                                   int64_t q_stride, const void* k, int64_t k_stride, void* q_out,
                                   int64_t q_out_stride, void* k_out, int64_t k_out_stride, void* stream) {
  TRY(check_rope(d));
  TRY(check_seqs(seqs));
  if (seqs->rows == 0) return LATTICE_OK;
  REQUIRE(seqs->span || d->positions, "neither span nor positions");
  TRY(check_tensor("q", q, q_stride, d->heads, d->head_dim));
  TRY(check_tensor("k", k, k_stride, d->kv_heads, d->head_dim));
  TRY(check_tensor("q_out", q_out, q_out_stride, d->heads, d->head_dim));
  TRY(check_tensor("k_out", k_out, k_out_stride, d->kv_heads, d->head_dim));
  RopeArgs a = rope_args(d, seqs);
  a.q = tensor(q, q_stride);
  a.k = tensor(k, k_stride);
  a.oq = tensor(q_out, q_out_stride);
  a.ok = tensor(k_out, k_out_stride);
  RopeTurns t;
  rope_turns(d->theta, d->rotary_dim, &t);
  HIPRET(rope_fwd(a, t, strm(stream)));
  return LATTICE_OK;
}

size_t lattice_qk_rope_bwd_workspace(const lattice_qk_rope_desc* d, int64_t rows) {
  if (check_rope(d) != LATTICE_OK || rows <= 0 || rows >= MAX_ROWS) return 0;
  return rope_bwd_workspace(rows, d->head_dim);
}

lattice_status lattice_qk_rope_bwd(const lattice_qk_rope_desc* d, const lattice_seqs* seqs, const void* q,
                                   int64_t q_stride, const void* k, int64_t k_stride, const void* d_q_out,
                                   int64_t d_q_out_stride, const void* d_k_out, int64_t d_k_out_stride, void* dq,
                                   int64_t dq_stride, void* dk, int64_t dk_stride, float* dgain_q, float* dgain_k,
                                   void* ws, size_t ws_bytes, void* stream) {
  TRY(check_rope(d));
  TRY(check_seqs(seqs));
  RopeArgs a = rope_args(d, seqs);
  a.dgain_q = dgain_q;
  a.dgain_k = dgain_k;
  if (seqs->rows > 0) {
    REQUIRE(seqs->span || d->positions, "neither span nor positions");
    TRY(check_tensor("q", q, q_stride, d->heads, d->head_dim));
    TRY(check_tensor("k", k, k_stride, d->kv_heads, d->head_dim));
    TRY(check_tensor("d_q_out", d_q_out, d_q_out_stride, d->heads, d->head_dim));
    TRY(check_tensor("d_k_out", d_k_out, d_k_out_stride, d->kv_heads, d->head_dim));
    TRY(check_tensor("dq", dq, dq_stride, d->heads, d->head_dim));
    TRY(check_tensor("dk", dk, dk_stride, d->kv_heads, d->head_dim));
    if (dgain_q || dgain_k) {
      const size_t need = rope_bwd_workspace(seqs->rows, d->head_dim);
      if (!ws || ws_bytes < need) FAIL(LATTICE_ERR_WORKSPACE, "workspace %zu < %zu", ws_bytes, need);
    }
  }
  a.q = tensor(q, q_stride);
  a.k = tensor(k, k_stride);
  a.gq = tensor(d_q_out, d_q_out_stride);
  a.gk = tensor(d_k_out, d_k_out_stride);
  a.oq = tensor(dq, dq_stride);
  a.ok = tensor(dk, dk_stride);
  RopeTurns t;
  rope_turns(d->theta, d->rotary_dim, &t);
  HIPRET(rope_bwd(a, t, ws, strm(stream)));
  return LATTICE_OK;
}

lattice_status lattice_seq_attn_fwd(const lattice_seq_attn_desc* d, const lattice_seqs* seqs, const void* q,
                                    int64_t q_stride, const void* k, int64_t k_stride, const void* v,
                                    int64_t v_stride, void* out, int64_t out_stride, float* lse, void* out_lo,
                                    void* stream) {
  TRY(check_attn(d));
  TRY(check_seqs(seqs));
  if (seqs->rows == 0 || seqs->num_seqs == 0) return LATTICE_OK;
  REQUIRE(seqs->span, "null span (lattice_seq_plan writes it)");
  TRY(check_tensor("q", q, q_stride, d->heads, d->head_dim));
  TRY(check_tensor("k", k, k_stride, d->kv_heads, d->head_dim));
  TRY(check_tensor("v", v, v_stride, d->kv_heads, d->head_dim));
  TRY(check_tensor("out", out, out_stride, d->heads, d->head_dim));
  REQUIRE((uintptr_t)out_lo % 16 == 0, "out_lo is not 16-byte aligned");
  TRY(check_attn_size(d, seqs));
  SeqAttnArgs a = attn_args(d, seqs);
  a.q = tensor(q, q_stride);
  a.k = tensor(k, k_stride);
  a.v = tensor(v, v_stride);
  a.o = tensor(out, out_stride);
  a.lse = lse;
  a.out_lo = out_lo;
  HIPRET(seq_attn_fwd(a, strm(stream)));
  return LATTICE_OK;
}

size_t lattice_seq_attn_bwd_workspace(const lattice_seq_attn_desc* d, const lattice_seqs* seqs) {
  if (check_attn(d) != LATTICE_OK || check_seqs(seqs) != LATTICE_OK) return 0;
  return seq_attn_bwd_workspace(attn_args(d, seqs));
}

lattice_status lattice_seq_attn_bwd(const lattice_seq_attn_desc* d, const lattice_seqs* seqs, const void* q,
                                    int64_t q_stride, const void* k, int64_t k_stride, const void* v,
                                    int64_t v_stride, const void* out, int64_t out_stride, const float* lse,
                                    const void* out_lo, const void* d_out, int64_t d_out_stride, void* dq,
                                    int64_t dq_stride, void* dk, int64_t dk_stride, void* dv, int64_t dv_stride,
                                    void* ws, size_t ws_bytes, void* stream) {
  TRY(check_attn(d));
  TRY(check_seqs(seqs));
  if (seqs->rows == 0 || seqs->num_seqs == 0) return LATTICE_OK;
  REQUIRE(seqs->span && seqs->offsets, "null span or offsets");
  REQUIRE(lse, "null lse");
  TRY(check_tensor("q", q, q_stride, d->heads, d->head_dim));
  TRY(check_tensor("k", k, k_stride, d->kv_heads, d->head_dim));
  TRY(check_tensor("v", v, v_stride, d->kv_heads, d->head_dim));
  TRY(check_tensor("out", out, out_stride, d->heads, d->head_dim));
  TRY(check_tensor("d_out", d_out, d_out_stride, d->heads, d->head_dim));
  TRY(check_tensor("dq", dq, dq_stride, d->heads, d->head_dim));
  TRY(check_tensor("dk", dk, dk_stride, d->kv_heads, d->head_dim));
  TRY(check_tensor("dv", dv, dv_stride, d->kv_heads, d->head_dim));
  REQUIRE((uintptr_t)out_lo % 16 == 0, "out_lo is not 16-byte aligned");
  TRY(check_attn_size(d, seqs));
  SeqAttnArgs a = attn_args(d, seqs);
  const size_t need = seq_attn_bwd_workspace(a);
  if (!ws || ws_bytes < need) FAIL(LATTICE_ERR_WORKSPACE, "workspace %zu < %zu", ws_bytes, need);
  REQUIRE((uintptr_t)ws % 16 == 0, "workspace is not 16-byte aligned");
  a.q = tensor(q, q_stride);
  a.k = tensor(k, k_stride);
  a.v = tensor(v, v_stride);
  a.o = tensor(out, out_stride);
  a.lse = const_cast<float*>(lse);
  a.out_lo = const_cast<void*>(out_lo);
  a.go = tensor(d_out, d_out_stride);
  a.gq = tensor(dq, dq_stride);
  a.gk = tensor(dk, dk_stride);
  a.gv = tensor(dv, dv_stride);
  HIPRET(seq_attn_bwd(a, ws, strm(stream)));
  return LATTICE_OK;
}

lattice_status lattice_seq_cache_fill(const lattice_seq_attn_desc* d, const lattice_seqs* seqs, const void* k,
                                      int64_t k_stride, const void* v, int64_t v_stride, const int32_t* first,
                                      const int32_t* cache_index, const lattice_seq_cache* cache, void* stream) {
  TRY(check_attn(d));
  REQUIRE(!d->key_mask, "a cache takes no key_mask");
  TRY(check_seqs(seqs));
  TRY(check_cache(d, cache));
  if (seqs->rows == 0 || seqs->num_seqs == 0 || cache->num_caches == 0) return LATTICE_OK;
  REQUIRE(seqs->offsets, "null offsets");
  TRY(check_tensor("k", k, k_stride, d->kv_heads, d->head_dim));
  TRY(check_tensor("v", v, v_stride, d->kv_heads, d->head_dim));
  HIPRET(seq_cache_fill(cache_args(d, cache, cache_index), seqs->rows, seqs->offsets, seqs->num_seqs, first,
                        tensor(k, k_stride), tensor(v, v_stride), strm(stream)));
  return LATTICE_OK;
}

size_t lattice_seq_step_workspace(const lattice_seq_attn_desc* d, int32_t batch) {
  if (check_attn(d) != LATTICE_OK || batch <= 0 || (int64_t)d->window + d->sinks > MAX_ROWS) return 0;
  return seq_step_workspace(batch, d->heads, d->kv_heads, d->head_dim, d->sinks + d->window);
}

lattice_status lattice_seq_step(const lattice_seq_attn_desc* d, const lattice_qk_rope_desc* rope, int32_t batch,
                                const void* q, int64_t q_stride, const void* k, int64_t k_stride, const void* v,
                                int64_t v_stride, const int32_t* lens, const int32_t* cache_index,
                                const lattice_seq_cache* cache, void* out, int64_t out_stride, void* ws,
                                size_t ws_bytes, void* stream) {
  TRY(check_step(d, rope, batch));
  TRY(check_cache(d, cache));
  if (batch == 0 || cache->num_caches == 0) return LATTICE_OK;
  SeqStepArgs a;
  RopeTurns t{};
  TRY(step_args(d, rope, batch, q, q_stride, k, k_stride, v, v_stride, lens, out, out_stride, &a, &t));
  const size_t need = seq_step_workspace(batch, d->heads, d->kv_heads, d->head_dim, d->sinks + d->window);
  if (need > 0 && (!ws || ws_bytes < need)) FAIL(LATTICE_ERR_WORKSPACE, "workspace %zu < %zu", ws_bytes, need);
  a.c = cache_args(d, cache, cache_index);
  HIPRET(seq_step(a, t, ws, strm(stream)));
  return LATTICE_OK;
}

lattice_status lattice_seq_cache8_fill(const lattice_seq_attn_desc* d, const lattice_seqs* seqs, const void* k,
                                       int64_t k_stride, const void* v, int64_t v_stride, const int32_t* first,
                                       const int32_t* cache_index, const lattice_seq_cache8* cache, void* stream) {
  TRY(check_attn(d));
  REQUIRE(!d->key_mask, "a cache takes no key_mask");
  TRY(check_seqs(seqs));
  TRY(check_cache8(d, cache));
  if (seqs->rows == 0 || seqs->num_seqs == 0 || cache->num_caches == 0) return LATTICE_OK;
  REQUIRE(seqs->offsets, "null offsets");
  TRY(check_tensor("k", k, k_stride, d->kv_heads, d->head_dim));
  TRY(check_tensor("v", v, v_stride, d->kv_heads, d->head_dim));
  HIPRET(seq_cache8_fill(cache8_args(d, cache, cache_index), seqs->rows, seqs->offsets, seqs->num_seqs,
                         seqs->max_len < seqs->rows ? seqs->max_len : seqs->rows, first,
                         tensor(k, k_stride), tensor(v, v_stride), strm(stream)));
  return LATTICE_OK;
}

size_t lattice_seq_step8_workspace(const lattice_seq_attn_desc* d, int32_t batch) {
  if (check_attn(d) != LATTICE_OK || batch <= 0 || (int64_t)d->window + d->sinks > MAX_ROWS) return 0;
  return seq_step8_workspace(batch, d->heads, d->kv_heads, d->head_dim, d->sinks + d->window);
}

lattice_status lattice_seq_step8(const lattice_seq_attn_desc* d, const lattice_qk_rope_desc* rope, int32_t batch,
                                 const void* q, int64_t q_stride, const void* k, int64_t k_stride, const void* v,
                                 int64_t v_stride, const int32_t* lens, const int32_t* cache_index,
                                 const lattice_seq_cache8* cache, void* out, int64_t out_stride, void* ws,
                                 size_t ws_bytes, void* stream) {
  TRY(check_step(d, rope, batch));
  TRY(check_cache8(d, cache));
  if (batch == 0 || cache->num_caches == 0) return LATTICE_OK;
  SeqStepArgs a;
  RopeTurns t{};
  TRY(step_args(d, rope, batch, q, q_stride, k, k_stride, v, v_stride, lens, out, out_stride, &a, &t));
  const size_t need = seq_step8_workspace(batch, d->heads, d->kv_heads, d->head_dim, d->sinks + d->window);
  if (need > 0 && (!ws || ws_bytes < need)) FAIL(LATTICE_ERR_WORKSPACE, "workspace %zu < %zu", ws_bytes, need);
  if (need > 0) REQUIRE((uintptr_t)ws % 4 == 0, "workspace is not 4-byte aligned");
  HIPRET(seq_step8(a, cache8_args(d, cache, cache_index), t, ws, strm(stream)));
  return LATTICE_OK;
}

}  // extern "C"
