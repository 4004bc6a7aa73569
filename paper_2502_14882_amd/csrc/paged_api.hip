// Host side of the paged 8-bit cache (include/cq_paged.h): argument checks, plans, launches.  Every check
// runs before the first HIP call, so a rejected call launches nothing.
#include <cmath>

#include "paged_internal.h"
#include "decode_meet.h"

namespace {

using cq::fail;

bool aligned(const void* p, unsigned n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

int hip_fail(hipError_t e, const char* what) { return fail(CQ_ERR_HIP, "%s: %s", what, hipGetErrorString(e)); }

int check_head_dim(int d) {
  if (d < 32 || d > 256 || d % 32 != 0)
    return fail(CQ_ERR_SHAPE, "head_dim=%d must be a multiple of 32 in [32, 256]", d);
  return CQ_OK;
}

int check_rows(int n_tokens, int dtype) {
  if (n_tokens < 0) return fail(CQ_ERR_SHAPE, "n_tokens=%d must be >= 0", n_tokens);
  if (dtype != CQP_F16 && dtype != CQP_BF16) return fail(CQ_ERR_UNSUPPORTED, "dtype=%d is not a CQP_* type", dtype);
  return CQ_OK;
}

// n_heads: 0 = any; written: the rows must not overlap
int check_heads(const char* which, const cqp_heads_t* t, int n_tokens, int d, int n_heads, bool written) {
  if (!t) return fail(CQ_ERR_NULL, "%s is NULL", which);
  if (t->n_heads < 1) return fail(CQ_ERR_SHAPE, "%s has n_heads=%d", which, t->n_heads);
  if (t->reserved != 0) return fail(CQ_ERR_SHAPE, "%s has reserved=%d, 0 is wanted", which, t->reserved);
  if (n_heads > 0 && t->n_heads != n_heads)
    return fail(CQ_ERR_SHAPE, "%s has %d heads, %d are wanted", which, t->n_heads, n_heads);
  if (n_tokens == 0) return CQ_OK;
  if (!t->data) return fail(CQ_ERR_NULL, "%s has a NULL data pointer", which);
  if (!aligned(t->data, 16)) return fail(CQ_ERR_ALIGN, "%s must be 16-byte aligned", which);
  if (t->token_stride < 0 || t->head_stride < 0 || t->token_stride % 8 != 0 || t->head_stride % 8 != 0)
    return fail(CQ_ERR_ALIGN, "the strides of %s (%lld, %lld) must be >= 0 and multiples of 8", which,
                (long long)t->token_stride, (long long)t->head_stride);
  const double span = (double)t->token_stride * n_tokens + (double)t->head_stride * t->n_heads;
  if (span >= 4.0e18) return fail(CQ_ERR_SHAPE, "%s is too large", which);
  if (written) {
    // one of the strides steps over all that lies along the other
    const long long heads = (long long)(t->n_heads - 1) * t->head_stride + d;
    const long long tokens = (long long)(n_tokens - 1) * t->token_stride + d;
    const bool heads_apart = t->n_heads == 1 || t->head_stride >= d, tokens_apart = n_tokens == 1 || t->token_stride >= d;
    const bool nested = n_tokens == 1 || t->n_heads == 1 || t->token_stride >= heads || t->head_stride >= tokens;
    if (!heads_apart || !tokens_apart || !nested)
      return fail(CQ_ERR_SHAPE, "rows of %s overlap (strides %lld, %lld)", which, (long long)t->token_stride,
                  (long long)t->head_stride);
  }
  return CQ_OK;
}

cq::HeadRows rows_of(const cqp_heads_t& t) { return cq::HeadRows{t.data, t.token_stride, t.head_stride, t.n_heads}; }

int check_cache(const cqp_cache_t* c, bool pointers, cq::PagedCacheArgs* out) {
  if (!c) return fail(CQ_ERR_NULL, "cache is NULL");
  if (c->n_pages < 1 || c->n_kv_heads < 1)
    return fail(CQ_ERR_SHAPE, "n_pages=%d and n_kv_heads=%d must be >= 1", c->n_pages, c->n_kv_heads);
  const int rc = check_head_dim(c->head_dim);
  if (rc != CQ_OK) return rc;
  int log2 = 4;
  while (log2 < 8 && (1 << log2) != c->page) ++log2;
  if ((1 << log2) != c->page) return fail(CQ_ERR_SHAPE, "page=%d is not 16, 32, 64, 128 or 256", c->page);
  if ((double)c->n_kv_heads * c->page * c->head_dim >= 2147483648.0)
    return fail(CQ_ERR_SHAPE, "a page of %d heads x %d tokens x %d channels is too large", c->n_kv_heads, c->page, c->head_dim);
  if ((double)c->n_pages * c->n_kv_heads * c->page * c->head_dim >= 4.0e18) return fail(CQ_ERR_SHAPE, "cache too large");
  if (pointers) {
    if (!c->k_codes || !c->v_codes || !c->k_scale || !c->v_scale) return fail(CQ_ERR_NULL, "cache has a NULL pointer");
    if (!aligned(c->k_codes, 16) || !aligned(c->v_codes, 16))
      return fail(CQ_ERR_ALIGN, "the cache's codes must be 16-byte aligned");
    if (!aligned(c->k_scale, 4) || !aligned(c->v_scale, 4))
      return fail(CQ_ERR_ALIGN, "the cache's scales must be 4-byte aligned");
  }
  *out = cq::PagedCacheArgs{c->k_codes, c->v_codes, c->k_scale, c->v_scale, c->n_pages, c->n_kv_heads, c->head_dim, c->page, log2};
  return CQ_OK;
}

int check_batch(const cqp_batch_t* s, const cq::PagedCacheArgs& c, int n_tokens, bool pointers, cq::PagedBatch* out) {
  if (!s) return fail(CQ_ERR_NULL, "batch is NULL");
  if (s->batch < 1 || s->max_pages < 1 || s->max_new < 1 || s->max_len < 1)
    return fail(CQ_ERR_SHAPE, "batch=%d, max_pages=%d, max_new=%d and max_len=%d must be >= 1", s->batch, s->max_pages,
                s->max_new, s->max_len);
  if (pointers) {
    if (!s->page_table || !s->seq_lens || !s->q_start) return fail(CQ_ERR_NULL, "batch has a NULL pointer");
    if (!aligned(s->page_table, 4) || !aligned(s->seq_lens, 4) || !aligned(s->q_start, 4))
      return fail(CQ_ERR_ALIGN, "the batch's arrays must be 4-byte aligned");
  }
  const long long held = (long long)s->max_pages * c.page;
  int bound = s->max_len < held ? s->max_len : (int)held;
  // places are counted in 32 bits, a step beyond the last one included
  if (bound > 0x7fffffff - 4096) return fail(CQ_ERR_SHAPE, "max_len=%d is too large", s->max_len);
  *out = cq::PagedBatch{s->page_table, s->seq_lens, s->q_start, s->batch, s->max_pages,
                        s->max_new < n_tokens || n_tokens < 1 ? s->max_new : n_tokens, n_tokens, bound};
  return CQ_OK;
}

int check_rope(const cqp_rope_t* r, const int32_t* positions, int n_tokens, int d, cq::RopeArgs* out) {
  if (!r) return fail(CQ_ERR_NULL, "rope is NULL");
  if (r->rot_dim < 16 || r->rot_dim > d || r->rot_dim % 16 != 0)
    return fail(CQ_ERR_SHAPE, "rot_dim=%d must be a multiple of 16 in [16, head_dim=%d]", r->rot_dim, d);
  if (r->n_axes < 1 || r->n_axes > 4) return fail(CQ_ERR_SHAPE, "n_axes=%d must be 1 to 4", r->n_axes);
  if (r->pairs != CQP_PAIRS_HALVES && r->pairs != CQP_PAIRS_ADJACENT)
    return fail(CQ_ERR_UNSUPPORTED, "pairs=%d is not a CQP_PAIRS_* value", r->pairs);
  if (r->reserved != 0) return fail(CQ_ERR_SHAPE, "rope has reserved=%d, 0 is wanted", r->reserved);
  *out = cq::RopeArgs{};
  for (int i = 0; i < r->rot_dim / 2; ++i) {
    if (r->axis_of[i] >= r->n_axes)
      return fail(CQ_ERR_SHAPE, "axis_of[%d]=%d, but n_axes=%d", i, r->axis_of[i], r->n_axes);
    out->axis_of[i] = r->axis_of[i];
  }
  if (!r->inv_freq) return fail(CQ_ERR_NULL, "rope has a NULL inv_freq");
  if (!positions && n_tokens > 0) return fail(CQ_ERR_NULL, "positions is NULL");
  if (!aligned(r->inv_freq, 4) || !aligned(positions, 4))
    return fail(CQ_ERR_ALIGN, "inv_freq and positions must be 4-byte aligned");
  out->inv_freq = r->inv_freq;
  out->positions = positions;
  out->half = r->rot_dim / 2;
  out->n_axes = r->n_axes;
  out->adjacent = r->pairs == CQP_PAIRS_ADJACENT;
  out->sign = 1.0f;
  return CQ_OK;
}

}  // namespace

extern "C" {

int cqp_rotate(const cqp_rope_t* rope, const int32_t* positions, int32_t n_tokens, int32_t head_dim, int32_t dtype,
               int32_t backward, const cqp_heads_t* in, const cqp_heads_t* out, int32_t n_tensors, void* stream) {
  cq::RopeArgs r;
  int rc = check_head_dim(head_dim);
  if (rc != CQ_OK) return rc;
  if ((rc = check_rows(n_tokens, dtype)) != CQ_OK) return rc;
  if ((rc = check_rope(rope, positions, n_tokens, head_dim, &r)) != CQ_OK) return rc;
  if (n_tensors < 1 || n_tensors > 2) return fail(CQ_ERR_SHAPE, "n_tensors=%d must be 1 or 2", n_tensors);
  if (backward != 0 && backward != 1) return fail(CQ_ERR_UNSUPPORTED, "backward=%d must be 0 or 1", backward);
  if (!in || !out) return fail(CQ_ERR_NULL, "in or out is NULL");
  cq::HeadRows from[2], to[2];
  for (int i = 0; i < n_tensors; ++i) {
    if ((rc = check_heads("in", &in[i], n_tokens, head_dim, 0, false)) != CQ_OK) return rc;
    if ((rc = check_heads("out", &out[i], n_tokens, head_dim, in[i].n_heads, true)) != CQ_OK) return rc;
    from[i] = rows_of(in[i]);
    to[i] = rows_of(out[i]);
  }
  if (n_tokens == 0) return CQ_OK;
  if (backward) r.sign = -1.0f;
  const hipError_t e = cq::launch_rotate(r, n_tokens, head_dim, dtype == CQP_BF16, from, to, n_tensors,
                                         static_cast<hipStream_t>(stream));
  if (e == hipErrorInvalidConfiguration) return fail(CQ_ERR_SHAPE, "%d tokens are too many for a launch", n_tokens);
  return e == hipSuccess ? CQ_OK : hip_fail(e, "rotate");
}

int cqp_append_kv(const cqp_cache_t* cache, const cqp_batch_t* batch, int32_t n_tokens, int32_t dtype, const cqp_heads_t* k,
                  const cqp_heads_t* v, const cqp_rope_t* rope, const int32_t* positions, const cqp_heads_t* q_in,
                  const cqp_heads_t* q_out, void* stream) {
  cq::PagedCacheArgs c;
  cq::PagedBatch s;
  cq::RopeArgs r = {};
  int rc = check_cache(cache, true, &c);
  if (rc != CQ_OK) return rc;
  if ((rc = check_rows(n_tokens, dtype)) != CQ_OK) return rc;
  if ((rc = check_batch(batch, c, n_tokens, true, &s)) != CQ_OK) return rc;
  if ((rc = check_heads("k", k, n_tokens, c.d, c.heads, false)) != CQ_OK) return rc;
  if ((rc = check_heads("v", v, n_tokens, c.d, c.heads, false)) != CQ_OK) return rc;
  if (!rope && positions) return fail(CQ_ERR_NULL, "positions without a rope");
  if (rope && (rc = check_rope(rope, positions, n_tokens, c.d, &r)) != CQ_OK) return rc;
  cq::HeadRows from = {}, to = {};
  if (q_in || q_out) {
    if (!q_in || !q_out) return fail(CQ_ERR_NULL, "q_in and q_out go together");
    if (!rope) return fail(CQ_ERR_NULL, "queries are given, but rope is NULL");
    if ((rc = check_heads("q_in", q_in, n_tokens, c.d, 0, false)) != CQ_OK) return rc;
    if ((rc = check_heads("q_out", q_out, n_tokens, c.d, q_in->n_heads, true)) != CQ_OK) return rc;
    from = rows_of(*q_in);
    to = rows_of(*q_out);
  }
  if (n_tokens == 0) return CQ_OK;
  const hipError_t e = cq::launch_append(c, s, dtype == CQP_BF16, rows_of(*k), rows_of(*v), r, from, to,
                                         static_cast<hipStream_t>(stream));
  if (e == hipErrorInvalidConfiguration) return fail(CQ_ERR_SHAPE, "%d tokens in %d sequences are too many for a launch", n_tokens, s.batch);
  return e == hipSuccess ? CQ_OK : hip_fail(e, "append");
}

size_t cqp_attn_workspace_bytes(const cqp_cache_t* cache, const cqp_batch_t* batch, int32_t n_tokens, int32_t n_q_heads) {
  cq::PagedCacheArgs c;
  cq::PagedBatch s;
  if (check_cache(cache, false, &c) != CQ_OK || n_tokens < 0 || check_batch(batch, c, n_tokens, false, &s) != CQ_OK ||
      n_q_heads < 1 || n_q_heads % c.heads != 0)
    return 0;
  const cq::PagedPlan plan = cq::make_paged_plan(c, s, n_q_heads);
  return plan.fits ? plan.ws_bytes : 0;
}

int cqp_attn(const cqp_cache_t* cache, const cqp_batch_t* batch, int32_t n_tokens, int32_t dtype, const cqp_heads_t* q,
             const cqp_heads_t* out, float* lse, int32_t causal, float softmax_scale, void* workspace,
             size_t workspace_bytes, void* stream) {
  cq::PagedAttention a = {};
  int rc = check_cache(cache, true, &a.cache);
  if (rc != CQ_OK) return rc;
  if ((rc = check_rows(n_tokens, dtype)) != CQ_OK) return rc;
  if ((rc = check_batch(batch, a.cache, n_tokens, true, &a.batch)) != CQ_OK) return rc;
  if ((rc = check_heads("q", q, n_tokens, a.cache.d, 0, false)) != CQ_OK) return rc;
  if ((rc = check_heads("out", out, n_tokens, a.cache.d, q->n_heads, true)) != CQ_OK) return rc;
  if (q->n_heads % a.cache.heads != 0)
    return fail(CQ_ERR_SHAPE, "q has %d heads, not a multiple of n_kv_heads=%d", q->n_heads, a.cache.heads);
  if (!aligned(lse, 4)) return fail(CQ_ERR_ALIGN, "lse must be 4-byte aligned");
  if (causal != 0 && causal != 1) return fail(CQ_ERR_UNSUPPORTED, "causal=%d must be 0 or 1", causal);
  if (!std::isfinite(softmax_scale) || softmax_scale < 0.f)
    return fail(CQ_ERR_SHAPE, "softmax_scale must be finite and >= 0");
  if (softmax_scale == 0.f) softmax_scale = 1.0f / std::sqrt((float)a.cache.d);
  a.plan = cq::make_paged_plan(a.cache, a.batch, q->n_heads);
  if (!a.plan.fits) return fail(CQ_ERR_SHAPE, "%d tokens of %d heads in %d sequences are too many for a launch", n_tokens, q->n_heads, batch->batch);
  if (!workspace) return fail(CQ_ERR_WORKSPACE, "workspace is NULL");
  if (!aligned(workspace, 256)) return fail(CQ_ERR_WORKSPACE, "workspace must be 256-byte aligned");
  if (workspace_bytes < a.plan.ws_bytes)
    return fail(CQ_ERR_WORKSPACE, "workspace has %zu bytes, %zu needed", workspace_bytes, a.plan.ws_bytes);
  if (n_tokens == 0) return CQ_OK;
  a.q = rows_of(*q);
  a.out = rows_of(*out);
  a.lse = lse;
  a.g = q->n_heads / a.cache.heads;
  a.causal = causal;
  a.scale_log2 = softmax_scale * 1.44269504088896340736f;
  a.counts = static_cast<unsigned long long*>(workspace);
  a.tag = a.plan.few_joins ? cq::meeting_tag() : 0;
  a.ml = static_cast<float*>(workspace) + a.plan.ws_ml_floats;
  a.acc = static_cast<float*>(workspace) + a.plan.ws_acc_floats;
  hipStream_t st = static_cast<hipStream_t>(stream);
  hipError_t e = a.plan.prompts ? cq::launch_paged_prompt(a, dtype == CQP_BF16, st) : hipSuccess;
  if (e == hipSuccess && a.plan.few) e = cq::launch_paged_few(a, dtype == CQP_BF16, st);
  if (e == hipSuccess && (a.plan.prompt_splits > 1 || (a.plan.few_splits > 1 && !a.plan.few_joins))) e = cq::launch_paged_combine(a, dtype == CQP_BF16, st);
  return e == hipSuccess ? CQ_OK : hip_fail(e, "attention");
}

}  // extern "C"
