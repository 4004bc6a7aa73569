/*
 * cq_paged.h - C ABI of libcq's paged 8-bit KV cache on MI355X (gfx950).
 *
 * What a serving step of a (multimodal) language model does around the packed visual cache of cq.h,
 * for tokens that arrive one by one or a prompt at a time:
 *   cqp_rotate     rotary positions with one to four axes (text position; time, height and
 *                  width of visual tokens) on queries and keys, and their gradient;
 *   cqp_append_kv  growth of the cache: new keys (rotated on the way) and values are coded
 *                  and written to their sequences' pages, the step's queries rotated beside them;
 *   cqp_attn       attention of the new tokens' queries over the cache, from single tokens over
 *                  long sequences to whole prompts.
 *
 * The conventions of cq.h hold: device pointers owned by the caller, nothing allocated or kept,
 * asynchronous on `stream`, host structs read before the call returns, cq_status values with
 * cq_last_error(), argument errors found on the host before any HIP call.  Lengths, offsets, page
 * tables and positions lie in DEVICE memory, so that a step can be recorded once into a HIP graph
 * and replayed while the sequences grow; the host gives upper bounds.  What the host cannot see the
 * kernels bound themselves: no content of these arrays makes them touch memory outside the tensors.
 * The device that holds the tensors must be the current one, and `stream` one of its streams.
 */
#ifndef CQ_PAGED_H_
#define CQ_PAGED_H_

#include "cq.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element type of queries, keys, values and outputs. */
enum { CQP_F16 = 0, CQP_BF16 = 1 };

/* Rows of heads [n_tokens, n_heads, head_dim], channels contiguous: `data` 16-byte aligned, the
 * strides (in elements) multiples of 8, >= 0 for inputs; rows of outputs must not overlap.  A
 * part of a fused projection is passed with the projection's token stride. */
typedef struct {
  void *data;
  int64_t token_stride, head_stride;
  int32_t n_heads;
  int32_t reserved; /* 0 */
} cqp_heads_t;

/*
 * The cache: n_pages pages of `page` tokens.  Element = code * scale, a code being an e4m3 float (OCP
 * FP8 without infinities, largest value 448) and the scale a power of two (cqp_append_kv writes no
 * others, and cqp_attn relies on it), one per page and KV head for the keys and one for the values.
 *   k_codes  [n_pages, n_kv_heads, page, head_dim]
 *   v_codes  [n_pages, n_kv_heads, head_dim, page]   (a channel's tokens lie together)
 *   k_scale, v_scale  fp32 [n_pages, n_kv_heads]
 * Code pointers are 16-byte, scale pointers 4-byte aligned.  Nothing needs to be cleared: slots
 * that hold no token, and the scales of pages that hold none, are never used.
 */
typedef struct {
  int32_t n_pages;    /* >= 1 */
  int32_t page;       /* 16, 32, 64, 128 or 256 */
  int32_t n_kv_heads; /* >= 1 */
  int32_t head_dim;   /* multiple of 32 in [32, 256] */
  uint8_t *k_codes, *v_codes;
  float *k_scale, *v_scale;
} cqp_cache_t;

/*
 * The sequences of a step.  The new tokens of all sequences lie behind each other: sequence b has the
 * rows q_start[b] <= t < q_start[b + 1] of every [n_tokens, ...] tensor, at most max_new of
 * them, none at all included.  seq_lens[b] counts the tokens of the sequence that the cache holds
 * with these, so row t is token seq_lens[b] - (q_start[b + 1] - t) of the sequence, and token j lies in
 * slot j % page of page page_table[b][j / page].  Rows behind q_start[batch] belong to nobody: they are
 * neither read nor written.  Values out of range are brought into it: q_start into [0,
 * n_tokens], a sequence's rows to max_new (its first ones), seq_lens into [0, min(max_len, max_pages * page)]; a page
 * table entry outside [0, n_pages) is a page that is not there.
 */
typedef struct {
  int32_t batch;                  /* >= 1 */
  int32_t max_pages;              /* entries of a row of the page table, >= 1 */
  int32_t max_new;                /* host bound of the new tokens of a sequence, >= 1 */
  int32_t max_len;                /* host bound of seq_lens, >= 1 */
  const int32_t *page_table;      /* [batch, max_pages] */
  const int32_t *seq_lens;        /* [batch] */
  const int32_t *q_start;         /* [batch + 1], not decreasing */
} cqp_batch_t;

/* How the channels of a pair lie, r = rot_dim. */
enum {
  CQP_PAIRS_HALVES = 0,  /* pair i = channels i and i + r / 2 */
  CQP_PAIRS_ADJACENT = 1 /* pair i = channels 2 i and 2 i + 1 */
};

/*
 * Rotary positions.  Pair i (0 <= i < rot_dim / 2) of every head of token t is turned by the angle
 *     positions[axis_of[i]][t] * inv_freq[i],
 * the product and its sine and cosine to fp64 accuracy, rounded to fp32; products and sums of the
 * rotation in fp32, each rounded; one rounding to the element type.  Channels from rot_dim on stay.
 * Text uses one axis; with several a token of an image or a video has a position on each, and
 * axis_of says which frequencies belong to which (any assignment).
 */
typedef struct {
  int32_t rot_dim;  /* multiple of 16, 16 <= rot_dim <= head_dim */
  int32_t n_axes;   /* 1 to 4 */
  int32_t pairs;    /* CQP_PAIRS_* */
  int32_t reserved; /* 0 */
  const float *inv_freq;   /* device [rot_dim / 2], 4-byte aligned */
  uint8_t axis_of[128];    /* [rot_dim / 2], each < n_axes */
} cqp_rope_t;

/*
 * Turns the heads of one or two tensors (queries and keys), in one launch.
 *   positions  in : device int32 [n_axes, n_tokens], 4-byte aligned, any values
 *   in, out       : host arrays of n_tensors (1 or 2) entries; out[i] may be in[i] (same data and strides: in
 *                   place), otherwise they must not overlap
 *   backward      : 0, or 1 for the rotation by the opposite angles - the inverse, and the
 *                   gradient (in = gradient of the result, out = gradient of the argument)
 * n_tokens == 0 is a successful no-op.  NaN and infinities stay in their pairs.
 * Errors: CQ_ERR_NULL, CQ_ERR_ALIGN, CQ_ERR_SHAPE, CQ_ERR_UNSUPPORTED (dtype, pairs), CQ_ERR_HIP.
 */
int cqp_rotate(const cqp_rope_t *rope, const int32_t *positions, int32_t n_tokens, int32_t head_dim,
               int32_t dtype, int32_t backward, const cqp_heads_t *in, const cqp_heads_t *out,
               int32_t n_tensors, void *stream);

/*
 * Appends the new tokens' keys and values to the cache, in one launch.
 *   k, v       in : [n_tokens, n_kv_heads, head_dim]
 *   rope, positions in : the keys are turned as by cqp_rotate before they are coded, without a
 *                   rounding between; both NULL: they are taken as they are
 *   q_in, q_out   : both NULL, or queries [n_tokens, n_q_heads, head_dim] to be turned as by cqp_rotate in the
 *                   same launch (in place or apart); needs rope
 * For a page of a sequence and a KV head: scale = the smallest power of two s >= 2^-100 with |x| <=
 * 448 s for every finite new element x of the page, or the page's present scale if that is larger and the page
 * held tokens before (its slot 0 is not among the new ones).  Where the scale grows, the page's codes
 * are brought to the new one (rounded to nearest even: exact but for codes that become subnormal).
 * Codes are rounded to nearest even; a NaN or an infinity becomes a NaN code and leaves the scale to the
 * others.  Slots of no new token keep their codes but for that growth.
 * Tokens whose page is not there, or whose place in the sequence is negative, are dropped.  Within a
 * call no page may be written by two sequences.
 * The result depends on the arguments alone, not on how the work is spread.  Tokens appended one by one
 * and at once get the same scales; their codes differ where a scale grew in between.
 * Errors: as cqp_rotate (CQ_ERR_SHAPE also for more work than a launch can hold: 2^32 threads).
 */
int cqp_append_kv(const cqp_cache_t *cache, const cqp_batch_t *batch, int32_t n_tokens, int32_t dtype,
                  const cqp_heads_t *k, const cqp_heads_t *v, const cqp_rope_t *rope,
                  const int32_t *positions, const cqp_heads_t *q_in, const cqp_heads_t *q_out,
                  void *stream);

/* Bytes of scratch cqp_attn needs (a multiple of 256, > 0) for this cache, these bounds, n_tokens and
 * n_q_heads; depends on nothing in device memory.  0 if an argument is invalid. */
size_t cqp_attn_workspace_bytes(const cqp_cache_t *cache, const cqp_batch_t *batch, int32_t n_tokens,
                                int32_t n_q_heads);

/*
 * out = softmax(softmax_scale * q K^T) V over the tokens of each row's sequence in the cache.
 *   q    in : [n_tokens, n_q_heads, head_dim], n_q_heads a multiple of n_kv_heads; query head hq
 *             reads KV head hq / (n_q_heads / n_kv_heads)
 *   out  out: the same shape and type; it must not overlap q
 *   lse  out: NULL, or fp32 [n_tokens, n_q_heads] (dense): the natural logarithm of the sum of
 *             exp(softmax_scale * q . k) - with it results over several caches are joined
 *   causal  : 1: a row sees the tokens of its sequence up to its own; 0: all seq_lens[b] tokens
 *   softmax_scale: 0 means 1/sqrt(head_dim)
 *   workspace: device, 256-byte aligned, at least cqp_attn_workspace_bytes(); contents undefined before and
 *             after; calls that overlap in time must not share it
 * Tokens of pages that are not there are not attended.  A row that sees no token gives zeros and
 * lse = -infinity.  A NaN in the key or value of a token reaches the rows that see that token - at
 * least their affected channels - and no others.
 * Products are exact in the fp16 matrix cores' fp32 sums (the queries of a row are
 * scaled by a power of two first); weights are rounded to fp16 for their products, to a pair of
 * fp16 where the element type is fp16 and max_new times the query heads of a KV head is at most
 * 64; their sums take them unrounded, in fp32.
 * The result depends on the arguments alone: the same call gives the same bits.
 * Errors: CQ_ERR_NULL, CQ_ERR_ALIGN, CQ_ERR_SHAPE (also for more work than a launch can hold),
 * CQ_ERR_UNSUPPORTED, CQ_ERR_WORKSPACE, CQ_ERR_HIP.
 */
int cqp_attn(const cqp_cache_t *cache, const cqp_batch_t *batch, int32_t n_tokens, int32_t dtype,
             const cqp_heads_t *q, const cqp_heads_t *out, float *lse, int32_t causal,
             float softmax_scale, void *workspace, size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* CQ_PAGED_H_ */
