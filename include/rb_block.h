/*
 * rb_block.h -- C ABI of what a block of a model computes between its matrix products (gfx950 / MI355X), library librb_block.so.
 *
 * The buffer (rb.h) makes the augmented mini-batch, rb_train.h has both ends of the training step on it.  Here is what lies between, for models that
 * have it: normalised rows, dropout, attention.
 *   rb_norm       layer norm of rows, alone or of the sum of a residual row and a row that goes through dropout, and its gradients.
 *   rb_dropout    dropout alone.
 *   rb_attention  attention of packed documents - fresh and rehearsed sequences of any lengths behind one another - and its gradients.
 *
 * Conventions are those of rb.h and rb_train.h: handles are host memory; device memory (inputs, outputs, workspace) and streams are the caller's and only
 * borrowed; the hot calls check what the host can see, enqueue on the given stream and return without synchronising; all functions return RB_OK or a
 * negative rb_status, nothing aborts or throws, and on an error of the arguments or of the handle's state nothing was enqueued.  Handles hold no results.
 * Calls on one handle share its workspace: they go to one stream, or the caller orders the streams, and no two host threads call at once.
 * Calls may be captured into a graph.  Every result is bit for bit reproducible (no sum depends on the order in which workgroups run).
 */
#ifndef RB_BLOCK_H
#define RB_BLOCK_H

#include "rb.h"

#ifdef __cplusplus
extern "C" {
#endif

#define RB_MAX_NORM_ROWS (1 << 23)     /* most rows of a call of rb_norm_* and rb_dropout         */
#define RB_MAX_NORM_WIDTH 32768        /* longest row of rb_norm                                  */
#define RB_MAX_DROP_WIDTH (1 << 27)    /* longest row of rb_dropout                               */
#define RB_MAX_HEADS 1024              /* most heads of queries                                   */
#define RB_MAX_HEAD_DIM 128            /* longest row of a head                                   */
#define RB_MAX_TOKENS (1 << 22)        /* most positions of a call                                */
#define RB_MAX_HEAD_ROWS (1 << 30)     /* most positions times heads of queries                   */
#define RB_MAX_DOCUMENTS (1 << 22)     /* most documents of a call                                */

/* ---- dropout ------------------------------------------------------------- */

/*
 * Dropout of rows.  The element in row i and column j stays if its 16 random bits, as a number, are at least P = p * 65536 to the nearest integer (half to even),
 * and is then multiplied by 65536 / (65536 - P), rounded to binary32: its expectation is the element's own, whatever p is rounded to.  Otherwise it is
 * 0, whatever it was.  The bits are the j % 8-th of the eight halves (low ones first) of the output words of Philox4x32-10 with
 *   counter = (i, 2^31 + j / 8, step's low half, step's high half), key = (seed's low half, seed's high half),
 * a function of (seed, step, row, column) alone: nothing is stored, the gradient's call is the same call on the gradients, and what rows lie
 * apart by, their type and who else is in the mini-batch do not matter.  The buffer's draws (rb.h) use other counters: one seed may serve both.
 * Layers of one training step have a `step` (or a seed) of their own each.  seed and step are read when a call is made: one that was captured into a graph
 * drops the same elements in every replay.  A graph that trains leaves dropout's calls out, is captured anew, or has p = 0.
 */
typedef struct rb_drop {
    double p;              /* 0 <= p <= 1; 1: nothing stays                          */
    uint64_t seed, step;
} rb_drop;

/*
 * out <- dropout(x): rows of `width` elements of type `dtype` (RB_F32, RB_BF16), row i `stride` * i elements behind the first; any alignment
 * that the element type allows.  out may be x with the same stride (otherwise the two must not overlap).  Products in binary32, rounded once.
 * rows = 0 is a no-op.
 * RB_EINVAL: null or misaligned pointers, unknown dtype, rows < 0 or > RB_MAX_NORM_ROWS, width < 1 or > RB_MAX_DROP_WIDTH, a stride < width,
 * p not in [0, 1].
 */
int rb_dropout(const void *x, int64_t x_stride, int64_t rows, int64_t width, int32_t dtype, const rb_drop *drop, void *out, int64_t out_stride,
               void *hip_stream);

/* ---- layer norm ---------------------------------------------------------- */

typedef struct rb_norm rb_norm;

/*
 * Describe rows of `width` elements of type `dtype`, weights (and biases) of type `weight_dtype` (RB_F32, RB_BF16), and what is added to the
 * variance.  Host-only.  RB_EINVAL: null out, width < 1 or > RB_MAX_NORM_WIDTH, unknown types, eps not positive and finite.
 */
int rb_norm_create(rb_norm **out, int64_t width, int32_t dtype, int32_t weight_dtype, float eps);

/* Bytes of workspace rb_norm_bind wants (4 KB for each column: sums of the weights' gradients; the forward pass uses none). */
int rb_norm_query(const rb_norm *n, size_t *workspace_bytes);

/* Attach the workspace (device, 256-byte aligned); nothing is enqueued.  It stays borrowed until rb_norm_destroy or the next bind. */
int rb_norm_bind(rb_norm *n, void *workspace);

/* Rows on the device: row i begins stride * i elements behind `data`; any alignment that the element type allows. */
typedef struct rb_rows {
    void *data;
    int64_t stride;
} rb_rows;

/*
 * For each of `rows` rows, in binary32:
 *   total = residual + dropout(x), rounded to dtype               -> total     (without residual: dropout(x); without drop: residual + x)
 *   mean = the mean of total, rstd = 1 / sqrt(mean of (total - mean)^2 + eps), of total as it was rounded    -> mean[row], rstd[row]
 *   y = (total - mean) * rstd * weight + bias, rounded to dtype   -> y
 * residual, drop, bias may be null (none).  total->data may be null only if there is neither residual nor drop: total is x then.
 * mean and rstd may be null.  weight and bias: `width` elements of weight_dtype, contiguous.  y or total may be x, or total residual
 * (same pointer and stride); otherwise what is written overlaps nothing.  A NaN or infinity in a row's total makes its y NaN and no other row's.
 * A row of equal elements has y = bias, but for what the rounding of its mean leaves.  rows = 0 is a no-op.
 * RB_EINVAL: null or misaligned pointers, rows < 0 or > RB_MAX_NORM_ROWS, a stride < width, p not in [0, 1].
 */
int rb_norm_forward(rb_norm *n, const rb_rows *x, const rb_rows *residual, const rb_drop *drop, int64_t rows, const void *weight, const void *bias,
                    const rb_rows *total, const rb_rows *y, float *mean, float *rstd, void *hip_stream);

/*
 * Gradients of a loss with the derivatives grad_y of y and grad_total of total (may be null: total goes nowhere else).  With h = (total - mean) * rstd
 * and g = grad_y * weight, in binary32:
 *   d = rstd * (g - mean(g) - h * mean(g * h)) + grad_total   -> grad_sum: the gradient of the sum, so of the residual (and of x without drop), rounded to dtype
 *   dropout(d)                                                -> grad_x, rounded to dtype (needed with drop, null without)
 *   sum over the rows of grad_y * h, of grad_y                -> grad_weight, grad_bias (each may be null), `width` elements of weight_dtype
 * mean and rstd are rb_norm_forward's for this total; what rounding the mean to one number has left is made again from total (of rows far from 0 it may be as large
 * as what they differ by).  grad_sum or grad_x may be grad_y or grad_total, but not both the same (same pointer and stride);
 * otherwise what is written overlaps nothing.  rows = 0: grad_weight and grad_bias become 0.
 * RB_EINVAL: as above; drop without grad_x or grad_x without drop.  RB_ESTATE: not bound.
 */
int rb_norm_grad(rb_norm *n, const rb_rows *grad_y, const rb_rows *total, const rb_rows *grad_total, const float *mean, const float *rstd, const rb_drop *drop,
                 int64_t rows, const void *weight, const rb_rows *grad_sum, const rb_rows *grad_x, void *grad_weight, void *grad_bias, void *hip_stream);

/* Free the host handle.  Device memory stays the caller's. */
int rb_norm_destroy(rb_norm *n);

/* ---- attention of packed documents ---------------------------------------- */

typedef struct rb_attention rb_attention;

/*
 * Describe attention with `heads` heads of queries and `kv_heads` of keys and values (head h reads kv head h / (heads / kv_heads)) of head_dim bfloat16
 * numbers each, for up to max_tokens positions.  causal != 0: a position does not see what is behind it, but for its document's prefix.
 * scale multiplies the products; cap > 0: scores are cap * tanh(score / cap), cap = 0: as they are.  Host-only.
 * RB_EINVAL: null out, heads < 1 or > RB_MAX_HEADS, kv_heads < 1 or no divisor of heads, head_dim < 8, > RB_MAX_HEAD_DIM or no multiple of 8,
 * max_tokens < 1, > RB_MAX_TOKENS or more than RB_MAX_HEAD_ROWS with the heads, scale not positive and finite, cap negative or not finite,
 * scale * log2 e, cap * log2 e or scale / cap beyond binary32's normal numbers (of scale / cap a third of the largest).
 */
int rb_attention_create(rb_attention **out, int64_t heads, int64_t kv_heads, int64_t head_dim, int64_t max_tokens, int32_t causal, float scale, float cap);

/* Bytes of workspace rb_attention_bind wants: 16 a position, 8 a position and head of queries, and what the gradients' parts may need at most, 64 KB (heads of up to
 * 64 numbers; else 128 KB) for each 128 positions of a head of keys times 16, no more than 2048 such (256 MiB).  The forward pass uses the positions' alone. */
int rb_attention_query(const rb_attention *a, size_t *workspace_bytes);

/* Attach the workspace (device, 256-byte aligned); nothing is enqueued.  It stays borrowed until rb_attention_destroy or the next bind. */
int rb_attention_bind(rb_attention *a, void *workspace);

/* Rows of heads on the device: head h of position t begins t * token_stride + h * head_stride elements behind `data`.  All are multiples of 16 bytes; strides
 * are not negative, token_stride is at most 2^26; what is written lies row by row or head by head, no two rows of heads overlap. */
typedef struct rb_heads {
    void *data;
    int64_t token_stride, head_stride;
} rb_heads;

/* Documents on the device.  Document d begins at position offsets[d] and ends before offsets[d + 1], or lengths[d] positions behind its begin if that is
 * nearer (lengths may be null: all positions).  The first prefixes[d] positions of a document are seen by all of it (null: none; means something only if
 * causal).  offsets: count + 1 numbers, none smaller than the one before.  What cannot be (offsets that fall, numbers outside of the positions, negative lengths)
 * is cut to the positions there are: which results such a call has is not specified, but it reads and writes nothing else.
 * The host sees `count` alone, so that is what chooses between the forms below, and documents of no positions count: offsets that are padded to a fixed number
 * with many of them make long documents be taken for short ones, which costs time (and precision only gains). */
typedef struct rb_documents {
    const int64_t *offsets, *lengths, *prefixes;
    int64_t count;
} rb_documents;

/*
 * For every head h and every position i of a document, over the positions j of that document that it sees (j <= i or j in the prefix if causal, else all):
 *   s[j] = scale * (q[i] . k[j]);  s[j] = cap * tanh(s[j] / cap) with a cap;  s[j] -= slopes[h] * |i - j| with slopes (device, `heads` numbers; may be null)
 *   lse = log of the sum of e^s[j]                -> lse[h * tokens + i]  (may be null)
 *   out = sum of e^(s[j] - lse) v[j]              -> out, rounded to bfloat16
 * Products of bfloat16 numbers with sums in binary32; e^(s - max) is rounded to bfloat16 for the product with v, its sum is not.  With less than 128 positions a
 * document in the mean (tokens < 128 * count) it is taken to 2^-17 of itself instead.  slopes may have either sign.  With a cap of up to 32 and more positions than that, scores are
 * off by up to cap * 2^-21; other capped scores are within 2^-20 of themselves.  Positions that belong to no document have out 0 and lse -inf, and what lies there in q, k and v does not matter.  What a position
 * does not see has no influence on it (but for how many positions and documents there are, which choose the form), infinities and NaN included; an infinity in a v[j] that it sees makes out that infinity (or NaN, where its weight is 0
 * in binary32), a NaN NaN.  out overlaps nothing that is read.  tokens = 0 is a no-op.
 * RB_EINVAL: null or misaligned pointers, strides that do not fit, tokens < 0 or > max_tokens, documents' count < 0 or > RB_MAX_DOCUMENTS.
 * RB_ESTATE: not bound.
 */
int rb_attention_forward(rb_attention *a, const rb_heads *q, const rb_heads *k, const rb_heads *v, int64_t tokens, const rb_documents *documents,
                         const float *slopes, const rb_heads *out, float *lse, void *hip_stream);

/*
 * Gradients with respect to q, k and v of a loss with the derivative grad_out of out; out and lse are rb_attention_forward's for the same arguments.  With p =
 * e^(s - lse), dp = grad_out[i] . v[j], ds = p * (dp - sum of p * dp), times the cap's slope and scale:
 *   grad_v[j] = sum over i of p grad_out[i],  grad_q[i] = sum over j of ds k[j],  grad_k[j] = sum over i of ds q[i]
 * (of keys and values over their heads of queries too), sums in binary32, p and ds rounded to bfloat16 for these products (or taken to 2^-17 of themselves,
 * as above), results rounded to bfloat16.  A position that sees one alone has a gradient of q of 0.
 * The sum of p * dp is made in binary32 from the first value grad_out[i] . out[i] on, so that out's rounding does not matter.
 * A position's gradients come of what it sees and of the positions that see it, with what these see; nothing else has an influence.  Where it sees or is seen by a
 * q, k, v or grad_out that is not finite, or one of the positions that see it has an out that is not finite, they are not finite (which of their numbers
 * is not specified).  An infinite k without weight (a score of -inf) matters to itself and to the gradients of q of who sees it, to no other.
 * Positions that belong to no document have gradients 0.  What is written overlaps nothing.  (The slopes have no gradient.)
 * RB_EINVAL, RB_ESTATE: as above.
 */
int rb_attention_grad(rb_attention *a, const rb_heads *q, const rb_heads *k, const rb_heads *v, int64_t tokens, const rb_documents *documents,
                      const float *slopes, const rb_heads *out, const float *lse, const rb_heads *grad_out, const rb_heads *grad_q, const rb_heads *grad_k,
                      const rb_heads *grad_v, void *hip_stream);

/* Free the host handle.  Device memory stays the caller's. */
int rb_attention_destroy(rb_attention *a);

#ifdef __cplusplus
}
#endif
#endif /* RB_BLOCK_H */
