/*
 * rb_train.h -- C ABI of the training step that the rehearsal buffer feeds (gfx950 / MI355X), library librb_train.so.
 *
 * The buffer (rb.h) augments every mini-batch with representatives (Listing 1 of the paper: train(m_augmented)).  Here is what a
 * training program computes at that augmented mini-batch at both ends of its model:
 *   rb_scorer  log probabilities of given tokens (or classes) under rows of logits, the rows' entropy and top alternatives, and the
 *              gradient of these with respect to the logits.  The alternatives of a sample are small enough to be kept in its row of
 *              the buffer; when the sample is rehearsed, its stored alternatives are given tokens and the weighted sum of their log
 *              probabilities is the distillation loss.
 *   rb_ortho   an update orthogonalised by Newton-Schulz products, alone or within the optimiser step that applies it.
 *
 * Conventions are those of rb.h: handles are host memory; device memory (inputs, outputs, workspace) and streams are the caller's and
 * only borrowed; the hot calls (score, grad, apply, step) check what the host can see, enqueue on the given stream and return without
 * synchronising; all functions return RB_OK or a negative rb_status, nothing aborts or throws, and on an error of the arguments or of
 * the handle's state nothing was enqueued.  Handles hold no results: every call computes from its arguments alone.  Calls on one handle
 * share its workspace: they go to one stream, or the caller orders the streams, and no two host threads call at once.
 * Every result is bit for bit reproducible (no sum depends on the order in which workgroups run).
 */
#ifndef RB_TRAIN_H
#define RB_TRAIN_H

#include "rb.h"

#ifdef __cplusplus
extern "C" {
#endif

#define RB_MAX_VOCAB (1 << 28)     /* largest number of logits in a row                        */
#define RB_MAX_ROWS (1 << 23)      /* most rows of one call                                    */
#define RB_MAX_GIVEN 64            /* most given tokens per row                                */
#define RB_MAX_TOP 64              /* most alternatives per row                                */
#define RB_MAX_DIM 65536           /* longest side of a matrix                                 */
#define RB_MAX_MATRICES 65535      /* most matrices of one handle                              */
#define RB_MAX_ORTHO_STEPS 16      /* most Newton-Schulz steps                                 */

/* ---- scores of tokens ---------------------------------------------------- */

typedef struct rb_scorer rb_scorer;

/*
 * Describe rows of `vocab` logits of type `dtype` (RB_F32, RB_BF16), `given` tokens per row to be scored and `top` alternatives to be
 * reported.  Host-only.  RB_EINVAL: null out, vocab < 1 or > RB_MAX_VOCAB, unknown dtype, given < 0 or > RB_MAX_GIVEN, top < 0,
 * > RB_MAX_TOP or > vocab.
 */
int rb_scorer_create(rb_scorer **out, int64_t vocab, int32_t dtype, int64_t given, int64_t top);

/* Bytes of workspace rb_scorer_bind wants (5 KB without alternatives, 2 KB more for each, whatever the number of rows: it serves calls of few
 * rows, whose rows are shared by several workgroups). */
int rb_scorer_query(const rb_scorer *s, size_t *workspace_bytes);

/* Attach the workspace (device, 256-byte aligned, of at least the queried size) and enqueue its clearing on hip_stream; it stays borrowed
 * until rb_scorer_destroy or the next bind.  RB_EINVAL: null or misaligned. */
int rb_scorer_bind(rb_scorer *s, void *workspace, void *hip_stream);

/*
 * For each of `rows` rows z[0..vocab) of `logits` (device; row i begins row_stride * i elements behind the first, row_stride >= vocab; any
 * alignment that the element type allows), in binary32:
 *   lse      log of the sum of e^z[j]                                                     -> lse[row]      (may be null)
 *   log probabilities  z[t] - lse of the given tokens t = tokens[row][0..given)           -> logp[row][given]
 *   entropy  -sum of p[j] log p[j] with p[j] = e^(z[j] - lse)                             -> entropy[row]  (may be null)
 *   the `top` largest logits, largest first, equal ones by lowest index: their indices    -> top_ids[row][top]
 *            and log probabilities                                                        -> top_logp[row][top]
 * A given token outside [0, vocab) is left out: its log probability is 0.  A logit of -inf is masked: probability 0, log probability
 * -inf, nothing added to the entropy.  A row whose logits are all -inf has lse -inf, entropy 0, log probabilities -inf.  A row that holds
 * a NaN or +inf has NaN everywhere and indices -1.  `tokens`, `logp` and the two of the alternatives may be null only if there are none.
 * The logits are read once.  rows = 0 is a no-op.  The time depends on the logits where there are alternatives: rows that rise along their
 * indices, in which every logit is one when it comes, take up to about twice that of rows in no order.
 * RB_EINVAL: null or misaligned pointers, rows < 0 or > RB_MAX_ROWS, row_stride < vocab.  RB_ESTATE: not bound.
 */
int rb_scorer_score(rb_scorer *s, const void *logits, int64_t rows, int64_t row_stride, const int64_t *tokens, float *logp, float *lse,
                    float *entropy, float *top_logp, int64_t *top_ids, void *hip_stream);

/*
 * The gradient with respect to the logits of a loss that depends on the log probabilities with the derivatives grad_logp[row][given] and
 * on the entropies with the derivatives grad_entropy[row] (may be null: not at all):
 *   grad_logits[j] = -p[j] * (W + grad_entropy * (log p[j] + entropy)) + sum of the grad_logp of the given tokens that are j,
 * W the sum of grad_logp over the given tokens that are not left out.  lse and entropy are rb_scorer_score's for these logits (entropy may
 * be null where grad_entropy is).  Computed in binary32, rounded once to the logits' type.  A masked logit's p is 0 (its gradient only what
 * is given for it).  p is as exact as the lse it is given: the rounding of lse to binary32, up to 2^-24 |lse|, is a relative error of p.  A row whose
 * lse is -inf has gradient 0, one whose lse is NaN has NaN.  grad_logits may be the logits themselves (the same
 * pointer and stride); otherwise the two must not overlap.  Logits are read once, gradients written once; rows of the two that lie alike
 * relative to 16 bytes are moved 16 bytes at a time, others element by element.
 * RB_EINVAL: as above, grad_stride < vocab, grad_entropy without entropy.  (The workspace is not used: bound or not.)
 */
int rb_scorer_grad(rb_scorer *s, const void *logits, int64_t rows, int64_t row_stride, const int64_t *tokens, const float *lse,
                   const float *entropy, const float *grad_logp, const float *grad_entropy, void *grad_logits, int64_t grad_stride,
                   void *hip_stream);

/* Free the host handle.  Device memory stays the caller's. */
int rb_scorer_destroy(rb_scorer *s);

/* ---- orthogonalised updates ---------------------------------------------- */

typedef struct rb_ortho rb_ortho;

/*
 * Describe `matrices` matrices of m x n, updates (gradients) of type `dtype`, results (weights) of type `out_dtype`, and `steps`
 * Newton-Schulz steps with the coefficients (a, b, c) = coefficients[3 i .. 3 i + 2] (HOST array) in step i.  Host-only.
 * The method, per matrix G with m <= n (otherwise of its transpose): X = G / (|G| + eps), |G| the Frobenius norm; in every step
 * A = X X^T, X <- a X + (b A + c A A) X.  Every singular value s of G / (|G| + eps) becomes the polynomials' value at s.
 * Operands of the products are held as sums of two binary16 numbers, sums in binary32; that holds singular values up to 4 in every step: RB_EINVAL for
 * coefficients that lead a value of [0, 1] beyond.
 * Precision.  Such a sum has 22 bits of an element but no steps finer than 2^-36 in X, 2^-35 in A and 2^-34 in what X is multiplied by, |G| + eps being
 * 1: elements of X under about 2^-14 have fewer bits.  In the norm of a whole matrix a result is as near the exact one as the same steps in binary32 are (at
 * most 4 times as far off; twice was seen, mostly nearer).  Relative to its own norm a row or column that is much smaller than the rest is not: one of k elements whose
 * norm is r times |G| + eps is off by about 2^-38 sqrt(k) / r of itself besides, and by no more than 2^-36 (sqrt(k) + 64) / r with the usual coefficients (the
 * same steps in binary32: by some 1e-6 whatever r is).  With rows whose sizes fall evenly from the first to the last, rows of 1/1000 of the first's size are
 * off by 3e-7 at 256 x 256 and 3e-6 at 4096 x 4096, of 1e-6 by 2e-4 and 3e-3.  (Matrices of up to 128 x 128: X itself is binary32, 1e-6 at 1e-6.)
 * So it is with all rows of a matrix whose |G| is far below eps.
 * A NaN or an infinity in a matrix makes all of its result NaN, and no other matrix's.
 * RB_EINVAL also: null pointers, matrices < 1 or > RB_MAX_MATRICES, m, n < 1 or > RB_MAX_DIM, unknown types, steps < 1 or >
 * RB_MAX_ORTHO_STEPS, a coefficient or eps that is not finite, eps < 0.
 */
int rb_ortho_create(rb_ortho **out, int64_t matrices, int64_t m, int64_t n, int32_t dtype, int32_t out_dtype,
                    const float *coefficients, int64_t steps, float eps);

/* Bytes of workspace rb_ortho_bind wants: about 20 bytes per element of the matrices for large ones. */
int rb_ortho_query(const rb_ortho *o, size_t *workspace_bytes);

/* Attach the workspace (device, 256-byte aligned); nothing is enqueued.  It stays borrowed until rb_ortho_destroy or the next bind. */
int rb_ortho_bind(rb_ortho *o, void *workspace);

/*
 * out <- the orthogonalised update, matrix by matrix.  Element (i, j) of matrix k is at k * matrix_stride + i * row_stride + j (strides in
 * elements; matrices may lie behind each other or side by side).  out may be the update itself if the types and strides are the same;
 * otherwise the two must not overlap, and no two elements of out may be at one place.
 * RB_EINVAL: null or misaligned pointers, row_stride < n, a negative matrix_stride, for out one under n with several matrices.  RB_ESTATE: not bound.
 */
int rb_ortho_apply(rb_ortho *o, const void *update, int64_t update_matrix_stride, int64_t update_row_stride, void *out,
                   int64_t out_matrix_stride, int64_t out_row_stride, void *hip_stream);

/*
 * A whole optimiser step with orthogonalised updates, in place, elementwise in binary32:
 *   momentum <- beta * momentum + grad;   U = grad + beta * momentum (nesterov != 0) or momentum;   O = U orthogonalised;
 *   weight <- (1 - lr * weight_decay) * weight - lr * scale * O
 * weight is of the handle's out_dtype, grad of its dtype, momentum binary32 and contiguous (matrices x m x n).  The three must not overlap.
 * RB_EINVAL: as above, a factor that is not finite.  RB_ESTATE: not bound.
 */
int rb_ortho_step(rb_ortho *o, void *weight, int64_t weight_matrix_stride, int64_t weight_row_stride, const void *grad,
                  int64_t grad_matrix_stride, int64_t grad_row_stride, float *momentum, float lr, float beta, int32_t nesterov,
                  float weight_decay, float scale, void *hip_stream);

/* Free the host handle.  Device memory stays the caller's. */
int rb_ortho_destroy(rb_ortho *o);

#ifdef __cplusplus
}
#endif
#endif /* RB_TRAIN_H */
