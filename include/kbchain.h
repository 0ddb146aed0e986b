/*
 * kbchain.h -- C ABI of the multi-hop chain glue (gfx950), a harness library
 * beside kbfollow.h, and of the operators before a hop: embedding lookup and
 * penalties, biases and masks on logits (below).
 *
 * The multi-hop question-answering model of Sec. 3.2 chains follow steps,
 * x^t = follow(x^{t-1}, r^t), takes a softmax of the last hop's entity
 * weights and a cross-entropy loss against the answer set written as a
 * distribution.  Between the follow calls the chain needs a few column-wise
 * operations, provided here so that a whole chain, forward and backward, runs
 * in this project's kernels:
 *   r^t = softmax(rho^t) over the relations (and its backward),
 *   x^t = u^t / sum(u^t) over the entities, one sum per example (and its
 *         backward),
 *   the softmax cross-entropy of the last hop (loss and gradient).
 *
 * Layout: every array is entity-major (or relation-major) and
 * batch-contiguous float32 [n][b], element (i, beta) at i * b + beta, as in
 * kbfollow.h; each of the b columns is one example and every reduction runs
 * over the n rows of a column.  Reductions are taken in double, in a fixed
 * order (bitwise reproducible), and every float output is rounded once.
 *
 * Streams and memory: every call only enqueues work on `stream` (hipStream_t,
 * NULL = null stream), allocates nothing and returns.  All pointers are
 * DEVICE pointers; input and output arrays must not overlap unless stated.
 * A workgroup reduces 4, 8 or 16 columns over all n rows.  Columns of more than a
 * few thousand rows are better cut into ranges of rows, whose partial values
 * need device scratch: the *_scratch forms take it (kbc_scratch_size bytes, 8-byte
 * aligned, used by that call alone until it has run), and are the plain forms
 * when it is NULL.
 *
 * Errors: arguments are checked before anything is enqueued; on failure
 * nothing is launched.  Returns KBC_OK, KBC_EINVAL (null pointer, n < 1 or
 * b < 1) or KBC_EHIP (launch failure).
 */
#ifndef KBCHAIN_H
#define KBCHAIN_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { KBC_OK = 0, KBC_EINVAL = 1, KBC_EHIP = 4 } kbc_status;

/* p[:, beta] = softmax(z[:, beta]) over the n rows:
 * exp(z - max) / sum(exp(z - max)), in double.  z, p: [n][b]. */
kbc_status kbc_softmax(int64_t n, int32_t b, const float *z, float *p, void *stream);

/* Backward of kbc_softmax: dz = p (.) (dp - <dp, p>), the inner product per
 * column.  p is softmax's output; dp the upstream gradient.  All [n][b]. */
kbc_status kbc_softmax_backward(int64_t n, int32_t b, const float *p, const float *dp, float *dz,
                                void *stream);

/* L1 normalisation per column: sums[beta] = sum_i u[i, beta] (double), and
 * x = u / sums.  u, x: [n][b]; sums: DEVICE double[b], written.  For
 * non-negative u (entity weights). */
kbc_status kbc_l1_normalize(int64_t n, int32_t b, const float *u, float *x, double *sums,
                            void *stream);

/* Backward of kbc_l1_normalize: du = (dx - <dx, x>) / sums, per column.
 * x: the normalised output; sums: as written by kbc_l1_normalize. */
kbc_status kbc_l1_normalize_backward(int64_t n, int32_t b, const float *x, const double *sums,
                                     const float *dx, float *du, void *stream);

/* Softmax cross-entropy of logits z against targets t (both [n][b]),
 * averaged over the b examples:
 *   col_loss[beta] = -sum_i t[i, beta] * log softmax(z[:, beta])[i]   (double[b])
 *   loss[0]        = (sum over beta of col_loss, in order) / b         (double[1])
 *   dz             = (softmax(z) * sum_i t[i, beta] - t) / b            ([n][b])
 * (dz is the gradient of loss[0]; with targets summing to 1 per column it is
 * (softmax(z) - t) / b). */
kbc_status kbc_softmax_xent(int64_t n, int32_t b, const float *z, const float *t,
                            double *col_loss, double *loss, float *dz, void *stream);

/* Scratch that the *_scratch forms use at this shape (0: none; any pointer,
 * NULL too, gives the plain form then).  A non-NULL scratch of fewer bytes is
 * KBC_EINVAL. */
size_t kbc_scratch_size(int64_t n, int32_t b);
kbc_status kbc_softmax_scratch(int64_t n, int32_t b, const float *z, float *p, void *scratch,
                               size_t bytes, void *stream);
kbc_status kbc_softmax_backward_scratch(int64_t n, int32_t b, const float *p, const float *dp,
                                        float *dz, void *scratch, size_t bytes, void *stream);
kbc_status kbc_l1_normalize_scratch(int64_t n, int32_t b, const float *u, float *x, double *sums,
                                    void *scratch, size_t bytes, void *stream);
kbc_status kbc_l1_normalize_backward_scratch(int64_t n, int32_t b, const float *x,
                                             const double *sums, const float *dx, float *du,
                                             void *scratch, size_t bytes, void *stream);
kbc_status kbc_softmax_xent_scratch(int64_t n, int32_t b, const float *z, const float *t,
                                    double *col_loss, double *loss, float *dz, void *scratch,
                                    size_t bytes, void *stream);

/* ------------------------------------------------------------------------
 * Embedding lookup with scaling
 * ------------------------------------------------------------------------
 *
 * The words of a question become the vector that its relation logits are taken
 * from: rows of a table, scaled, one output row per token or pooled per question.
 * Rows are row-major here, [rows][dim], the transpose of the arrays above:
 *   ids    : `tokens` ids, id_bytes 4 (int32) or 8 (int64) each.  An id outside
 *            [0, rows) stands for padding: a row of zeros, no term of a sum, no
 *            gradient.
 *   table  : [rows][dim] of `type`, row r at r * stride elements (stride >= dim).
 *   out, dout, dtable : contiguous, of `type`.
 * Any element alignment will do.  1 <= rows < 2^31 - 1, tokens <= 2^30, bags <
 * 2^31 - 1 (2^25 with mean), 1 <= dim <= 65536, else KBC_EINVAL.  Sums are taken in double, in a
 * fixed order (partial sums of float16 outputs in float); an output is rounded to
 * float, and to a 16-bit type from there.
 */
typedef enum { KBC_F32 = 0, KBC_BF16 = 1, KBC_F16 = 2 } kbc_type;

/* out[t] = scale * table[ids[t]], [tokens][dim]. */
kbc_status kbc_embed(int64_t tokens, const void *ids, int32_t id_bytes, int64_t rows, int32_t dim,
                     const void *table, int64_t stride, kbc_type type, float scale, void *out,
                     void *stream);

/* out[g] = scale * sum over the tokens t of bag g of table[ids[t]], [bags][dim];
 * mean != 0: divided by the number of those that are no padding.  A bag without
 * any is zeros.
 *   offsets : bags + 1 of them, of the ids' integer type, not decreasing: bag g is
 *             tokens [offsets[g], offsets[g + 1]) (values outside [0, tokens] are
 *             taken as the nearer end).  NULL: every bag has tokens / bags tokens,
 *             which has to be whole.
 *   scratch : kbc_embed_pool_scratch_size bytes (ragged: offsets are given), 16-byte
 *             aligned, used by this call alone until it has run. */
size_t kbc_embed_pool_scratch_size(int64_t tokens, int64_t bags, int32_t ragged, int32_t dim,
                                   kbc_type type, int32_t mean);
kbc_status kbc_embed_pool(int64_t tokens, const void *ids, int32_t id_bytes, int64_t bags,
                          const void *offsets, int64_t rows, int32_t dim, const void *table,
                          int64_t stride, kbc_type type, float scale, int32_t mean, void *out,
                          void *scratch, size_t bytes, void *stream);

/* Gradient of either with respect to the table, fully written, [rows][dim]:
 *   dtable[v] = sum over t with ids[t] == v of scale * dout[t]          (bags == 0)
 *               ... of scale (/ tokens of the bag) * dout[bag of t]     (bags > 0)
 * Rows that no token names are zeros. */
size_t kbc_embed_backward_scratch_size(int64_t tokens, int64_t bags, int32_t dim, kbc_type type,
                                       int32_t mean);
kbc_status kbc_embed_backward(int64_t tokens, const void *ids, int32_t id_bytes, int64_t bags,
                              const void *offsets, int64_t rows, int32_t dim, const void *dout,
                              kbc_type type, float scale, int32_t mean, void *dtable,
                              void *scratch, size_t bytes, void *stream);

/* ------------------------------------------------------------------------
 * Penalties, biases and masks on logits
 * ------------------------------------------------------------------------
 *
 * What a column of logits z [n][b] may still take, before its softmax: relations
 * or words that it has had already are made less likely, biases are added, what a
 * type, a grammar or a question rules out is masked.  With c the number of times
 * row i is in column beta's history:
 *   v = z[i][beta]
 *   c > 0:  v = v > 0 ? v / repeat : v * repeat;  v -= presence + frequency * c
 *   v += bias
 *   not allowed:  v = fill, whatever z holds there
 */
typedef struct {
  const float *bias;      /* DEVICE [n], or [n][b] with bias_each; NULL: none */
  const void *allowed;    /* DEVICE bytes (0: not allowed), or with allowed_bits 32-bit words, of
                             which bit i % 32 of word i / 32 is row i's: [rows], or [rows][b] with
                             allowed_each (rows: n, or words, ceil(n / 32)); NULL: all */
  int32_t bias_each, allowed_bits, allowed_each;
  int32_t id_bytes;       /* of history and offsets: 4 (int32) or 8 (int64) */
  int64_t entries;        /* ids in all histories, at most 2^30; 0: none */
  const void *history;    /* DEVICE ids; those outside [0, n) are padding */
  const void *offsets;    /* DEVICE [b + 1], not decreasing: column beta's are [offsets[beta],
                             offsets[beta + 1]); NULL: entries / b of each column */
  const float *repeat, *presence, *frequency; /* DEVICE [b], one a column, or NULL: */
  float repeat_all, presence_all, frequency_all; /* for all columns (none: 1, 0, 0) */
} kbc_limits;

/* out [n][b], float, of logits z [n][b] of `type`; out must not overlap z.  Every
 * element is rounded to float once, n < 2^31 - 1.  KBC_EINVAL also where a penalty of
 * all columns is not finite or repeat_all not positive (a column's own repeat has to
 * be positive too; it is not checked).  With a frequency a column may have up to 2^26
 * ids (with offsets: all of them together), else KBC_EINVAL. */
kbc_status kbc_constrain(int64_t n, int32_t b, const void *z, kbc_type type, const kbc_limits *l,
                         float fill, float *out, void *stream);

/* Gradients for the upstream gradient dout [n][b]: dz [n][b] of `type`,
 *   dz = not allowed ? 0 : dout * (c > 0 ? (z > 0 ? 1 / repeat : repeat) : 1),
 * and unless NULL dbias, [n][b] with bias_each, else [n], summed over the columns in
 * double, in a fixed order.  z may be NULL where no repeat is given.  The outputs
 * must not overlap each other or any input. */
kbc_status kbc_constrain_backward(int64_t n, int32_t b, const void *z, kbc_type type,
                                  const kbc_limits *l, const float *dout, void *dz, float *dbias,
                                  void *stream);

#ifdef __cplusplus
}
#endif

#endif /* KBCHAIN_H */
