/*
 * ps_soft — operators over a whole item table on one MI355X (gfx950): softmax cross
 * entropy, distillation from a teacher's top scores (both with the gradients of both
 * tables) and each row's k best items.  None of them stores the rows x items matrix of
 * scores.  C ABI: plain pointers and sizes only.
 *
 * A row (a user of a factor model, a token) holds K numbers x_i, an item holds K numbers
 * w_j, and s_ij = x_i . w_j is the row's score of the item:
 *   ps_soft_xent     row i has target items j with values v.  With lse_i = log sum_j exp s_ij
 *                      loss_i = sum over its targets of v (lse_i - s_ij)
 *                    and, of sum_i weight_i loss_i,
 *                      dX_i = weight_i (V_i sum_j p_ij w_j - sum over its targets of v w_j)
 *                      dW_j = sum_i weight_i V_i p_ij x_i - sum over targets (i, j) of weight_i v x_i
 *                    with p_ij = exp(s_ij - lse_i) and V_i the sum of the row's values.
 *   ps_soft_distill  a teacher scored k items of each row; with q its softmax at temperature
 *                    tau (over the k, or over all its items if its log-sum-exp is given),
 *                    p_ij = exp(s_ij / tau - lse_i), lse_i = log sum_j exp(s_ij / tau):
 *                      loss_i = tau^2 sum over the k of q (log q - log p)
 *                    and the gradients of sum_i weight_i loss_i: those above with v = q,
 *                    V_i = sum q and weight_i tau for weight_i.
 *   ps_soft_top      the k items of the largest scores, in decreasing order, equal scores by
 *                    increasing item.  The order is that of the scores in 64 bits (products
 *                    of the given numbers exact, sums rounded to 53 bits): it does not depend
 *                    on how the work was split.
 *
 * Conventions for every call:
 *   - returns PS_SOFT_OK (0) or a negative code; ps_soft_last_error() gives the message;
 *   - data pointers are DEVICE memory on the handle's device; the caller owns them.  X and W
 *     are row-major with a row stride in elements (ldx, ldw >= K); rows need no alignment
 *     beyond their type's (rows whose address and stride are multiples of 16 bytes are read
 *     fastest).  Outputs must not overlap inputs or each other;
 *   - calls are asynchronous on the handle's stream (ps_soft_set_stream) and read nothing
 *     back: n, entries, k are the host's, ids and row pointers are checked by the kernels.  An
 *     item id >= items makes its row's loss NaN and counts as no target (ps_soft_top: excludes
 *     nothing); so does a row pointer that decreases or lies outside [0, entries] (its row has no
 *     list then; where rows' lists overlap, dW is unspecified); nothing outside the arrays is touched;
 *   - the handle owns a workspace that grows to the largest call seen (growing synchronizes the
 *     stream).  A call that is being captured into a graph cannot grow it: run the same call
 *     once before, or ps_soft_reserve; else PS_SOFT_ESTATE.  A handle that has been captured
 *     keeps every workspace until it is destroyed;
 *   - a handle is not thread-safe, and calls on one handle, replays of graphs that hold its
 *     calls among them, must not overlap: they share the workspace.  Use a handle each;
 *   - the losses scale each table by a power of two and round its numbers: fp32 to 22 bits, but to no
 *     less than 2^-38 of the table's largest finite number (felt below 2^-16 of it; bf16 and f16
 *     numbers are exact above 2^-28 of it).  The softmax's weights have 22 bits, those of a row or of an
 *     item that are far below its largest to 2^-31 of that one (an item's beside targets: to 2^-38 of
 *     the sum of these);
 *     A score is off by about 2^-22 of sum |x_k w_k|, in the same way for rows and items: beyond 10^5 that
 *     is felt where several items share a row's softmax, and dW loses its meaning beyond 10^7;
 *   - equal calls give equal bits: sums have a fixed order, whatever runs beside them.
 */
#ifndef PS_SOFT_H
#define PS_SOFT_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct ps_soft ps_soft_t;

/* return codes */
#define PS_SOFT_OK 0
#define PS_SOFT_EINVAL (-1)  /* bad argument: sizes, null pointers, unknown keys */
#define PS_SOFT_ENOMEM (-2)  /* host or device allocation failed; the handle stays usable */
#define PS_SOFT_EDEVICE (-3) /* a HIP call failed */
#define PS_SOFT_ESTATE (-4)  /* the call cannot be made now (see the workspace above) */

/* element types of X, W, dX and dW */
#define PS_SOFT_F32 0
#define PS_SOFT_BF16 1
#define PS_SOFT_F16 2

/* option keys (ps_soft_set_option) */
#define PS_SOFT_OPT_DEVICE 1 /* HIP device ordinal; -1 (default): the device current at the
                                handle's first device call.  Before that call */
#define PS_SOFT_OPT_SPLITS 2 /* pieces that the reduced axis (items for rows, rows for items) is cut
                                into, in [1, 1024]; 0 (default): by the sizes.  Sums are joined in a
                                fixed order; other pieces round otherwise */
#define PS_SOFT_OPT_SEARCH 3 /* how ps_soft_top searches: 0 all scores in 64 bits; 1 candidates by matrix
                                instructions first (below 2^30 items); -1 (default): the form estimated
                                faster.  Same results, bit for bit */

/*
 * Create a handle for tables of `items` items of K numbers of type `type`.  No device memory
 * is touched.  Limits: 1 <= items <= 2^31 - 65; 1 <= K <= 512.  EINVAL otherwise; *out is NULL
 * on failure.
 */
int ps_soft_create(int64_t items, int32_t K, int32_t type, ps_soft_t **out);

/* Set an option (keys above); EINVAL for an unknown key or value. */
int ps_soft_set_option(ps_soft_t *h, int32_t key, int64_t value);

/* Launch on this HIP stream from now on (a hipStream_t); NULL (the default) is HIP's null stream.
   The new stream waits for the handle's work on the old one, unless it is being captured: then
   that work must be done before.  The caller keeps both alive. */
int ps_soft_set_stream(ps_soft_t *h, void *hip_stream);

/* Grow the workspace to what any call with at most n rows, `entries` targets or exclusions and
   `top` items per row needs. */
int ps_soft_reserve(ps_soft_t *h, int64_t n, int64_t entries, int32_t top);

/*
 * Softmax cross entropy of n rows X (n x K, stride ldx) over the items W (items x K, stride
 * ldw), and its gradients.
 *   row_ptr, item, value, entries: the targets of row i are entries row_ptr[i] .. row_ptr[i+1]
 *     of item and value (value NULL: all 1); row_ptr NULL: one target per row, entries = n.  An
 *     item < 0 is no target (its value is not read as a number); an item twice counts twice.
 *   weight [n], or NULL: all 1.  A row without target or of weight 0 is masked: it is read as a
 *     row of zeros (whatever it holds), its loss and gradient are 0.
 *   loss [n], lse [n]: fp32; NULL: not wanted.
 *   dX (n x K, stride lddx), dW (items x K, stride lddw): of the handle's type, sums in fp32
 *     rounded once; NULL: not wanted.  Written, not added to; the space between rows is left.
 * 0 <= n <= 2^26 (n = 0: dW is zero); entries <= 2^31 - 65.
 */
int ps_soft_xent(ps_soft_t *h, int64_t n, const void *X, int64_t ldx, const void *W, int64_t ldw,
                 const int64_t *row_ptr, const int32_t *item, const float *value, int64_t entries,
                 const float *weight, float *loss, float *lse, void *dX, int64_t lddx, void *dW, int64_t lddw);

/*
 * Distillation from a teacher's top scores.
 *   item, score (n x k, row stride ldt >= k): the teacher's k items of each row and its scores of
 *     them (not divided by tau).  An item < 0 (its score is not read as a number) or a score of
 *     -inf is no entry, so shorter lists are padded with either.  k >= 1.
 *   tlse [n], or NULL: the teacher's log sum exp(score / tau) over all its items; with it q does not
 *     add up to 1, and the rest of the teacher's mass is left out of the loss.
 *   tau > 0, finite.
 * The other arguments are those of ps_soft_xent; lse is that of the student's scores / tau; rows
 * without entry are masked.
 */
int ps_soft_distill(ps_soft_t *h, int64_t n, const void *X, int64_t ldx, const void *W, int64_t ldw, int32_t k,
                    const int32_t *item, const float *score, int64_t ldt, float tau, const float *tlse,
                    const float *weight, float *loss, float *lse, void *dX, int64_t lddx, void *dW, int64_t lddw);

/*
 * The k best items of n rows, 1 <= k <= 256.
 *   row_ptr, item, entries: items that row i excludes, as for ps_soft_xent (an item twice is
 *     excluded once, an id outside [0, items) excludes nothing); row_ptr NULL: none.
 *   top_item, top_score (n x k, row stride ldo >= k): int32 and fp32 (the 64-bit score rounded).
 *     Where fewer than k items are left: item -1, score -inf.  A score that is NaN ranks above all.
 */
int ps_soft_top(ps_soft_t *h, int64_t n, const void *X, int64_t ldx, const void *W, int64_t ldw, int32_t k,
                const int64_t *row_ptr, const int32_t *item, int64_t entries, int32_t *top_item, float *top_score,
                int64_t ldo);

/* Message of the last failed call on this handle (never NULL). */
const char *ps_soft_last_error(const ps_soft_t *h);

/* Free everything the handle owns (synchronizes its stream); NULL-safe. */
void ps_soft_destroy(ps_soft_t *h);

#ifdef __cplusplus
}
#endif

#endif /* PS_SOFT_H */
