/*
 * tag_policy.h -- C ABI of the operators on the decision head's scores: the
 * raw scores themselves, priors under constraints that the caller knows and
 * the network does not, and the loss that balances the decisions over the
 * devices, with its gradient.
 *
 * Rows are queries, columns the S slices of a table.  Conventions follow
 * tag.h: caller-owned DEVICE buffers, asynchronous on hip_stream, arguments
 * validated before anything is enqueued, no allocation.  Row strides are in
 * elements and at least S; rows may start at any element.  A workspace is
 * scratch for the duration of a call (calls that share one must be ordered);
 * nothing in it needs to start at zero.  But where a call says so, no array that
 * it writes overlaps another of its arrays.
 */
#ifndef TAG_POLICY_H
#define TAG_POLICY_H

#include "tag.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Raw scores of tag_gnn_decide, before its softmax: scores [Q][S] fp32,
 * everything else (arguments, workspace, errors) as in tag_gnn_decide.  An
 * out-of-range query's row is filled with -inf. */
tag_status tag_gnn_scores(const tag_graph *g, const tag_model_dims *dims, const tag_weights *w,
                          int32_t n_replicas, const float *E_op, const float *E_dev, const tag_slices *slices,
                          int32_t n_query, const int32_t *query_rep, const int32_t *query_graph,
                          const int32_t *query_op, float *scores, void *workspace, size_t ws_bytes,
                          void *hip_stream);

/*
 * What a caller knows about the slices of each query.  Every array is DEVICE
 * and may be NULL; a row stride of 0 shares one row among all queries.
 *   allow        bit a % 32 of word a / 32 of a row is set where slice a is
 *                allowed; rows of (S + 31) / 32 words (NULL: all allowed)
 *   bias         added to the scores (NULL: none); -inf forbids too
 *   history      rows of n_history slice ids the query took before, of which
 *                the first history_len[q] count (NULL: all n_history; values
 *                are clamped to [0, n_history], which is at most 2^30); ids
 *                outside [0, S) are ignored
 *   repetition   [Q] divides a taken slice's positive score and multiplies a
 *                negative one (NULL: 1)
 *   presence     [Q] subtracted from a taken slice's score (NULL: 0)
 *   frequency    [Q] subtracted once per time it was taken (NULL: 0)
 */
typedef struct tag_constraints {
    const uint32_t *allow;
    int64_t allow_stride;
    const float *bias;
    int64_t bias_stride;
    const int32_t *history;
    int64_t history_stride;
    int32_t n_history;
    const int32_t *history_len;
    const float *repetition, *presence, *frequency;
} tag_constraints;

/*
 * Constrained priors.  With c_a the number of times slice a stands in the
 * query's history, in fp32, each operation rounded:
 *   y = score                                        (widened from bf16)
 *   y = y > 0 ? y / repetition : y * repetition      if c_a > 0
 *   y = y - frequency * c_a ;  y = y - presence      if c_a > 0
 *   y = y + bias ;  y = -inf                         if a is not allowed
 *   prior = softmax(y),  argmax = lowest index among maxima,  best = max y
 * A row with nothing left (every y = -inf) has an all-zero prior, argmax -1
 * and best -inf.  Whatever stands in a slice that is not allowed (infinities,
 * NaN) has no effect.  A NaN elsewhere gives a prior of NaN, argmax -1 and
 * best NaN; a y of +inf is found by argmax and best, with a prior of NaN.
 *
 *   scores       [Q] rows of S, dtype TAG_F32 or TAG_BF16 (base aligned to its
 *                element)
 *   constrained  y, same type as scores, rounded to it (may be NULL; may be
 *                `scores` itself with its row stride; no other overlap)
 *   prior        fp32 (may be NULL)
 *   argmax, best [Q] int32, fp32
 */
tag_status tag_constrain_workspace(int32_t n_query, int32_t n_slices, size_t *bytes);
tag_status tag_constrain(int32_t n_query, int32_t n_slices, int32_t dtype, const void *scores, int64_t score_stride,
                         const tag_constraints *constraints, void *constrained, int64_t constrained_stride,
                         float *prior, int64_t prior_stride, int32_t *argmax, float *best, void *workspace,
                         size_t ws_bytes, void *hip_stream);

/*
 * Balance loss.  A slice's work is shared equally by its devices:
 * A_ad = [d in mask_a] / popcount(mask_a) over devices d < M = n_dev (other
 * bits are ignored; a slice without a device counts for none).  Over the n
 * rows that are used (use[q] != 0, or use NULL, and some score > -inf):
 *   p      = softmax(scores)                      count_a = #{q : argmax p_q = a}
 *   load_d = 1/n sum_a count_a A_ad               (lowest index among maxima)
 *   loss   = coef M sum_d load_d mean_q sum_a p_qa A_ad
 *   grad   = d loss / d scores with load held:
 *            coef M / n p_qa (h_a - sum_b p_qb h_b),  h_a = sum_d load_d A_ad
 * Evenly spread decisions over M devices give the least, coef.  Rows that are
 * not used have a zero gradient (their scores are not read where use[q] = 0);
 * with no used row the loss is 0.  A used row with a NaN counts for no slice
 * and makes the loss and its own gradient NaN; so does one of +inf, which counts
 * for its slice.
 *
 *   scores  [Q] rows of S <= 16384, TAG_F32 or TAG_BF16
 *   mask    [S] device masks (tag_slices.mask)
 *   grad    same type as scores; overwritten, or with accumulate != 0 (TAG_F32
 *           only) added to; must not overlap scores
 *   loss [1] fp32, count [S] int32, load [M] fp32
 * Sums run in a fixed order: a call is bitwise repeatable.
 */
tag_status tag_balance_workspace(int32_t n_query, int32_t n_slices, size_t *bytes);
tag_status tag_balance(int32_t n_query, int32_t n_slices, int32_t dtype, const void *scores, int64_t score_stride,
                       const uint64_t *mask, int32_t n_dev, const uint8_t *use, float coef, void *grad,
                       int64_t grad_stride, int32_t accumulate, float *loss, int32_t *count, float *load,
                       void *workspace, size_t ws_bytes, void *hip_stream);

#ifdef __cplusplus
}
#endif

#endif /* TAG_POLICY_H */
