/*
 * tag_beam.h -- C ABI of beam search over the decision head's scores: one
 * level of the search (the best continuations of every beam's slices) and the
 * reordering of the beams' states after it.
 *
 * n_search independent searches run side by side.  Before a level each has
 * width_in beams, after it width beams.  Conventions follow tag.h: caller-owned
 * DEVICE buffers, asynchronous on hip_stream, arguments validated before
 * anything is enqueued, no allocation.  A workspace is scratch for the duration
 * of a call (calls that share one must be ordered); nothing in it needs to
 * start at zero.  But where a call says so, no array that it writes overlaps
 * another of its arrays.
 */
#ifndef TAG_BEAM_H
#define TAG_BEAM_H

#include "tag.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * One level.  Beam v of a search has the row x_v of S scores and the log
 * probability total_v so far.  Its continuations, in 64 bits, are
 *   c_va = x_va + (total_v - log sum_b exp x_vb)       for every x_va > -inf
 * and those of a finished beam (done[v] != 0; its scores do not matter) the one
 * candidate c = total_v, which counts as slice 0 where ties are broken.  The
 * `width` best candidates of all beams of a search, best first, equal ones in
 * the order of (beam, slice), become its new beams:
 *   total   c, rounded to fp32 (below its range: -inf)     parent  v
 *   slice   a, or -1 of a finished beam
 * A beam has no candidates if its total is not finite, or if a NaN or +inf
 * stands among its scores (which a finished beam may have); what is left
 * over of the width has total -inf, parent -1 and slice -1.  A search starts
 * from width_in = 1, or from totals of -inf but for one beam.
 *
 *   scores    n_search * width_in rows of S, TAG_F32 or TAG_BF16, row stride in
 *             elements, at least S; rows may start at any element
 *   total_in  [n_search][width_in] fp32
 *   done      [n_search][width_in], or NULL: none is finished
 *   total     [n_search][width] fp32; may be total_in where width_in = width
 *   parent, slice  [n_search][width] int32
 * width and width_in are at most 256, width_in * S at most 2^30, n_search *
 * width_in * stride at most 2^58 (TAG_ESHAPE).
 * A call is bitwise repeatable.
 */
tag_status tag_beam_workspace(int32_t n_search, int32_t width_in, int32_t width, int32_t n_slices, size_t *bytes);
tag_status tag_beam_select(int32_t n_search, int32_t width_in, int32_t width, int32_t n_slices, int32_t dtype,
                           const void *scores, int64_t score_stride, const float *total_in, const uint8_t *done,
                           float *total, int32_t *parent, int32_t *slice, void *workspace, size_t ws_bytes,
                           void *hip_stream);

/*
 * One array of states, a row of row_bytes for every beam: beam v of search b
 * at in + b in_search + v in_beam, where its successors' rows are written at
 * out + b out_search + w out_beam (strides in bytes, any alignment).  Rows of
 * `out` do not overlap one another.  out may be in, with its strides (then the
 * search stride also covers the larger of both widths).
 */
typedef struct tag_beam_state {
    const void *in;
    void *out;
    int64_t row_bytes, in_search, in_beam, out_search, out_beam;
} tag_beam_state;

/*
 * Reorders states: row w of each search's `out` becomes row parent[b][w] of its
 * `in`, as it was before the call.  Rows whose parent is outside [0, width_in)
 * are left as they were.  `states` is a HOST array, read during the call, of at
 * most 64 arrays.  parent: DEVICE [n_search][width].
 */
tag_status tag_beam_reorder(int32_t n_search, int32_t width_in, int32_t width, const int32_t *parent,
                            const tag_beam_state *states, int32_t n_states, void *hip_stream);

#ifdef __cplusplus
}
#endif

#endif /* TAG_BEAM_H */
