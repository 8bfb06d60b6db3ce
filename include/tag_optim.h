/*
 * tag_optim.h -- C ABI of the orthogonalised optimiser step: Newton-Schulz
 * products that bring a matrix's singular values near one, and the update of
 * weight matrices by the orthogonalised momentum of their gradients, the
 * matrix counterpart of the SGD update of tag_train_step; and the clipping of
 * gradients by their global norm.
 *
 * Conventions follow tag.h: caller-owned DEVICE buffers, asynchronous on
 * hip_stream, arguments validated before anything is enqueued, no allocation.
 * The groups themselves are HOST arrays, read during the call.  A workspace is
 * scratch for the duration of a call (calls that share one must be ordered);
 * nothing in it needs to start at zero.  Sums run in a fixed order: a call is
 * bitwise repeatable.
 */
#ifndef TAG_OPTIM_H
#define TAG_OPTIM_H

#include "tag.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * The iteration.  With G of n x m (transposed first where rows > cols, so
 * n <= m):
 *   X = G / (||G||_F + eps)
 *   `steps` times:  A = X X^T,  B = b A + c A A,  X = a X + B X
 * so that a singular value s becomes a s + b s^3 + c s^5 in each step.  eps is
 * positive; steps is 1..32.  Coefficients under which a singular value in
 * [0, 1] may leave [0, 3.5] on the way, or an eigenvalue of B [-15, 15], are
 * refused (TAG_EINVAL): the products are scaled for that range.
 * A matrix with an infinity or a NaN gives NaN everywhere; a matrix of zeros
 * gives zeros.
 */
typedef struct tag_newton_schulz {
    int32_t steps;
    float a, b, c, eps;
} tag_newton_schulz;

/* `count` matrices of one shape: matrix i, row r, column c of an array at
 * base[i matrix_stride + r row_stride + c] (strides in elements; count times
 * matrix_stride and rows times row_stride at most 2^58, TAG_ESHAPE). */
typedef struct tag_matrices {
    void *base;
    int64_t row_stride, matrix_stride;
} tag_matrices;

typedef struct tag_ortho_group {
    int32_t count, rows, cols;     /* sides up to 32768, at most 2^19 tiles of 64 x 64 in all */
    tag_matrices in, out;          /* out may be in, with its strides; otherwise written arrays overlap nothing */
} tag_ortho_group;

/*
 * Orthogonalises every matrix of every group.  dtype: of in and out.
 * Products of two-part splits that hold every operand to 2^-22, with fp32
 * accumulation, about as near the exact iteration as fp32 products; TAG_BF16
 * results are rounded once, from the same accuracy.  That is relative to
 * the largest values of X, which is at most of norm one at first: where
 * ||G||_F is far below eps, what is left of it is held to 2^-37 of one.  Which
 * order a matrix's sums take depends on the sizes of the call's other groups.
 */
tag_status tag_orthogonalise_workspace(const tag_ortho_group *groups, int32_t n_groups, size_t *bytes);
tag_status tag_orthogonalise(const tag_ortho_group *groups, int32_t n_groups, int32_t dtype,
                             const tag_newton_schulz *ns, void *workspace, size_t ws_bytes, void *hip_stream);

/*
 * One optimiser step (all fp32).  For every matrix of a group
 *   m = momentum m + g
 *   u = nesterov ? g + momentum m : m
 *   w = (1 - lr weight_decay) w - lr sqrt(max(1, rows / cols)) O(u)
 * with O the iteration above; for a group with plain != 0 (biases, vectors:
 * give them as one row) O(u) = u with factor 1.  w, g and m are three
 * different arrays, and no w or m is part of another group.
 */
typedef struct tag_muon_group {
    int32_t count, rows, cols, plain;   /* as above; plain: up to 2^31 elements, each matrix's rounded up to 4,096 */
    tag_matrices w, g, m;          /* w and m written, g read */
} tag_muon_group;

typedef struct tag_muon_options {
    float lr, momentum, weight_decay;   /* lr >= 0, momentum in [0, 1), weight_decay >= 0 */
    int32_t nesterov;
} tag_muon_options;

tag_status tag_muon_workspace(const tag_muon_group *groups, int32_t n_groups, size_t *bytes);
tag_status tag_muon_step(const tag_muon_group *groups, int32_t n_groups, const tag_newton_schulz *ns,
                         const tag_muon_options *options, void *workspace, size_t ws_bytes, void *hip_stream);

/*
 * The step from clipped gradients, which stay as they are.  clip: DEVICE
 * {norm, scale} as tag_clip writes them for these gradients, no part of a w or
 * m.  The step takes scale g for g (one more rounding of fp32); with a norm that
 * is not finite it leaves weights and momentum as they are.
 */
tag_status tag_muon_step_clipped(const tag_muon_group *groups, int32_t n_groups, const tag_newton_schulz *ns,
                                 const tag_muon_options *options, const float *clip, void *workspace,
                                 size_t ws_bytes, void *hip_stream);

/*
 * Clipping by the global norm, over all elements of all arrays of a plan:
 *   norm  = sqrt(sum g^2)                          (64 bits; result: fp32)
 *   scale = norm > max_norm ? max_norm / norm : 1  (rounded to fp32)
 *   out   = scale g                                (rounded to fp32, then to the array's type)
 * A norm that is not finite as fp32 (an infinity or a NaN among the gradients, or
 * values near the end of fp32's range) gives scale 0 and an out of zeros: the
 * gradients of that step are dropped, as norm tells.
 *
 * Row r, column c of an array stand at g[r g_stride + c] and out[r out_stride + c]
 * (strides in elements, at least cols; a vector is one row).  out may be g, with
 * its stride (then nothing is written where scale is 1), or NULL: the array
 * counts for the norm only.  Arrays of both types may stand in one plan; any
 * alignment of their elements will do.  What is written overlaps nothing else.
 */
typedef struct tag_clip_array {
    const void *g;
    void *out;
    int64_t rows, cols, g_stride, out_stride;   /* rows, cols >= 0 */
    int32_t dtype;                 /* TAG_F32 or TAG_BF16 */
} tag_clip_array;

/* A plan of the arrays, on the HOST; filled by tag_clip_prepare, read by tag_clip. */
typedef struct tag_clip_plan {
    const void *table;             /* the DEVICE table */
    int64_t chunks;                /* entries of it */
    int32_t writes;                /* 1: some array has an out elsewhere than at g, 2: none has, but some at g */
} tag_clip_plan;

/*
 * Lays the table out that tag_clip reads, tag_clip_table_bytes of DEVICE memory,
 * which outlives the plan.  `arrays` (HOST) is read during the call; their
 * addresses stay those of the plan.  Synchronises hip_stream once (so it cannot
 * be captured; tag_clip can).
 */
tag_status tag_clip_table_bytes(const tag_clip_array *arrays, int32_t n_arrays, size_t *bytes);
tag_status tag_clip_prepare(const tag_clip_array *arrays, int32_t n_arrays, void *table, size_t table_bytes,
                            void *hip_stream, tag_clip_plan *plan);

/* Clips.  max_norm >= 0 (infinity: the norm alone, scale 1).  result: DEVICE [2],
 * norm and scale. */
tag_status tag_clip_workspace(size_t *bytes);
tag_status tag_clip(const tag_clip_plan *plan, double max_norm, float *result, void *workspace, size_t ws_bytes,
                    void *hip_stream);

#ifdef __cplusplus
}
#endif

#endif /* TAG_OPTIM_H */
