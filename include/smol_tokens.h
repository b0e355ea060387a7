/*
 * smol_tokens.h -- from preprocessed images and token ids to the rows of a
 * sequence model, with gradients (libsmol, MI355X gfx950).
 *
 * The preprocessing calls (smol.h) end at the network's input tensor. When
 * the network is a transformer, its first layers read that tensor once and
 * turn it into rows: images are cut into patches, each projected to one row
 * of the sequence; token ids look their rows up in a table; both kinds of
 * rows stand in one sequence buffer, which is then normalised. These calls
 * are those layers: patch embedding, embedding lookup and layer norm, each
 * with the backward pass that training needs (section 5.3 fine-tunes on
 * low-resolution inputs).
 *
 * Conventions of all calls:
 *   - Every matrix is given by a DEVICE pointer, a number of rows and a row
 *     stride in elements (>= its width; >= 0 for one that is only read, so
 *     that one row can stand for all); elements of a row are consecutive.
 *     Pointers need the alignment of one element only. Outputs overlap no
 *     input unless the call says so ("may be x itself": the same pointer and
 *     stride).
 *   - Element types are SMOL_ELEM_*. Products and sums are held in fp32
 *     whatever the types, and rounded once (to nearest even) when an output
 *     is written. Results do not depend on scheduling: the same inputs give
 *     the same bits.
 *   - Argument structures are HOST memory read during the call; reserved
 *     fields must be zero. Work is enqueued on `stream` (a hipStream_t of
 *     the current device, or NULL), nothing is synchronised and nothing is
 *     allocated: calls that need room take a workspace of the caller.
 *   - Calls return SMOL_OK, SMOL_ERR_INVALID_ARG, SMOL_ERR_UNSUPPORTED (past
 *     a limit below, or more workgroups than one launch takes: 2^24 tiles of
 *     a patch embedding, 2^32 values of its gradients together) or
 *     SMOL_ERR_HIP; on an error found by validation nothing is enqueued.
 *     smol_last_error() has the detail.
 */
#ifndef SMOL_TOKENS_H
#define SMOL_TOKENS_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* Element types (the first two are numbered as SMOL_OUT_F32, SMOL_OUT_F16). */
#define SMOL_ELEM_F32 0
#define SMOL_ELEM_F16 1
#define SMOL_ELEM_BF16 2

/* Token id types. */
#define SMOL_IDS_I32 0
#define SMOL_IDS_I64 1

/* Limits. */
#define SMOL_MAX_NORM_DIM 8192       /* columns of a layer norm               */
#define SMOL_MAX_EMBED_DIM 65536     /* columns of an embedding table         */
#define SMOL_MAX_PATCH_DIM 65536     /* rows of a patch embedding's weight    */
#define SMOL_MAX_PATCH 256           /* side of a patch                       */
#define SMOL_MAX_PATCH_VALUES 262144 /* values of a patch: channels * side^2  */
#define SMOL_MAX_ROWS 1073741824     /* rows, ids, vocabulary (2^30)          */

/* ------------------------------------------------------------------------
 * Patch embedding.
 *
 * Image i of n is cut into th x tw patches, th = floor(height / patch), tw =
 * floor(width / patch) (trailing pixels are not used), in row order; patch
 * t's values, in the order of one weight row, are a[i][t][k]:
 *
 *   out[i][t][d] = sum_k r(a[i][t][k]) * weight[d][k] + bias[d] + pos[t][d]
 *
 * r rounds a pixel to the weight's type, as a matrix product's operands
 * share one type (no rounding when the types agree or the weight is fp32).
 * ------------------------------------------------------------------------ */

/* The images and the projection.
 *   images      n images as the preprocessing calls write them: channels x
 *               height x width (SMOL_LAYOUT_NCHW) or height x width x
 *               channels (SMOL_LAYOUT_NHWC), dense
 *   image_type  SMOL_ELEM_F32 or SMOL_ELEM_F16 with any type; SMOL_ELEM_BF16
 *               with type SMOL_ELEM_BF16 only
 *   type        of weight, bias, pos, out and grad_out
 *   patch, dim  side of a patch; width of an output row */
typedef struct smol_patch_shape {
    int32_t n, channels, height, width;
    int32_t patch, dim;
    int32_t layout;
    int32_t image_type;
    int32_t type;
    int32_t reserved[3];
} smol_patch_shape;

/* smol_patch_embed.
 *   weight  dim x channels x patch x patch (NCHW) or dim x patch x patch x
 *           channels (NHWC): the layout of the images; dense
 *   bias    dim, or NULL
 *   pos     th * tw x dim, dense, or NULL
 *   out     patch t of image i at out + i * image_stride + t * row_stride
 *           (strides in elements): the rows may stand in a longer sequence.
 *           No two rows may overlap. */
typedef struct smol_patch_args {
    smol_patch_shape shape;
    const void *images;
    const void *weight;
    const void *bias;
    const void *pos;
    void *out;
    int64_t image_stride;
    int64_t row_stride;
} smol_patch_args;

int smol_patch_embed(const smol_patch_args *a, void *stream);

/* smol_patch_embed_backward -- the parameters' gradients (the pixels come
 * from a decoder and have none):
 *
 *   grad_weight[d][k] (+)= sum_{i,t} grad_out[i][t][d] * r(a[i][t][k])
 *   grad_bias[d]      (+)= sum_{i,t} grad_out[i][t][d]
 *   grad_pos[t][d]    (+)= sum_i     grad_out[i][t][d]
 *
 *   grad_out     strided as out of smol_patch_embed
 *   grad_weight, grad_bias, grad_pos  of grad_type, dense; each may be NULL
 *                (not computed)
 *   grad_type    SMOL_ELEM_F32 or the shape's type
 *   accumulate   0: the gradients are overwritten; 1: added to
 *   workspace    16-byte aligned, at least smol_patch_workspace_bytes(shape)
 *                bytes, not needed once the call's work is done */
typedef struct smol_patch_grad_args {
    smol_patch_shape shape;
    const void *grad_out;
    int64_t image_stride;
    int64_t row_stride;
    const void *images;
    void *grad_weight;
    void *grad_bias;
    void *grad_pos;
    void *workspace;
    int64_t workspace_bytes;
    int32_t grad_type;
    int32_t accumulate;
} smol_patch_grad_args;

int smol_patch_embed_backward(const smol_patch_grad_args *a, void *stream);

/* Bytes of workspace the backward call needs (0 for an invalid shape). */
int64_t smol_patch_workspace_bytes(const smol_patch_shape *shape);

/* ------------------------------------------------------------------------
 * Embedding lookup.
 *
 *   out[i][c] = scale * table[ids[i]][c]
 *
 * An id outside 0 .. vocab - 1 names no token (the place of an image's row,
 * padding of a batch): its row is zeros, or, with keep = 1, left as it is.
 * The ids are device data, so the host cannot check them; no id is read or
 * written out of bounds.
 * ------------------------------------------------------------------------ */
typedef struct smol_embed_args {
    const void *ids; /* n ids of ids_type                        */
    const void *table; /* vocab x dim, rows table_stride apart     */
    void *out; /* n x dim, rows out_stride apart           */
    int64_t n, vocab, table_stride, out_stride;
    int32_t dim;
    int32_t ids_type;
    int32_t table_type, out_type;
    float scale; /* finite */
    int32_t keep;
    int32_t reserved[2];
} smol_embed_args;

int smol_embed(const smol_embed_args *a, void *stream);

/* smol_embed_backward -- the table's gradient, all vocab rows:
 *
 *   grad_table[v][c] (+)= scale * sum_{i: ids[i] = v} grad_out[i][c]
 *
 * Each sum runs over its rows in their order, in pieces that are then joined
 * in order; where the pieces begin depends on the sizes and the ids alone. (Few
 * rows are found by their ids directly, more by sorting the ids, stably.) With
 * accumulate = 0 rows that no id names are zeros; with 1 they are not touched.
 *   padding      an id whose row gets no gradient (-1: none; with accumulate
 *                = 0 its row is zeros)
 *   grad_type    any element type
 *   workspace    16-byte aligned, at least smol_embed_workspace_bytes(n,
 *                vocab, dim) bytes */
typedef struct smol_embed_grad_args {
    const void *grad_out; /* n x dim, rows grad_stride apart */
    const void *ids;
    void *grad_table; /* vocab x dim, rows table_stride apart */
    void *workspace;
    int64_t workspace_bytes;
    int64_t n, vocab, grad_stride, table_stride;
    int64_t padding;
    int32_t dim;
    int32_t ids_type;
    int32_t out_type; /* of grad_out */
    int32_t grad_type;
    float scale;
    int32_t accumulate;
} smol_embed_grad_args;

int smol_embed_backward(const smol_embed_grad_args *a, void *stream);

/* Bytes of workspace the backward call needs (0 for sizes out of range). */
int64_t smol_embed_workspace_bytes(int64_t n, int64_t vocab, int32_t dim);

/* ------------------------------------------------------------------------
 * Layer norm, with a residual sum before it.
 *
 *   h    = x, or x + residual rounded to the type
 *   mean = (1/dim) sum_c h[c],  rstd = 1 / sqrt((1/dim) sum_c (h[c] - mean)^2 + eps)
 *   out  = (h - mean) * rstd * weight + bias
 *
 * The variance is that of the differences from the mean, not a difference
 * of squares. A NaN or infinity makes its own row NaN and no other.
 * ------------------------------------------------------------------------ */
typedef struct smol_norm_args {
    const void *x; /* rows x dim of type                                */
    const void *residual; /* rows x dim of type, or NULL                       */
    const void *weight; /* dim of weight_type, or NULL (ones)                */
    const void *bias; /* dim of weight_type, or NULL (zeros)               */
    void *out; /* rows x dim of type; may be x or residual itself   */
    void *sum; /* h, rows x dim of type, or NULL; may be x or       */
               /* residual itself                                   */
    float *mean; /* rows, or NULL                                     */
    float *rstd; /* rows, or NULL                                     */
    int64_t rows;
    int64_t x_stride, residual_stride, out_stride, sum_stride;
    int32_t dim;
    int32_t type;
    int32_t weight_type; /* SMOL_ELEM_F32 or type */
    float eps; /* >= 0, finite */
    int32_t reserved[2];
} smol_norm_args;

int smol_layer_norm(const smol_norm_args *a, void *stream);

/* smol_layer_norm_backward, for each row with xh = (h - mean) * rstd and g =
 * grad_out * weight:
 *
 *   grad_x       = grad_sum + rstd * (g - mean(g) - xh * mean(g * xh))
 *   grad_weight (+)= sum over rows of grad_out * xh
 *   grad_bias   (+)= sum over rows of grad_out
 *
 * grad_x is the gradient of h: of x and of residual alike. */
typedef struct smol_norm_grad_args {
    const void *grad_out; /* rows x dim of type                              */
    const void *h; /* rows x dim of type (x, or sum of the forward)   */
    const void *grad_sum; /* rows x dim of type: the gradient that reaches h */
                          /* past the norm, or NULL                         */
    const void *weight; /* dim of weight_type, or NULL                     */
    const float *mean; /* rows                                            */
    const float *rstd; /* rows                                            */
    void *grad_x; /* rows x dim of type; may be grad_out, h or       */
                  /* grad_sum itself                                 */
    void *grad_weight; /* dim of weight_type, or NULL                     */
    void *grad_bias; /* dim of weight_type, or NULL                     */
    void *workspace; /* 16-byte aligned                                 */
    int64_t workspace_bytes;
    int64_t rows;
    int64_t grad_stride, h_stride, sum_stride, x_stride;
    int32_t dim;
    int32_t type;
    int32_t weight_type;
    int32_t accumulate; /* of grad_weight and grad_bias                    */
} smol_norm_grad_args;

int smol_layer_norm_backward(const smol_norm_grad_args *a, void *stream);

/* Bytes of workspace the backward call needs (0 for sizes out of range). */
int64_t smol_norm_workspace_bytes(int64_t rows, int32_t dim);

#ifdef __cplusplus
}
#endif

#endif /* SMOL_TOKENS_H */
