/*
 * smol_attention.h -- from the normalised rows of a sequence model to rows
 * that have looked at each other, with gradients (libsmol, MI355X gfx950).
 *
 * The token calls (smol_tokens.h) end at normalised rows; a projection makes
 * queries, keys and values of them. These calls are what follows: rotary
 * positions, norms of queries and keys head by head with the rotation in the
 * same pass, and attention, with the backward passes that training needs and
 * the forms for single tokens that answering needs.
 *
 * Conventions are those of smol_tokens.h (element types, fp32 sums, one
 * rounding per output, results that do not depend on scheduling, host
 * argument structures, streams, errors), and:
 *   - A matrix of heads has rows (tokens), heads within a row and `dim`
 *     consecutive elements within a head; rows and heads have a stride of
 *     their own in elements, so queries, keys and values may stand beside each
 *     other in one projection's rows. A stride of 0 lets one row or head of
 *     an input stand for all. No two heads of an output may overlap; an
 *     output that begins where another matrix of the call does is refused
 *     unless the call says that it may (then with the same strides).
 */
#ifndef SMOL_ATTENTION_H
#define SMOL_ATTENTION_H

#include <stdint.h>

#include "smol_tokens.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Limits. */
#define SMOL_MAX_HEAD_DIM 256    /* values of a head: rotation, head norm       */
#define SMOL_MAX_ATTEND_DIM 128  /* values of a head: attention (multiple of 8) */
#define SMOL_MAX_HEADS 1024      /* heads of a row                              */
#define SMOL_MAX_ATTEND_BATCH 65536     /* sequences of an attention call       */
#define SMOL_MAX_ATTEND_ROWS 16777216   /* rows of a sequence (2^24)            */

/* ------------------------------------------------------------------------
 * Rotary frequencies (HOST computation; nothing is enqueued).
 *
 * freqs[i], i = 0 .. dim / 2 - 1, in radians a position, in fp64:
 *   SMOL_ROTARY_NONE    base^(-2 i / dim)
 *   SMOL_ROTARY_LINEAR  that divided by factor (positions squeezed)
 *   SMOL_ROTARY_BASE    with base * factor^(dim / (dim - 2)) in place of base
 *                       (the slowest frequency divided by factor; dim 2: none)
 *   SMOL_ROTARY_PARTS   f keep + (f / factor) (1 - keep), keep = (turns - low) /
 *                       (high - low) within 0 .. 1, turns = f length / (2 pi):
 *                       frequencies of many turns within `length` positions
 *                       stay, those of few are squeezed
 * gain, the factor of cosines and sines: 0.1 ln(factor) + 1 for
 * SMOL_ROTARY_PARTS, else 1.
 * ------------------------------------------------------------------------ */
#define SMOL_ROTARY_NONE 0
#define SMOL_ROTARY_LINEAR 1
#define SMOL_ROTARY_BASE 2
#define SMOL_ROTARY_PARTS 3

typedef struct smol_rotary_plan {
    double base;    /* > 0, finite                                            */
    double factor;  /* >= 1, finite (unused: SMOL_ROTARY_NONE)                 */
    double length;  /* > 0, finite (the three: SMOL_ROTARY_PARTS alone)        */
    double low, high; /* turns, low < high                                     */
    int32_t dim;    /* rotated values of a head: even, 2 .. SMOL_MAX_HEAD_DIM  */
    int32_t scaling;
} smol_rotary_plan;

int smol_rotary_frequencies(const smol_rotary_plan *p, double *freqs, float *gain);

/* ------------------------------------------------------------------------
 * Rotation by positions. With angle p freqs[i] (p the row's position; formed
 * and reduced in fp64), c = gain cos, s = gain sin of it:
 *
 *   out[a] = x[a] c - x[b] s,   out[b] = x[b] c + x[a] s
 *
 * where pair i is (a, b) = (i, i + rot / 2), or (2 i, 2 i + 1) interleaved,
 * i = 0 .. rot / 2 - 1. Values from rot on are copied.
 *
 * smol_rotate_backward is the gradient: x holds that of the rotated values,
 * out gets that of the values (the transposed rotation, gain included).
 * ------------------------------------------------------------------------ */
typedef struct smol_rotate_args {
    const void *x;   /* rows x heads x dim of type                             */
    void *out;       /* the same; may be x itself                              */
    const void *positions; /* rows, of positions_type (SMOL_IDS_*), any value  */
    const double *freqs;   /* rot / 2, on the DEVICE                           */
    int64_t rows;
    int64_t x_row_stride, x_head_stride, out_row_stride, out_head_stride;
    int32_t heads, dim;
    int32_t rot;     /* even, 2 .. dim                                         */
    int32_t type;
    int32_t positions_type;
    int32_t interleaved;
    float gain;      /* finite                                                 */
    int32_t reserved;
} smol_rotate_args;

int smol_rotate(const smol_rotate_args *a, void *stream);
int smol_rotate_backward(const smol_rotate_args *a, void *stream);

/* ------------------------------------------------------------------------
 * Norm of each head of queries and keys, then the rotation, in one pass:
 *
 *   r = 1 / sqrt((1/dim) sum_c x[c]^2 + eps),   out = rotation(x r weight)
 *
 * Squares are formed in fp32: values past 2^63 / sqrt(dim) overflow, and those
 * below 2^-75 count as zeros (with eps 0, a head of such values alone is not
 * finite).
 * ------------------------------------------------------------------------ */

/* The queries or the keys. heads may be 0: this side is then absent. */
typedef struct smol_head_side {
    const void *x;      /* rows x heads x dim of type                          */
    void *out;          /* the same; may be x itself                           */
    const void *weight; /* dim of weight_type, or NULL (ones)                  */
    int64_t x_row_stride, x_head_stride, out_row_stride, out_head_stride;
    int32_t heads;
    int32_t reserved;
} smol_head_side;

/* What both directions share. rot 0: no rotation, positions and freqs unused. */
typedef struct smol_head_shape {
    const void *positions;
    const double *freqs;
    int64_t rows;
    int32_t dim, rot;
    int32_t type;
    int32_t weight_type; /* SMOL_ELEM_F32 or type */
    int32_t positions_type;
    int32_t interleaved;
    float eps;           /* >= 0, finite */
    float gain;
    int32_t reserved[2];
} smol_head_shape;

typedef struct smol_head_norm_args {
    smol_head_shape shape;
    smol_head_side q, k;
} smol_head_norm_args;

int smol_head_norm(const smol_head_norm_args *a, void *stream);

/* smol_head_norm_backward: with g = transposed rotation of grad_out, u = g
 * weight, xh = x r,
 *
 *   grad_x         = r (u - xh mean(u xh))
 *   grad_weight (+)= sum over rows and heads of g xh */
typedef struct smol_head_grad_side {
    const void *grad_out; /* rows x heads x dim of type                        */
    const void *x;
    const void *weight;   /* or NULL (ones)                                    */
    void *grad_x;         /* may be grad_out or x itself                       */
    void *grad_weight;    /* dim of weight_type, or NULL (not computed)        */
    int64_t grad_out_row_stride, grad_out_head_stride;
    int64_t x_row_stride, x_head_stride;
    int64_t grad_x_row_stride, grad_x_head_stride;
    int32_t heads;
    int32_t reserved;
} smol_head_grad_side;

typedef struct smol_head_norm_grad_args {
    smol_head_shape shape;
    smol_head_grad_side q, k;
    void *workspace;      /* 16-byte aligned                                   */
    int64_t workspace_bytes;
    int32_t accumulate;   /* 0: grad_weight is overwritten; 1: added to        */
    int32_t reserved;
} smol_head_norm_grad_args;

int smol_head_norm_backward(const smol_head_norm_grad_args *a, void *stream);

/* Bytes of workspace the backward call needs (0 for sizes out of range). */
int64_t smol_head_norm_workspace_bytes(int64_t rows, int32_t q_heads, int32_t k_heads,
                                       int32_t dim);

/* ------------------------------------------------------------------------
 * Attention.
 *
 * `batch` sequences of `queries` rows of queries and `keys` rows of keys and
 * values; query head h reads key head floor(h kv_heads / heads). Of sequence
 * b the first q_length rows of queries and k_length rows of keys exist (all,
 * where the lengths are NULL; lengths are clamped to 0 .. queries, keys).
 * The queries are the sequence's last rows: query i stands at position p =
 * k_length - q_length + i and sees key j, 0 <= j < k_length,
 *   causal 0: always
 *   causal 1: if j <= p, and j > p - window or j < sinks (window 0: any)
 *
 *   s[j] = scale q . k[j],   lse = ln sum_j exp(s[j]),
 *   out  = sum_j exp(s[j] - lse) v[j]             over the keys it sees
 *
 * A query that sees no key, or does not exist, has out 0 and lse minus
 * infinity. What a query does not see takes no part, whatever it holds: NaN
 * and infinities there are harmless. Of the scores that it sees, a NaN or plus
 * infinity makes its row and lse NaN; minus infinity has no weight, and a row of
 * nothing else is NaN with lse minus infinity. A NaN or an infinity among the
 * values that it sees is in its row, however small the weight; finite values up
 * to 2^127 give finite rows. The weights exp(s - m), m near the row's maximum,
 * are rounded to the type before the product with v, as matrix operands are
 * (fp16: those below 2^-32 of the largest are then zero). A call some of whose
 * sums are not finite forms them twice, in a few times its time.
 *
 * Single tokens, prompts and pieces of prompts are the same call: new tokens
 * are the last `queries` rows of a cache whose first k_length rows are filled.
 * ------------------------------------------------------------------------ */
typedef struct smol_attend_shape {
    const int32_t *q_lengths; /* batch, on the DEVICE, or NULL                 */
    const int32_t *k_lengths; /* batch, on the DEVICE, or NULL                 */
    int32_t batch, queries, keys;
    int32_t heads, kv_heads;  /* heads a multiple of kv_heads                  */
    int32_t dim;              /* a multiple of 8                               */
    int32_t type;             /* of all matrices                               */
    int32_t causal;
    int32_t window, sinks;    /* >= 0; 0 unless causal                         */
    float scale;              /* 2^-60 .. 2^60                                 */
    int32_t reserved;
} smol_attend_shape;

/* A matrix of heads of each sequence: row r, head h of sequence b at data +
 * b batch_stride + r row_stride + h head_stride. */
typedef struct smol_attend_rows {
    const void *data;
    int64_t batch_stride, row_stride, head_stride;
} smol_attend_rows;

/* The same, written. */
typedef struct smol_attend_out {
    void *data;
    int64_t batch_stride, row_stride, head_stride;
} smol_attend_out;

/* smol_attend.
 *   lse   batch x queries x heads, dense, or NULL
 *   rest  batch x queries x heads x dim of the type, dense, or NULL: what
 *         rounding took from out, rounded itself. smol_attend_backward needs
 *         it for gradients as exact as their rounding where few keys have
 *         most of a query's weight. */
typedef struct smol_attend_args {
    smol_attend_shape shape;
    smol_attend_rows q, k, v;
    smol_attend_out out;
    float *lse;
    void *rest;
    void *workspace; /* 16-byte aligned, smol_attend_workspace_bytes(shape) bytes */
    int64_t workspace_bytes;
} smol_attend_args;

int smol_attend(const smol_attend_args *a, void *stream);

/* Bytes of workspace the forward call needs: room for sums of parts of the
 * keys, where there are few queries (0 for an invalid shape). */
int64_t smol_attend_workspace_bytes(const smol_attend_shape *shape);

/* smol_attend_backward: with p[i][j] = exp(s[i][j] - lse[i]), over pairs of a
 * query and a key that it sees,
 *
 *   d[i][j]   = p[i][j] (grad_out[i] . v[j] - grad_out[i] . (out[i] + rest[i]))
 *   grad_v[j] = sum_i p[i][j] grad_out[i]       (over all heads that read j)
 *   grad_q[i] = scale sum_j d[i][j] k[j],   grad_k[j] = scale sum_i d[i][j] q[i]
 *
 * p and d are rounded to the type before these products (fp16: times powers of
 * two, so that p down to 2^-30 and d of any size are held; a call some of whose d
 * pass 2^10 forms sums twice in 2 to 3 times its time, as one with a NaN or an
 * infinity does). A query that is NaN, or whose lse is, makes the gradients of
 * all keys that it sees NaN. Rows that do not exist get zeros. */
typedef struct smol_attend_grad_args {
    smol_attend_shape shape;
    smol_attend_rows grad_out, q, k, v, out;
    const void *rest;  /* of the forward pass, or NULL (zeros)                 */
    const float *lse;  /* of the forward pass                                  */
    smol_attend_out grad_q, grad_k, grad_v;
    void *workspace;   /* 16-byte aligned                                      */
    int64_t workspace_bytes;
} smol_attend_grad_args;

int smol_attend_backward(const smol_attend_grad_args *a, void *stream);

/* smol_attend_backward_kept: the same, with lse and rest where a program keeps
 * them, at strides of their own (of sequences, rows and heads, in elements; 0 lets
 * one stand for all) instead of dense. */
typedef struct smol_attend_kept {
    int64_t lse_batch_stride, lse_row_stride, lse_head_stride;
    int64_t rest_batch_stride, rest_row_stride, rest_head_stride; /* unused: rest NULL */
} smol_attend_kept;

int smol_attend_backward_kept(const smol_attend_grad_args *a, const smol_attend_kept *kept,
                              void *stream);

/* Bytes of workspace a backward call needs (0 for an invalid shape). */
int64_t smol_attend_backward_workspace_bytes(const smol_attend_shape *shape);

#ifdef __cplusplus
}
#endif

#endif /* SMOL_ATTENTION_H */
