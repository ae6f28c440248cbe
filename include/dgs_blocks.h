/*
 * libdgs, training blocks -- the memory-bound part of a transformer worker's step, around the hot path of dgs.h: what lies
 * between two blocks (norm, gate, residual sum, norm), the 8-bit checkpoints that the forward pass keeps for the backward
 * pass, and the gradients that are read from them; and what lies behind the last block: the output layer with its loss, and
 * updates orthogonalised before they are sent.  Parameters and their gradients are fp32, as in the flat buffers of
 * dgs.h, and gradients can be added to what such a buffer holds.
 *
 * Conventions as in dgs.h: the caller owns every device buffer; a call enqueues its work on `hip_stream` (a hipStream_t,
 * NULL = the default stream) of the current device and returns without waiting; 0 or a negative DGS_E* code; nothing is
 * thrown, and nothing is enqueued when an argument is refused.  There is no context and no state: calls on different
 * streams are independent as long as their buffers are.  Every call may be captured into a HIP graph (kernels only).
 *
 * Matrices are row-major with contiguous columns; a stride is the distance of two rows in elements, at least `cols` and below
 * 2^32.  Pointers need the alignment of their element type only.  More than 2^31 - 1 rows: DGS_ENOTSUP.
 */
#ifndef DGS_BLOCKS_H
#define DGS_BLOCKS_H

#include "dgs.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { DGS_F32 = 0, DGS_F16 = 1, DGS_BF16 = 2 };            /* element types */
enum { DGS_NORM_NONE = 0, DGS_NORM_RMS = 1, DGS_NORM_LAYER = 2 };

/* Columns that dgs_edge_forward / _backward take. */
#define DGS_EDGE_MAX_COLS 16384
/* Columns that share an exponent in a checkpoint. */
#define DGS_CHECKPOINT_RUN 32

/*
 * A checkpoint of a rows x cols matrix: one signed code a value and one exponent byte for every run of 32 columns of a row
 * (the last run of a row may be shorter).  A run's values are code * 2^(byte - 127); the byte is the smallest in [1, 248]
 * for which the run's largest magnitude rounds to at most 127, and codes are rounded to nearest, halfway cases to even.
 * (Only above 127.5 * 2^121 are codes cut to 127.)  Byte 255: the run held an infinity or NaN and reads as NaN; its
 * codes are 0.  Every value of a checkpoint is exact in bfloat16.
 */
typedef struct dgs_codes {
    int8_t *codes;          /* rows x cols */
    uint64_t codes_stride;  /* >= cols */
    uint8_t *exps;          /* rows x ceil(cols / 32) */
    uint64_t exps_stride;   /* >= ceil(cols / 32) */
} dgs_codes;

typedef struct dgs_matrix {
    void *data;             /* NULL: absent */
    uint64_t stride;
} dgs_matrix;

/*
 * The edge between two blocks.  Per row, with N(v) = (v - mean) * rstd, rstd = 1 / sqrt(mean((v - mean)^2) + eps), and mean
 * taken as 0 for DGS_NORM_RMS:
 *
 *     fh    = N_post(f)                      (f itself for DGS_NORM_NONE)
 *     x_out = skip * x + branch * gate * (fh * post_weight + post_bias)
 *     xh    = N_pre(x_out)
 *     u     = xh * pre_weight + pre_bias
 *
 * everything in fp32, x_out and u rounded once; xh is taken of the sum before it is rounded.  Absent weights are 1, absent
 * biases 0, an absent gate 1.  Row r takes gate row r / rows_per_gate, of ceil(rows / rows_per_gate).
 */
typedef struct dgs_edge {
    uint32_t cols;          /* 1 .. DGS_EDGE_MAX_COLS */
    int32_t post, pre;      /* DGS_NORM_* */
    float post_eps, pre_eps; /* > 0 */
    float skip, branch;
    const float *post_weight, *post_bias, *pre_weight, *pre_bias; /* cols floats each, or NULL */
} dgs_edge;

/*
 * dgs_edge_forward.  Types: `stream_type` is that of x and x_out, `type` that of f and u: equal, or the stream DGS_F32.
 * The gate has `gate_type`: DGS_F32 or `type`.
 *   f absent     no branch: x_out is x and is not written; u = N_pre(x).  post must be DGS_NORM_NONE, no gate.
 *   pre = NONE   u must be absent.
 *   post_saved, pre_saved   checkpoints of fh and xh, or codes = NULL.
 *   stats        rows x 4 floats, or NULL: post mean, post rstd, pre mean, pre rstd (0 for a norm that is NONE, mean 0 for RMS).
 * x_out may be x and u may be f (same stride); other outputs overlap nothing.
 */
typedef struct dgs_edge_forward_args {
    uint32_t rows, rows_per_gate;
    int32_t stream_type, type, gate_type, reserved;
    dgs_matrix x, f, gate, x_out, u;
    dgs_codes post_saved, pre_saved;
    float *stats;
} dgs_edge_forward_args;

int dgs_edge_forward(const dgs_edge *edge /*host*/, const dgs_edge_forward_args *args /*host*/, void *hip_stream);

/*
 * dgs_edge_backward.  dx_out and du are the gradients that arrive at x_out and u (either may be absent: zero).  With
 * p = du * pre_weight and the row means written <.>,
 *
 *     d  = dx_out + rstd_pre * (p - [<p>] - xh <p xh>)      ([..]: DGS_NORM_LAYER only)
 *     m  = branch * gate * d,   k = m * post_weight
 *     dx = skip * d,            df = rstd_post * (k - [<k>] - fh <k fh>)     (df = k for DGS_NORM_NONE)
 *     dgate = branch * sum over the gate row's rows of d * (fh * post_weight + post_bias)
 *     post_weight' = sum_rows m fh,  post_bias' = sum_rows m,  pre_weight' = sum_rows du xh,  pre_bias' = sum_rows du
 *
 * fh and xh come from the checkpoints, or are computed from `f` and `x_out` (which then have `type` and `stream_type`,
 * and are as the forward pass read and wrote them: of an f that u was written over, nothing is left) and the stats; both
 * norms the same way.  stats: as dgs_edge_forward wrote them.  du absent or pre = NONE: nothing is
 * read of xh; neither f nor post_saved: an edge without a branch (df, dgate, post gradients must be absent).
 * Any output may be absent.  dgate has gate_type.  accumulate != 0: the four parameter gradients, and a dgate of
 * DGS_F32, are added to; otherwise written.  All sums are taken in fp32, in an order that is fixed by the sizes.
 * dx may be dx_out, df may be du (same stride).
 * workspace: device memory of at least dgs_edge_backward_workspace() bytes, 16-byte aligned, whose contents do not matter;
 * not to be used by another call at the same time.  (No rows: none is needed.)
 */
typedef struct dgs_edge_backward_args {
    uint32_t rows, rows_per_gate;
    int32_t stream_type, type, gate_type, accumulate;
    dgs_matrix dx_out, du, gate, f, x_out;
    dgs_codes post_saved, pre_saved;
    const float *stats;
    dgs_matrix dx, df, dgate;
    float *post_weight_grad, *post_bias_grad, *pre_weight_grad, *pre_bias_grad;
    void *workspace;
    uint64_t workspace_bytes;
} dgs_edge_backward_args;

/* Bytes for `rows` rows and, of an edge with a gate, rows_per_gate (0: no gate).  Pure host computation; 0 on invalid arguments too. */
size_t dgs_edge_backward_workspace(uint32_t rows, uint32_t cols, uint32_t rows_per_gate);
int dgs_edge_backward(const dgs_edge *edge /*host*/, const dgs_edge_backward_args *args /*host*/, void *hip_stream);

/*
 * Checkpoint of a matrix, and back: out = value * scale + shift (scale, shift: cols floats, or NULL), rounded to `type`;
 * without them what a finite checkpoint value rounds to beyond the largest DGS_F16 is that largest.
 */
int dgs_checkpoint_encode(uint32_t rows, uint32_t cols, int type, const void *x, uint64_t x_stride,
                          const dgs_codes *to /*host*/, void *hip_stream);
int dgs_checkpoint_decode(uint32_t rows, uint32_t cols, const dgs_codes *from /*host*/, const float *scale,
                          const float *shift, int type, void *out, uint64_t out_stride, void *hip_stream);

/*
 * Gradient of a linear layer y = u W^T + b (W: outs x cols) whose input is u = value * scale + shift of a checkpoint:
 *
 *     dw = dy^T u = (dy^T values) * scale + (sum_rows dy) shift^T        outs x cols floats, rows dw_stride apart
 *     db = sum_rows dy                                                    outs floats, or NULL
 *
 * dy: rows x outs of `type`.  Every product of dy and a checkpoint value is exact in fp32 -- DGS_F16 and DGS_F32 values go
 * through the matrix units as two and three bfloat16 parts -- and sums are fp32, in an order that is fixed by the sizes.  (Of a
 * DGS_F32 value below 2^-110, what is no multiple of 2^-133 is left out.)
 * accumulate != 0: dw and db are added to.  workspace: at least dgs_checkpoint_weight_grad_workspace() bytes, 16-byte
 * aligned; as above.  Rows of dy or of the checkpoint 2^27 bytes or more apart: DGS_ENOTSUP.
 */
typedef struct dgs_weight_grad_args {
    uint32_t rows, outs, cols;
    int32_t type, accumulate, reserved;
    dgs_matrix dy;
    dgs_codes saved;
    const float *scale, *shift;
    float *dw;
    uint64_t dw_stride;
    float *db;
    void *workspace;
    uint64_t workspace_bytes;
} dgs_weight_grad_args;

size_t dgs_checkpoint_weight_grad_workspace(uint32_t rows, uint32_t outs, uint32_t cols, int type);
int dgs_checkpoint_weight_grad(const dgs_weight_grad_args *args /*host*/, void *hip_stream);

/*
 * The output layer with its loss: logits z = x W^T + bias (W: vocab x cols), softmax cross entropy against one target a row.
 *
 *     lse_t  = log sum_v exp z_tv
 *     loss_t = lse_t - z_t[target_t]               0 where the target is no entry of the vocabulary (negative: padding)
 *
 * and for gradients dloss_t and dlse_t that arrive at them (NULL: 1 for every row, and 0), dloss_t taken as 0 for a row whose
 * target is no entry,
 *
 *     dz_t = (dloss_t + dlse_t) softmax_t - dloss_t onehot(target_t)
 *     dx = dz W,   dweight = dz^T x,   dbias = sum_t dz_t
 *
 * Logits are not kept: the backward pass computes them again, a piece of the vocabulary at a time.
 *
 * x, weight and dx have `type`; bias, loss, lse, dweight and dbias are fp32.  Sums, exponentials and statistics are fp32, of
 * products that are exact (DGS_F32: 2^-22 off; of more than 32 rows, x and W in 22 bits, below 2^-20 of the largest of their row
 * in steps of 2^-41 of it).  dz is held in 22 bits, below
 * 2^-28 of its row's incoming gradients in steps of 2^-49 of them; a dx of DGS_BF16 takes 11 bits, and steps of 2^-38 (of at
 * most 16 rows all).  dbias is summed from fp32.  Of the other operands of the gradients' products, magnitudes below 2^-39 (DGS_F32: 2^-50) of
 * the largest (of W; of x times its row's gradients) are lost.  A bias of -infinity takes an entry out; where all of them are out, and where logits are infinite or
 * NaN, lse is what the formula gives or NaN.
 * A row that nothing arrives at (dloss and dlse 0) leaves no gradient, whatever it holds.
 *
 *   forward    reads x, weight, bias, targets; writes loss (or NULL) and lse.
 *   backward   reads those and lse; writes dx, dweight (rows dweight_stride apart) and dbias, each or none of them.
 *              accumulate != 0: dweight and dbias are added to.
 * Outputs overlap nothing (a loss that overlaps lse: DGS_EINVAL).  workspace: at least dgs_head_workspace() bytes for the same arguments (of the pointers their
 * alignment counts), 16-byte aligned; as above.  More than 2^20 columns, 2^24 rows or entries, 2^34
 * values of x or 2^38 logits: DGS_ENOTSUP.
 */
typedef struct dgs_head_args {
    uint32_t rows, cols, vocab;
    int32_t type, target_bytes, accumulate;     /* targets: 4 or 8 bytes each, signed */
    dgs_matrix x, weight;
    const float *bias;
    const void *targets;
    float *loss, *lse;
    const float *dloss, *dlse;
    dgs_matrix dx;
    float *dweight;
    uint64_t dweight_stride;
    float *dbias;
    void *workspace;
    uint64_t workspace_bytes;
} dgs_head_args;

size_t dgs_head_workspace(const dgs_head_args *args /*host*/, int backward);
int dgs_head_forward(const dgs_head_args *args /*host*/, void *hip_stream);
int dgs_head_backward(const dgs_head_args *args /*host*/, void *hip_stream);

/*
 * Updates of weight matrices, orthogonalised: for each of `count` matrices of one shape, X = G / (|G| + eps) with the Frobenius
 * norm, `steps` times with A = X X^T (X^T in place of X where rows > cols)
 *
 *     X = a X + (b A + c A^2) X
 *
 * and out = scale * X, or with accumulate != 0 out + scale * X, rounded once.  Sums are fp32, the norm's in 64 bits.  Results of
 * DGS_F32 and DGS_F16 take 22 bits of X, A and the polynomial to the products, of DGS_BF16 11; what lies below 2^-15 is held in
 * steps of 2^-37 (of an update whose norm is below eps, in steps as much smaller).  Values of X, A and the polynomial
 * must stay below 16, as they do with coefficients that take singular values up to 1 to such near 1.  A matrix that holds an
 * infinity or NaN leaves NaN; of zeros (with eps > 0) zeros.
 * in, out: host arrays of `count` matrices each, read before the call returns.  out[i] may be in[i] (same type and stride);
 * otherwise outputs overlap nothing.  More than 65536 rows or columns: DGS_ENOTSUP.
 */
typedef struct dgs_orthogonalise_args {
    uint32_t count, rows, cols, steps;          /* steps >= 1 */
    int32_t type, out_type, accumulate, reserved;
    float a, b, c, eps, scale;                  /* eps >= 0 */
    const dgs_matrix *in, *out;
    void *workspace;
    uint64_t workspace_bytes;
} dgs_orthogonalise_args;

size_t dgs_orthogonalise_workspace(const dgs_orthogonalise_args *args /*host*/);
int dgs_orthogonalise(const dgs_orthogonalise_args *args /*host*/, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* DGS_BLOCKS_H */
