/*
 * libdgs, training blocks -- the memory-bound part of a transformer worker's step, around the hot path of dgs.h: what lies
 * between two blocks (norm, gate, residual sum, norm), the 8-bit checkpoints that the forward pass keeps for the backward
 * pass, and the gradients that are read from them.  Parameters and their gradients are fp32, as in the flat buffers of
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

#ifdef __cplusplus
}
#endif
#endif /* DGS_BLOCKS_H */
