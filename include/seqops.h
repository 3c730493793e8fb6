/*
 * seqops.h -- C ABI of the operators around a depthwise convolution over a token sequence, for MI355X (gfx950), in libdwconv.so:
 *
 *   lnorm_*   layer norm over the channels of each token, forward and backward, with the residual's sum;
 *   cconv_*   the short causal depthwise convolution over tokens, forward, backward and one token at a time;
 *   sscan_*   the selective state space scan that reads the convolution's output, forward, backward and one token at a time.
 *
 * Types, status codes, streams, workspaces and errors are those of dwconv.h: every data pointer is a device pointer owned by the caller, the
 * library never allocates, copies or synchronises, all work is enqueued on `stream` (a hipStream_t, NULL = the default stream; its device
 * must be the current one), arguments are checked on the host before the first HIP call, every output is overwritten, no output may alias an
 * input (the state of a step, which is updated in place, aside), and no atomics are used: results are bit-identical from run to run.
 *
 * Tokens and sequences.  A call takes T >= 0 tokens (rows) packed one after the other into `sequences` >= 1 sequences.  With `starts` NULL
 * the sequences have equal lengths, T / sequences (which has to divide).  Otherwise `starts` points to sequences + 1 ascending int32 on the device,
 * the first 0 and the last T: sequence s is the tokens starts[s] .. starts[s+1] - 1, and may be empty.  Other contents give
 * unspecified values, but nothing outside the tensors is read or written.  With T == 0 the tensors of tokens may be NULL.
 *
 * Rows.  A tensor of tokens is T rows of its width, `stride` elements from one row's start to the next (at least the width where T > 1); a gradient's
 * rows have the stride of the tensor that it is the gradient of.  Offsets are formed in 64 bits.  Pointers need only the alignment
 * of their elements, except workspaces and `kept`, which have to be 16-byte aligned.  Rows that start at a multiple of 16 bytes are the fastest.
 *
 * dtype F32: all tensors are fp32.  dtype BF16: tensors marked "stored" hold bf16, everything else is fp32 (int32 for `starts` and `slots`).
 * Sums, statistics and states are held in fp32 inside the kernels; a stored output is rounded once, to nearest-even.
 */
#ifndef SEQOPS_H
#define SEQOPS_H

#include "dwconv.h"

#ifdef __cplusplus
extern "C" {
#endif

/* What a descriptor may ask for at most; more is DWCONV_ERR_TOO_LARGE (more channels of lnorm, taps of cconv or states of sscan than their own maxima:
 * DWCONV_ERR_UNSUPPORTED; numbers that do not divide, or below their least: DWCONV_ERR_BAD_DIM). */
#define SEQOPS_MAX_T 0x7fff0000      /* tokens, sequences, slots                    */
#define SEQOPS_MAX_C (1 << 24)       /* channels of cconv and sscan                 */
#define SEQOPS_MAX_STRIDE (1 << 25)  /* elements from one row to the next           */

/* ---- layer norm --------------------------------------------------------------------------------
 *
 *   s[t,c] = x[t,c] + residual[t,c]        (residual may be NULL: s = x)
 *   mean[t] = sum_c s / C,  rstd[t] = 1 / sqrt(sum_c (s - mean)^2 / C + eps)
 *   y[t,c] = (s - mean) * rstd * w[c] + b[c]
 * and, with g = dy * w and xhat = (s - mean) * rstd,
 *   dx[t,c] = rstd * (g - sum_c g / C - xhat * sum_c (g * xhat) / C) + dtotal[t,c]     (dtotal may be NULL)
 *   dw[c] = sum_t dy * xhat,  db[c] = sum_t dy
 * dx is the gradient of x and of residual alike.  Rows are dense. */
#define LNORM_MAX_C 16384
typedef struct lnorm_desc {
    int32_t T, C;   /* tokens >= 0, 1 <= channels <= LNORM_MAX_C */
    int32_t dtype;  /* enum dwconv_dtype          */
    float eps;      /* >= 0                       */
} lnorm_desc;

/* What a call does not name is ignored. */
typedef struct lnorm_tensors {
    const void *x;        /* stored [T,C]; the backward pass takes s here (total, or x where there was no residual)   */
    const void *residual; /* stored [T,C], may be NULL; needs total                                                   */
    const void *w, *b;    /* stored [C]; each may be NULL (ones, zeros)                                               */
    void *y;              /* stored [T,C]                                                                             */
    void *total;          /* stored [T,C]: s, rounded; may be NULL without residual, and is not written then           */
    void *mean, *rstd;    /* fp32 [T]: outputs of the forward pass (may be NULL together), inputs of the backward pass */
    const void *dy;       /* stored [T,C]                                                                             */
    const void *dtotal;   /* stored [T,C], the gradient that arrives at total; may be NULL                            */
    void *dx;             /* stored [T,C]                                                                             */
    void *dw, *db;        /* fp32 [C]; may be NULL together                                                           */
} lnorm_tensors;

/* x, residual, w, b: read.  y, total, mean, rstd: written. */
int lnorm_fwd(const lnorm_desc *desc, const lnorm_tensors *tensors, void *stream);
/* Device scratch of lnorm_bwd; host-only; 0 for an invalid desc. */
size_t lnorm_bwd_workspace_bytes(const lnorm_desc *desc);
/* x, w, mean, rstd, dy, dtotal: read.  dx, dw, db: written. */
int lnorm_bwd(const lnorm_desc *desc, const lnorm_tensors *tensors, void *workspace, size_t workspace_bytes, void *stream);

/* ---- causal depthwise convolution over tokens ---------------------------------------------------
 *
 *   p[t,c] = b[c] + sum_{k<K} w[k,c] * x[t-(K-1)+k, c]
 *   y = p, or p / (1 + exp(-p)) where `silu` is set
 * Rows before a sequence's first token are the sequence's row of `init` ([sequences,K-1,C], the last of the K-1 next to the token), or zero.
 * `final` gets the last K-1 rows of each sequence in the same form, rows of init among them where the sequence is shorter.
 *   dx[t,c] = sum_k w[k,c] * dp[t+K-1-k, c] inside the sequence, with dp = dy * dy/dp
 *   dw[k,c] = sum_t dp[t,c] * x[t-(K-1)+k, c],  db[c] = sum_t dp[t,c]
 * init is a constant of the backward pass. */
#define CCONV_MAX_K 8
typedef struct cconv_desc {
    int32_t T, C;               /* tokens >= 0, channels >= 1                                             */
    int32_t K;                  /* taps, 2 <= K <= CCONV_MAX_K                                            */
    int32_t sequences;          /* >= 1; a step: the number of slots of `state`                           */
    int32_t dtype;              /* enum dwconv_dtype                                                      */
    int32_t silu;               /* 0 or 1                                                                 */
    int64_t x_stride, y_stride; /* of the rows of x and dx, and of y and dy, in elements                  */
} cconv_desc;

typedef struct cconv_tensors {
    const void *x;       /* stored, T rows of C                                                   */
    const void *w;       /* stored [K,C]                                                          */
    const void *b;       /* stored [C], may be NULL (zeros)                                       */
    const void *starts;  /* int32 [sequences+1], may be NULL                                      */
    const void *init;    /* stored [sequences,K-1,C], may be NULL                                 */
    void *y;             /* stored, T rows of C                                                   */
    void *final;         /* stored [sequences,K-1,C], may be NULL                                 */
    const void *slots;   /* int32 [T], may be NULL                                                */
    void *state;         /* stored [sequences,K-1,C]                                              */
    const void *dy;      /* stored, T rows of C                                                   */
    void *dx;            /* stored, T rows of C                                                   */
    void *dw, *db;       /* fp32 [K,C] and [C]; db may be NULL                                    */
} cconv_tensors;

/* x, w, b, starts, init: read.  y, final: written. */
int cconv_fwd(const cconv_desc *desc, const cconv_tensors *tensors, void *stream);
/* Device scratch of cconv_bwd; host-only; 0 for an invalid desc. */
size_t cconv_bwd_workspace_bytes(const cconv_desc *desc);
/* x, w, b, starts, init, dy: read.  dx, dw, db: written. */
int cconv_bwd(const cconv_desc *desc, const cconv_tensors *tensors, void *workspace, size_t workspace_bytes, void *stream);
/* One new token for each of T rows: row t takes slot slots[t] of `state` (slot t without slots; T <= sequences then), convolves its K-1 rows and
 * x[t], and moves the slot on by one row.  A row whose slot is outside 0 .. sequences - 1 is padding: its y is zero.  No slot may appear twice.
 * x, w, b, slots: read.  y: written.  state: read and written. */
int cconv_step(const cconv_desc *desc, const cconv_tensors *tensors, void *stream);

/* ---- selective state space scan ------------------------------------------------------------------
 *
 * C channels with N states each; the channels are split into `groups` runs of C / groups that share their rows of B and C (below: g(c)).
 *   delta[t,c] = softplus(dt[t,c] + dt_bias[c])   (without softplus: the sum itself)
 *   h[t,c,n] = exp(delta * A[c,n]) * h[t-1,c,n] + delta * x[t,c] * B[t,g(c),n]
 *   v[t,c] = sum_n C[t,g(c),n] * h[t,c,n] + D[c] * x[t,c]
 *   y = v, or v * z / (1 + exp(-z)) with a gate z
 * h before a sequence's first token is the sequence's row of `init` ([sequences,C,N]), or zero; `final` gets h after each sequence's last token
 * (init's row, or zero, where the sequence is empty).  init is a constant of the backward pass. */
#define SSCAN_MAX_N 64
typedef struct sscan_desc {
    int32_t T, C;      /* tokens >= 0, channels >= 1                                       */
    int32_t N;         /* states of a channel, 1 <= N <= SSCAN_MAX_N                       */
    int32_t groups;    /* >= 1, divides C                                                  */
    int32_t sequences; /* >= 1; a step: the number of slots of `state`                     */
    int32_t dtype;     /* enum dwconv_dtype                                                */
    int32_t softplus;  /* 0 or 1                                                           */
    int32_t reserved;  /* 0                                                                */
    int64_t x_stride, dt_stride, z_stride, b_stride, c_stride, y_stride; /* of the rows of x, dt, z, B, C and y (and their gradients) */
} sscan_desc;

typedef struct sscan_tensors {
    const void *x, *dt;     /* stored, T rows of C                                                    */
    const void *A;          /* fp32 [C,N]                                                             */
    const void *B, *C;      /* stored, T rows of groups * N                                           */
    const void *D;          /* fp32 [C], may be NULL (zeros)                                          */
    const void *z;          /* stored, T rows of C, may be NULL (no gate)                             */
    const void *dt_bias;    /* fp32 [C], may be NULL (zeros)                                          */
    const void *starts;     /* int32 [sequences+1], may be NULL                                       */
    const void *init;       /* fp32 [sequences,C,N], may be NULL                                      */
    void *y;                /* stored, T rows of C                                                    */
    void *final;            /* fp32 [sequences,C,N], may be NULL                                      */
    void *kept;             /* sscan_kept_bytes(desc), what a backward pass needs of the states: written by the forward pass (NULL where
                             * no backward pass follows), read by the backward pass                   */
    const void *slots;      /* int32 [T], may be NULL                                                 */
    void *state;            /* fp32 [sequences,C,N]                                                   */
    const void *dy;         /* stored, T rows of C                                                    */
    void *dx, *ddt;         /* stored, T rows of C                                                    */
    void *dA;               /* fp32 [C,N]                                                             */
    void *dB, *dC;          /* stored, T rows of groups * N                                           */
    void *dD;               /* fp32 [C], NULL where D is                                              */
    void *dz;               /* stored, T rows of C, NULL where z is                                   */
    void *ddt_bias;         /* fp32 [C], may be NULL                                                  */
} sscan_tensors;

/* Bytes of `kept` and of the two passes' device scratch; host-only; 0 for an invalid desc (a workspace of 0 bytes may be NULL). */
size_t sscan_kept_bytes(const sscan_desc *desc);
size_t sscan_fwd_workspace_bytes(const sscan_desc *desc);
size_t sscan_bwd_workspace_bytes(const sscan_desc *desc);
/* x, dt, A, B, C, D, z, dt_bias, starts, init: read.  y, final, kept: written. */
int sscan_fwd(const sscan_desc *desc, const sscan_tensors *tensors, void *workspace, size_t workspace_bytes, void *stream);
/* What the forward pass read, kept and dy: read.  dx, ddt, dA, dB, dC, dD, dz, ddt_bias: written. */
int sscan_bwd(const sscan_desc *desc, const sscan_tensors *tensors, void *workspace, size_t workspace_bytes, void *stream);
/* One new token for each of T rows, on the slots of `state` as in cconv_step.
 * x, dt, A, B, C, D, z, dt_bias, slots: read.  y: written.  state: read and written. */
int sscan_step(const sscan_desc *desc, const sscan_tensors *tensors, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* SEQOPS_H */
