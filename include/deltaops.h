/*
 * deltaops.h -- C ABI of the operators of a block that learns by the gated delta rule, for MI355X (gfx950), in libdwconv.so:
 *
 *   gdelta_*  the gated delta rule over packed token sequences, forward, backward and one token at a time;
 *   hnorm_*   the RMS norm of each head with a gate, forward and backward (what follows the rule);
 *   rnorm_*   the RMS norms after a block and before the next one, with the block's gate, the residual's scale and sum, forward and backward.
 *
 * Types, status codes, streams, workspaces, errors, tokens, sequences and rows are those of seqops.h: every data pointer is a device pointer owned by the caller, the
 * library never allocates, copies or synchronises, all work is enqueued on `stream`, arguments are checked on the host before the first HIP call, every output is
 * overwritten, no output may alias an input (the state of a step, which is updated in place, aside), and no atomics are used: results are bit-identical
 * from run to run.  A workspace is scratch of one call: calls that may run at the same time, and graphs that may be replayed at the same time, need one each.
 *
 * dtype F32: all tensors are fp32.  dtype BF16: tensors marked "stored" hold bf16, everything else is fp32 (int32 for `starts` and `slots`).
 * Sums, statistics and states are held in fp32 or wider; a stored output is rounded once, to nearest-even.  Sums of squares are fp32: where one passes its range (numbers
 * of 1e19 and more in a row) what is divided by its root is not specified.
 */
#ifndef DELTAOPS_H
#define DELTAOPS_H

#include "seqops.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- gated delta rule ----------------------------------------------------------------------------
 *
 * H value heads with a state S of K x V numbers each; H / key_heads neighbouring value heads share a key head (h / (H / key_heads), below: their q and k).
 *   g[t,h] = A[h] * softplus(a[t,h] + a_bias[h])     (without softplus: A * the sum itself)
 *   beta[t,h] = 1 / (1 + exp(-b[t,h]))               (without sigmoid: b itself)
 *   qn = q / sqrt(sum q^2 + eps), kn likewise        (without norm: q and k themselves)
 *   S[t] = exp(g) * S[t-1] + beta * kn (v[t] - exp(g) * S[t-1]^T kn)^T
 *   y[t,h] = scale * S[t]^T qn
 * S before a sequence's first token is the sequence's row of `init` ([sequences,H,K,V]), or zero; `final` gets S after each sequence's last token (init's row, or
 * zero, where the sequence is empty).  init is a constant of the backward pass.  g is taken as -256 where it is less: its decay is zero in fp32 long before.
 * A number that is not finite leaves the outputs of its head before its token, of the other heads, and of other sequences as they were; which of the head's outputs from
 * its token on are not finite is not specified.  The same holds for the gradients of other sequences, and of heads of other key heads.
 * Decays may grow (with A > 0, or without softplus): over any run of neighbouring tokens of a sequence g may add up to 87 - ln(max(r, 1000)), which is 80, or less where r is over
 * 1000: with norm the largest of 1 / |k| and |scale| / (|q| |k|), where |x| = sqrt(sum x^2 + eps), without it the largest of |scale|, |scale| |q| |k| and |beta| |k|^2.  Where it adds up
 * to more, the head's answers from that run's end on, the sequence's `final` and its gradients may be NaN though the formula's numbers are finite.  Answers before that, or before the
 * first number that passes fp32, other heads and other sequences keep their bits.  What decays by more than e^-87 over a run of tokens may count as nothing, however large it was.
 * gdelta_step has neither bound.
 *
 * T / 64 + sequences must be less than 2^31.  What is computed between tokens holds 24 bits with bf16 tensors too, and y has the same bits whatever else a call is
 * asked for.  A backward pass takes `starts` where its forward pass did, with the same values, and the same value of DWCONV_TUNE_GDELTA_PIECE (the chunks of 64 tokens
 * that a piece of a long sequence has, by default chosen from the sizes; kept's layout goes by it). */
#define GDELTA_MAX_K 256
#define GDELTA_MAX_V 256
#define GDELTA_MAX_H 65535          /* value heads */
#define GDELTA_MAX_STRIDE (1 << 22) /* elements from one row to the next */
typedef struct gdelta_desc {
    int32_t T, H;               /* tokens >= 0, value heads >= 1                                            */
    int32_t K, V;               /* 1 <= K <= GDELTA_MAX_K, 1 <= V <= GDELTA_MAX_V                           */
    int32_t key_heads;          /* >= 1, divides H                                                          */
    int32_t sequences;          /* >= 1; a step: the number of slots of `state`                             */
    int32_t dtype;              /* enum dwconv_dtype                                                        */
    int32_t softplus, sigmoid, norm; /* 0 or 1 each                                                         */
    float scale, eps;           /* finite; eps >= 0                                                         */
    int64_t q_stride, k_stride, v_stride, a_stride, b_stride, y_stride; /* of the rows of q, k, v, a, b and y (and their gradients) */
} gdelta_desc;

typedef struct gdelta_tensors {
    const void *q, *k;      /* stored, T rows of key_heads * K                                              */
    const void *v;          /* stored, T rows of H * V                                                      */
    const void *a, *b;      /* stored, T rows of H                                                          */
    const void *A, *a_bias; /* fp32 [H]; each may be NULL (minus ones, zeros)                               */
    const void *starts;     /* int32 [sequences+1], may be NULL                                             */
    const void *init;       /* fp32 [sequences,H,K,V], may be NULL                                          */
    void *y;                /* stored, T rows of H * V                                                      */
    void *final;            /* fp32 [sequences,H,K,V], may be NULL                                          */
    void *kept;             /* gdelta_kept_bytes(desc), what a backward pass needs of the forward one: written by the forward pass (NULL where
                             * no backward pass follows), read by the backward pass                         */
    const void *slots;      /* int32 [T], may be NULL                                                       */
    void *state;            /* fp32 [sequences,H,K,V]                                                       */
    const void *dy;         /* stored, T rows of H * V                                                      */
    void *dq, *dk;          /* stored, T rows of key_heads * K                                              */
    void *dv;               /* stored, T rows of H * V                                                      */
    void *da, *db;          /* stored, T rows of H                                                          */
    void *dA, *da_bias;     /* fp32 [H], each may be NULL                                                   */
} gdelta_tensors;

/* Bytes of `kept` and of the two passes' device scratch; host-only; 0 for an invalid desc (a workspace of 0 bytes may be NULL). */
size_t gdelta_kept_bytes(const gdelta_desc *desc);
size_t gdelta_fwd_workspace_bytes(const gdelta_desc *desc);
size_t gdelta_bwd_workspace_bytes(const gdelta_desc *desc);
/* q, k, v, a, b, A, a_bias, starts, init: read.  y, final, kept: written.  Where kept is given no workspace is used (it may be NULL). */
int gdelta_fwd(const gdelta_desc *desc, const gdelta_tensors *tensors, void *workspace, size_t workspace_bytes, void *stream);
/* What the forward pass read (init aside, whose part kept holds), kept and dy: read.  dq, dk, dv, da, db, dA, da_bias: written. */
int gdelta_bwd(const gdelta_desc *desc, const gdelta_tensors *tensors, void *workspace, size_t workspace_bytes, void *stream);
/* One new token for each of T rows: row t takes slot slots[t] of `state` (slot t without slots; T <= sequences then) and moves it on by its token.  A row whose slot
 * is outside 0 .. sequences - 1 is padding: its y is zero.  No slot may appear twice.
 * q, k, v, a, b, A, a_bias, slots: read.  y: written.  state: read and written. */
int gdelta_step(const gdelta_desc *desc, const gdelta_tensors *tensors, void *stream);

/* ---- norm of heads with a gate --------------------------------------------------------------------
 *
 * Rows of H runs of D channels, each run normalised by itself; w is shared by the runs.
 *   rstd[t,h] = 1 / sqrt(sum_d x^2 / D + eps),  n = x * rstd
 *   y = n * w[d] * act(z)             act(z) = z / (1 + exp(-z)) with silu, else 1 / (1 + exp(-z)); without z: 1
 *   dx = rstd * (g - n * sum_d (g * n) / D) with g = dy * act(z) * w,  dz = dy * n * w * act'(z),  dw[d] = sum_{t,h} dy * act(z) * n */
#define HNORM_MAX_D 1024
typedef struct hnorm_desc {
    int32_t T, H, D;   /* tokens >= 0, runs >= 1, 1 <= D <= HNORM_MAX_D                */
    int32_t dtype;     /* enum dwconv_dtype                                            */
    int32_t silu;      /* 0 or 1                                                       */
    float eps;         /* >= 0                                                         */
    int64_t x_stride, z_stride, y_stride; /* of the rows of x and dx, z and dz, y and dy */
} hnorm_desc;

typedef struct hnorm_tensors {
    const void *x;     /* stored, T rows of H * D                                      */
    const void *z;     /* stored, T rows of H * D, may be NULL (no gate)               */
    const void *w;     /* stored [D], may be NULL (ones)                               */
    void *y;           /* stored, T rows of H * D                                      */
    void *rstd;        /* fp32 [T,H]: output of the forward pass (may be NULL), input of the backward pass */
    const void *dy;    /* stored, T rows of H * D                                      */
    void *dx;          /* stored, T rows of H * D                                      */
    void *dz;          /* stored, T rows of H * D, NULL where z is                     */
    void *dw;          /* fp32 [D], may be NULL                                        */
} hnorm_tensors;

/* x, z, w: read.  y, rstd: written. */
int hnorm_fwd(const hnorm_desc *desc, const hnorm_tensors *tensors, void *stream);
/* Device scratch of hnorm_bwd; host-only; 0 for an invalid desc. */
size_t hnorm_bwd_workspace_bytes(const hnorm_desc *desc);
/* x, z, w, rstd, dy: read.  dx, dz, dw: written. */
int hnorm_bwd(const hnorm_desc *desc, const hnorm_tensors *tensors, void *workspace, size_t workspace_bytes, void *stream);

/* ---- norms around a block ------------------------------------------------------------------------
 *
 *   p = x * rstd1 * w1[c] with rstd1[t] = 1 / sqrt(sum_c x^2 / C + eps)     (without post: p = x)
 *   s = residual + alpha * scale[c] * p * act(z)                           (act as for hnorm; what is NULL is left out)
 *   y = s * rstd2 * w2[c] with rstd2[t] = 1 / sqrt(sum_c s^2 / C + eps)     (y may be NULL: no block follows)
 * and, with n2 = s * rstd2 and g2 = dy * w2,
 *   dresidual = ds = rstd2 * (g2 - n2 * sum_c (g2 * n2) / C) + dtotal,  dw2[c] = sum_t dy * n2
 *   dscale[c] = sum_t alpha * ds * p * act(z),  dz = alpha * scale * ds * p * act'(z)
 *   dx = rstd1 * (g1 - n1 * sum_c (g1 * n1) / C) with g1 = alpha * scale * ds * act(z) * w1 and n1 = x * rstd1 (without post: alpha * scale * ds * act(z)),
 *   dw1[c] = sum_t alpha * scale * ds * act(z) * n1
 * Rows are dense but for those of x and dx, z and dz. */
#define RNORM_MAX_C 8192
typedef struct rnorm_desc {
    int32_t T, C;      /* tokens >= 0, 1 <= channels <= RNORM_MAX_C                    */
    int32_t dtype;     /* enum dwconv_dtype                                            */
    int32_t post;      /* 0 or 1: whether the block's output is normalised             */
    int32_t silu;      /* 0 or 1                                                       */
    float eps;         /* >= 0                                                         */
    float alpha;       /* finite                                                       */
    int32_t reserved;  /* 0                                                            */
    int64_t x_stride, z_stride; /* of the rows of x and dx, z and dz                   */
} rnorm_desc;

typedef struct rnorm_tensors {
    const void *x;             /* stored, T rows of C; the backward pass needs it with post, z or scale                                             */
    const void *z;             /* stored, T rows of C, may be NULL (no gate)                                                                        */
    const void *residual;      /* stored [T,C], may be NULL (zeros)                                                                                 */
    const void *w1, *scale, *w2; /* stored [C]; each may be NULL (ones); w1 needs post                                                              */
    void *total;               /* stored [T,C]: s, rounded; output of the forward pass, input of the backward pass (where there is dy)              */
    void *y;                   /* stored [T,C], may be NULL                                                                                         */
    void *rstd1, *rstd2;       /* fp32 [T]: outputs of the forward pass (each may be NULL), inputs of the backward pass with post and with dy       */
    const void *dy;            /* stored [T,C], NULL where y was                                                                                    */
    const void *dtotal;        /* stored [T,C], the gradient that arrives at total; may be NULL where there is dy                                   */
    void *dx;                  /* stored, T rows of C                                                                                               */
    void *dz;                  /* stored, T rows of C, NULL where z is                                                                              */
    void *dresidual;           /* stored [T,C], may be NULL                                                                                         */
    void *dw1, *dscale, *dw2;  /* fp32 [C], each may be NULL; dw1 needs post, dw2 needs dy, dscale needs scale                                      */
} rnorm_tensors;

/* x, z, residual, w1, scale, w2: read.  total, y, rstd1, rstd2: written. */
int rnorm_fwd(const rnorm_desc *desc, const rnorm_tensors *tensors, void *stream);
/* Device scratch of rnorm_bwd; host-only; 0 for an invalid desc. */
size_t rnorm_bwd_workspace_bytes(const rnorm_desc *desc);
/* x, z, w1, scale, w2, total, rstd1, rstd2, dy, dtotal: read.  dx, dz, dresidual, dw1, dscale, dw2: written. */
int rnorm_bwd(const rnorm_desc *desc, const rnorm_tensors *tensors, void *workspace, size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* DELTAOPS_H */
