/*
 * arena_layer.h - C ABI of the layer operators: the training step of a gated
 * feed-forward sub-layer on one MI355X.
 *
 * The estimator of arena.h prices plans from per-layer tables: the seconds of
 * a layer's forward and backward pass, its parameter, activation and boundary
 * bytes (the profiled operators of Sec. 3.4 of the paper).  The operators here
 * are such a layer's parts as kernels of this library, so the rows of a job can
 * be measured on the machine (paper_2403_16125_amd/layer_profile.py).
 *
 *   arena_norm_forward, arena_norm_backward    norms before and after a block,
 *                                              its gate and the residual scale
 *   arena_ffn_forward, arena_ffn_backward      gated feed-forward block
 *   arena_orthogonal_update                    orthogonalised weight update
 *
 * Conventions of arena.h: every function returns an arena_status and never
 * throws; arguments are validated on the host before anything is enqueued, on
 * error nothing is written and arena_last_error() says why.  The context names
 * the device and carries the error text; it holds no state of these calls, so
 * one context serves any number of streams (one thread at a time).  All
 * pointers are caller-owned DEVICE memory.  Matrices are row-major; ld_* is
 * the distance of two rows in elements.  Calls are asynchronous on `stream` (a
 * hipStream_t; NULL is the null stream), allocate nothing and synchronise
 * nothing, so a captured stream records them.  Outputs must not overlap inputs or
 * each other, except where said.  The same inputs give the same bits.
 *
 * Workspace: arena_*_workspace gives the bytes that a call with the same
 * descriptor needs (its pointers' values matter only in being NULL or not and
 * in their alignment); the caller passes that much device memory, aligned to
 * 256 bytes, for the time of the call on the stream.  0 bytes: may be NULL.
 *
 * Types: ARENA_BF16 and ARENA_F16 (and ARENA_F32 where said).  Products take
 * 16-bit operands and sum in 32 bits; sums, statistics and activation
 * functions are in 32 bits (sums of squares of an update in 64).
 */
#ifndef ARENA_LAYER_H
#define ARENA_LAYER_H

#include "arena.h"

#ifdef __cplusplus
extern "C" {
#endif

#define ARENA_F32 0
#define ARENA_BF16 1
#define ARENA_F16 2

/* Limits (ARENA_ERR_UNSUPPORTED beyond them). */
#define ARENA_LAYER_MAX_LD ((1 << 22) - 8)  /* row stride and width of a product's matrix, elements */
#define ARENA_LAYER_MAX_TOKENS 0x3fffffff   /* tokens of a call */
#define ARENA_NORM_MAX_WIDTH 16384          /* values of a row that a norm covers */
#define ARENA_UPDATE_MAX_SIDE 32768         /* rows and columns of an orthogonalised matrix */
#define ARENA_UPDATE_MAX_STEPS 16
#define ARENA_UPDATE_MAX_BATCH 4096

/* ------------------------------------------------------------------ */
/* Norms around a block                                                 */
/* ------------------------------------------------------------------ */

#define ARENA_NORM_RMS 0
#define ARENA_NORM_LAYER 1

/* For each token (row):
 *   v = norm(y) w_post + b_post,  r = x + scale gate v,  n = norm(r) w_pre + b_pre
 *   norm(z) = (z - mu) / sqrt(mean((z - mu)^2) + eps), mu = mean(z) (LAYER) or 0 (RMS)
 * x is the residual stream before a block and y the block's output; r is the
 * stream after it and n the input of the next block.  y NULL: no block before
 * (r = x, not written).  n NULL: no block after.  The weights, biases and the gate
 * are optional (1, 0, 1).  Gate rows: row t / gate_rows scales token t;
 * gate_rows 0 is one row for all tokens.  n is formed from r in 32 bits, before r is rounded;
 * the backward pass starts from r as it is stored, so a 16-bit stream costs it that rounding. */
typedef struct arena_norm_desc {
    int32_t dtype;            /* of y, n, gate, weights, biases: ARENA_F32, BF16 or F16 */
    int32_t stream_dtype;     /* of x and r: dtype or ARENA_F32 */
    int32_t kind;             /* ARENA_NORM_RMS or ARENA_NORM_LAYER */
    int32_t width;            /* 1..ARENA_NORM_MAX_WIDTH */
    int64_t tokens;           /* 0 is allowed */
    int64_t gate_rows;
    float eps;                /* >= 0, finite */
    float scale;              /* finite */
    const void* x; int64_t ld_x;
    const void* y; int64_t ld_y;
    const void* gate; int64_t ld_gate;
    const void *w_post, *b_post, *w_pre, *b_pre;
    void* r; int64_t ld_r;    /* may be x itself (same pointer and stride) */
    void* n; int64_t ld_n;
    float* stats;             /* [tokens][4], nullable: the rows' means and 1 / deviations for the backward pass */
} arena_norm_desc;

arena_status arena_norm_forward(arena_ctx* ctx, const arena_norm_desc* d, void* stream);

/* Gradients.  `f` is the forward's descriptor (x and n are not read; r is, or x
 * where y is NULL; stats is required).  Given dn and dr, the gradients of n and
 * r (either may be NULL: none), writes those of x (dx, of stream_dtype), y, the
 * gate (dense rows of `width`), weights and biases (of dtype); NULL outputs are
 * not computed.  dx may be dr itself (same pointer and stride), with the same bits. */
typedef struct arena_norm_grads {
    const void* dn; int64_t ld_dn;
    const void* dr; int64_t ld_dr;
    void* dx; int64_t ld_dx;
    void* dy; int64_t ld_dy;
    void *dgate, *dw_post, *db_post, *dw_pre, *db_pre;
    void* workspace; int64_t workspace_bytes;
} arena_norm_grads;

arena_status arena_norm_backward_workspace(arena_ctx* ctx, const arena_norm_desc* f, int64_t* bytes);
arena_status arena_norm_backward(arena_ctx* ctx, const arena_norm_desc* f, const arena_norm_grads* g, void* stream);

/* ------------------------------------------------------------------ */
/* Gated feed-forward block                                             */
/* ------------------------------------------------------------------ */

#define ARENA_ACT_SILU 0   /* z / (1 + exp(-z)) */
#define ARENA_ACT_GELU 1   /* z (1 + erf(z / sqrt 2)) / 2 */
#define ARENA_ACT_RELU 2   /* max(z, 0) */

/* g = x w_gate^T, u = x w_up^T, h = act(g) u, y = h w_down^T, with x [tokens, model],
 * w_gate and w_up [inner, model], w_down [model, inner], y [tokens, model].  h
 * has `tokens` rows of ld_inner values; g and u, kept in 24 bits a value for the backward
 * pass, take 3 tokens ld_inner bytes each (rows of 16-bit heads, then rows of
 * 8-bit tails).  All three are 16-byte aligned, ld_inner is a multiple of 8 and
 * at least `inner`; columns past `inner` up to the next multiple of 8 are
 * written as zeros.  g and u NULL (both): not kept, as where no backward pass follows.
 * h, and the gradients of g and u that the backward pass forms, are rounded to dtype as
 * the next products' operands: in float16 an h past 65504 is infinite and gradients below
 * 6e-5 lose bits, whatever the type of the weights' gradients.  Any alignment and stride of x, y and the
 * weights; 16-byte aligned ones with widths and strides of multiples of 8 are
 * read in place, others are copied to the workspace first. */
typedef struct arena_ffn_desc {
    int32_t dtype;            /* ARENA_BF16 or ARENA_F16 */
    int32_t activation;       /* ARENA_ACT_* */
    int64_t tokens;           /* 0 is allowed */
    int32_t model, inner;     /* >= 1 */
    const void* x; int64_t ld_x;
    const void* w_gate; int64_t ld_gate;
    const void* w_up; int64_t ld_up;
    const void* w_down; int64_t ld_down;
    void *g, *u, *h; int64_t ld_inner;
    void* y; int64_t ld_y;    /* not used by the backward pass */
    void* workspace; int64_t workspace_bytes;
} arena_ffn_desc;

arena_status arena_ffn_forward_workspace(arena_ctx* ctx, const arena_ffn_desc* d, int64_t* bytes);
arena_status arena_ffn_forward(arena_ctx* ctx, const arena_ffn_desc* d, void* stream);

/* Gradients of x and the weights from dy, with the forward's x, weights, g, u
 * and h.  grad_dtype is the type of the weights' gradients: dtype, or ARENA_F32;
 * accumulate != 0 adds to what they hold (micro-batches of one step).  NULL
 * outputs are not computed. */
typedef struct arena_ffn_grads {
    int32_t grad_dtype, accumulate;
    const void* dy; int64_t ld_dy;
    void* dx; int64_t ld_dx;
    void* dw_gate; int64_t ld_dw_gate;
    void* dw_up; int64_t ld_dw_up;
    void* dw_down; int64_t ld_dw_down;
} arena_ffn_grads;

arena_status arena_ffn_backward_workspace(arena_ctx* ctx, const arena_ffn_desc* f, const arena_ffn_grads* g,
                                          int64_t* bytes);
arena_status arena_ffn_backward(arena_ctx* ctx, const arena_ffn_desc* f, const arena_ffn_grads* g, void* stream);

/* ------------------------------------------------------------------ */
/* Orthogonalised update                                                */
/* ------------------------------------------------------------------ */

/* For each of `batch` matrices:
 *   M' = mu M + G,  U = G + mu M' (nesterov) or M'    (momentum NULL: U = G)
 *   X = U / (|U|_F + eps);  `steps` times  X <- a X + (b A + c A^2) X, A = X X^T
 *   out = scale X
 * with (a, b, c) = coefficients[step].  A is formed on the smaller side.  The
 * products' operands are float16 scaled by 2^12, whatever the gradient's type; what
 * rounding takes off X goes along beside it (but for the last two steps), as its
 * share on small singular values would grow by `a` a step.  Polynomials whose iterates can
 * leave the magnitudes that holds (15, starting from singular values of at most
 * 1) are refused as UNSUPPORTED.  Out of bfloat16 or float16 type
 * (a float16 out overflows past 65504, as any conversion). */
typedef struct arena_update_desc {
    int32_t dtype;                 /* of the gradient: ARENA_F32, BF16 or F16 */
    int32_t out_dtype;             /* ARENA_BF16 or ARENA_F16 */
    int32_t batch, rows, cols;     /* >= 1 */
    int32_t steps;                 /* 0..ARENA_UPDATE_MAX_STEPS */
    int32_t nesterov;
    float mu, eps, scale;          /* finite; eps >= 0 */
    const float* coefficients;     /* HOST [steps][3], read during the call */
    const void* grad; int64_t ld_grad, stride_grad;              /* stride: elements between matrices */
    const float* momentum; int64_t ld_momentum, stride_momentum; /* nullable */
    float* momentum_out; int64_t ld_momentum_out, stride_momentum_out; /* M'; may be momentum itself */
    void* out; int64_t ld_out, stride_out;
    void* workspace; int64_t workspace_bytes;
} arena_update_desc;

arena_status arena_orthogonal_update_workspace(arena_ctx* ctx, const arena_update_desc* d, int64_t* bytes);
arena_status arena_orthogonal_update(arena_ctx* ctx, const arena_update_desc* d, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* ARENA_LAYER_H */
