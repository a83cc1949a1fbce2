/*
 * arena_experts.h - C ABI of the operators of a mixture-of-experts layer on one
 * MI355X, beside those of arena_layer.h: the jobs of the estimator have such layers
 * (all-to-all bytes on every other one), and these make their cost measurable.
 *
 *   arena_route_forward, arena_route_backward   each token's k experts and weights
 *   arena_sort_by_expert                        where each choice's row lies
 *   arena_dispatch                              tokens to their experts' rows
 *   arena_combine, arena_combine_backward       and back, with the weights applied
 *   arena_experts_forward, arena_experts_backward   gated blocks of groups of rows
 *
 * The conventions, types, workspaces and limits of arena_layer.h hold here.  Index
 * and offset values lie in device memory, where the host cannot check them: the
 * kernels hold every one inside its range, as said at each call, so none of them can
 * lead a read or write out of a tensor.  Outputs overlap neither inputs nor each other.
 */
#ifndef ARENA_EXPERTS_H
#define ARENA_EXPERTS_H

#include "arena_layer.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Limits (ARENA_ERR_UNSUPPORTED beyond them). */
#define ARENA_MAX_EXPERTS 1024
#define ARENA_ROUTE_MAX_CHOICES 16         /* experts that the router chooses for a token */
#define ARENA_MAX_CHOICES 64               /* rows that a token is sent to */

/* Types of whole numbers. */
#define ARENA_I32 3
#define ARENA_I64 4

/* ------------------------------------------------------------------ */
/* Router                                                               */
/* ------------------------------------------------------------------ */

/* Of each token's logits the k largest in falling order, of equal ones the lowest
 * index first (both zeros are equal; NaN is larger than every number):
 *   index[t, j] = e_j,  weight[t, j] = scale p_{e_j} / (normalise ? sum_i p_{e_i} : 1)
 * with p the softmax over all experts.  An expert whose logit is -inf is never
 * chosen; choices that are left over have index -1 and weight 0.  A logit of NaN or
 * +inf makes the token's weights NaN. */
typedef struct arena_route_desc {
    int32_t dtype;            /* of the logits: ARENA_F32, BF16 or F16 */
    int32_t experts;          /* 1..ARENA_MAX_EXPERTS */
    int32_t k;                /* 1..min(experts, ARENA_ROUTE_MAX_CHOICES) */
    int32_t normalise;
    int64_t tokens;           /* 0 is allowed */
    float scale;              /* finite */
    const void* logits; int64_t ld_logits;
    int32_t* index;           /* [tokens][k] */
    float* weight;            /* [tokens][k]; not used by the backward pass */
} arena_route_desc;

arena_status arena_route_forward(arena_ctx* ctx, const arena_route_desc* d, void* stream);

/* dlogits (of dtype, rows of ld_dlogits) from the weights' gradient dweight
 * (float32, rows of ld_dweight), the forward's logits and its index: the choice
 * itself has no gradient.  Indices outside of 0..experts-1 are choices left over. */
arena_status arena_route_backward(arena_ctx* ctx, const arena_route_desc* f, const float* dweight, int64_t ld_dweight,
                                  void* dlogits, int64_t ld_dlogits, void* stream);

/* ------------------------------------------------------------------ */
/* Tokens to experts and back                                           */
/* ------------------------------------------------------------------ */

/* Choices (t, j) in order of their expert, within one in order of t and j:
 *   offsets[e] .. offsets[e + 1] - 1  are expert e's rows,  row[t, j] that of a choice.
 * An index outside of 0..experts-1 (the router's -1) is dropped: row -1. */
typedef struct arena_sort_desc {
    int32_t index_dtype;      /* ARENA_I32 or ARENA_I64 */
    int32_t experts;          /* 1..ARENA_MAX_EXPERTS */
    int64_t tokens;           /* 0 is allowed */
    int32_t k;                /* 1..ARENA_MAX_CHOICES */
    const void* index;        /* [tokens][k] */
    int32_t* offsets;         /* [experts + 1] */
    int32_t* row;             /* [tokens][k] */
    void* workspace; int64_t workspace_bytes;
} arena_sort_desc;

arena_status arena_sort_by_expert_workspace(arena_ctx* ctx, const arena_sort_desc* d, int64_t* bytes);
arena_status arena_sort_by_expert(arena_ctx* ctx, const arena_sort_desc* d, void* stream);

/* Matrices of a row a token (x, y, dy, dx: [tokens, model]) and of a row a choice
 * (xs, ys, dys, dxs: [rows, model]), all of dtype.  A row index outside of 0..rows-1 is a
 * dropped choice.  Rows of choices that none names are not written. */
typedef struct arena_move_desc {
    int32_t dtype;            /* ARENA_F32, BF16 or F16 */
    int32_t model;            /* >= 1 */
    int64_t tokens, rows;     /* 0 is allowed */
    int32_t k;                /* 1..ARENA_MAX_CHOICES */
    const int32_t* row;       /* [tokens][k], no row twice */
    const float* weight; int64_t ld_weight;   /* float32 [tokens][k] */
} arena_move_desc;

/* xs[row[t, j]] = x[t]; weight is not used.  Its gradient is arena_combine without weights. */
arena_status arena_dispatch(arena_ctx* ctx, const arena_move_desc* d, const void* x, int64_t ld_x, void* xs,
                            int64_t ld_xs, void* stream);

/* y[t] = sum_j weight[t, j] ys[row[t, j]] over the choices that are not dropped, in
 * 32 bits, rounded once; weight NULL: 1. */
arena_status arena_combine(arena_ctx* ctx, const arena_move_desc* d, const void* ys, int64_t ld_ys, void* y,
                           int64_t ld_y, void* stream);

/* dys[row[t, j]] = weight[t, j] dy[t] and dweight[t, j] = <dy[t], ys[row[t, j]]>
 * (float32 [tokens][k]; 0 of a dropped choice). */
arena_status arena_combine_backward(arena_ctx* ctx, const arena_move_desc* d, const void* dy, int64_t ld_dy,
                                    const void* ys, int64_t ld_ys, void* dys, int64_t ld_dys, float* dweight,
                                    void* stream);

/* ------------------------------------------------------------------ */
/* Experts' gated blocks                                                */
/* ------------------------------------------------------------------ */

/* The gated block of arena_layer.h for groups of rows: rows offsets[e] ..
 * offsets[e + 1] - 1 of x and y meet matrix e of w_gate and w_up [experts, inner, model] and
 * w_down [experts, model, inner], stride_* values apart.  Rows outside of all groups
 * are neither read nor written, whatever they hold.  offsets is [experts + 1] in device memory,
 * 0 <= offsets[e] <= offsets[e + 1] <= rows (values past that are held to it; groups
 * that overlap leave shared rows to either).  g, u and h as there, with `rows` in the
 * place of `tokens`; an expert without rows is allowed, as is no row at all. */
typedef struct arena_experts_desc {
    int32_t dtype;            /* ARENA_BF16 or ARENA_F16 */
    int32_t activation;       /* ARENA_ACT_* */
    int64_t rows;             /* 0 is allowed */
    int32_t model, inner;     /* >= 1 */
    int32_t experts;          /* 1..ARENA_MAX_EXPERTS */
    const int32_t* offsets;
    const void* x; int64_t ld_x;
    const void* w_gate; int64_t ld_gate, stride_gate;
    const void* w_up; int64_t ld_up, stride_up;
    const void* w_down; int64_t ld_down, stride_down;
    void *g, *u, *h; int64_t ld_inner;
    void* y; int64_t ld_y;    /* not used by the backward pass */
    void* workspace; int64_t workspace_bytes;
} arena_experts_desc;

arena_status arena_experts_forward_workspace(arena_ctx* ctx, const arena_experts_desc* d, int64_t* bytes);
arena_status arena_experts_forward(arena_ctx* ctx, const arena_experts_desc* d, void* stream);

/* Gradients as of arena_ffn_backward.  The weights' are zero (with accumulate: as they
 * were) for an expert without rows. */
typedef struct arena_experts_grads {
    int32_t grad_dtype, accumulate;
    const void* dy; int64_t ld_dy;
    void* dx; int64_t ld_dx;
    void* dw_gate; int64_t ld_dw_gate, stride_dw_gate;
    void* dw_up; int64_t ld_dw_up, stride_dw_up;
    void* dw_down; int64_t ld_dw_down, stride_dw_down;
} arena_experts_grads;

arena_status arena_experts_backward_workspace(arena_ctx* ctx, const arena_experts_desc* f,
                                              const arena_experts_grads* g, int64_t* bytes);
arena_status arena_experts_backward(arena_ctx* ctx, const arena_experts_desc* f, const arena_experts_grads* g,
                                    void* stream);

#ifdef __cplusplus
}
#endif

#endif /* ARENA_EXPERTS_H */
