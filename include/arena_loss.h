/*
 * arena_loss.h - C ABI of the cross entropy over a vocabulary on one MI355X: a language
 * model's last layer, which ends every stack that the estimator cuts into stages.
 *
 * The conventions, types, workspaces and limits of arena_layer.h hold here.
 */
#ifndef ARENA_LOSS_H
#define ARENA_LOSS_H

#include "arena_experts.h"

#ifdef __cplusplus
extern "C" {
#endif

#define ARENA_MAX_VOCABULARY (1 << 24)

/* l = x w^T with x [tokens, model] and w [vocabulary, model],
 *   lse[t] = log sum_v exp(l[t, v]),  loss[t] = lse[t] - l[t, target[t]],
 * in 32 bits from the products' sums on.  The logits are formed tile by tile and not
 * kept.  loss is 0 where target[t] = ignore_index (whether or not that is an entry of
 * the vocabulary), NaN where it is any other value outside of 0..vocabulary-1. */
typedef struct arena_loss_desc {
    int32_t dtype;            /* of x and w: ARENA_BF16 or ARENA_F16 */
    int32_t target_dtype;     /* ARENA_I32 or ARENA_I64 */
    int64_t tokens;           /* 0 is allowed */
    int32_t model;            /* >= 1 */
    int32_t vocabulary;       /* 1..ARENA_MAX_VOCABULARY */
    int64_t ignore_index;
    const void* x; int64_t ld_x;
    const void* w; int64_t ld_w;
    const void* target;       /* [tokens] */
    float* loss;              /* [tokens], nullable; not used by the backward pass */
    float* lse;               /* [tokens]: written by the forward pass, read by the backward pass */
    void* workspace; int64_t workspace_bytes;
} arena_loss_desc;

arena_status arena_cross_entropy_forward_workspace(arena_ctx* ctx, const arena_loss_desc* d, int64_t* bytes);
arena_status arena_cross_entropy_forward(arena_ctx* ctx, const arena_loss_desc* d, void* stream);

/* With dloss the losses' gradient (element t at t stride_dloss; 0: one for all),
 *   dl[t, v] = dloss[t] (exp(l[t, v] - lse[t]) - [v = target[t]]),  dx = dl w,  dw = dl^T x.
 * The logits are formed again, in pieces of the vocabulary whose gradient takes at most 256 MB
 * (or 4096 entries), rounded to dtype as the products' operand; in float16 after a power of
 * two that brings the largest dloss to about 2^10.  Of up to 32 tokens there are two operands, the
 * second what rounding took off the first; of more a token's dx and dw are off by the rounding of
 * its entries, most of all its target's: 2^-8 of that in bfloat16, 2^-11 in float16.  dx is
 * summed over the pieces in 32 bits.  A token whose target is ignore_index has a dx of 0 and no
 * part in dw, whatever its x, lse and dloss hold; any other target outside of the vocabulary makes
 * both NaN.  dw is of grad_dtype (dtype or ARENA_F32), accumulate != 0 adds to what it holds.
 * NULL outputs are not computed.
 *
 * exp(l - lse) is off by lse's own rounding, 2^-24 |lse| of it, so the target's entry of dl is off
 * by as much of dloss: of a token whose target has all but 1e-6 of the sum, at an lse of 30, it is
 * rounding for the greater part, and its row of dl need not add up to 0.  loss does not have this
 * error: it is formed from the sum, not from lse. */
typedef struct arena_loss_grads {
    int32_t grad_dtype, accumulate;
    const float* dloss; int64_t stride_dloss;
    void* dx; int64_t ld_dx;
    void* dw; int64_t ld_dw;
} arena_loss_grads;

arena_status arena_cross_entropy_backward_workspace(arena_ctx* ctx, const arena_loss_desc* f,
                                                    const arena_loss_grads* g, int64_t* bytes);
arena_status arena_cross_entropy_backward(arena_ctx* ctx, const arena_loss_desc* f, const arena_loss_grads* g,
                                          void* stream);

#ifdef __cplusplus
}
#endif

#endif /* ARENA_LOSS_H */
