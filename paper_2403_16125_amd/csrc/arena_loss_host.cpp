// Host side of the C ABI declared in include/arena_loss.h: argument checks, pieces of the
// tokens and the vocabulary, workspace layout and launches.  No call allocates device
// memory or synchronises.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>

#include "arena_loss.h"
#include "arena_layer_internal.h"
#include "arena_layer_plan.h"

using namespace arena::plan;
using arena::ctx_clear;
using arena::ctx_fail;
using arena::LossArgs;
using arena::mm::GroupArgs;

namespace {

// Of a forward product: bounds its statistics.  65536 tokens, 32768 x 512, in pieces of 8192 to
// 65536: 2.13 to 2.16 ms, no order in it.
constexpr int64_t kTokenPiece = 32768;
// Of the logits' gradient that a backward pass holds at once, which the last-level cache can hold between
// the products.  With 64, 128, 256, 512 and 1024 MB: 8192 tokens, 131072 x 4096, 27.7, 26.9, 26.8, 26.8 and
// 26.8 ms; 50001 x 1024, 3.31, 3.20, 3.03, 3.08 and 3.21; 2000 tokens, 131072 x 2048, 4.22, 3.96, 3.78,
// 3.69 and 3.70.
constexpr int64_t kGradientBytes = 256 << 20;
// Entries of a piece of the vocabulary, however many tokens.  65536 tokens, 32768 x 1024, with 2048, 4096,
// 8192 and 16384: 17.0, 16.0, 15.4 and 15.3 ms, each twice the memory of the one before (0.5 GB with 4096).
constexpr int64_t kLeastPiece = 4096;

arena_status check_loss(arena_ctx* c, const char* who, const arena_loss_desc* d)
{
    if (!d) return ctx_fail(c, ARENA_ERR_INVALID_ARG, "%s: descriptor is NULL", who);
    if (d->dtype != ARENA_BF16 && d->dtype != ARENA_F16)
        return ctx_fail(c, ARENA_ERR_INVALID_ARG, "%s: dtype=%d is neither bfloat16 nor float16", who, d->dtype);
    if (d->target_dtype != ARENA_I32 && d->target_dtype != ARENA_I64)
        return ctx_fail(c, ARENA_ERR_INVALID_ARG, "%s: target_dtype=%d is neither int32 nor int64", who, d->target_dtype);
    if (d->tokens < 0 || d->model < 1 || d->vocabulary < 1)
        return ctx_fail(c, ARENA_ERR_INVALID_ARG, "%s: tokens=%lld model=%d vocabulary=%d", who, (long long)d->tokens,
                        d->model, d->vocabulary);
    if (d->tokens > ARENA_LAYER_MAX_TOKENS || d->model > ARENA_LAYER_MAX_LD || d->vocabulary > ARENA_MAX_VOCABULARY)
        return ctx_fail(c, ARENA_ERR_UNSUPPORTED, "%s: tokens=%lld model=%d vocabulary=%d (max %d, %d, %d)", who,
                        (long long)d->tokens, d->model, d->vocabulary, ARENA_LAYER_MAX_TOKENS, ARENA_LAYER_MAX_LD,
                        ARENA_MAX_VOCABULARY);
    if (ceil_div(d->vocabulary, 64) * ceil_div(d->model, 64) > 0x7fffffff ||
        ceil_div(d->tokens, 64) * ceil_div(std::max<int64_t>(d->model, kLeastPiece), 64) > 0x7fffffff)
        return ctx_fail(c, ARENA_ERR_UNSUPPORTED, "%s: tokens=%lld model=%d vocabulary=%d make too many tiles", who,
                        (long long)d->tokens, d->model, d->vocabulary);
    arena_status s;
    if ((s = check_matrix(c, who, "w", d->w, d->ld_w, d->model, 2))) return s;
    if (d->tokens == 0) return ARENA_OK;
    if ((s = check_matrix(c, who, "x", d->x, d->ld_x, d->model, 2))) return s;
    const size_t wide = d->target_dtype == ARENA_I64 ? 8 : 4;
    if (!d->target || !d->lse)
        return ctx_fail(c, ARENA_ERR_INVALID_ARG, "%s: %s is NULL", who, d->target ? "lse" : "target");
    if (!aligned(d->target, wide) || !aligned(d->lse, 4) || !aligned(d->loss, 4))
        return ctx_fail(c, ARENA_ERR_INVALID_ARG, "%s: target, loss or lse is not aligned to its values", who);
    return ARENA_OK;
}

arena_status check_loss_grads(arena_ctx* c, const char* who, const arena_loss_desc* d, const arena_loss_grads* g)
{
    if (!g) return ctx_fail(c, ARENA_ERR_INVALID_ARG, "%s: gradient descriptor is NULL", who);
    if (g->grad_dtype != d->dtype && g->grad_dtype != ARENA_F32)
        return ctx_fail(c, ARENA_ERR_INVALID_ARG, "%s: grad_dtype=%d is neither dtype nor float32", who, g->grad_dtype);
    arena_status s;
    if (g->dw && (s = check_matrix(c, who, "dw", g->dw, g->ld_dw, d->model, bytes_of(g->grad_dtype)))) return s;
    if (d->tokens == 0) return ARENA_OK;
    if (!g->dloss) return ctx_fail(c, ARENA_ERR_INVALID_ARG, "%s: dloss is NULL", who);
    if (!aligned(g->dloss, 4) || g->stride_dloss < 0)
        return ctx_fail(c, ARENA_ERR_INVALID_ARG, "%s: dloss is not aligned to its values, or stride_dloss < 0", who);
    if (g->dx && (s = check_matrix(c, who, "dx", g->dx, g->ld_dx, d->model, 2))) return s;
    return ARENA_OK;
}

// The kind of tile for a product with k whole; bytes: what the epilogue moves for a value.
int choose_whole(int64_t M, int64_t N, int64_t steps, double bytes, bool any)
{
    return choose_groups(M, N, steps, 1, bytes, false, 1.0, true, any).kind;
}

LossArgs loss_args(const arena_loss_desc* d)
{
    LossArgs A;
    std::memset(&A, 0, sizeof(A));
    A.tokens = d->tokens;
    A.vocabulary = d->vocabulary;
    A.model = d->model;
    A.target = d->target;
    A.target_wide = d->target_dtype == ARENA_I64;
    A.ignore = d->ignore_index;
    return A;
}

// Whether a forward pass takes the kernel for few tokens, which has more reads of the weights
// in flight than the tiles (one token, 131072 x 4096: 227 us on tiles).
bool few_tokens(const arena_loss_desc* d) { return d->tokens <= 16; }

struct LossPlan {
    Pieces w;
    bool skinny, any;
    int64_t piece;            // tokens
    int kind;
    int64_t columns;          // of tiles
    void *stats, *picked;
    LossPlan(const arena_loss_desc* d, void* base)
        : w(base), skinny(few_tokens(d)),
          any(!Operand::direct(d->x, d->ld_x, d->model) || !Operand::direct(d->w, d->ld_w, d->model)),
          piece(std::min(d->tokens, kTokenPiece)),
          kind(choose_whole(piece, d->vocabulary, ceil_div(d->model, arena::mm::kBK), 0.5, any)),
          columns(ceil_div(d->vocabulary, skinny ? arena::mm::kSkinnyCols : arena::mm::kGroupCols[kind]))
    {
        stats = w.take(8 * piece * columns);
        picked = w.take(4 * piece);
    }
};

// Up to how many tokens the logits' gradient is kept in two operands of 16 bits, the second what
// rounding took off the first.  One entry of a token, its target's, is most of dx and of
// dw[target], so its rounding would be as much as the results' own.  Both operands' rows are
// those of one tile of 64, and one step of 64 of the weights' gradient, so the products read and
// multiply no more (loss with gradients, 131072 x 4096: one token 886 us with one operand, 892 with
// two; 8 tokens 947 and 971; 32 tokens 980 and 1040; 32 tokens, 5000 x 1024, 54 and 58).  Past that they would.
constexpr int64_t kFineTokens = 32;

struct LossBackPlan {
    Pieces w;
    bool any;                         // the weight's rows start on any value
    bool fine;
    int64_t count;                    // rows of the logits' gradient
    int64_t piece, ld_x, ld_g;        // entries of a piece; rows of the copy of x and of the logits' gradient
    bool many;                        // pieces: dx is summed in 32 bits
    void *rows, *scale, *x, *g, *sum, *part;
    LossBackPlan(const arena_loss_desc* d, const arena_loss_grads* o, void* base)
        : w(base), any(!Operand::direct(d->w, d->ld_w, d->model))
    {
        const int64_t T = d->tokens, V = d->vocabulary, D = d->model;
        fine = T > 0 && T <= kFineTokens;
        count = fine ? 2 * T : T;
        piece = V;
        if (2 * count * pad8(V) > kGradientBytes)
            piece = std::min(V, std::max(kLeastPiece, kGradientBytes / (2 * count) / 256 * 256));
        many = piece < V;
        ld_x = pad8(D);
        ld_g = pad8(piece);
        rows = w.take(T * (int64_t)sizeof(arena::mm::LossRow));
        scale = w.take(T > 0 && d->dtype == ARENA_F16 ? 8 : 0);
        x = w.take(2 * count * ld_x);
        g = w.take(2 * count * ld_g);
        sum = w.take((many || fine) && o->dx ? 4 * count * D : 0);
        int64_t most = 0;
        for (int64_t n : {piece, V - (V - 1) / piece * piece}) {
            if (o->dx && T > 0) most = std::max(most, cut_dx(count, D, n, any).part);
            if (o->dw) most = std::max(most, cut_dw(count, D, n).part);
        }
        part = w.take(most);
    }
    static GroupCut cut_dx(int64_t T, int64_t D, int64_t n, bool any)
    {
        return choose_groups(T, D, ceil_div(n, arena::mm::kBK), 1, 4.0, true, 1.0, true, any);
    }
    static GroupCut cut_dw(int64_t T, int64_t D, int64_t n)
    {
        return choose_groups(n, D, ceil_div(T, arena::mm::kBK), 1, 2.0, true, 1.0, true, false);
    }
};

}  // namespace

extern "C" {

arena_status arena_cross_entropy_forward_workspace(arena_ctx* c, const arena_loss_desc* d, int64_t* bytes)
{
    if (!c) return ARENA_ERR_INVALID_ARG;
    ctx_clear(c);
    if (!bytes) return ctx_fail(c, ARENA_ERR_INVALID_ARG, "cross entropy: bytes is NULL");
    const arena_status s = check_loss(c, "cross entropy", d);
    if (s) return s;
    *bytes = d->tokens ? LossPlan(d, nullptr).w.used : 0;
    return ARENA_OK;
}

arena_status arena_cross_entropy_forward(arena_ctx* c, const arena_loss_desc* d, void* stream)
{
    if (!c) return ARENA_ERR_INVALID_ARG;
    ctx_clear(c);
    const char* who = "cross entropy";
    arena_status st = check_loss(c, who, d);
    if (st || d->tokens == 0) return st;
    const LossPlan P(d, d->workspace);
    if ((st = check_workspace(c, who, d->workspace, d->workspace_bytes, P.w.used))) return st;
    DeviceScope scope(arena::ctx_device(c));
    if (scope.status != hipSuccess) return hip_error(c, scope.status, "hipSetDevice");
    hipStream_t s = (hipStream_t)stream;
    hipError_t e;
    const int wide = d->target_dtype == ARENA_I64 ? 8 : 4;
    for (int64_t t = 0; t < d->tokens; t += P.piece) {
        const int64_t n = std::min(P.piece, d->tokens - t);
        GroupArgs A = new_args<GroupArgs>(n, d->vocabulary, d->model);
        A.any = P.any;
        A.a[0] = (const char*)d->x + 2 * t * d->ld_x; A.lda = d->ld_x;
        A.b[0] = d->w; A.ldb = d->ld_w;
        A.target = (const char*)d->target + t * wide;
        A.target_wide = wide == 8;
        A.stats = (float*)P.stats;
        A.picked = (float*)P.picked;
        A.splits = 1;
        e = P.skinny ? arena::mm::launch_skinny_groups(A, d->dtype, arena::mm::kLossLogits, s)
                     : arena::mm::launch_loss(A, d->dtype, arena::mm::kLossLogits, P.kind, s);
        if (e) return hip_error(c, e, "cross entropy logits launch");
        LossArgs L = loss_args(d);
        L.tokens = n;
        L.target = A.target;
        L.stats = (const float*)P.stats;
        L.picked = (const float*)P.picked;
        L.columns = (int)P.columns;
        L.loss = d->loss ? d->loss + t : nullptr;
        L.lse = d->lse + t;
        if ((e = arena::launch_loss_join(L, s))) return hip_error(c, e, "cross entropy join launch");
    }
    return ARENA_OK;
}

arena_status arena_cross_entropy_backward_workspace(arena_ctx* c, const arena_loss_desc* f, const arena_loss_grads* g,
                                                    int64_t* bytes)
{
    if (!c) return ARENA_ERR_INVALID_ARG;
    ctx_clear(c);
    const char* who = "cross entropy backward";
    if (!bytes) return ctx_fail(c, ARENA_ERR_INVALID_ARG, "%s: bytes is NULL", who);
    arena_status s;
    if ((s = check_loss(c, who, f)) || (s = check_loss_grads(c, who, f, g))) return s;
    *bytes = LossBackPlan(f, g, nullptr).w.used;
    return ARENA_OK;
}

arena_status arena_cross_entropy_backward(arena_ctx* c, const arena_loss_desc* f, const arena_loss_grads* g, void* stream)
{
    if (!c) return ARENA_ERR_INVALID_ARG;
    ctx_clear(c);
    const char* who = "cross entropy backward";
    arena_status st;
    if ((st = check_loss(c, who, f)) || (st = check_loss_grads(c, who, f, g))) return st;
    const LossBackPlan P(f, g, f->workspace);
    if ((st = check_workspace(c, who, f->workspace, f->workspace_bytes, P.w.used))) return st;
    const int64_t T = f->tokens, V = f->vocabulary, D = f->model, count = P.count;
    const bool dx = g->dx && T > 0, scaled = f->dtype == ARENA_F16 && T > 0;
    if (!dx && !g->dw) return ARENA_OK;
    DeviceScope scope(arena::ctx_device(c));
    if (scope.status != hipSuccess) return hip_error(c, scope.status, "hipSetDevice");
    hipStream_t s = (hipStream_t)stream;
    using namespace arena::mm;
    hipError_t e;
    LossArgs L = loss_args(f);
    L.dloss = g->dloss;
    L.s_dloss = g->stride_dloss;
    L.lse_in = f->lse;
    L.rows = (LossRow*)P.rows;
    L.scale = scaled ? (float*)P.scale : nullptr;
    L.x = f->x; L.ld_x = f->ld_x;
    L.x_to = P.x; L.ld_to = P.ld_x;
    L.twice = P.fine;
    if ((e = arena::launch_loss_rows(L, s))) return hip_error(c, e, "cross entropy rows launch");
    const float* factor = scaled ? (const float*)P.scale + 1 : nullptr;
    const int size = bytes_of(g->grad_dtype);
    for (int64_t v = 0; v < V; v += P.piece) {
        const int64_t n = std::min(P.piece, V - v);
        const void* w = (const char*)f->w + 2 * v * f->ld_w;
        if (T > 0) {
            GroupArgs A = new_args<GroupArgs>(T, n, D);
            A.any = P.any;
            A.a[0] = P.x; A.lda = P.ld_x;
            A.b[0] = w; A.ldb = f->ld_w;
            A.c[0] = P.g; A.ldc = P.ld_g;
            A.pad = (int)pad8(n);
            A.rows = (const LossRow*)P.rows;
            A.first_col = (int)v;
            A.splits = 1;
            A.low = P.fine ? (int)T : 0;
            const int kind = P.fine ? (int)kGroup64x128 : choose_whole(T, n, ceil_div(D, kBK), 2.0, P.any);
            if ((e = launch_loss(A, f->dtype, kLossGradient, kind, s)))
                return hip_error(c, e, "cross entropy logits' gradient launch");
        }
        if (dx) {
            const bool first = v == 0, last = v + n == V && !P.fine;
            GroupArgs X = new_args<GroupArgs>(count, D, n);
            X.any = P.any;
            X.a[0] = P.g; X.lda = P.ld_g;
            X.b[0] = w; X.ldb = f->ld_w;
            X.c[0] = last ? g->dx : P.sum; X.ldc = last ? g->ld_dx : D;
            X.out = last ? kOut16 : kOutF32;
            X.e[0] = P.sum; X.lde = D; X.e_f32 = 1;
            X.beta = first ? 0.0f : 1.0f;
            X.factor = factor;
            X.part = (float*)P.part;
            const GroupCut cut = P.cut_dx(count, D, n, P.any);
            X.splits = cut.splits;
            if ((e = launch_loss(X, f->dtype, kRowsCols, cut.kind, s)))
                return hip_error(c, e, "cross entropy input gradient launch");
        }
        if (g->dw) {
            char* dw = (char*)g->dw + size * v * g->ld_dw;
            GroupArgs W = new_args<GroupArgs>(n, D, count);
            W.a[0] = P.g; W.lda = P.ld_g;
            W.b[0] = P.x; W.ldb = P.ld_x;
            W.c[0] = dw; W.ldc = g->ld_dw;
            W.out = g->grad_dtype == ARENA_F32 ? kOutF32 : kOut16;
            if (g->accumulate) {
                W.beta = 1.0f;
                W.e[0] = dw; W.lde = g->ld_dw;
                W.e_f32 = g->grad_dtype == ARENA_F32;
            }
            W.factor = factor;
            W.part = (float*)P.part;
            const GroupCut cut = P.cut_dw(count, D, n);
            W.splits = cut.splits;
            if ((e = launch_loss(W, f->dtype, kColsCols, cut.kind, s)))
                return hip_error(c, e, "cross entropy weight gradient launch");
        }
    }
    if (dx && P.fine &&
        (e = arena::launch_loss_fold((const float*)P.sum, g->dx, g->ld_dx, T, (int)D, f->dtype, s)))
        return hip_error(c, e, "cross entropy input gradient fold launch");
    return ARENA_OK;
}

}  // extern "C"
