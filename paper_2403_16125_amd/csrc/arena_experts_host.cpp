// Host side of the C ABI declared in include/arena_experts.h: argument checks, the choice
// of tiles, workspace layout and launches.  No call allocates device memory or
// synchronises.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>

#include "arena_experts.h"
#include "arena_layer_internal.h"
#include "arena_layer_plan.h"

using namespace arena::plan;
using arena::ctx_clear;
using arena::ctx_fail;
using arena::MoveArgs;
using arena::RouteArgs;
using arena::SortArgs;
using arena::mm::GroupArgs;

static_assert(ARENA_MAX_EXPERTS == arena::kRouteMaxExperts, "experts of the header and the kernels");
static_assert(ARENA_ROUTE_MAX_CHOICES == arena::kRouteMaxChoices, "choices of the header and the kernels");

namespace {

arena_status check_tokens(arena_ctx* c, const char* who, const char* name, int64_t n)
{
    if (n < 0) return ctx_fail(c, ARENA_ERR_INVALID_ARG, "%s: %s=%lld", who, name, (long long)n);
    if (n > ARENA_LAYER_MAX_TOKENS)
        return ctx_fail(c, ARENA_ERR_UNSUPPORTED, "%s: %s=%lld (max %d)", who, name, (long long)n,
                        ARENA_LAYER_MAX_TOKENS);
    return ARENA_OK;
}

// A dense array of values of `size` bytes.
arena_status check_array(arena_ctx* c, const char* who, const char* name, const void* p, size_t size)
{
    if (!p) return ctx_fail(c, ARENA_ERR_INVALID_ARG, "%s: %s is NULL", who, name);
    if (!aligned(p, size)) return ctx_fail(c, ARENA_ERR_INVALID_ARG, "%s: %s is not aligned to its values", who, name);
    return ARENA_OK;
}

arena_status check_experts_number(arena_ctx* c, const char* who, int experts)
{
    if (experts < 1) return ctx_fail(c, ARENA_ERR_INVALID_ARG, "%s: experts=%d", who, experts);
    if (experts > ARENA_MAX_EXPERTS)
        return ctx_fail(c, ARENA_ERR_UNSUPPORTED, "%s: experts=%d (max %d)", who, experts, ARENA_MAX_EXPERTS);
    return ARENA_OK;
}

arena_status check_choices(arena_ctx* c, const char* who, int64_t tokens, int k, int most)
{
    if (k < 1) return ctx_fail(c, ARENA_ERR_INVALID_ARG, "%s: k=%d", who, k);
    if (k > most) return ctx_fail(c, ARENA_ERR_UNSUPPORTED, "%s: k=%d (max %d)", who, k, most);
    if (tokens * k > 0x7fffffff)
        return ctx_fail(c, ARENA_ERR_UNSUPPORTED, "%s: %lld choices (max 2^31 - 1)", who, (long long)(tokens * k));
    return ARENA_OK;
}

bool is_float(int dtype) { return dtype == ARENA_F32 || dtype == ARENA_BF16 || dtype == ARENA_F16; }

// ---------------------------------------------------------------- router

arena_status check_route(arena_ctx* c, const char* who, const arena_route_desc* d, bool backward)
{
    if (!d) return ctx_fail(c, ARENA_ERR_INVALID_ARG, "%s: descriptor is NULL", who);
    if (!is_float(d->dtype)) return ctx_fail(c, ARENA_ERR_INVALID_ARG, "%s: dtype=%d", who, d->dtype);
    arena_status s;
    if ((s = check_experts_number(c, who, d->experts)) || (s = check_tokens(c, who, "tokens", d->tokens)) ||
        (s = check_choices(c, who, d->tokens, d->k, ARENA_ROUTE_MAX_CHOICES)))
        return s;
    if (d->k > d->experts)
        return ctx_fail(c, ARENA_ERR_INVALID_ARG, "%s: k=%d of %d experts", who, d->k, d->experts);
    if (!std::isfinite(d->scale)) return ctx_fail(c, ARENA_ERR_INVALID_ARG, "%s: scale is not finite", who);
    if (d->tokens == 0) return ARENA_OK;
    if ((s = check_matrix(c, who, "logits", d->logits, d->ld_logits, d->experts, bytes_of(d->dtype))) ||
        (s = check_array(c, who, "index", d->index, 4)) || (!backward && (s = check_array(c, who, "weight", d->weight, 4))))
        return s;
    return ARENA_OK;
}

RouteArgs route_args(const arena_route_desc* d)
{
    RouteArgs A;
    std::memset(&A, 0, sizeof(A));
    A.tokens = d->tokens;
    A.experts = d->experts;
    A.k = d->k;
    A.normalise = d->normalise != 0;
    A.scale = d->scale;
    A.logits = d->logits;
    A.ld_logits = d->ld_logits;
    A.index = d->index;
    A.weight = d->weight;
    return A;
}

// ---------------------------------------------------------------- sort and moves

arena_status check_sort(arena_ctx* c, const char* who, const arena_sort_desc* d)
{
    if (!d) return ctx_fail(c, ARENA_ERR_INVALID_ARG, "%s: descriptor is NULL", who);
    if (d->index_dtype != ARENA_I32 && d->index_dtype != ARENA_I64)
        return ctx_fail(c, ARENA_ERR_INVALID_ARG, "%s: index_dtype=%d is neither int32 nor int64", who, d->index_dtype);
    arena_status s;
    if ((s = check_experts_number(c, who, d->experts)) || (s = check_tokens(c, who, "tokens", d->tokens)) ||
        (s = check_choices(c, who, d->tokens, d->k, ARENA_MAX_CHOICES)) ||
        (s = check_array(c, who, "offsets", d->offsets, 4)))
        return s;
    if (d->tokens > 0 && ((s = check_array(c, who, "index", d->index, d->index_dtype == ARENA_I64 ? 8 : 4)) ||
                          (s = check_array(c, who, "row", d->row, 4))))
        return s;
    return ARENA_OK;
}

SortArgs sort_args(const arena_sort_desc* d, int64_t* bytes)
{
    SortArgs A;
    std::memset(&A, 0, sizeof(A));
    A.choices = d->tokens * d->k;
    A.experts = d->experts;
    A.wide = d->index_dtype == ARENA_I64;
    A.index = d->index;
    A.offsets = d->offsets;
    A.row = d->row;
    A.counts = (int32_t*)d->workspace;
    arena::sort_plan(A.choices, &A.blocks, &A.each);
    *bytes = A.blocks > 1 ? pad256(4 * (int64_t)A.blocks * A.experts) : 0;
    return A;
}

arena_status check_move(arena_ctx* c, const char* who, const arena_move_desc* d)
{
    if (!d) return ctx_fail(c, ARENA_ERR_INVALID_ARG, "%s: descriptor is NULL", who);
    if (!is_float(d->dtype)) return ctx_fail(c, ARENA_ERR_INVALID_ARG, "%s: dtype=%d", who, d->dtype);
    if (d->model < 1) return ctx_fail(c, ARENA_ERR_INVALID_ARG, "%s: model=%d", who, d->model);
    if (d->model > ARENA_LAYER_MAX_LD)
        return ctx_fail(c, ARENA_ERR_UNSUPPORTED, "%s: model=%d (max %d)", who, d->model, ARENA_LAYER_MAX_LD);
    arena_status s;
    if ((s = check_tokens(c, who, "tokens", d->tokens)) || (s = check_choices(c, who, d->tokens, d->k, ARENA_MAX_CHOICES)))
        return s;
    if (d->rows < 0 || d->rows > 0x7fffffff)
        return ctx_fail(c, ARENA_ERR_INVALID_ARG, "%s: rows=%lld", who, (long long)d->rows);
    if (d->tokens == 0) return ARENA_OK;
    if ((s = check_array(c, who, "row", d->row, 4))) return s;
    if (!aligned(d->weight, 4)) return ctx_fail(c, ARENA_ERR_INVALID_ARG, "%s: weight is not aligned to its values", who);
    return ARENA_OK;
}

// Row strides here only enter 64-bit products, but the limit is that of all operators.
arena_status check_rows(arena_ctx* c, const char* who, const char* name, const void* p, int64_t ld, int64_t rows,
                        const arena_move_desc* d)
{
    if (rows == 0) return ARENA_OK;
    return check_matrix(c, who, name, p, ld, d->model, bytes_of(d->dtype));
}

MoveArgs move_args(const arena_move_desc* d)
{
    MoveArgs A;
    std::memset(&A, 0, sizeof(A));
    A.tokens = d->tokens;
    A.rows = d->rows;
    A.model = d->model;
    A.k = d->k;
    A.row = d->row;
    A.weight = d->weight;
    A.ld_weight = d->ld_weight;
    return A;
}

arena_status check_weight(arena_ctx* c, const char* who, const arena_move_desc* d)
{
    if (d->tokens > 0 && d->ld_weight < d->k)
        return ctx_fail(c, ARENA_ERR_INVALID_ARG, "%s: row stride %lld of weight is less than its width %d", who,
                        (long long)d->ld_weight, d->k);
    return ARENA_OK;
}

// ---------------------------------------------------------------- experts

arena_status check_stack(arena_ctx* c, const char* who, const char* name, const void* p, int64_t ld, int64_t stride,
                         int64_t rows, int64_t width, int experts, size_t size)
{
    const arena_status s = check_matrix(c, who, name, p, ld, width, size);
    if (s) return s;
    if (experts > 1 && stride < (rows - 1) * ld + width)
        return ctx_fail(c, ARENA_ERR_INVALID_ARG, "%s: stride %lld between the matrices of %s is less than a matrix", who,
                        (long long)stride, name);
    return ARENA_OK;
}

arena_status check_experts(arena_ctx* c, const char* who, const arena_experts_desc* d, bool backward)
{
    if (!d) return ctx_fail(c, ARENA_ERR_INVALID_ARG, "%s: descriptor is NULL", who);
    if (d->dtype != ARENA_BF16 && d->dtype != ARENA_F16)
        return ctx_fail(c, ARENA_ERR_INVALID_ARG, "%s: dtype=%d is neither bfloat16 nor float16", who, d->dtype);
    if (d->activation != ARENA_ACT_SILU && d->activation != ARENA_ACT_GELU && d->activation != ARENA_ACT_RELU)
        return ctx_fail(c, ARENA_ERR_INVALID_ARG, "%s: activation=%d", who, d->activation);
    if (d->model < 1 || d->inner < 1)
        return ctx_fail(c, ARENA_ERR_INVALID_ARG, "%s: model=%d inner=%d", who, d->model, d->inner);
    if (d->model > ARENA_LAYER_MAX_LD || d->inner > ARENA_LAYER_MAX_LD)
        return ctx_fail(c, ARENA_ERR_UNSUPPORTED, "%s: model=%d inner=%d (max %d)", who, d->model, d->inner,
                        ARENA_LAYER_MAX_LD);
    arena_status s;
    if ((s = check_experts_number(c, who, d->experts)) || (s = check_tokens(c, who, "rows", d->rows)) ||
        (s = check_stack(c, who, "w_gate", d->w_gate, d->ld_gate, d->stride_gate, d->inner, d->model, d->experts, 2)) ||
        (s = check_stack(c, who, "w_up", d->w_up, d->ld_up, d->stride_up, d->inner, d->model, d->experts, 2)) ||
        (s = check_stack(c, who, "w_down", d->w_down, d->ld_down, d->stride_down, d->model, d->inner, d->experts, 2)))
        return s;
    // a launch has a block for each tile that there can be
    const int64_t tiles = arena::mm::group_tiles(d->rows, d->experts, 256) * ceil_div(std::max(d->model, d->inner), 128);
    if (tiles > 0x7fffffff)
        return ctx_fail(c, ARENA_ERR_UNSUPPORTED, "%s: rows=%lld of %d and %d values make too many tiles", who,
                        (long long)d->rows, d->model, d->inner);
    if (2 * (int64_t)d->experts * ceil_div(d->model, 256) * ceil_div(d->inner, 256) > 0x7fffffff)
        return ctx_fail(c, ARENA_ERR_UNSUPPORTED, "%s: %d experts of %d x %d make too many tiles", who, d->experts,
                        d->model, d->inner);
    if (d->rows == 0) return ARENA_OK;
    if ((s = check_array(c, who, "offsets", d->offsets, 4)) || (s = check_matrix(c, who, "x", d->x, d->ld_x, d->model, 2)) ||
        (s = check_matrix(c, who, "h", d->h, d->ld_inner, pad8(d->inner), 2)) ||
        (!backward && (s = check_matrix(c, who, "y", d->y, d->ld_y, d->model, 2))))
        return s;
    if (!d->g != !d->u || (backward && !d->g))
        return ctx_fail(c, ARENA_ERR_INVALID_ARG, "%s: g and u are given together%s", who,
                        backward ? " (the backward pass needs them)" : " or not at all");
    if (d->ld_inner % 8 || !aligned(d->h, 16) || !aligned(d->g, 16) || !aligned(d->u, 16))
        return ctx_fail(c, ARENA_ERR_INVALID_ARG,
                        "%s: g, u and h need 16-byte alignment and ld_inner a multiple of 8 (got %lld)", who,
                        (long long)d->ld_inner);
    return ARENA_OK;
}

arena_status check_experts_grads(arena_ctx* c, const char* who, const arena_experts_desc* d, const arena_experts_grads* g)
{
    if (!g) return ctx_fail(c, ARENA_ERR_INVALID_ARG, "%s: gradient descriptor is NULL", who);
    if (g->grad_dtype != d->dtype && g->grad_dtype != ARENA_F32)
        return ctx_fail(c, ARENA_ERR_INVALID_ARG, "%s: grad_dtype=%d is neither dtype nor float32", who, g->grad_dtype);
    const size_t size = bytes_of(g->grad_dtype);
    const int e = d->experts;
    arena_status s;
    if ((g->dw_gate && (s = check_stack(c, who, "dw_gate", g->dw_gate, g->ld_dw_gate, g->stride_dw_gate, d->inner, d->model, e, size))) ||
        (g->dw_up && (s = check_stack(c, who, "dw_up", g->dw_up, g->ld_dw_up, g->stride_dw_up, d->inner, d->model, e, size))) ||
        (g->dw_down && (s = check_stack(c, who, "dw_down", g->dw_down, g->ld_dw_down, g->stride_dw_down, d->model, d->inner, e, size))))
        return s;
    if (d->rows == 0) return ARENA_OK;
    if ((s = check_matrix(c, who, "dy", g->dy, g->ld_dy, d->model, 2)) ||
        (g->dx && (s = check_matrix(c, who, "dx", g->dx, g->ld_dx, d->model, 2))))
        return s;
    return ARENA_OK;
}

// Whether the loads that write to the LDS can read matrices: rows on 16 bytes.
bool even(const void* p, int64_t ld, int64_t cols, int64_t stride, int experts)
{
    return Operand::direct(p, ld, cols) && (experts == 1 || stride % 8 == 0);
}

// The kind of tile and the parts of k for a product of groups of rows: how they fall is not
// known here, so each group that can have rows is taken to waste half a tile.  The parts are
// matrices of all rows.
GroupCut choose_rows(int64_t rows, int64_t groups, int64_t N, int64_t steps, bool dual, double bytes, bool any,
                     bool gated = false)
{
    using namespace arena::mm;
    GroupCut best = {any ? kGroup128 : kGroup256, 1, 0, 0};
    double least = INFINITY;
    for (int kind = 0; kind < kGroupKinds; ++kind) {
        const int64_t some = std::min(groups, rows), tn = ceil_div(N, dual ? kGroupCols[kind] / 2 : kGroupCols[kind]);
        const double tm = std::max((double)some, (double)rows / kGroupRows[kind] + 0.5 * some);
        if (group_tiles(rows, groups, kGroupRows[kind]) * tn > 0x7fffffff) continue;
        for (int s = 1; s <= 64 && (s == 1 || (!dual && kind != kGroup256 && s * 4 <= steps)); ++s) {
            if (s > 1 && tm * tn * s > 2.0 * kUnits) break;      // more blocks than there is room for
            const int64_t part = s > 1 ? 4 * s * rows * pad8(N) : 0;
            const double t = group_time(tm * tn * s, std::ceil((double)steps / s), kind, 1, s > 1 ? 4.0 : bytes, 1.0, false,
                                        any) + (s > 1 ? kJoin + part * 1e-6 / kJoinRate : 0.0);
            if (t < least) {
                least = t;
                best = {kind, s, part, 0};
            }
        }
        if (!dual && !gated && !(any && kind == kGroup256)) {
            int tail;
            int64_t part;
            const double t = tail_time(tm * tn, (double)steps, kind, bytes, &tail, &part);
            if (t < least) {
                least = t;
                best = {kind, 1, part, tail};
            }
        }
    }
    return best;
}

// The kind of tile and the parts of k for a product of groups of steps, taken to be of
// one length but for the longest, half as long again.  (How much is of little weight: with 1, 1.25, 1.5 and 2
// times, training takes the same to 1 % at 200 to 16384 rows of 8 experts 1024 x 2752, 1000 to 16384 of 64 experts
// 2048 x 1408 and 3000 of 8 experts 4096 x 10944.)
GroupCut choose_steps(int64_t M, int64_t N, int64_t rows, int64_t groups, int pairs, double bytes,
                      bool any)
{
    return choose_groups(M, N, std::max<int64_t>(1, ceil_div(rows, groups * arena::mm::kBK)), groups * pairs, bytes, true,
                         1.5, false, any);
}

// Whether a forward pass takes the kernel for few rows, which streams the weights and has no
// tiles to fill, but reads those of a group again for every 16 rows.  Up to 16 rows it is
// faster at all sizes (one row of 8 experts 4096 x 10944: 64 us, on tiles 73; 16 rows of 64
// experts 2048 x 1408: 60 and 65).  Past that where an expert has about 12 rows at most and its
// matrices stay in the caches (32 rows of 4 experts 4096 x 512: 23 and 39; 64 rows of 64 experts
// 2048 x 1408: 148 and 161), not with larger ones (32 rows of 8 experts 4096 x 10944: 387 and
// 371) or more rows (32 rows of 2 experts 2048 x 5461: 69 and 44).
bool few_rows(const arena_experts_desc* d)
{
    return d->rows <= 16 || (d->rows <= 64 && d->rows <= 12 * (int64_t)d->experts &&
                             (int64_t)d->model * d->inner <= 1 << 22);
}

// Which matrices the loads that write to the LDS cannot take: their products load to
// registers first.
struct Uneven {
    bool x, up, down;         // up: or the gate weights, or their row strides differ
    explicit Uneven(const arena_experts_desc* d)
        : x(!even(d->x, d->ld_x, d->model, 0, 1)),
          up(!even(d->w_gate, d->ld_gate, d->model, d->stride_gate, d->experts) ||
             !even(d->w_up, d->ld_up, d->model, d->stride_up, d->experts) || d->ld_gate != d->ld_up),
          down(!even(d->w_down, d->ld_down, d->inner, d->stride_down, d->experts))
    {
    }
};

struct ExpertsPlan {
    Pieces w;
    Uneven any;
    GroupCut up, down;
    void* part;
    ExpertsPlan(const arena_experts_desc* d, void* base) : w(base), any(d), up{0, 1, 0, 0}, down{0, 1, 0, 0}, part(nullptr)
    {
        if (d->rows == 0 || few_rows(d)) return;
        using arena::mm::kBK;
        up = choose_rows(d->rows, d->experts, d->inner, ceil_div(d->model, kBK), true, d->g ? 4.0 : 1.0, any.x || any.up);
        down = choose_rows(d->rows, d->experts, d->model, ceil_div(d->inner, kBK), false, 2.0, any.down);
        part = w.take(down.part);
    }
};

struct ExpertsBackPlan {
    Pieces w;
    Uneven any;
    bool dy_any;
    int64_t ld;               // rows of dg and du
    void *dg, *du, *part;
    bool pair;                // both weight gradients of the first products in one launch
    GroupCut cut_h, cut_x, cut_up, cut_down;
    ExpertsBackPlan(const arena_experts_desc* d, const arena_experts_grads* g, void* base)
        : w(base), any(d), dy_any(!even(g->dy, g->ld_dy, d->model, 0, 1))
    {
        ld = pad8(d->inner);
        dg = w.take(2 * d->rows * ld);
        du = w.take(2 * d->rows * ld);
        pair = g->dw_gate && g->dw_up && g->ld_dw_gate == g->ld_dw_up &&
               (d->experts == 1 || g->stride_dw_gate == g->stride_dw_up);
        const double bytes = bytes_of(g->grad_dtype) * (g->accumulate ? 2.0 : 1.0);
        cut_up = choose_steps(d->inner, d->model, d->rows, d->experts, pair ? 2 : 1, bytes, any.x);
        cut_down = choose_steps(d->model, d->inner, d->rows, d->experts, 1, bytes, dy_any);
        cut_h = cut_x = {0, 1, 0, 0};
        if (d->rows > 0 && (g->dx || g->dw_gate || g->dw_up))
            cut_h = choose_rows(d->rows, d->experts, d->inner, ceil_div(d->model, arena::mm::kBK), false, 10.0,
                                dy_any || any.down, true);
        if (d->rows > 0 && g->dx)
            cut_x = choose_rows(d->rows, d->experts, d->model, 2 * ceil_div(d->inner, arena::mm::kBK), false, 2.0, any.up);
        part = w.take(std::max({g->dw_gate || g->dw_up ? cut_up.part : 0, g->dw_down ? cut_down.part : 0, cut_h.part,
                                cut_x.part}));
    }
};

}  // namespace

extern "C" {

arena_status arena_route_forward(arena_ctx* c, const arena_route_desc* d, void* stream)
{
    if (!c) return ARENA_ERR_INVALID_ARG;
    ctx_clear(c);
    const arena_status s = check_route(c, "route", d, false);
    if (s || d->tokens == 0) return s;
    DeviceScope scope(arena::ctx_device(c));
    if (scope.status != hipSuccess) return hip_error(c, scope.status, "hipSetDevice");
    const hipError_t e = arena::launch_route_forward(route_args(d), d->dtype, (hipStream_t)stream);
    return e == hipSuccess ? ARENA_OK : hip_error(c, e, "route launch");
}

arena_status arena_route_backward(arena_ctx* c, const arena_route_desc* f, const float* dweight, int64_t ld_dweight,
                                  void* dlogits, int64_t ld_dlogits, void* stream)
{
    if (!c) return ARENA_ERR_INVALID_ARG;
    ctx_clear(c);
    const char* who = "route backward";
    arena_status s = check_route(c, who, f, true);
    if (s || f->tokens == 0) return s;
    if ((s = check_matrix(c, who, "dweight", dweight, ld_dweight, f->k, 4)) ||
        (s = check_matrix(c, who, "dlogits", dlogits, ld_dlogits, f->experts, bytes_of(f->dtype))))
        return s;
    RouteArgs A = route_args(f);
    A.dweight = dweight;
    A.ld_dweight = ld_dweight;
    A.dlogits = dlogits;
    A.ld_dlogits = ld_dlogits;
    DeviceScope scope(arena::ctx_device(c));
    if (scope.status != hipSuccess) return hip_error(c, scope.status, "hipSetDevice");
    const hipError_t e = arena::launch_route_backward(A, f->dtype, (hipStream_t)stream);
    return e == hipSuccess ? ARENA_OK : hip_error(c, e, "route backward launch");
}

arena_status arena_sort_by_expert_workspace(arena_ctx* c, const arena_sort_desc* d, int64_t* bytes)
{
    if (!c) return ARENA_ERR_INVALID_ARG;
    ctx_clear(c);
    if (!bytes) return ctx_fail(c, ARENA_ERR_INVALID_ARG, "sort by expert: bytes is NULL");
    const arena_status s = check_sort(c, "sort by expert", d);
    if (!s) (void)sort_args(d, bytes);
    return s;
}

arena_status arena_sort_by_expert(arena_ctx* c, const arena_sort_desc* d, void* stream)
{
    if (!c) return ARENA_ERR_INVALID_ARG;
    ctx_clear(c);
    arena_status s = check_sort(c, "sort by expert", d);
    if (s) return s;
    int64_t need;
    const SortArgs A = sort_args(d, &need);
    if ((s = check_workspace(c, "sort by expert", d->workspace, d->workspace_bytes, need))) return s;
    DeviceScope scope(arena::ctx_device(c));
    if (scope.status != hipSuccess) return hip_error(c, scope.status, "hipSetDevice");
    const hipError_t e = arena::launch_sort(A, (hipStream_t)stream);
    return e == hipSuccess ? ARENA_OK : hip_error(c, e, "sort by expert launch");
}

arena_status arena_dispatch(arena_ctx* c, const arena_move_desc* d, const void* x, int64_t ld_x, void* xs, int64_t ld_xs,
                            void* stream)
{
    if (!c) return ARENA_ERR_INVALID_ARG;
    ctx_clear(c);
    const char* who = "dispatch";
    arena_status s = check_move(c, who, d);
    if (s || d->tokens == 0 || d->rows == 0) return s;
    if ((s = check_rows(c, who, "x", x, ld_x, d->tokens, d)) || (s = check_rows(c, who, "xs", xs, ld_xs, d->rows, d)))
        return s;
    MoveArgs A = move_args(d);
    A.token = x; A.ld_token = ld_x;
    A.to_choice = xs; A.ld_to_choice = ld_xs;
    DeviceScope scope(arena::ctx_device(c));
    if (scope.status != hipSuccess) return hip_error(c, scope.status, "hipSetDevice");
    const hipError_t e = arena::launch_dispatch(A, d->dtype, (hipStream_t)stream);
    return e == hipSuccess ? ARENA_OK : hip_error(c, e, "dispatch launch");
}

arena_status arena_combine(arena_ctx* c, const arena_move_desc* d, const void* ys, int64_t ld_ys, void* y, int64_t ld_y,
                           void* stream)
{
    if (!c) return ARENA_ERR_INVALID_ARG;
    ctx_clear(c);
    const char* who = "combine";
    arena_status s = check_move(c, who, d);
    if (s || d->tokens == 0) return s;
    if ((d->weight && (s = check_weight(c, who, d))) || (s = check_rows(c, who, "ys", ys, ld_ys, d->rows, d)) ||
        (s = check_rows(c, who, "y", y, ld_y, d->tokens, d)))
        return s;
    MoveArgs A = move_args(d);
    A.choice = ys; A.ld_choice = ld_ys;
    A.to_token = y; A.ld_to_token = ld_y;
    DeviceScope scope(arena::ctx_device(c));
    if (scope.status != hipSuccess) return hip_error(c, scope.status, "hipSetDevice");
    const hipError_t e = arena::launch_combine(A, d->dtype, (hipStream_t)stream);
    return e == hipSuccess ? ARENA_OK : hip_error(c, e, "combine launch");
}

arena_status arena_combine_backward(arena_ctx* c, const arena_move_desc* d, const void* dy, int64_t ld_dy, const void* ys,
                                    int64_t ld_ys, void* dys, int64_t ld_dys, float* dweight, void* stream)
{
    if (!c) return ARENA_ERR_INVALID_ARG;
    ctx_clear(c);
    const char* who = "combine backward";
    arena_status s = check_move(c, who, d);
    if (s || d->tokens == 0) return s;
    if (!d->weight) return ctx_fail(c, ARENA_ERR_INVALID_ARG, "%s: weight is NULL", who);
    if ((s = check_weight(c, who, d)) || (s = check_rows(c, who, "dy", dy, ld_dy, d->tokens, d)) ||
        (s = check_rows(c, who, "ys", ys, ld_ys, d->rows, d)) || (s = check_rows(c, who, "dys", dys, ld_dys, d->rows, d)) ||
        (s = check_array(c, who, "dweight", dweight, 4)))
        return s;
    MoveArgs A = move_args(d);
    A.token = dy; A.ld_token = ld_dy;
    A.choice = ys; A.ld_choice = ld_ys;
    A.to_choice = dys; A.ld_to_choice = ld_dys;
    A.dweight = dweight;
    DeviceScope scope(arena::ctx_device(c));
    if (scope.status != hipSuccess) return hip_error(c, scope.status, "hipSetDevice");
    const hipError_t e = arena::launch_combine_backward(A, d->dtype, (hipStream_t)stream);
    return e == hipSuccess ? ARENA_OK : hip_error(c, e, "combine backward launch");
}

arena_status arena_experts_forward_workspace(arena_ctx* c, const arena_experts_desc* d, int64_t* bytes)
{
    if (!c) return ARENA_ERR_INVALID_ARG;
    ctx_clear(c);
    if (!bytes) return ctx_fail(c, ARENA_ERR_INVALID_ARG, "experts forward: bytes is NULL");
    const arena_status s = check_experts(c, "experts forward", d, false);
    if (s) return s;
    *bytes = ExpertsPlan(d, nullptr).w.used;
    return ARENA_OK;
}

arena_status arena_experts_forward(arena_ctx* c, const arena_experts_desc* d, void* stream)
{
    if (!c) return ARENA_ERR_INVALID_ARG;
    ctx_clear(c);
    arena_status st = check_experts(c, "experts forward", d, false);
    if (st || d->rows == 0) return st;
    const ExpertsPlan P(d, d->workspace);
    if ((st = check_workspace(c, "experts forward", d->workspace, d->workspace_bytes, P.w.used))) return st;
    DeviceScope scope(arena::ctx_device(c));
    if (scope.status != hipSuccess) return hip_error(c, scope.status, "hipSetDevice");
    hipStream_t s = (hipStream_t)stream;
    const int64_t R = d->rows;
    const Uneven& any = P.any;
    const bool few = few_rows(d);
    GroupArgs A = new_args<GroupArgs>(R, d->inner, d->model);
    A.offsets = d->offsets; A.groups = d->experts;
    A.splits = 1;
    A.any = any.x || any.up;
    A.a[0] = d->x; A.lda = d->ld_x;
    A.b[0] = d->w_gate; A.ldb = d->ld_gate; A.sb = d->stride_gate;
    A.b[1] = d->w_up; A.ldb1 = d->ld_up; A.sb1 = d->stride_up;
    A.c[0] = d->h; A.ldc = d->ld_inner;
    A.g = d->g; A.u = d->u; A.ldg = d->ld_inner;
    A.act = d->activation;
    A.pad = (int)pad8(d->inner);
    hipError_t e = few ? arena::mm::launch_skinny_groups(A, d->dtype, arena::mm::kGateUp, s)
                       : arena::mm::launch_groups(A, d->dtype, arena::mm::kGateUp, P.up.kind, s);
    if (e) return hip_error(c, e, "experts gate and up launch");
    GroupArgs B = new_args<GroupArgs>(R, d->model, d->inner);
    B.offsets = d->offsets; B.groups = d->experts;
    B.splits = P.down.splits;
    B.tail = P.down.tail;
    B.part = (float*)P.part;
    B.any = any.down;
    B.a[0] = d->h; B.lda = d->ld_inner;
    B.b[0] = d->w_down; B.ldb = d->ld_down; B.sb = d->stride_down;
    B.c[0] = d->y; B.ldc = d->ld_y;
    e = few ? arena::mm::launch_skinny_groups(B, d->dtype, arena::mm::kRowsRows, s)
            : arena::mm::launch_groups(B, d->dtype, arena::mm::kRowsRows, P.down.kind, s);
    return e == hipSuccess ? ARENA_OK : hip_error(c, e, "experts down launch");
}

arena_status arena_experts_backward_workspace(arena_ctx* c, const arena_experts_desc* f, const arena_experts_grads* g,
                                              int64_t* bytes)
{
    if (!c) return ARENA_ERR_INVALID_ARG;
    ctx_clear(c);
    const char* who = "experts backward";
    if (!bytes) return ctx_fail(c, ARENA_ERR_INVALID_ARG, "%s: bytes is NULL", who);
    arena_status s;
    if ((s = check_experts(c, who, f, true)) || (s = check_experts_grads(c, who, f, g))) return s;
    *bytes = ExpertsBackPlan(f, g, nullptr).w.used;
    return ARENA_OK;
}

arena_status arena_experts_backward(arena_ctx* c, const arena_experts_desc* f, const arena_experts_grads* g, void* stream)
{
    if (!c) return ARENA_ERR_INVALID_ARG;
    ctx_clear(c);
    const char* who = "experts backward";
    arena_status st;
    if ((st = check_experts(c, who, f, true)) || (st = check_experts_grads(c, who, f, g))) return st;
    const ExpertsBackPlan P(f, g, f->workspace);
    if ((st = check_workspace(c, who, f->workspace, f->workspace_bytes, P.w.used))) return st;
    DeviceScope scope(arena::ctx_device(c));
    if (scope.status != hipSuccess) return hip_error(c, scope.status, "hipSetDevice");
    hipStream_t s = (hipStream_t)stream;
    const int64_t R = f->rows, D = f->model, F = f->inner, E = f->experts;
    using namespace arena::mm;
    hipError_t e;
    if (R > 0 && (g->dx || g->dw_gate || g->dw_up)) {
        GroupArgs H = new_args<GroupArgs>(R, F, D);
        H.offsets = f->offsets; H.groups = f->experts;
        H.splits = P.cut_h.splits;
        H.part = (float*)P.part;
        H.any = P.dy_any || P.any.down;
        H.a[0] = g->dy; H.lda = g->ld_dy;
        H.b[0] = f->w_down; H.ldb = f->ld_down; H.sb = f->stride_down;
        H.g = f->g; H.u = f->u; H.ldg = f->ld_inner;
        H.c[0] = P.dg; H.c[1] = P.du; H.ldc = P.ld;
        H.act = f->activation;
        H.pad = (int)P.ld;
        if ((e = launch_groups(H, f->dtype, kGateUpBack, P.cut_h.kind, s)))
            return hip_error(c, e, "experts inner gradient launch");
    }
    // of every group C[m, n] = sum over its rows of a(t, m) b(t, n), beside what accumulate keeps
    auto weight = [&](const void* a0, const void* a1, int64_t lda, const void* b, int64_t ldb, int64_t M, int64_t N,
                      void* c0, void* c1, int64_t ldc, int64_t sc, const GroupCut& cut, bool any) {
        GroupArgs A = new_args<GroupArgs>(M, N, R);
        A.any = any;
        A.offsets = f->offsets; A.groups = f->experts;
        A.pairs = c1 != nullptr;
        A.batch = (int)E * (c1 ? 2 : 1);
        A.a[0] = a0; A.a[1] = a1; A.lda = lda;
        A.b[0] = A.b[1] = b; A.ldb = ldb;
        A.c[0] = c0; A.c[1] = c1; A.ldc = ldc; A.sc = sc;
        A.out = g->grad_dtype == ARENA_F32 ? kOutF32 : kOut16;
        if (g->accumulate) {
            A.beta = 1.0f;
            A.e[0] = c0; A.e[1] = c1; A.lde = ldc; A.se = sc;
            A.e_f32 = g->grad_dtype == ARENA_F32;
        }
        A.splits = cut.splits;
        A.part = (float*)P.part;
        return launch_groups(A, f->dtype, kColsCols, cut.kind, s);
    };
    if (g->dw_down && (e = weight(g->dy, nullptr, g->ld_dy, f->h, f->ld_inner, D, F, g->dw_down, nullptr, g->ld_dw_down,
                                  g->stride_dw_down, P.cut_down, P.dy_any)))
        return hip_error(c, e, "experts down gradient launch");
    if (P.pair) {
        if ((e = weight(P.dg, P.du, P.ld, f->x, f->ld_x, F, D, g->dw_gate, g->dw_up, g->ld_dw_gate, g->stride_dw_gate,
                        P.cut_up, P.any.x)))
            return hip_error(c, e, "experts gate and up gradient launch");
    } else {
        if (g->dw_gate && (e = weight(P.dg, nullptr, P.ld, f->x, f->ld_x, F, D, g->dw_gate, nullptr, g->ld_dw_gate,
                                      g->stride_dw_gate, P.cut_up, P.any.x)))
            return hip_error(c, e, "experts gate gradient launch");
        if (g->dw_up && (e = weight(P.du, nullptr, P.ld, f->x, f->ld_x, F, D, g->dw_up, nullptr, g->ld_dw_up,
                                    g->stride_dw_up, P.cut_up, P.any.x)))
            return hip_error(c, e, "experts up gradient launch");
    }
    if (R > 0 && g->dx) {
        GroupArgs X = new_args<GroupArgs>(R, D, F);
        X.offsets = f->offsets; X.groups = f->experts;
        X.splits = P.cut_x.splits;
        X.tail = P.cut_x.tail;
        X.part = (float*)P.part;
        X.a[0] = P.dg; X.a[1] = P.du; X.lda = P.ld;
        X.any = P.any.up;
        X.b[0] = f->w_gate; X.ldb = f->ld_gate; X.sb = f->stride_gate;
        X.b[1] = f->w_up; X.ldb1 = f->ld_up; X.sb1 = f->stride_up;
        X.c[0] = g->dx; X.ldc = g->ld_dx;
        if ((e = launch_groups(X, f->dtype, kRowsCols, P.cut_x.kind, s)))
            return hip_error(c, e, "experts input gradient launch");
    }
    return ARENA_OK;
}

}  // extern "C"
