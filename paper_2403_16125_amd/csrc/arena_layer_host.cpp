// Host side of the C ABI declared in include/arena_layer.h: argument checks,
// the choice of tiles and splits, workspace layout and launches.  No call
// allocates device memory or synchronises.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <initializer_list>

#include "arena_layer.h"
#include "arena_layer_internal.h"

using arena::ctx_clear;
using arena::ctx_fail;
using arena::NormArgs;
using arena::UpdateArgs;
using arena::mm::GemmArgs;

static_assert(ARENA_NORM_MAX_WIDTH == arena::kNormMaxWidth, "norm width of the header and the kernels");
static_assert(ARENA_LAYER_MAX_LD < arena::mm::kMaxLd, "row stride limit of the header and the kernels");

namespace {

struct DeviceScope {
    int before = -1;
    hipError_t status;
    explicit DeviceScope(int device)
    {
        status = hipGetDevice(&before);
        if (status == hipSuccess && before != device) status = hipSetDevice(device);
        else before = -1;
    }
    ~DeviceScope()
    {
        if (before >= 0) (void)hipSetDevice(before);
    }
};

arena_status hip_error(arena_ctx* c, hipError_t e, const char* what)
{
    return ctx_fail(c, ARENA_ERR_DEVICE, "%s: %s", what, hipGetErrorString(e));
}

int64_t pad8(int64_t n) { return (n + 7) / 8 * 8; }
int64_t pad256(int64_t n) { return (n + 255) / 256 * 256; }
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
bool aligned(const void* p, size_t bytes) { return ((uintptr_t)p & (bytes - 1)) == 0; }
int bytes_of(int dtype) { return dtype == ARENA_F32 ? 4 : 2; }

// Hands out pieces of the workspace, 256-byte aligned; without a base it only counts.
struct Pieces {
    char* base;
    int64_t used = 0;
    explicit Pieces(void* p) : base((char*)p) {}
    void* take(int64_t bytes)
    {
        void* p = base ? base + used : nullptr;
        used += pad256(bytes);
        return p;
    }
};

arena_status check_workspace(arena_ctx* c, const char* who, const void* p, int64_t have, int64_t need)
{
    if (need == 0) return ARENA_OK;
    if (!p) return ctx_fail(c, ARENA_ERR_INVALID_ARG, "%s: workspace is NULL (%lld bytes needed)", who, (long long)need);
    if (!aligned(p, 256)) return ctx_fail(c, ARENA_ERR_INVALID_ARG, "%s: workspace is not aligned to 256 bytes", who);
    if (have < need)
        return ctx_fail(c, ARENA_ERR_INVALID_ARG, "%s: workspace of %lld bytes, %lld needed", who, (long long)have,
                        (long long)need);
    return ARENA_OK;
}

// A matrix argument: present, rows apart by at least their width, within the
// strides that the kernels' 32-bit offsets take.
arena_status check_matrix(arena_ctx* c, const char* who, const char* name, const void* p, int64_t ld, int64_t width,
                          size_t size)
{
    if (!p) return ctx_fail(c, ARENA_ERR_INVALID_ARG, "%s: %s is NULL", who, name);
    if (!aligned(p, size)) return ctx_fail(c, ARENA_ERR_INVALID_ARG, "%s: %s is not aligned to its values", who, name);
    if (ld < width)
        return ctx_fail(c, ARENA_ERR_INVALID_ARG, "%s: row stride %lld of %s is less than its width %lld", who,
                        (long long)ld, name, (long long)width);
    if (ld > ARENA_LAYER_MAX_LD)
        return ctx_fail(c, ARENA_ERR_UNSUPPORTED, "%s: row stride %lld of %s (max %d)", who, (long long)ld, name,
                        ARENA_LAYER_MAX_LD);
    return ARENA_OK;
}

// ---------------------------------------------------------------- products

using arena::mm::Cut;

// What a kind of tile costs in microseconds (measured on one MI355X): a step
// of 64 of k with every slot of the compute units taken and with at most one
// block on each, a block's start, and how many blocks a compute unit holds.  A
// compute unit moves about 40 KB of an epilogue's bytes a microsecond.
struct TileCost {
    double full, alone, start;
    int slots;
};
constexpr TileCost kTileCost[arena::mm::kTileKinds] = {
    {1.60, 1.30, 5.0, 1}, {0.90, 0.67, 2.6, 2}, {0.60, 0.55, 3.2, 1}, {0.41, 0.35, 1.0, 2}};
constexpr double kEpilogueRate = 40e3;
constexpr double kLaunch = 3.0;             // a launch
constexpr double kSeam = 8.0;               // and the compute units that idle before it for others' last tiles
constexpr double kJoin = 4.0, kJoinRate = 3.0;     // joining parts: the launch, and megabytes a microsecond
constexpr int64_t kUnits = 256;             // compute units

// `tiles` tiles of a kind in one launch, k in `splits` parts.  bytes: what the
// epilogue moves for a value of the tile.  Whole rounds over the compute units,
// then one that is not full.
double launch_time(int64_t tiles, int64_t steps, int kind, int64_t splits, double bytes)
{
    const TileCost& k = kTileCost[kind];
    const int64_t per = ceil_div(steps, splits), blocks = tiles * splits, round = kUnits * k.slots;
    const double values = (double)arena::mm::kTileSide[kind] * arena::mm::kTileSide[kind];
    const double end = values * (splits > 1 ? 4.0 : bytes) / kEpilogueRate;
    const int64_t rounds = blocks / round, rest = blocks % round;
    double t = kLaunch + rounds * (per * k.full + k.start + end * k.slots);
    if (rest > kUnits) t += per * k.full + k.start + end * k.slots;
    else if (rest > 0) t += per * k.alone + k.start + end;
    return t + (splits > 1 ? kJoin + blocks * values * 4e-6 / kJoinRate : 0.0);
}

// The cheapest cut of a product: every kind of tile for whole rounds over the
// compute units or for none, and every smaller kind and split of k for the
// rest.  A last round that is nearly empty costs as much as a full one: 136
// tiles of 256 on 256 compute units (the Gram matrix of 4096 rows) would leave
// half of them idle for the whole product.
// dual: gate and up share a tile, which then covers half as many columns.
// sym: only the tiles on and below the diagonal.
Cut choose_cut(int64_t M, int64_t N, int64_t steps, int64_t batch, bool dual, bool sym, double bytes,
               double* time = nullptr)
{
    using namespace arena::mm;
    Cut best = {k256, k256, 0, 1, (int)steps};
    double least = INFINITY;
    for (int main = 0; main < kTileKinds; ++main) {
        const int64_t side = kTileSide[main], tm = ceil_div(M, side), tn = ceil_div(N, dual ? side / 2 : side);
        const int64_t all = (sym ? tm * (tm + 1) / 2 : tm * tn) * batch, round = kUnits * kTileCost[main].slots;
        for (int64_t first : {all / round * round, (int64_t)0}) {
            const double begin = first ? launch_time(first, steps, main, 1, bytes) + (first < all ? kSeam : 0.0) : 0.0;
            if (first == all && begin < least) {
                least = begin;
                best = {main, main, first, 1, (int)steps};
            }
            if (first == all) continue;
            for (int tail = 0; tail < kTileKinds; ++tail) {
                if (kTileSide[tail] > side || (first == 0 && tail != main)) continue;
                const int64_t ratio = side / kTileSide[tail], tiles = (all - first) * ratio * ratio;
                for (int s = 1; s <= 16 && (s == 1 || s * 4 <= steps); ++s) {
                    const double t = begin + launch_time(tiles, steps, tail, s, bytes);
                    if (t < least) {
                        least = t;
                        best = {main, tail, first, s, (int)ceil_div(steps, s)};
                    }
                }
            }
        }
    }
    if (best.per > 0) best.splits = (int)std::max<int64_t>(1, ceil_div(steps, best.per));
    if (time) *time = least;
    return best;
}

// Whether two independent products are faster in one launch, and over how many
// parts of the first one's k (the cut's splits; 0: they are not).  The blocks of
// 128 x 128 share the compute units: their work over all slots and the longest
// block's end bound the time.  first, second: what each takes by itself.
struct Half {
    int64_t M, N, steps, batch;
    double bytes, alone;
};

Cut choose_pair(const Half& a, const Half& b)
{
    using namespace arena::mm;
    Cut best = {k128, k128, 0, 0, 0};
    double least = a.alone + b.alone;
    const TileCost& k = kTileCost[k128];
    const int64_t na = ceil_div(a.M, 128) * ceil_div(a.N, 128) * a.batch;
    const int64_t nb = ceil_div(b.M, 128) * ceil_div(b.N, 128) * b.batch, slots = kUnits * k.slots;
    const double value = 128.0 * 128.0 / kEpilogueRate * k.slots;
    if (na + nb > (1 << 20)) return best;
    for (int s = 1; s <= 16 && (s == 1 || s * 4 <= a.steps); ++s) {
        const int64_t per = ceil_div(a.steps, s), blocks = na * ceil_div(a.steps, per);
        const double step = blocks + nb > kUnits ? k.full : k.alone;
        const double ta = per * step + k.start + value * (s > 1 ? 4.0 : a.bytes);
        const double tb = b.steps * step + k.start + value * b.bytes;
        const double work = (blocks * ta + nb * tb) / slots, longest = std::max(ta, tb);
        // a last round leaves some slots idle, fewer than of equal blocks
        const double t = kLaunch + std::max(longest, work + (blocks + nb > slots ? 0.25 * longest : 0.0)) +
                         (s > 1 ? kJoin + blocks * 128.0 * 128.0 * 4e-6 / kJoinRate : 0.0);
        if (t < least) {
            least = t;
            best = {k128, k128, 0, s, (int)per};
        }
    }
    if (best.splits > 0) best.splits = (int)ceil_div(a.steps, best.per);
    return best;
}

// A symmetric product: the tiles on and below the diagonal, each written twice,
// unless all tiles once are no slower (as where they fit the compute units at
// once).  bytes: what an epilogue reads and writes for a value written once.
Cut choose_symmetric(int64_t n, int64_t steps, int64_t batch, double bytes, bool* sym)
{
    double all, half;
    const Cut a = choose_cut(n, n, steps, batch, false, false, bytes, &all);
    const Cut h = choose_cut(n, n, steps, batch, false, true, bytes + 2.0, &half);
    *sym = half < all;
    return *sym ? h : a;
}

int64_t part_bytes(const Cut& cut, int64_t M, int64_t N, int64_t batch, bool dual, bool sym)
{
    if (cut.splits <= 1) return 0;
    const int64_t side = arena::mm::kTileSide[cut.main], tm = ceil_div(M, side), tn = ceil_div(N, dual ? side / 2 : side);
    const int64_t all = (sym ? tm * (tm + 1) / 2 : tm * tn) * batch;
    return 4 * cut.splits * (all - cut.first) * side * side;
}

GemmArgs new_args(int64_t M, int64_t N, int64_t K)
{
    GemmArgs A;
    std::memset(&A, 0, sizeof(A));
    A.M = (int)M;
    A.N = (int)N;
    A.K = (int)K;
    A.nseg = 1;
    A.batch = 1;
    A.alpha = 1.0f;
    return A;
}

// A matrix as the tiled kernels take it: in place, or a copy in the workspace.
struct Operand {
    const void* p;
    int64_t ld;
    const void* from = nullptr;
    int64_t ld_from = 0, rows = 0, cols = 0;
    void* copy = nullptr;

    static bool direct(const void* p, int64_t ld, int64_t cols) { return aligned(p, 16) && ld % 8 == 0 && cols % 8 == 0; }

    Operand(Pieces& w, const void* q, int64_t ld_q, int64_t rows_, int64_t cols_, bool in_place)
    {
        p = q;
        ld = ld_q;
        if (in_place) return;
        from = q;
        ld_from = ld_q;
        rows = rows_;
        cols = cols_;
        ld = pad8(cols);
        copy = w.take(2 * rows * ld);
        p = copy;
    }

};

// Fills the copies among some operands.
hipError_t pack(std::initializer_list<const Operand*> operands, hipStream_t s)
{
    arena::mm::Pack packs[arena::mm::kMaxPacks];
    int n = 0;
    for (const Operand* o : operands)
        if (o->copy && n < arena::mm::kMaxPacks)
            packs[n++] = {o->from, o->copy, o->ld_from, o->ld, o->rows, o->cols};
    return n ? arena::mm::launch_packs(packs, n, s) : hipSuccess;
}

// ---------------------------------------------------------------- norms

arena_status check_norm(arena_ctx* c, const char* who, const arena_norm_desc* d, bool backward)
{
    if (!d) return ctx_fail(c, ARENA_ERR_INVALID_ARG, "%s: descriptor is NULL", who);
    if (d->dtype != ARENA_F32 && d->dtype != ARENA_BF16 && d->dtype != ARENA_F16)
        return ctx_fail(c, ARENA_ERR_INVALID_ARG, "%s: dtype=%d", who, d->dtype);
    if (d->stream_dtype != d->dtype && d->stream_dtype != ARENA_F32)
        return ctx_fail(c, ARENA_ERR_INVALID_ARG, "%s: stream_dtype=%d is neither dtype nor float32", who,
                        d->stream_dtype);
    if (d->kind != ARENA_NORM_RMS && d->kind != ARENA_NORM_LAYER)
        return ctx_fail(c, ARENA_ERR_INVALID_ARG, "%s: kind=%d", who, d->kind);
    if (d->width < 1) return ctx_fail(c, ARENA_ERR_INVALID_ARG, "%s: width=%d", who, d->width);
    if (d->width > ARENA_NORM_MAX_WIDTH)
        return ctx_fail(c, ARENA_ERR_UNSUPPORTED, "%s: width=%d (max %d)", who, d->width, ARENA_NORM_MAX_WIDTH);
    if (d->tokens < 0 || d->gate_rows < 0)
        return ctx_fail(c, ARENA_ERR_INVALID_ARG, "%s: tokens=%lld gate_rows=%lld", who, (long long)d->tokens,
                        (long long)d->gate_rows);
    if (d->tokens > ARENA_LAYER_MAX_TOKENS)
        return ctx_fail(c, ARENA_ERR_UNSUPPORTED, "%s: tokens=%lld (max %d)", who, (long long)d->tokens,
                        ARENA_LAYER_MAX_TOKENS);
    if (!(d->eps >= 0.0f) || !std::isfinite(d->eps) || !std::isfinite(d->scale))
        return ctx_fail(c, ARENA_ERR_INVALID_ARG, "%s: eps must be finite and >= 0, scale finite", who);
    if (d->tokens > 0 && !d->y && (d->gate || d->w_post || d->b_post))
        return ctx_fail(c, ARENA_ERR_INVALID_ARG, "%s: gate, w_post and b_post need y", who);
    if (d->tokens > 0 && !d->n && !backward && (d->w_pre || d->b_pre))
        return ctx_fail(c, ARENA_ERR_INVALID_ARG, "%s: w_pre and b_pre need n", who);
    const size_t size = bytes_of(d->dtype), stream = bytes_of(d->stream_dtype);
    const void* vectors[] = {d->gate, d->w_post, d->b_post, d->w_pre, d->b_pre};
    for (const void* v : vectors)
        if (!aligned(v, size)) return ctx_fail(c, ARENA_ERR_INVALID_ARG, "%s: a weight is not aligned to its values", who);
    if (!aligned(d->stats, 4)) return ctx_fail(c, ARENA_ERR_INVALID_ARG, "%s: stats is not aligned to its values", who);
    arena_status s;
    if (d->gate && (s = check_matrix(c, who, "gate", d->gate, d->ld_gate, d->width, size))) return s;
    if (d->tokens == 0) return ARENA_OK;
    if (d->y && (s = check_matrix(c, who, "y", d->y, d->ld_y, d->width, size))) return s;
    if (!backward) {
        if (!d->y && !d->n) return ctx_fail(c, ARENA_ERR_INVALID_ARG, "%s: neither y nor n: nothing to do", who);
        if ((s = check_matrix(c, who, "x", d->x, d->ld_x, d->width, stream))) return s;
        if (d->y && (s = check_matrix(c, who, "r", d->r, d->ld_r, d->width, stream))) return s;
        if (d->n && (s = check_matrix(c, who, "n", d->n, d->ld_n, d->width, size))) return s;
    }
    return ARENA_OK;
}

NormArgs norm_args(const arena_norm_desc* d)
{
    NormArgs A;
    std::memset(&A, 0, sizeof(A));
    A.x = d->x; A.ld_x = d->ld_x;
    A.y = d->y; A.ld_y = d->ld_y;
    A.gate = d->gate; A.ld_gate = d->ld_gate;
    A.w_post = d->w_post; A.b_post = d->b_post; A.w_pre = d->w_pre; A.b_pre = d->b_pre;
    A.r = d->r; A.ld_r = d->ld_r;
    A.n = d->n; A.ld_n = d->ld_n;
    A.stats = d->stats;
    A.tokens = d->tokens;
    // a gate row of more tokens than there are is one of all of them
    const int64_t all = std::max<int64_t>(1, d->tokens);
    A.gate_rows = d->gate_rows > 0 ? std::min(d->gate_rows, all) : all;
    A.width = d->width;
    A.layer = d->kind == ARENA_NORM_LAYER;
    A.eps = d->eps;
    A.scale = d->scale;
    return A;
}

arena_status norm_workspace(arena_ctx* c, const char* who, const arena_norm_desc* d, int64_t* bytes, int64_t* sums,
                            int* workers, int* rows_each)
{
    arena_status s = check_norm(c, who, d, true);
    if (s) return s;
    const NormArgs A = norm_args(d);
    arena::norm_plan(A.tokens, A.gate_rows, A.width, workers, rows_each);
    *sums = pad256((int64_t)*workers * arena::kNormSums * A.width * 4);
    *bytes = *sums + (A.width > arena::kNormSumsWidth ? pad256(A.tokens * 8) : 0);
    return ARENA_OK;
}

// ---------------------------------------------------------------- feed-forward

arena_status check_ffn(arena_ctx* c, const char* who, const arena_ffn_desc* d, bool backward)
{
    if (!d) return ctx_fail(c, ARENA_ERR_INVALID_ARG, "%s: descriptor is NULL", who);
    if (d->dtype != ARENA_BF16 && d->dtype != ARENA_F16)
        return ctx_fail(c, ARENA_ERR_INVALID_ARG, "%s: dtype=%d is neither bfloat16 nor float16", who, d->dtype);
    if (d->activation != ARENA_ACT_SILU && d->activation != ARENA_ACT_GELU && d->activation != ARENA_ACT_RELU)
        return ctx_fail(c, ARENA_ERR_INVALID_ARG, "%s: activation=%d", who, d->activation);
    if (d->tokens < 0 || d->model < 1 || d->inner < 1)
        return ctx_fail(c, ARENA_ERR_INVALID_ARG, "%s: tokens=%lld model=%d inner=%d", who, (long long)d->tokens,
                        d->model, d->inner);
    if (d->tokens > ARENA_LAYER_MAX_TOKENS)
        return ctx_fail(c, ARENA_ERR_UNSUPPORTED, "%s: tokens=%lld (max %d)", who, (long long)d->tokens,
                        ARENA_LAYER_MAX_TOKENS);
    if (d->model > ARENA_LAYER_MAX_LD || d->inner > ARENA_LAYER_MAX_LD)
        return ctx_fail(c, ARENA_ERR_UNSUPPORTED, "%s: model=%d inner=%d (max %d)", who, d->model, d->inner,
                        ARENA_LAYER_MAX_LD);
    arena_status s;
    if ((s = check_matrix(c, who, "w_gate", d->w_gate, d->ld_gate, d->model, 2)) ||
        (s = check_matrix(c, who, "w_up", d->w_up, d->ld_up, d->model, 2)) ||
        (s = check_matrix(c, who, "w_down", d->w_down, d->ld_down, d->inner, 2)))
        return s;
    if (d->tokens == 0) return ARENA_OK;
    if ((s = check_matrix(c, who, "x", d->x, d->ld_x, d->model, 2)) ||
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

// The operands of a call and the pieces of its workspace.
struct FfnPlan {
    Pieces w;
    bool skinny, gate_ok;
    Operand x, gate, up, down;
    FfnPlan(const arena_ffn_desc* d, bool skinny_, void* base)
        : w(base), skinny(skinny_),
          gate_ok(Operand::direct(d->w_gate, d->ld_gate, d->model) && Operand::direct(d->w_up, d->ld_up, d->model) &&
                  d->ld_gate == d->ld_up),
          x(w, d->x, d->ld_x, d->tokens, d->model, skinny || Operand::direct(d->x, d->ld_x, d->model)),
          gate(w, d->w_gate, d->ld_gate, d->inner, d->model, skinny || gate_ok),
          up(w, d->w_up, d->ld_up, d->inner, d->model, skinny || gate_ok),
          down(w, d->w_down, d->ld_down, d->model, d->inner, skinny || Operand::direct(d->w_down, d->ld_down, d->inner))
    {
    }
};

// Whether a forward pass takes the kernel for few tokens, which streams the
// weights past them.  Past 16 tokens it reads as much of the tokens as of the
// weights, and the tiled products are faster where the weights are large (24
// tokens, 4096 x 10944: 87 us against 75; 4096 x 1368: 23 us against 27).
bool few_tokens(const arena_ffn_desc* d)
{
    return d->tokens <= 16 || (d->tokens <= arena::mm::kSkinnyRows && (int64_t)d->model * d->inner <= 1 << 23);
}

struct ForwardPlan : FfnPlan {
    Cut cut_up, cut_down;
    void* part;
    ForwardPlan(const arena_ffn_desc* d, void* base) : FfnPlan(d, few_tokens(d), base)
    {
        cut_up = choose_cut(d->tokens, d->inner, ceil_div(d->model, arena::mm::kBK), 1, true, false, d->g ? 4.0 : 1.0);
        cut_down = choose_cut(d->tokens, d->model, ceil_div(d->inner, arena::mm::kBK), 1, false, false, 2.0);
        part = w.take(skinny ? 0 : std::max(part_bytes(cut_up, d->tokens, d->inner, 1, true, false),
                                            part_bytes(cut_down, d->tokens, d->model, 1, false, false)));
    }
};

struct BackwardPlan : FfnPlan {
    Operand dy;
    int64_t ld;               // rows of dg and du
    void *dg, *du, *part;
    bool pair;                // both weight gradients of the first products in one launch
    Cut cut_dh, cut_dx, cut_down, cut_up;
    Cut pair_dh, pair_dx;     // the inner gradient with dw_down, dx with dw_gate and dw_up, if splits > 0
    BackwardPlan(const arena_ffn_desc* d, const arena_ffn_grads* g, void* base)
        : FfnPlan(d, false, base),
          dy(w, g->dy, g->ld_dy, d->tokens, d->model, Operand::direct(g->dy, g->ld_dy, d->model))
    {
        const int64_t T = d->tokens, D = d->model, F = d->inner, bk = arena::mm::kBK;
        ld = pad8(F);
        dg = w.take(2 * T * ld);
        du = w.take(2 * T * ld);
        pair = g->dw_gate && g->dw_up && g->ld_dw_gate == g->ld_dw_up;
        const int pairs = pair ? 2 : 1;
        const double bytes = bytes_of(g->grad_dtype) * (g->accumulate ? 2.0 : 1.0);
        Half dh = {T, F, ceil_div(D, bk), 1, 10.0, 0.0}, dx = {T, D, 2 * ceil_div(F, bk), 1, 2.0, 0.0};
        Half down = {D, F, ceil_div(T, bk), 1, bytes, 0.0}, up = {F, D, ceil_div(T, bk), pairs, bytes, 0.0};
        auto alone = [](Half& h) { return choose_cut(h.M, h.N, h.steps, h.batch, false, false, h.bytes, &h.alone); };
        cut_dh = alone(dh);
        cut_dx = alone(dx);
        cut_down = alone(down);
        cut_up = alone(up);
        pair_dh = pair_dx = Cut{arena::mm::k128, arena::mm::k128, 0, 0, 0};
        const bool inner_grad = g->dx || g->dw_gate || g->dw_up;
        if (T > 0 && inner_grad && g->dw_down) pair_dh = choose_pair(dh, down);
        if (T > 0 && g->dx && pair) pair_dx = choose_pair(dx, up);
        int64_t most = 0;
        auto need = [&](const Half& h, const Cut& cut) {
            most = std::max(most, part_bytes(cut, h.M, h.N, h.batch, false, false));
        };
        need(dh, pair_dh.splits ? pair_dh : cut_dh);
        need(dx, pair_dx.splits ? pair_dx : cut_dx);
        if (!pair_dh.splits) need(down, cut_down);
        if (!pair_dx.splits) need(up, cut_up);
        part = w.take(most);
    }
};

arena_status check_ffn_grads(arena_ctx* c, const char* who, const arena_ffn_desc* d, const arena_ffn_grads* g)
{
    if (!g) return ctx_fail(c, ARENA_ERR_INVALID_ARG, "%s: gradient descriptor is NULL", who);
    if (g->grad_dtype != d->dtype && g->grad_dtype != ARENA_F32)
        return ctx_fail(c, ARENA_ERR_INVALID_ARG, "%s: grad_dtype=%d is neither dtype nor float32", who, g->grad_dtype);
    const size_t size = bytes_of(g->grad_dtype);
    arena_status s;
    if (g->dw_gate && (s = check_matrix(c, who, "dw_gate", g->dw_gate, g->ld_dw_gate, d->model, size))) return s;
    if (g->dw_up && (s = check_matrix(c, who, "dw_up", g->dw_up, g->ld_dw_up, d->model, size))) return s;
    if (g->dw_down && (s = check_matrix(c, who, "dw_down", g->dw_down, g->ld_dw_down, d->inner, size))) return s;
    if (d->tokens == 0) return ARENA_OK;
    if ((s = check_matrix(c, who, "dy", g->dy, g->ld_dy, d->model, 2))) return s;
    if (g->dx && (s = check_matrix(c, who, "dx", g->dx, g->ld_dx, d->model, 2))) return s;
    return ARENA_OK;
}

// ---------------------------------------------------------------- orthogonalised update

constexpr double kHalfScale = 4096.0;      // 2^12: what float16 operands of an update are scaled by
constexpr double kHalfMost = 15.5;         // magnitudes that holds, with room for rounding
// The Gram matrix A is held as C = A - 1/2, and b A + c A^2 as the constant
// b/2 + c/4 and the rest (b + c) C + c C^2, whose constant joins a: the same
// polynomial, but what is rounded to float16 is small on the diagonal both
// while singular values are small and once they lie about 1.  The update's
// error against 64 bits fell from 1.3-1.9e-3 to 0.7-1.1e-3 (64 to 1000 rows).
constexpr double kCentre = 0.5;

// Whether every matrix of the iteration stays within kHalfMost: bounds over the
// singular values from 0 (a normalised matrix of some size has nearly all of them
// there, the padding of a small one exactly) to their largest, at both ends and the
// stationary points of the polynomials.
bool polynomial_holds(const float* k, int steps)
{
    double s = 1.0;
    for (int i = 0; i < steps; ++i) {
        const double a = k[3 * i], b = k[3 * i + 1], c = k[3 * i + 2];
        const double t = s * s;
        auto B = [&](double v) { return std::fabs((b + 2.0 * c * kCentre) * (v - kCentre) + c * (v - kCentre) * (v - kCentre)); };
        auto X = [&](double v) { return std::sqrt(v) * std::fabs(a + b * v + c * v * v); };
        double most_b = std::max(B(0.0), B(t)), most_x = X(t);
        if (c != 0.0) {
            const double v = -b / (2.0 * c);
            if (v > 0.0 && v < t) most_b = std::max(most_b, B(v));
        }
        // d/ds (a s + b s^3 + c s^5) = a + 3 b v + 5 c v^2 with v = s^2
        const double disc = 9.0 * b * b - 20.0 * a * c;
        if (c != 0.0 && disc >= 0.0) {
            for (double sign : {-1.0, 1.0}) {
                const double v = (-3.0 * b + sign * std::sqrt(disc)) / (10.0 * c);
                if (v > 0.0 && v < t) most_x = std::max(most_x, X(v));
            }
        } else if (c == 0.0 && b != 0.0) {
            const double v = -a / (3.0 * b);
            if (v > 0.0 && v < t) most_x = std::max(most_x, X(v));
        }
        if (!(t <= kHalfMost) || !(most_b <= kHalfMost) || !(most_x <= kHalfMost)) return false;
        s = most_x * 1.005;                // roundings of a step
    }
    return true;
}

arena_status check_update(arena_ctx* c, const char* who, const arena_update_desc* d)
{
    if (!d) return ctx_fail(c, ARENA_ERR_INVALID_ARG, "%s: descriptor is NULL", who);
    if (d->dtype != ARENA_F32 && d->dtype != ARENA_BF16 && d->dtype != ARENA_F16)
        return ctx_fail(c, ARENA_ERR_INVALID_ARG, "%s: dtype=%d", who, d->dtype);
    if (d->out_dtype != ARENA_BF16 && d->out_dtype != ARENA_F16)
        return ctx_fail(c, ARENA_ERR_INVALID_ARG, "%s: out_dtype=%d is neither bfloat16 nor float16", who, d->out_dtype);
    if (d->batch < 1 || d->rows < 1 || d->cols < 1 || d->steps < 0)
        return ctx_fail(c, ARENA_ERR_INVALID_ARG, "%s: batch=%d rows=%d cols=%d steps=%d", who, d->batch, d->rows,
                        d->cols, d->steps);
    if (d->rows > ARENA_UPDATE_MAX_SIDE || d->cols > ARENA_UPDATE_MAX_SIDE || d->steps > ARENA_UPDATE_MAX_STEPS ||
        d->batch > ARENA_UPDATE_MAX_BATCH)
        return ctx_fail(c, ARENA_ERR_UNSUPPORTED, "%s: batch=%d rows=%d cols=%d steps=%d (max %d, %d, %d, %d)", who,
                        d->batch, d->rows, d->cols, d->steps, ARENA_UPDATE_MAX_BATCH, ARENA_UPDATE_MAX_SIDE,
                        ARENA_UPDATE_MAX_SIDE, ARENA_UPDATE_MAX_STEPS);
    if (!(d->eps >= 0.0f) || !std::isfinite(d->eps) || !std::isfinite(d->mu) || !std::isfinite(d->scale))
        return ctx_fail(c, ARENA_ERR_INVALID_ARG, "%s: eps must be finite and >= 0, mu and scale finite", who);
    if (d->steps > 0 && !d->coefficients) return ctx_fail(c, ARENA_ERR_INVALID_ARG, "%s: coefficients is NULL", who);
    for (int i = 0; i < 3 * d->steps; ++i)
        if (!std::isfinite(d->coefficients[i]))
            return ctx_fail(c, ARENA_ERR_INVALID_ARG, "%s: a coefficient is not finite", who);
    if (!polynomial_holds(d->coefficients, d->steps))
        return ctx_fail(c, ARENA_ERR_UNSUPPORTED, "%s: the polynomials leave the magnitudes that float16 operands hold",
                        who);
    if (!d->momentum != !d->momentum_out)
        return ctx_fail(c, ARENA_ERR_INVALID_ARG, "%s: momentum and momentum_out are given together", who);
    arena_status s;
    if ((s = check_matrix(c, who, "grad", d->grad, d->ld_grad, d->cols, bytes_of(d->dtype))) ||
        (d->momentum && (s = check_matrix(c, who, "momentum", d->momentum, d->ld_momentum, d->cols, 4))) ||
        (d->momentum && (s = check_matrix(c, who, "momentum_out", d->momentum_out, d->ld_momentum_out, d->cols, 4))) ||
        (s = check_matrix(c, who, "out", d->out, d->ld_out, d->cols, 2)))
        return s;
    if (d->batch > 1) {
        const int64_t last = d->rows - 1;
        if (d->stride_grad < last * d->ld_grad + d->cols || d->stride_out < last * d->ld_out + d->cols ||
            (d->momentum && (d->stride_momentum < last * d->ld_momentum + d->cols ||
                             d->stride_momentum_out < last * d->ld_momentum_out + d->cols)))
            return ctx_fail(c, ARENA_ERR_INVALID_ARG, "%s: a stride between matrices is less than a matrix", who);
    }
    return ARENA_OK;
}

// Whether step i adds what rounding took off its X: all but the last two do.
bool keeps_rest(const arena_update_desc* d, int i) { return i + 2 < d->steps; }

struct UpdatePlan {
    Pieces w;
    int64_t rows, cols, side;       // padded to multiples of 8
    bool tall;                      // more rows than columns: the Gram matrix is X^T X
    int blocks;
    void *x[2], *rest, *gram, *poly, *sums, *part;
    Cut cut_gram, cut_square, cut_x;
    bool sym_gram, sym_square;

    UpdatePlan(const arena_update_desc* d, void* base) : w(base)
    {
        const int64_t bk = arena::mm::kBK, n = d->batch;
        rows = pad8(d->rows);
        cols = pad8(d->cols);
        tall = d->rows > d->cols;
        side = tall ? cols : rows;
        const int64_t values = (int64_t)d->rows * pad8(d->cols) / 8;
        blocks = (int)std::max<int64_t>(1, std::min<int64_t>(arena::kUpdateBlocks, ceil_div(values, 1024)));
        for (void*& p : x) p = w.take(2 * n * rows * cols);
        rest = w.take(keeps_rest(d, 0) ? 2 * n * rows * cols : 0);
        gram = w.take(2 * n * side * side);
        poly = w.take(2 * n * side * side);
        sums = w.take(8 * n * blocks);
        cut_gram = choose_symmetric(side, ceil_div(tall ? rows : cols, bk), n, 2.0, &sym_gram);
        cut_square = choose_symmetric(side, ceil_div(side, bk), n, 4.0, &sym_square);
        cut_x = choose_cut(rows, cols, ceil_div(side, bk), n, false, false, 4.0);
        part = w.take(std::max(std::max(part_bytes(cut_gram, side, side, n, false, sym_gram),
                                        part_bytes(cut_square, side, side, n, false, sym_square)),
                               part_bytes(cut_x, rows, cols, n, false, false)));
    }
};

}  // namespace

extern "C" {

arena_status arena_norm_forward(arena_ctx* c, const arena_norm_desc* d, void* stream)
{
    if (!c) return ARENA_ERR_INVALID_ARG;
    ctx_clear(c);
    arena_status s = check_norm(c, "norm forward", d, false);
    if (s || d->tokens == 0) return s;
    DeviceScope scope(arena::ctx_device(c));
    if (scope.status != hipSuccess) return hip_error(c, scope.status, "hipSetDevice");
    const hipError_t e = arena::launch_norm_forward(norm_args(d), d->dtype, d->stream_dtype, (hipStream_t)stream);
    return e == hipSuccess ? ARENA_OK : hip_error(c, e, "norm forward launch");
}

arena_status arena_norm_backward_workspace(arena_ctx* c, const arena_norm_desc* f, int64_t* bytes)
{
    if (!c) return ARENA_ERR_INVALID_ARG;
    ctx_clear(c);
    if (!bytes) return ctx_fail(c, ARENA_ERR_INVALID_ARG, "norm backward: bytes is NULL");
    int64_t sums;
    int workers, rows;
    return norm_workspace(c, "norm backward", f, bytes, &sums, &workers, &rows);
}

arena_status arena_norm_backward(arena_ctx* c, const arena_norm_desc* f, const arena_norm_grads* g, void* stream)
{
    if (!c) return ARENA_ERR_INVALID_ARG;
    ctx_clear(c);
    const char* who = "norm backward";
    int64_t need, sums_bytes;
    int workers, rows;
    arena_status s = norm_workspace(c, who, f, &need, &sums_bytes, &workers, &rows);
    if (s) return s;
    if (!g) return ctx_fail(c, ARENA_ERR_INVALID_ARG, "%s: gradient descriptor is NULL", who);
    const size_t size = bytes_of(f->dtype), wide = bytes_of(f->stream_dtype);
    if (f->tokens > 0 && !f->y && (g->dy || g->dgate || g->dw_post || g->db_post))
        return ctx_fail(c, ARENA_ERR_INVALID_ARG, "%s: dy, dgate, dw_post and db_post need y", who);
    if (g->dgate && !f->gate) return ctx_fail(c, ARENA_ERR_INVALID_ARG, "%s: dgate needs gate", who);
    const void* sums[] = {g->dgate, g->dw_post, g->db_post, g->dw_pre, g->db_pre};
    for (const void* v : sums)
        if (!aligned(v, size)) return ctx_fail(c, ARENA_ERR_INVALID_ARG, "%s: a gradient is not aligned to its values", who);
    if (f->tokens > 0) {
        if (!g->dn && !g->dr) return ctx_fail(c, ARENA_ERR_INVALID_ARG, "%s: neither dn nor dr", who);
        if (!f->stats) return ctx_fail(c, ARENA_ERR_INVALID_ARG, "%s: stats is NULL", who);
        const void* res = f->y ? f->r : f->x;
        if ((g->dn && (s = check_matrix(c, who, "dn", g->dn, g->ld_dn, f->width, size))) ||
            (g->dn && (s = check_matrix(c, who, f->y ? "r" : "x", res, f->y ? f->ld_r : f->ld_x, f->width, wide))) ||
            (g->dr && (s = check_matrix(c, who, "dr", g->dr, g->ld_dr, f->width, wide))) ||
            (g->dx && (s = check_matrix(c, who, "dx", g->dx, g->ld_dx, f->width, wide))) ||
            (g->dy && (s = check_matrix(c, who, "dy", g->dy, g->ld_dy, f->width, size))) ||
            (s = check_workspace(c, who, g->workspace, g->workspace_bytes, need)))
            return s;
    }
    NormArgs A = norm_args(f);
    A.dn = g->dn; A.ld_dn = g->ld_dn;
    A.dr = g->dr; A.ld_dr = g->ld_dr;
    A.res = f->y ? f->r : f->x;
    A.ld_res = f->y ? f->ld_r : f->ld_x;
    A.dx = g->dx; A.ld_dx = g->ld_dx;
    A.dy = g->dy; A.ld_dy = g->ld_dy;
    A.dgate = f->tokens > 0 || f->gate_rows == 0 ? g->dgate : nullptr;
    A.dw_post = g->dw_post; A.db_post = g->db_post;
    A.dw_pre = g->dw_pre; A.db_pre = g->db_pre;
    A.part = (float*)g->workspace;
    A.means = (float*)((char*)g->workspace + sums_bytes);
    A.workers = workers;
    A.rows_each = rows;
    DeviceScope scope(arena::ctx_device(c));
    if (scope.status != hipSuccess) return hip_error(c, scope.status, "hipSetDevice");
    const hipError_t e = arena::launch_norm_backward(A, f->dtype, f->stream_dtype, (hipStream_t)stream);
    return e == hipSuccess ? ARENA_OK : hip_error(c, e, "norm backward launch");
}

arena_status arena_ffn_forward_workspace(arena_ctx* c, const arena_ffn_desc* d, int64_t* bytes)
{
    if (!c) return ARENA_ERR_INVALID_ARG;
    ctx_clear(c);
    if (!bytes) return ctx_fail(c, ARENA_ERR_INVALID_ARG, "ffn forward: bytes is NULL");
    const arena_status s = check_ffn(c, "ffn forward", d, false);
    if (s) return s;
    *bytes = d->tokens ? ForwardPlan(d, nullptr).w.used : 0;
    return ARENA_OK;
}

arena_status arena_ffn_forward(arena_ctx* c, const arena_ffn_desc* d, void* stream)
{
    if (!c) return ARENA_ERR_INVALID_ARG;
    ctx_clear(c);
    arena_status st = check_ffn(c, "ffn forward", d, false);
    if (st || d->tokens == 0) return st;
    const ForwardPlan P(d, d->workspace);
    if ((st = check_workspace(c, "ffn forward", d->workspace, d->workspace_bytes, P.w.used))) return st;
    DeviceScope scope(arena::ctx_device(c));
    if (scope.status != hipSuccess) return hip_error(c, scope.status, "hipSetDevice");
    hipStream_t s = (hipStream_t)stream;
    hipError_t e = pack({&P.x, &P.gate, &P.up, &P.down}, s);
    if (e) return hip_error(c, e, "ffn forward copies");

    GemmArgs A = new_args(d->tokens, d->inner, d->model);
    A.a[0] = P.x.p; A.lda = P.x.ld;
    A.b[0] = P.gate.p; A.b[1] = P.up.p; A.ldb = P.gate.ld; A.ldb1 = P.up.ld;
    A.c[0] = d->h; A.ldc = d->ld_inner;
    A.g = d->g; A.u = d->u; A.ldg = d->ld_inner;
    A.act = d->activation;
    A.pad = (int)pad8(d->inner);
    A.part = (float*)P.part;
    e = P.skinny ? arena::mm::launch_skinny(A, d->dtype, true, s)
                 : arena::mm::launch_gemm(A, d->dtype, arena::mm::kGateUp, P.cut_up, s);
    if (e) return hip_error(c, e, "ffn gate and up launch");

    GemmArgs B = new_args(d->tokens, d->model, d->inner);
    B.a[0] = d->h; B.lda = d->ld_inner;
    B.b[0] = P.down.p; B.ldb = P.down.ld;
    B.c[0] = d->y; B.ldc = d->ld_y;
    B.part = (float*)P.part;
    e = P.skinny ? arena::mm::launch_skinny(B, d->dtype, false, s)
                 : arena::mm::launch_gemm(B, d->dtype, arena::mm::kRowsRows, P.cut_down, s);
    return e == hipSuccess ? ARENA_OK : hip_error(c, e, "ffn down launch");
}

arena_status arena_ffn_backward_workspace(arena_ctx* c, const arena_ffn_desc* f, const arena_ffn_grads* g,
                                          int64_t* bytes)
{
    if (!c) return ARENA_ERR_INVALID_ARG;
    ctx_clear(c);
    if (!bytes) return ctx_fail(c, ARENA_ERR_INVALID_ARG, "ffn backward: bytes is NULL");
    arena_status s;
    if ((s = check_ffn(c, "ffn backward", f, true)) || (s = check_ffn_grads(c, "ffn backward", f, g))) return s;
    *bytes = BackwardPlan(f, g, nullptr).w.used;
    return ARENA_OK;
}

arena_status arena_ffn_backward(arena_ctx* c, const arena_ffn_desc* f, const arena_ffn_grads* g, void* stream)
{
    if (!c) return ARENA_ERR_INVALID_ARG;
    ctx_clear(c);
    const char* who = "ffn backward";
    arena_status st;
    if ((st = check_ffn(c, who, f, true)) || (st = check_ffn_grads(c, who, f, g))) return st;
    const BackwardPlan P(f, g, f->workspace);
    if ((st = check_workspace(c, who, f->workspace, f->workspace_bytes, P.w.used))) return st;
    DeviceScope scope(arena::ctx_device(c));
    if (scope.status != hipSuccess) return hip_error(c, scope.status, "hipSetDevice");
    hipStream_t s = (hipStream_t)stream;
    const int64_t T = f->tokens, D = f->model, F = f->inner;
    const int out = g->grad_dtype == ARENA_F32 ? arena::mm::kOutF32 : arena::mm::kOut16;
    hipError_t e = pack({&P.x, &P.gate, &P.up, &P.down, &P.dy}, s);
    if (e) return hip_error(c, e, "ffn backward copies");

    // the inner gradient, dx, and the weight gradients C[m, n] = sum over tokens
    // of a(t, m) b(t, n) beside what accumulate keeps
    GemmArgs H = new_args(T, F, D);
    H.a[0] = P.dy.p; H.lda = P.dy.ld;
    H.b[0] = P.down.p; H.ldb = P.down.ld;
    H.g = f->g; H.u = f->u; H.ldg = f->ld_inner;
    H.c[0] = P.dg; H.c[1] = P.du; H.ldc = P.ld;
    H.act = f->activation;
    H.pad = (int)P.ld;
    H.part = (float*)P.part;
    GemmArgs X = new_args(T, D, F);
    X.nseg = 2;
    X.a[0] = P.dg; X.a[1] = P.du; X.lda = P.ld;
    X.b[0] = P.gate.p; X.b[1] = P.up.p; X.ldb = P.gate.ld;
    X.c[0] = g->dx; X.ldc = g->ld_dx;
    X.part = (float*)P.part;
    auto weight = [&](const void* a0, const void* a1, int64_t lda, const void* b, int64_t ldb, int64_t M, int64_t N,
                      void* c0, void* c1, int64_t ldc) {
        GemmArgs A = new_args(M, N, T);
        A.pairs = c1 != nullptr;
        A.batch = c1 ? 2 : 1;
        A.a[0] = a0; A.a[1] = a1; A.lda = lda;
        A.b[0] = A.b[1] = b; A.ldb = ldb;
        A.c[0] = c0; A.c[1] = c1; A.ldc = ldc;
        A.out = out;
        if (g->accumulate) {
            A.beta = 1.0f;
            A.e[0] = c0; A.e[1] = c1; A.lde = ldc;
        }
        A.part = (float*)P.part;
        return A;
    };
    const GemmArgs down = weight(P.dy.p, nullptr, P.dy.ld, f->h, f->ld_inner, D, F, g->dw_down, nullptr, g->ld_dw_down);
    const bool inner_grad = T > 0 && (g->dx || g->dw_gate || g->dw_up);
    using namespace arena::mm;
    if (P.pair_dh.splits) {
        if ((e = launch_pair(H, f->dtype, kGateUpBack, down, P.pair_dh, s)))
            return hip_error(c, e, "ffn inner and down gradients launch");
    } else {
        if (inner_grad && (e = launch_gemm(H, f->dtype, kGateUpBack, P.cut_dh, s)))
            return hip_error(c, e, "ffn inner gradient launch");
        if (g->dw_down && (e = launch_gemm(down, f->dtype, kColsCols, P.cut_down, s)))
            return hip_error(c, e, "ffn down gradient launch");
    }
    if (P.pair) {
        const GemmArgs up = weight(P.dg, P.du, P.ld, P.x.p, P.x.ld, F, D, g->dw_gate, g->dw_up, g->ld_dw_gate);
        if (P.pair_dx.splits) {
            if ((e = launch_pair(X, f->dtype, kRowsCols, up, P.pair_dx, s)))
                return hip_error(c, e, "ffn input, gate and up gradients launch");
            return ARENA_OK;
        }
        if ((e = launch_gemm(up, f->dtype, kColsCols, P.cut_up, s)))
            return hip_error(c, e, "ffn gate and up gradient launch");
    } else {
        if (g->dw_gate && (e = launch_gemm(weight(P.dg, nullptr, P.ld, P.x.p, P.x.ld, F, D, g->dw_gate, nullptr,
                                                  g->ld_dw_gate), f->dtype, kColsCols, P.cut_up, s)))
            return hip_error(c, e, "ffn gate gradient launch");
        if (g->dw_up && (e = launch_gemm(weight(P.du, nullptr, P.ld, P.x.p, P.x.ld, F, D, g->dw_up, nullptr,
                                                g->ld_dw_up), f->dtype, kColsCols, P.cut_up, s)))
            return hip_error(c, e, "ffn up gradient launch");
    }
    if (T > 0 && g->dx && (e = launch_gemm(X, f->dtype, kRowsCols, P.cut_dx, s)))
        return hip_error(c, e, "ffn input gradient launch");
    return ARENA_OK;
}

arena_status arena_orthogonal_update_workspace(arena_ctx* c, const arena_update_desc* d, int64_t* bytes)
{
    if (!c) return ARENA_ERR_INVALID_ARG;
    ctx_clear(c);
    if (!bytes) return ctx_fail(c, ARENA_ERR_INVALID_ARG, "orthogonal update: bytes is NULL");
    const arena_status s = check_update(c, "orthogonal update", d);
    if (s) return s;
    *bytes = UpdatePlan(d, nullptr).w.used;
    return ARENA_OK;
}

arena_status arena_orthogonal_update(arena_ctx* c, const arena_update_desc* d, void* stream)
{
    if (!c) return ARENA_ERR_INVALID_ARG;
    ctx_clear(c);
    const char* who = "orthogonal update";
    arena_status st = check_update(c, who, d);
    if (st) return st;
    const UpdatePlan P(d, d->workspace);
    if ((st = check_workspace(c, who, d->workspace, d->workspace_bytes, P.w.used))) return st;
    DeviceScope scope(arena::ctx_device(c));
    if (scope.status != hipSuccess) return hip_error(c, scope.status, "hipSetDevice");
    hipStream_t s = (hipStream_t)stream;

    UpdateArgs U;
    std::memset(&U, 0, sizeof(U));
    U.grad = d->grad; U.ld_grad = d->ld_grad; U.s_grad = d->stride_grad;
    U.momentum = d->momentum; U.ld_mom = d->ld_momentum; U.s_mom = d->stride_momentum;
    U.momentum_out = d->momentum_out; U.ld_mom_out = d->ld_momentum_out; U.s_mom_out = d->stride_momentum_out;
    U.rows = d->rows; U.cols = d->cols; U.batch = d->batch;
    U.nesterov = d->nesterov != 0;
    U.mu = d->mu; U.eps = d->eps;
    U.x = P.x[0];
    U.rest = keeps_rest(d, 0) ? P.rest : nullptr;
    U.rows_p = (int)P.rows; U.ld_x = (int)P.cols;
    U.part = (double*)P.sums;
    U.blocks = P.blocks;
    hipError_t e;
    if ((e = arena::launch_update_sum(U, d->dtype, s)) || (e = arena::launch_update_scale(U, d->dtype, s)))
        return hip_error(c, e, "update scaling launch");

    const int64_t sx = P.rows * P.cols, sg = P.side * P.side;
    const float inv = (float)(1.0 / kHalfScale);
    auto run = [&](GemmArgs& A, const Cut& cut, bool sym, arena::mm::Product what) {
        A.batch = d->batch;
        A.sym = sym;
        A.part = (float*)P.part;
        return arena::mm::launch_gemm(A, ARENA_F16, what, cut, s);
    };
    int at = 0;
    for (int i = 0; i < std::max(1, (int)d->steps); ++i) {
        const bool last = i + 1 >= d->steps;
        const float* k = d->steps ? d->coefficients + 3 * i : nullptr;
        void* x = P.x[at];
        if (k) {
            // 2^12 C = 2^-12 (2^12 X)(2^12 X)^T - 2^11
            GemmArgs A = new_args(P.side, P.side, P.tall ? P.rows : P.cols);
            A.a[0] = A.b[0] = x; A.lda = A.ldb = P.cols; A.sa = A.sb = sx;
            A.c[0] = P.gram; A.ldc = P.side; A.sc = sg;
            A.alpha = inv;
            A.diag = (float)(kCentre * kHalfScale);
            if ((e = run(A, P.cut_gram, P.sym_gram, P.tall ? arena::mm::kColsCols : arena::mm::kRowsRows)))
                return hip_error(c, e, "update Gram launch");
            // 2^12 ((b + c) C + c C^2); C is symmetric, so its rows serve as columns
            GemmArgs B = new_args(P.side, P.side, P.side);
            B.a[0] = B.b[0] = P.gram; B.lda = B.ldb = P.side; B.sa = B.sb = sg;
            B.c[0] = P.poly; B.ldc = P.side; B.sc = sg;
            B.e[0] = P.gram; B.lde = P.side; B.se = sg;
            B.alpha = k[2] * inv;
            B.beta = (float)(k[1] + 2.0 * kCentre * k[2]);
            if ((e = run(B, P.cut_square, P.sym_square, arena::mm::kRowsRows)))
                return hip_error(c, e, "update square launch");
        }
        // 2^12 ((a + b/2 + c/4) X + B X), or X B where X is tall; the last step writes scale times it
        GemmArgs X = new_args(last ? d->rows : P.rows, last ? d->cols : P.cols, k ? P.side : 0);
        if (P.tall) {
            X.a[0] = x; X.lda = P.cols; X.sa = sx;
            X.b[0] = P.poly; X.ldb = P.side; X.sb = sg;
        } else {
            X.a[0] = P.poly; X.lda = P.side; X.sa = sg;
            X.b[0] = x; X.ldb = P.cols; X.sb = sx;
        }
        X.e[0] = x; X.lde = P.cols; X.se = sx;
        X.alpha = inv;
        X.beta = k ? (float)(k[0] + kCentre * k[1] + kCentre * kCentre * k[2]) : 1.0f;
        arena::mm::Product what = P.tall ? arena::mm::kRowsRows : arena::mm::kRowsCols;
        if (keeps_rest(d, i)) {
            what = P.tall ? arena::mm::kRowsRowsRest : arena::mm::kRowsColsRest;
            X.rest = P.rest;
            X.rest_in = k[0] * (1.0f / 2048.0f);
            X.rest_out = keeps_rest(d, i + 1);
            X.pad = X.N;
        }
        if (last) {
            X.alpha *= d->scale * inv;
            X.beta *= d->scale * inv;
            X.c[0] = d->out; X.ldc = d->ld_out; X.sc = d->stride_out;
            X.out = d->out_dtype == ARENA_BF16 ? arena::mm::kOutBf16 : arena::mm::kOut16;
        } else {
            X.c[0] = P.x[at ^ 1]; X.ldc = P.cols; X.sc = sx;
        }
        if ((e = run(X, P.cut_x, false, what)))
            return hip_error(c, e, "update product launch");
        at ^= 1;
    }
    return ARENA_OK;
}

}  // extern "C"
