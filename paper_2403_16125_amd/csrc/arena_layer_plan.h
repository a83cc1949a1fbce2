// What the host sides of the layer operators share: checks of arguments, pieces of a
// workspace, and the choice of tiles and splits for a product.
#pragma once

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <initializer_list>

#include "arena_layer.h"
#include "arena_layer_internal.h"

namespace arena {
namespace plan {

using mm::GemmArgs;

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

inline arena_status hip_error(arena_ctx* c, hipError_t e, const char* what)
{
    return ctx_fail(c, ARENA_ERR_DEVICE, "%s: %s", what, hipGetErrorString(e));
}

inline int64_t pad8(int64_t n) { return (n + 7) / 8 * 8; }
inline int64_t pad256(int64_t n) { return (n + 255) / 256 * 256; }
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline bool aligned(const void* p, size_t bytes) { return ((uintptr_t)p & (bytes - 1)) == 0; }
inline int bytes_of(int dtype) { return dtype == ARENA_F32 ? 4 : 2; }

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

inline arena_status check_workspace(arena_ctx* c, const char* who, const void* p, int64_t have, int64_t need)
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
inline arena_status check_matrix(arena_ctx* c, const char* who, const char* name, const void* p, int64_t ld, int64_t width,
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

using mm::Cut;

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
inline double launch_time(int64_t tiles, int64_t steps, int kind, int64_t splits, double bytes)
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
inline Cut choose_cut(int64_t M, int64_t N, int64_t steps, int64_t batch, bool dual, bool sym, double bytes,
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

inline Cut choose_pair(const Half& a, const Half& b)
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
inline Cut choose_symmetric(int64_t n, int64_t steps, int64_t batch, double bytes, bool* sym)
{
    double all, half;
    const Cut a = choose_cut(n, n, steps, batch, false, false, bytes, &all);
    const Cut h = choose_cut(n, n, steps, batch, false, true, bytes + 2.0, &half);
    *sym = half < all;
    return *sym ? h : a;
}

inline int64_t part_bytes(const Cut& cut, int64_t M, int64_t N, int64_t batch, bool dual, bool sym)
{
    if (cut.splits <= 1) return 0;
    const int64_t side = arena::mm::kTileSide[cut.main], tm = ceil_div(M, side), tn = ceil_div(N, dual ? side / 2 : side);
    const int64_t all = (sym ? tm * (tm + 1) / 2 : tm * tn) * batch;
    return 4 * cut.splits * (all - cut.first) * side * side;
}

template <typename Args = GemmArgs>
inline Args new_args(int64_t M, int64_t N, int64_t K)
{
    Args A;
    std::memset((void*)&A, 0, sizeof(A));
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
inline hipError_t pack(std::initializer_list<const Operand*> operands, hipStream_t s)
{
    arena::mm::Pack packs[arena::mm::kMaxPacks];
    int n = 0;
    for (const Operand* o : operands)
        if (o->copy && n < arena::mm::kMaxPacks)
            packs[n++] = {o->from, o->copy, o->ld_from, o->ld, o->rows, o->cols};
    return n ? arena::mm::launch_packs(packs, n, s) : hipSuccess;
}

// ---------------------------------------------------------------- products of groups

// What a kind of tile costs in microseconds (measured on one MI355X): a step of 64 of k
// with every slot of the compute units taken and with at most one block on each, a tile
// beside its steps, and how many blocks a compute unit holds.
struct GroupCost {
    double full, alone, start;
    int slots;
};
constexpr GroupCost kGroupCost[mm::kGroupKinds] = {
    {1.75, 1.30, 4.0, 1}, {1.00, 0.75, 3.0, 2}, {0.80, 0.60, 2.0, 2}};

// uneven: how much longer than the average one the longest of few tiles takes.  exact: how
// many tiles there are is known, and the last round counts as what it is; otherwise half a
// round more than they fill.
inline double group_time(double tiles, double steps, int kind, int64_t splits, double bytes, double uneven,
                         bool exact, bool any)
{
    if (any && kind == mm::kGroup256) return INFINITY;
    const GroupCost& k = kGroupCost[kind];
    const double per = std::ceil(steps / splits), values = (double)mm::kGroupRows[kind] * mm::kGroupCols[kind];
    const double end = values * (splits > 1 ? 4.0 : bytes) / kEpilogueRate;
    const double blocks = tiles * splits, round = kUnits * k.slots;
    const double alone = per * uneven * k.alone + k.start + end, full = per * k.full + k.start + end * k.slots;
    const double whole = std::floor(blocks / round), rest = blocks - whole * round;
    const double t = blocks <= kUnits  ? alone
                     : blocks <= round ? full + per * (uneven - 1.0) * k.full
                     : exact           ? whole * full + (rest > kUnits ? full : rest > 0 ? alone : 0.0)
                                       : (blocks / round + 0.5) * full;
    return kLaunch + t + (splits > 1 ? kJoin + blocks * values * 4e-6 / kJoinRate : 0.0);
}

// The kind of tile, and the parts of k if it may be split, for a product on resident blocks.
struct GroupCut {
    int kind, splits;
    int64_t part;             // bytes
    int tail;                 // most parts of the last round's tiles
};

constexpr double kTailJoin = 15.0;          // its launch and reads

// Whether the tiles past the last whole round are worth parts of their own: they cost a join.
// Sets *tail and the bytes of the parts (not more tiles than there are blocks); returns the time.
inline double tail_time(double tiles, double steps, int kind, double bytes, int* tail, int64_t* part)
{
    const GroupCost& k = kGroupCost[kind];
    const double values = (double)mm::kGroupRows[kind] * mm::kGroupCols[kind], round = kUnits * k.slots;
    const double full = steps * k.full + k.start + values * bytes / kEpilogueRate * k.slots;
    *tail = (int)std::min(8.0, steps / 8);
    *part = (int64_t)(4 * round * values);
    if (*tail < 2 || tiles < round) return INFINITY;
    return kLaunch + (tiles / round + 0.25) * full + kTailJoin;
}

inline GroupCut choose_groups(int64_t M, int64_t N, int64_t steps, int64_t batch, double bytes, bool split, double uneven,
                              bool exact, bool any)
{
    using namespace mm;
    GroupCut best = {any ? kGroup128 : kGroup256, 1, 0, 0};
    double least = INFINITY;
    for (int kind = 0; kind < kGroupKinds; ++kind) {
        const int64_t tiles = ceil_div(M, kGroupRows[kind]) * ceil_div(N, kGroupCols[kind]) * batch;
        for (int s = 1; s <= 64 && (s == 1 || (split && s * 4 <= steps)); ++s) {
            if (tiles * s > 0x7fffffff) continue;
            const double t = group_time((double)tiles, (double)steps, kind, s, bytes, uneven, exact, any);
            if (t < least) {
                least = t;
                best = {kind, s, s > 1 ? 4 * s * tiles * kGroupRows[kind] * kGroupCols[kind] : 0, 0};
            }
        }
    }
    return best;
}

}  // namespace plan
}  // namespace arena
