// Matrix products of groups (experts): rows offsets[g] .. offsets[g + 1] - 1 of A and C
// meet matrix g of B, or those steps of k of both operands make matrix g of C.  The products
// of a loss are of one group.  Loaders, fragments and the gated epilogues' formulas are those
// of arena_gemm.h.
//
// The groups are short and many, so what a tile costs beside its steps decides.  Blocks
// are resident: each takes tile after tile, and starts the next one's first loads before it
// writes the last.  For that the epilogue leaves the LDS alone: a lane holds four
// neighbouring columns of a row in each fragment, and a swap of rows of lanes between two
// fragments makes them eight of one.
//
// Waves whose rows all lie past the group's end only load for the others: they share a
// SIMD with waves that do not, so such a step takes little more than half the time.
//
// Large products are bound by the matrix cores and the clock under load, and by last rounds
// that do not fill the card.  In bfloat16, 16384 rows of 8 experts 4096 x 10944 (medians of six passes;
// other runs' differ by up to 4 %): gate and up 2.74 ms (1070 TFLOP/s), down 1.24 (1190), inner gradients
// 1.64 (890), weights' gradients 1.35 and 2.57 (1090 and 1140), dx 2.38 (1230), matrix cores busy in 48 to
// 66 % of the cycles.  A loss of 8192 tokens, 131072 x 4096: logits 6.63 ms (1330), a piece of 16384 entries
// 0.85 ms for their gradient, 0.84 for dx, 0.82 for dw (1290 to 1340).  With 256 rows an expert (64 of 2048 x 1408)
// the weights are read or written once for every two to four tiles and groups waste half a tile:
// 323 us, 157, 215, 238 + 445 and 297 (400 to 640), matrix cores busy in 25 to 34 %.  Small ones are
// bound by latency: about 8 us for the launch, the table, the first loads and the epilogue, and
// 0.6 to 0.8 for a step.
#pragma once

#include <algorithm>

#include "arena_gemm.h"

namespace arena {
namespace mm {

template <typename T_, int BM_, int BN_, int WM_, int WN_, bool ATR_, bool BTR_, int EPI_, int GROUP_, bool DIRECT_>
struct GroupTile {
    typedef T_ T;
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_;
    static constexpr bool ATR = ATR_, BTR = BTR_, DUAL = EPI_ == kGatedFwd;
    static constexpr int EPI = EPI_, GROUP = GROUP_;
    static constexpr bool kUpToN = EPI_ == kPlain || EPI_ == kWide;
    static constexpr bool kDirect = DIRECT_;
    static constexpr int kThreads = 64 * WM * WN;
    static constexpr int FM = BM / WM / 16, FN = BN / WN / 16;
    static constexpr int kCols = DUAL ? BN / 2 : BN;
    static constexpr bool kLean = BM == 256 && (EPI == kGatedBwd || EPI == kWide);
    // k in parts: of few rows the tiles do not fill the compute units
    static constexpr bool kSplit = EPI == kWide || (GROUP == kRowGroups && BM < 256 && (EPI == kPlain || EPI == kGatedBwd));
    static constexpr bool kTail = GROUP == kRowGroups && EPI == kPlain;      // the last round's tiles too
    static constexpr int kSegs = GROUP == kRowGroups && EPI == kPlain && BTR ? 2 : 1;    // both halves of dx
    // Buffers.  The smallest tiles are those of products with few: there a step is as long as
    // a load's way, unless it starts a step earlier.
    static constexpr int kStages = BM == 64 && DIRECT_ ? 3 : 2;
    // blocks on a compute unit, by their LDS (the groups' table is at most 12 KB)
    static constexpr int kBlocks = kStages * (BM + BN) * 128 <= 73728 ? 2 : 1;
    static constexpr int kWavesEach = kThreads / 256 * kBlocks;
    static constexpr int kRun = 32 * kBlocks;            // tiles that an XCD has in work at once
    // bytes of a row that the epilogue reads, brought to the LDS with the tile's first step:
    // read in the epilogue they would wait for the next tile's loads
    static constexpr int kRowBytes = EPI == kLossGrad ? 16 : EPI == kLossStats ? 4 : 0;
};

// The q-th tile of XCD x, -1 past its last: runs of RUN tiles go to the XCDs in turn, and
// what is left in eighths.  An eighth of all tiles to each would give the XCD with the longest
// groups of steps half as much again to do (8 experts of 16384 rows, 4096 x 10944: 1988 us
// so, in runs 1455), and takes 5 to 7 % longer with groups of rows too, where the XCDs then
// read different experts at a time.
template <int RUN>
__device__ __forceinline__ int tile_of_xcd(int x, int q, int tiles)
{
    const int whole = tiles / (8 * RUN);
    if (q < whole * RUN) return (q / RUN * 8 + x) * RUN + q % RUN;
    const int r = q - whole * RUN, rest = tiles - whole * 8 * RUN, per = rest >> 3, more = rest & 7;
    return r < per + (x < more ? 1 : 0) ? whole * 8 * RUN + x * per + min(x, more) + r : -1;
}

// Of every group its first row or step and its end, and of rows how many tile rows end with
// the group; in the LDS behind the buffers, as long as there are groups.
struct GroupTable {
    int *first, *end, *tiles;
    __device__ __forceinline__ GroupTable(int* p, int groups) : first(p), end(p + groups), tiles(p + 2 * groups) {}
    static int bytes(int group, int groups) { return group == kOneGroup ? 0 : (group == kRowGroups ? 12 : 8) * groups; }
};

// Offset g, held inside 0 .. rows whatever the offsets are.
__device__ __forceinline__ int group_end(const int32_t* offsets, int g, int rows)
{
    return min(max(offsets[g], 0), rows);
}

// Rows of group g and the tile rows that they make.
template <int BM>
__device__ __forceinline__ int tile_rows(const GroupArgs& A, int g, int* lo, int* hi)
{
    *lo = *hi = 0;
    if (g < A.groups) {
        *lo = group_end(A.offsets, g, A.M);
        *hi = max(*lo, group_end(A.offsets, g + 1, A.M));
    }
    return (*hi - *lo + BM - 1) / BM;
}

// Fills the table (one wave) and returns how many tile rows there are, at most `most`:
// groups that overlap could have more than a launch counts.
template <int BM>
__device__ __forceinline__ int fill_table(const GroupArgs& A, const GroupTable* table, int lane, int most)
{
    int total = 0;
    for (int g0 = 0; g0 < A.groups; g0 += 64) {
        int lo, hi;
        const int mine = tile_rows<BM>(A, g0 + lane, &lo, &hi);
        int sum = mine;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int w = __shfl_up(sum, d, 64);
            sum += lane >= d ? w : 0;
        }
        if (g0 + lane < A.groups) {
            table->first[g0 + lane] = lo;
            table->end[g0 + lane] = hi;
            table->tiles[g0 + lane] = min(most, total + sum);
        }
        total = min(most, total + __builtin_amdgcn_readlane(sum, 63));
    }
    return total;
}

// wide: as plain, the added matrix of a type of its own and of a group.
template <typename T>
struct Side<T, kWide> {
    u32x4 raw[2];
    __device__ __forceinline__ void load(const GroupArgs& A, int z, int m, int n)
    {
        if (A.beta == 0.0f) return;
        const char* p = (const char*)A.e[A.pairs ? z & 1 : 0];
        const int64_t from = (z >> A.pairs) * A.se + (int64_t)m * A.lde + n;
        const int left = A.N - n;
        if (A.e_f32) {
            const uint32_t* q = (const uint32_t*)p + from;
            if (left >= 8) __builtin_memcpy(raw, q, 32);
            else
#pragma unroll
                for (int r = 0; r < 8; ++r) raw[r >> 2][r & 3] = r < left ? q[r] : 0;
        } else {
            const uint16_t* q = (const uint16_t*)p + from;
            if (left >= 8) __builtin_memcpy(raw, q, 16);
            else
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    raw[0][r] = (2 * r < left ? q[2 * r] : 0) | (2 * r + 1 < left ? (uint32_t)q[2 * r + 1] << 16 : 0);
        }
    }
    __device__ __forceinline__ float get(int r, bool f32) const
    {
        typedef typename T::E E;
        if (f32) return __uint_as_float(raw[r >> 2][r & 3]);
        const uint16_t h = (uint16_t)(raw[0][r >> 1] >> (16 * (r & 1)));
        E e;
        __builtin_memcpy(&e, &h, 2);
        return (float)e;
    }
};

template <typename T>
__device__ __forceinline__ void plain_out(const GroupArgs& A, int z, int m, int n, float (&v)[8],
                                          const Side<T, kWide>& side)
{
    typedef typename T::E E;
    const int left = A.N - n;
    const int64_t at = (z >> A.pairs) * A.sc + (int64_t)m * A.ldc + n;
    void* c = A.c[A.pairs ? z & 1 : 0];
    const float alpha = A.factor ? A.alpha * A.factor[0] : A.alpha;
#pragma unroll
    for (int r = 0; r < 8; ++r) v[r] *= alpha;
    if (A.beta != 0.0f)
#pragma unroll
        for (int r = 0; r < 8; ++r) v[r] += A.beta * side.get(r, A.e_f32);
    if (A.out == kOutF32) put((float*)c + at, v, left);
    else put((E*)c + at, v, left);
}

// factor (exp(l - lse) - [column is the target]), zero for tokens left out of the loss,
// whatever their logits: rounded to 16 bits as the next two products' operand.
// LOW: for few tokens, what that rounding took off too, as rows of their own.
template <typename T, bool LOW>
__device__ __forceinline__ void loss_grad_out(const GroupArgs& A, int m, int n, const float (&v)[8], const LossRow& row)
{
    typedef typename T::E E;
    const float lse = row.lse, factor = row.factor;
    const int target = row.target, at = target - A.first_col - n;
    float g[8];
#pragma unroll
    for (int r = 0; r < 8; ++r) {
        const float p = __expf(v[r] - lse) - (r == at ? 1.0f : 0.0f);
        g[r] = n + r < A.N && target >= 0 ? factor * p : 0.0f;
    }
    put((E*)A.c[0] + (int64_t)m * A.ldc + n, g, 8);
    if (LOW && A.low) {
#pragma unroll
        for (int r = 0; r < 8; ++r) {
            const float high = (float)(E)g[r];
            g[r] = __builtin_fabsf(high) < INFINITY ? g[r] - high : 0.0f;
        }
        put((E*)A.c[0] + (int64_t)(m + A.low) * A.ldc + n, g, 8);
    }
}

// The statistics of a row's logits as they lie in the sums: a lane has columns 4 (lane >> 4) +
// 0..3 of each fragment, from column n on; four lanes share the row.  Of those below N the
// largest, the sum of exponentials beside it, and the target's (in A.picked[m]), if it is
// among them.
template <typename P>
__device__ __forceinline__ f32x2 row_stats(const GroupArgs& A, const f32x4 (&row)[P::FN], int m, int n, int target)
{
    float most = -INFINITY, sum = 0.0f;
    const bool whole = __all(n + (P::FN - 1) * 16 + 4 <= A.N);
    if (whole) {
#pragma unroll
        for (int j = 0; j < P::FN; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q) most = fmaxf(most, row[j][q]);
    } else {
#pragma unroll
        for (int j = 0; j < P::FN; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                if (n + j * 16 + q < A.N) most = fmaxf(most, row[j][q]);
    }
    most = fmaxf(most, __shfl_xor(most, 16, 64));
    most = fmaxf(most, __shfl_xor(most, 32, 64));
    const float by = most == -INFINITY ? 0.0f : most;       // of nothing but -inf the sum is 0
#pragma unroll
    for (int j = 0; j < P::FN; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const float e = __expf(row[j][q] - by);
            sum += whole || n + j * 16 + q < A.N ? e : 0.0f;
        }
    sum += __shfl_xor(sum, 16, 64);
    sum += __shfl_xor(sum, 32, 64);
    const int at = target - n;
    if (m < A.M && at >= 0 && at < P::FN * 16 && (at & 12) == 0) {
        float l = 0.0f;
#pragma unroll
        for (int j = 0; j < P::FN; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                if (at == j * 16 + q) l = row[j][q];
        A.picked[m] = l;
    }
    return f32x2{most, sum};
}

struct OneFragment {
    static constexpr int FN = 1;
};

// A tile: its place, its steps and its operands' first addresses.
struct Work {
    int m0, n0, m_end, z;       // z: group, or with pairs twice that and which of the two
    int part, parts;            // of a split k
    int slot;                   // of the last round's tiles
    int steps, sps, K;          // steps of all segments, of one, and k of a segment
    int s0;                     // first step of the part
};

// The tiles past the last whole round of `blocks` resident ones, and in how many parts of k
// they are shared out among all blocks (16384 rows of 8 experts 4096 x 10944, 4.25 rounds: down
// 1365 us whole, 1245 with the last 64 tiles in four parts; dx 2642 and 2341).
struct Tail {
    int tiles, parts;
    __device__ __forceinline__ Tail(int all, int blocks, int most)
    {
        tiles = most > 1 ? all % blocks : 0;
        parts = tiles > 0 ? min(most, blocks / tiles) : 1;
        if (parts < 2) tiles = 0, parts = 1;
    }
};

// Group and place of a tile, counted without parts.
template <typename P>
__device__ __forceinline__ void locate(const GroupArgs& A, const GroupTable& table, int lane, int tile, Work* w)
{
    constexpr bool kRows = P::GROUP == kRowGroups;
    int band_rows, in;
    if constexpr (kRows) {
        int below = 0;
        for (int g0 = 0;; g0 += 64) {
            const int ends = g0 + lane < A.groups ? table.tiles[g0 + lane] : 0x7fffffff;
            const int first = g0 + lane < A.groups ? table.first[g0 + lane] : 0;
            const uint64_t past = __ballot(tile < (int64_t)ends * A.tiles_n);
            if (past) {
                const int l = __ffsll((unsigned long long)past) - 1;
                if (l > 0) below = __builtin_amdgcn_readlane(ends, l - 1);
                w->z = g0 + l;
                w->m0 = __builtin_amdgcn_readlane(first, l);
                band_rows = __builtin_amdgcn_readlane(ends, l) - below;
                break;
            }
            below = __builtin_amdgcn_readlane(ends, 63);
        }
        in = tile - below * A.tiles_n;
    } else {
        const int each = A.tiles_m * A.tiles_n;
        w->z = quotient(tile, each);
        w->m0 = 0;
        band_rows = A.tiles_m;
        in = tile - w->z * each;
    }
    // bands of 8 tile rows
    const int band = 8 * A.tiles_n, b = quotient(in, band), at = in - b * band;
    const int high = min(8, band_rows - b * 8), tn = quotient(at, high);
    const int tm = b * 8 + at - tn * high;
    w->n0 = tn * P::kCols;
    w->m_end = A.M;
    if constexpr (kRows) w->m_end = __builtin_amdgcn_readfirstlane(table.end[w->z]);
    w->m0 += tm * P::BM;
}

// The loader of arena_gemm.h, with its lanes' part apart.
template <typename P, int R, bool TR, bool DUAL>
struct GroupLoader : Loader<P, R, TR, DUAL> {
    typedef Loader<P, R, TR, DUAL> Base;
    __device__ __forceinline__ void lanes(int) {}
    __device__ __forceinline__ void start(int tid, int first, int n, int64_t ld) { Base::init(tid, first, n, ld); }
    __device__ __forceinline__ int64_t pitch() const { return Base::step; }
};

// The same in two registers a lane: where a lane's chunks lie is worked out again for every
// load.  That costs a tenth of the plain products' time, but with the gated backward epilogue
// a 256 x 256 tile (128 sums, 96 of fragments) would fetch them from memory in every step,
// behind the loads in flight.
template <typename P, int R, bool TR, bool DUAL>
struct LeanLoader {
    static constexpr int kThreads = P::kThreads;
    static constexpr int kChunks = R * 8 / kThreads;
    static constexpr int kEach = TR ? kThreads * 8 / R : kThreads / 8;       // rows of the tile (of k: TR) that one load covers
    static constexpr int kGran = R / 16;
    int lane_row, lane_at;       // row within a load; byte offset of the chunk in it (TR: its column before the swizzle of `it`)
    int row0, ld, last;

    __device__ __forceinline__ void lanes(int tid)
    {
        if (TR) {
            lane_row = tid / (R / 8);
            const int pos = tid % (R / 8), f = ((lane_row & 3) | (lane_row >> 3 & 3) << 2) & (kGran - 1);
            lane_at = ((pos >> 1 ^ f) << 4) + ((pos & 1) << 3);
        } else {
            const int r = tid >> 3;
            static_assert(!DUAL || kEach % (P::BN / P::WN / 2) == 0, "a load's rows are of the gate or of the up matrix, or of both alike");
            lane_row = DUAL ? Dual<P::BN / P::WN>::row(r) : r;
            lane_at = ((tid & 7) ^ (r & 7)) << 4;
        }
    }
    __device__ __forceinline__ void start(int, int first, int n, int64_t ld_)
    {
        ld = (int)ld_;
        row0 = first;
        last = n - first;
    }
    __device__ __forceinline__ int64_t pitch() const { return TR ? (int64_t)ld * (2 * kBK) : 2 * kBK; }
    __device__ __forceinline__ const char* base(const void* p, int64_t from) const
    {
        return base_of(p, from, ld);
    }
    __device__ __forceinline__ const char* base_of(const void* p, int64_t from, int64_t ld_) const
    {
        const char* q = (const char*)p + 2 * from;
        return TR ? q + 2 * (int64_t)row0 : q + 2 * (int64_t)row0 * ld_;
    }
    template <bool TAIL>
    __device__ __forceinline__ void fetch(const char* p0, const char* p1, char* lds, int tid, int left) const
    {
        const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
        int row = lane_row, at = lane_at;
        asm volatile("" : "+v"(row), "+v"(at));       // not kept over the steps
#pragma unroll
        for (int it = 0; it < kChunks; ++it) {
            const char* p = p0;
            if (DUAL) p = Dual<P::BN / P::WN>::up(it * kEach + wave * 8) ? p1 : p0;
            uint32_t off;
            int k;
            if (TR) {
                k = row + it * kEach;
                // f of row + it kEach differs from that of row in the bits that kEach moves
                static_assert(kEach % 4 == 0 && (kEach % 32 == 0 || kEach == 16 || kEach == 8), "f over the loads");
                const int col = at ^ (kEach % 32 == 0 ? 0 : ((it * kEach >> 3 & 3) << 2 & (kGran - 1)) << 4);
                off = (uint32_t)k * (uint32_t)(ld * 2) + (uint32_t)(col < last ? col : 0) * 2;
            } else {
                k = at >> 1;
                const int r = DUAL ? Dual<P::BN / P::WN>::row(it * kEach) : it * kEach;
                off = (uint32_t)min(row + r, last - 1) * (uint32_t)(ld * 2) + (uint32_t)at;
            }
            const char* src = p + off;
            if (TAIL && k >= left) src = (const char*)&g_zero_chunk;
            load_to_lds(src, lds + (it * kThreads + wave * 64) * 16);
        }
    }
};

// Operands whose rows start on any value: loads to registers, which are unaligned, and from
// there to the LDS once the step before is multiplied.  Lays the same chunks in the same
// places.  A chunk that a row's end cuts is read whole where another row follows in the matrix
// (a row further on along k it is masked; columns past the last make columns of C that are not
// written), and value by value in the matrix's last row, or in every row where rows are
// shorter than a chunk: there the next one may not hold what is left of it.  The up matrix has a
// row stride of its own.
template <typename P, int R, bool TR, bool DUAL>
struct StagedLoader : LeanLoader<P, R, TR, DUAL> {
    typedef LeanLoader<P, R, TR, DUAL> Base;
    using Base::kChunks;
    using Base::kEach;
    u32x4 v[kChunks];

    static __device__ __forceinline__ u32x4 whole(const char* p)
    {
        u32x4 w;
        __builtin_memcpy(&w, p, 16);
        return w;
    }
    // n of eight values, zeros behind them
    static __device__ __forceinline__ u32x4 some(const char* p, int n)
    {
        const uint16_t* q = (const uint16_t*)p;
        u32x4 w = {0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) w[i >> 1] |= (uint32_t)q[i] << (16 * (i & 1));
        return w;
    }
    static __device__ __forceinline__ u32x4 masked(u32x4 w, int n)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] &= n >= 2 * i + 2 ? 0xffffffffu : n == 2 * i + 1 ? 0xffffu : 0u;
        return w;
    }
    __device__ __forceinline__ void load(const char* p0, const char* p1, int ld0, int ld1, int tid, int left)
    {
        const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
        int row = Base::lane_row, at = Base::lane_at;
        asm volatile("" : "+v"(row), "+v"(at));       // not kept over the steps
#pragma unroll
        for (int it = 0; it < kChunks; ++it) {
            const bool up = DUAL && Dual<P::BN / P::WN>::up(it * kEach + wave * 8);
            const char* p = up ? p1 : p0;
            const uint32_t pitch = (uint32_t)(up ? ld1 : ld0) * 2;
            const bool slim = pitch < 16;
            if (TR) {
                const int k = row + it * kEach;
                int col = at ^ (kEach % 32 == 0 ? 0 : ((it * kEach >> 3 & 3) << 2 & (Base::kGran - 1)) << 4);
                col = col < Base::last ? col : 0;
                const char* src = p + (uint32_t)k * pitch + (uint32_t)col * 2;
                if (left > kBK && !slim) v[it] = whole(src);
                else if (k >= left) v[it] = u32x4{0, 0, 0, 0};
                else if ((slim || k == left - 1) && col + 8 > Base::last) v[it] = some(src, Base::last - col);
                else v[it] = whole(src);
            } else {
                const int r = min(row + (DUAL ? Dual<P::BN / P::WN>::row(it * kEach) : it * kEach), Base::last - 1);
                const int n = left - (at >> 1);
                const char* src = p + (uint32_t)r * pitch + (uint32_t)at;
                if (left >= kBK) v[it] = whole(src);
                else if (n <= 0) v[it] = u32x4{0, 0, 0, 0};
                else if (n < 8 && (slim || r == Base::last - 1)) v[it] = some(src, n);
                else v[it] = masked(whole(src), n);
            }
        }
    }
    __device__ __forceinline__ void store(char* lds, int tid) const
    {
#pragma unroll
        for (int it = 0; it < kChunks; ++it) *(u32x4*)(lds + (it * P::kThreads + tid) * 16) = v[it];
    }
};

// LEAN: 0, 1, or 2 for operands of any alignment.
template <typename P, int R, bool TR, bool DUAL, int LEAN>
struct LoaderOf {
    typedef GroupLoader<P, R, TR, DUAL> Type;
};

template <typename P, int R, bool TR, bool DUAL>
struct LoaderOf<P, R, TR, DUAL, 1> {
    typedef LeanLoader<P, R, TR, DUAL> Type;
};

template <typename P, int R, bool TR, bool DUAL>
struct LoaderOf<P, R, TR, DUAL, 2> {
    typedef StagedLoader<P, R, TR, DUAL> Type;
};

// Four columns of two fragments j and j + 1 in lanes of rows of 16 (columns 4 r + 0..3 of
// row r) become eight of one: rows 0 and 2 hold columns 0..7 and 8..15 of fragment j, rows
// 1 and 3 those of fragment j + 1.
__device__ __forceinline__ void eight_columns(const f32x4& a, const f32x4& b, float (&v)[8])
{
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const u32x2 w = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane16_swap(__float_as_uint(a[q]),
                                                                                   __float_as_uint(b[q]), false, false));
        v[q] = __uint_as_float(w[0]);
        v[4 + q] = __uint_as_float(w[1]);
    }
}

// tiles: of a part, of groups of rows the most that there can be.
template <typename P>
__global__ __launch_bounds__(P::kThreads, P::kWavesEach) void groups_kernel(const GroupArgs A, const int tiles)
{
    typedef typename P::T T;
    constexpr bool kRows = P::GROUP == kRowGroups, kSteps = P::GROUP == kStepGroups;
    __shared__ __attribute__((aligned(16))) char sa0[P::BM * 128];
    __shared__ __attribute__((aligned(16))) char sa1[P::BM * 128];
    __shared__ __attribute__((aligned(16))) char sa2[P::kStages > 2 ? P::BM * 128 : 16];
    __shared__ __attribute__((aligned(16))) char sb0[P::BN * 128];
    __shared__ __attribute__((aligned(16))) char sb1[P::BN * 128];
    __shared__ __attribute__((aligned(16))) char sb2[P::kStages > 2 ? P::BN * 128 : 16];
    constexpr int kRowsEach = P::BM * P::kRowBytes;
    __shared__ __attribute__((aligned(16))) char row_data[P::kRowBytes ? 2 * kRowsEach : 16];
    __shared__ f32x2 stats[P::EPI == kLossStats ? P::BM * P::WN : 1];
    extern __shared__ int table_data[];
    const GroupTable table(table_data, A.groups);
    auto bufa = [&](int i) { return i == 0 ? sa0 : i == 1 ? sa1 : sa2; };
    auto bufb = [&](int i) { return i == 0 ? sb0 : i == 1 ? sb1 : sb2; };

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / P::WN, wn = wave % P::WN;
    int part_tiles = tiles;
    if constexpr (kRows) {
        __shared__ int rows;
        if (wave == 0) {
            const int total = fill_table<P::BM>(A, &table, lane, quotient(tiles, A.tiles_n));
            if (lane == 0) rows = total;
        }
        __syncthreads();
        part_tiles = __builtin_amdgcn_readfirstlane(rows) * A.tiles_n;
    }
    if constexpr (kSteps) {
        for (int g = tid; g < A.groups; g += P::kThreads) {
            // of no steps there need be no offsets
            const int lo = A.K > 0 ? group_end(A.offsets, g, A.K) : 0;
            table.first[g] = lo;
            table.end[g] = A.K > 0 ? max(lo, group_end(A.offsets, g + 1, A.K)) : 0;
        }
        __syncthreads();
    }

    const Tail tail(part_tiles, (int)gridDim.x, P::kTail ? A.tail : 0);
    const int n_tiles = (P::kSplit ? part_tiles * A.splits : part_tiles) + tail.tiles * (tail.parts - 1);
    const int xcd = blockIdx.x & 7;
    int q = blockIdx.x >> 3;
    // The tile that comes next; false if there is none.
    auto next_work = [&](Work* w) {
        int tile = tile_of_xcd<P::kRun>(xcd, q, n_tiles);
        q += gridDim.x >> 3;
        if (tile < 0) return false;
        w->part = 0;
        w->parts = 1;
        w->K = A.K;
        if (P::kSplit && A.splits > 1) {
            w->parts = A.splits;
            w->part = quotient(tile, part_tiles);
            tile -= w->part * part_tiles;
        } else if (P::kTail && tile >= part_tiles - tail.tiles && tail.parts > 1) {
            const int in = tile - (part_tiles - tail.tiles);
            w->parts = tail.parts;
            w->part = quotient(in, tail.tiles);
            w->slot = in - w->part * tail.tiles;
            tile = part_tiles - tail.tiles + w->slot;
        }
        locate<P>(A, table, lane, tile, w);
        return true;
    };

    constexpr int kLoader = P::kDirect ? P::kLean : 2;
    typename LoaderOf<P, P::BM, P::ATR, false, kLoader>::Type la;
    typename LoaderOf<P, P::BN, P::BTR, P::DUAL, kLoader>::Type lb;
    la.lanes(tid);
    lb.lanes(tid);
    Frags<P, P::BM, P::ATR> fa;
    Frags<P, P::BN, P::BTR> fb;
    fa.init(lane, wm * (P::BM / P::WM));
    fb.init(lane, wn * (P::BN / P::WN));
    const char *a0, *a1, *b0, *b1;        // of the segments, or b1 of the up matrix
    auto begin = [&](Work* w) {
        int k_from = 0;
        if constexpr (kSteps) {
            const int g = w->z >> A.pairs;
            k_from = __builtin_amdgcn_readfirstlane(table.first[g]);
            w->K = __builtin_amdgcn_readfirstlane(table.end[g]) - k_from;
        }
        w->sps = (w->K + kBK - 1) / kBK;
        w->steps = w->sps * P::kSegs;
        w->s0 = 0;
        if ((P::kSplit || P::kTail) && w->parts > 1) {
            const int per = quotient(w->steps + w->parts - 1, w->parts);
            w->s0 = min(w->part * per, w->steps);
            w->steps = min(per, w->steps - w->s0);
        }
        la.start(tid, w->m0, w->m_end, A.lda);
        lb.start(tid, w->n0, A.N, A.ldb);
        const int sel = !kRows && A.pairs ? w->z & 1 : 0;
        a0 = la.base(A.a[sel], kRows ? 0 : k_from * A.lda);
        b0 = lb.base(A.b[sel], kRows ? w->z * A.sb : k_from * A.ldb);
        a1 = P::kSegs == 2 ? la.base(A.a[1], 0) : a0;
        if constexpr (P::kSegs == 1 && !P::DUAL) b1 = b0;
        else if constexpr (P::kDirect) b1 = lb.base(A.b[1], w->z * A.sb1);      // of the same row stride
        else b1 = lb.base_of(A.b[1], w->z * A.sb1, A.ldb1);
    };
    auto fetch_rows = [&](const Work& w, char* to) {
        if (P::kRowBytes == 0 || wave >= P::BM / 64) return;
        const int m = min(w.m0 + wave * 64 + lane, A.M - 1);
        if (P::kRowBytes == 16) {
            load_to_lds((const char*)(A.rows + m), to + wave * 1024);
        } else {
            // the lower half of a wide target: one past 32 bits is no entry and picks nothing
            const char* p = (const char*)A.target + ((int64_t)m << (A.target_wide ? 3 : 2));
            __builtin_amdgcn_global_load_lds((GlobalVoid*)p, (LdsVoid*)(to + wave * 256), 4, 0, 0);
        }
    };
    auto fetch = [&](const Work& w, int step, char* sa, char* sb) {
        int at = w.s0 + step;
        const char *pa = a0, *pb = b0;
        bool second = false;
        if (P::kSegs == 2 && at >= w.sps) {
            at -= w.sps;
            pa = a1;
            pb = b1;
            second = true;
        }
        const int left = w.K - at * kBK;
        pa += at * la.pitch();
        if constexpr (!P::kDirect) {
            const int ld = (int)(second ? A.ldb1 : A.ldb);
            pb += P::BTR ? at * (int64_t)ld * (2 * kBK) : at * (2 * kBK);
            la.load(pa, pa, (int)A.lda, (int)A.lda, tid, left);
            lb.load(pb, P::DUAL ? b1 + at * (2 * kBK) : pb, ld, (int)A.ldb1, tid, left);
        } else {
            pb += at * lb.pitch();
            const char* pu = P::DUAL ? b1 + at * lb.pitch() : pb;
            if (left < kBK) {
                la.template fetch<true>(pa, pa, sa, tid, left);
                lb.template fetch<true>(pb, pu, sb, tid, left);
            } else {
                la.template fetch<false>(pa, pa, sa, tid, left);
                lb.template fetch<false>(pb, pu, sb, tid, left);
            }
        }
    };

    // what was loaded to registers goes to the LDS
    auto commit = [&](char* sa, char* sb) {
        if constexpr (!P::kDirect) {
            la.store(sa, tid);
            lb.store(sb, tid);
        }
    };

    f32x4 acc[P::FM][P::FN];
    typename T::V8 fa0[P::FM], fb0[P::FN], fa1[P::FM], fb1[P::FN];    // fragments of the step's halves
    auto read = [&](const char* sa, const char* sb, int kk, typename T::V8* a, typename T::V8* b) {
#pragma unroll
        for (int j = 0; j < P::FN; ++j) b[j] = fb.get(sb, j, kk);
#pragma unroll
        for (int i = 0; i < P::FM; ++i) a[i] = fa.get(sa, i, kk);
    };
    auto multiply = [&](const typename T::V8* a, const typename T::V8* b) {
#pragma unroll
        for (int i = 0; i < P::FM; ++i)
#pragma unroll
            for (int j = 0; j < P::FN; ++j) acc[i][j] = T::mfma(b[j], a[i], acc[i][j]);
    };
    auto weave = [&]() {
        constexpr int reads = P::FM * (P::ATR ? 2 : 1) + P::FN * (P::BTR ? 2 : 1), products = P::FM * P::FN;
        constexpr int each = products / reads > 0 ? products / reads : 1;
#pragma unroll
        for (int i = 0; i < reads; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);          // an LDS read
            __builtin_amdgcn_sched_group_barrier(0x008, each, 0);       // products
        }
    };
    // Waits for a step's loads.  After them the loads of the step behind may be in flight (three
    // buffers) and, in the first steps of a tile, the stores of the tile before, which were
    // issued later: operations complete in order, so that many may be left.  kStores is the
    // least that a whole tile's epilogue issues; after another one everything is awaited.
    constexpr int kAhead = P::kStages - 1, kLoads = la.kChunks + lb.kChunks;
    constexpr int kStores = P::FM * P::FN / (P::DUAL ? 4 : 2);
    static_assert(P::FM % 2 == 0 && kLoads + kStores < 64, "rows in pairs, operations counted in six bits");
    bool stored = false, idle = false;
    auto arrive = [&](int step, int steps) {
        asm volatile("" ::: "memory");
        if (!P::kDirect && !(P::kRowBytes && step == 0)) {
            __builtin_amdgcn_s_waitcnt(15 | 3 << 14 | 7 << 4);    // LDS writes
        } else if (kAhead == 2 && step + 1 < steps) {
            if (stored && step < 2) wait_loads<kLoads + kStores>();
            else wait_loads<kLoads>();
        } else {
            if (stored && step < kAhead) wait_loads<kStores>();
            else wait_loads<0>();
        }
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    // One step, from buffer u: see tile_product in arena_gemm.h.
    auto turn = [&](const Work& w, int step, int u, bool first) {
        arrive(step, w.steps);
        constexpr int kNext = P::kStages;
        if (step + kAhead < w.steps) fetch(w, step + kAhead, bufa((u + kAhead) % kNext), bufb((u + kAhead) % kNext));
        if (!(kRows && idle)) {
            __builtin_amdgcn_sched_barrier(0);
            read(bufa(u), bufb(u), 0, fa0, fb0);
            if (!first) multiply(fa1, fb1);
            weave();
            __builtin_amdgcn_sched_barrier(0);
            read(bufa(u), bufb(u), 1, fa1, fb1);
            multiply(fa0, fb0);
            weave();
            __builtin_amdgcn_sched_barrier(0);
        }
        if (!P::kDirect && step + 1 < w.steps) commit(bufa(u ^ 1), bufb(u ^ 1));
    };

    Work w;
    if (!next_work(&w)) return;
    begin(&w);
    fetch_rows(w, row_data);
    auto fetch_first = [&](const Work& w) {
        if (w.steps > 0) fetch(w, 0, bufa(0), bufb(0));
        if (kAhead == 2 && w.steps > 1) fetch(w, 1, bufa(1), bufb(1));
    };
    fetch_first(w);
    if (w.steps > 0) commit(bufa(0), bufb(0));
    bool odd = false;             // which rows are the tile's
    for (;;) {
#pragma unroll
        for (int i = 0; i < P::FM; ++i)
#pragma unroll
            for (int j = 0; j < P::FN; ++j) acc[i][j] = f32x4{0, 0, 0, 0};
        const int steps = w.steps;
        idle = kRows && w.m0 + wm * (P::BM / P::WM) >= w.m_end;
        if (steps > 0) {
            turn(w, 0, 0, true);
            for (int s = 1; s < steps; s += P::kStages)
#pragma unroll
                for (int u = 0; u < P::kStages; ++u)
                    if (s + u < steps) turn(w, s + u, (u + 1) % P::kStages, false);
        }
        // every wave holds its last fragments: the buffers are free for the next tile
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(15 | 3 << 14 | 7 << 4);         // LDS reads
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        if (steps > 0 && !idle) multiply(fa1, fb1);
        const Work done = w;
        const bool more = next_work(&w);
        if (more) {
            begin(&w);
            fetch_rows(w, row_data + (odd ? 0 : kRowsEach));
            fetch_first(w);
        }
        __builtin_amdgcn_sched_barrier(0);

        // A lane holds row lane & 15 and columns 4 (lane >> 4) + 0..3 of each fragment.
        constexpr int kAcross = P::DUAL ? P::FN / 4 : P::FN / 2;
        int l = lane;
        asm volatile("" : "+v"(l));       // places are worked out here, not kept over the steps
        const int mw = done.m0 + wm * (P::BM / P::WM) + (l & 15);
        const int nw = done.n0 + wn * (P::DUAL ? P::BN / P::WN / 2 : P::BN / P::WN) + 16 * (l >> 4 & 1) + 8 * (l >> 5);
        const int n_end = P::kUpToN ? A.N : A.pad;
        const char* const rows = row_data + (odd ? kRowsEach : 0);
        odd = !odd;
        auto row_out = [&](int m, const f32x4 (&row)[P::FN]) {
            constexpr int kSide = P::EPI == kLossGrad || P::EPI == kLossStats ? kPlain : P::EPI;
            Side<T, kSide> side[kAcross];
            LossRow record;
            if constexpr (P::EPI == kLossGrad) record = ((const LossRow*)rows)[m - done.m0];
            if ((P::EPI == kGatedBwd || (P::EPI == kWide && A.beta != 0.0f)) && !(P::kSplit && A.splits > 1))
#pragma unroll
                for (int j = 0; j < kAcross; ++j)
                    if (m < done.m_end && nw + j * 32 < n_end) side[j].load(A, done.z, m, nw + j * 32);
#pragma unroll
            for (int j = 0; j < kAcross; ++j) {
                const int n = nw + j * 32;
                float v[8], u[8];
                eight_columns(row[2 * j], row[2 * j + 1], v);
                if constexpr (P::DUAL) eight_columns(row[2 * (j + kAcross)], row[2 * (j + kAcross) + 1], u);
                if (m >= done.m_end || n >= n_end) continue;
                if (P::kTail && A.tail > 1 && done.parts > 1) {
                    put(A.part + ((int64_t)done.part * tail.tiles + done.slot) * (P::BM * P::BN) +
                            (m - done.m0) * P::kCols + n - done.n0, v, 8);
                } else if (kRows && P::kSplit && A.splits > 1) {
                    put(A.part + ((int64_t)done.part * A.M + m) * ((A.N + 7) & ~7) + n, v, 8);
                } else if (!kRows && P::kSplit && A.splits > 1) {
                    const int64_t t = ((int64_t)done.part * A.batch + done.z) * (A.tiles_m * A.tiles_n) +
                                      done.m0 / P::BM * A.tiles_n + done.n0 / P::kCols;
                    put(A.part + t * (P::BM * P::BN) + (m - done.m0) * P::kCols + n - done.n0, v, 8);
                } else if constexpr (P::EPI == kGatedFwd) {
                    gated_fwd_out<T, kGeluShort>(A, m, n, v, u);
                } else if constexpr (P::EPI == kGatedBwd) {
                    gated_bwd_out<T, kGeluShort>(A, m, n, v, side[j]);
                } else if constexpr (P::EPI == kWide) {
                    plain_out<T>(A, done.z, m, n, v, side[j]);
                } else if constexpr (P::EPI == kLossGrad) {
                    loss_grad_out<T, P::BM == 64>(A, m, n, v, record);
                } else {
                    put((typename T::E*)A.c[0] + (int64_t)m * A.ldc + n, v, A.N - n);
                }
            }
        };
        if constexpr (P::EPI == kLossStats) {
            // the block's WN waves share a row
            const int n = done.n0 + wn * (P::BN / P::WN) + 4 * (l >> 4);
#pragma unroll
            for (int i = 0; i < P::FM; ++i) {
                const int r = wm * (P::BM / P::WM) + i * 16 + (l & 15);
                const f32x2 e = row_stats<P>(A, acc[i], done.m0 + r, n, ((const int32_t*)rows)[r] - A.first_col);
                if (l < 16) stats[r * P::WN + wn] = e;
            }
            asm volatile("" ::: "memory");
            __builtin_amdgcn_s_waitcnt(15 | 3 << 14 | 7 << 4);         // LDS writes
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            for (int r = tid; r < P::BM; r += P::kThreads) {
                if (done.m0 + r >= A.M) continue;
                float most = -INFINITY, sum = 0.0f;
#pragma unroll
                for (int x = 0; x < P::WN; ++x) most = fmaxf(most, stats[r * P::WN + x][0]);
                const float by = most == -INFINITY ? 0.0f : most;
#pragma unroll
                for (int x = 0; x < P::WN; ++x) {
                    const f32x2 e = stats[r * P::WN + x];
                    sum += e[0] == -INFINITY ? e[1] : e[1] * __expf(e[0] - by);
                }
                ((f32x2*)A.stats)[(int64_t)(done.n0 / P::kCols) * A.M + done.m0 + r] = f32x2{most, sum};
            }
        } else if constexpr (P::EPI == kGatedFwd || P::EPI == kGatedBwd) {
            // Unrolled over all rows the activations would not fit the instruction cache:
            // two rows at a time, the others move up.
#pragma unroll 1
            for (int i = 0; i < P::FM; i += 2) {
                row_out(mw + i * 16, acc[0]);
                row_out(mw + i * 16 + 16, acc[1]);
#pragma unroll
                for (int k = 0; k + 2 < P::FM; ++k)
#pragma unroll
                    for (int j = 0; j < P::FN; ++j) acc[k][j] = acc[k + 2][j];
            }
        } else {
#pragma unroll
            for (int i = 0; i < P::FM; ++i) row_out(mw + i * 16, acc[i]);
        }
        if (!more) return;
        if (w.steps > 0) commit(bufa(0), bufb(0));
        stored = P::EPI != kLossStats && done.m0 + P::BM <= done.m_end && done.n0 + P::kCols <= A.N;
    }
}

// Joins the parts of a split product: a thread takes eight columns of
// a row of C, all parts in their order.
template <typename P>
__global__ __launch_bounds__(256) void groups_join_kernel(const GroupArgs A)
{
    typedef typename P::T T;
    const int chunks = (A.N + 7) / 8;
    const int64_t n = (int64_t)A.batch * A.M * chunks;
    const int64_t each = (int64_t)A.batch * A.tiles_m * A.tiles_n * (P::BM * P::BN);
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
        const int64_t row = i / chunks;
        const int c = (int)(i - row * chunks) * 8, z = (int)(row / A.M), m = (int)(row - (int64_t)z * A.M);
        const float* p = A.part + (((int64_t)z * A.tiles_m + m / P::BM) * A.tiles_n + c / P::kCols) * (P::BM * P::BN) +
                         (m % P::BM) * P::kCols + c % P::kCols;
        float v[8] = {};
        for (int s = 0; s < A.splits; ++s) {
            float w[8];
            get(p + s * each, w, 8);
#pragma unroll
            for (int r = 0; r < 8; ++r) v[r] += w[r];
        }
        Side<T, P::EPI> side;
        side.load(A, z, m, c);
        plain_out<T>(A, z, m, c, v, side);
    }
}

// The same of groups of rows, whose parts are matrices of all rows: a wave takes 512 columns of
// a row, if it is a group's.  Bound by its launch: 5 us for 50 rows of 1024 columns in 14 parts.
template <typename T, int EPI>
__global__ __launch_bounds__(256) void rows_join_kernel(const GroupArgs A)
{
    const int lane = threadIdx.x & 63, stretches = (A.N + 511) / 512, ld = (A.N + 7) & ~7;
    const int64_t i = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int m = (int)(i / stretches), n = (int)(i % stretches) * 512 + lane * 8;
    if (m >= A.M) return;
    bool some = false;
    for (int g = lane; g < A.groups; g += 64)
        some |= m >= group_end(A.offsets, g, A.M) && m < group_end(A.offsets, g + 1, A.M);
    if (!__any(some) || n >= ld) return;
    float v[8] = {};
    for (int s = 0; s < A.splits; ++s) {
        float w[8];
        get(A.part + ((int64_t)s * A.M + m) * ld + n, w, 8);
#pragma unroll
        for (int r = 0; r < 8; ++r) v[r] += w[r];
    }
    if constexpr (EPI == kGatedBwd) {
        Side<T, kGatedBwd> side;
        side.load(A, 0, m, n);
        gated_bwd_out<T, kGeluShort>(A, m, n, v, side);
    } else {
        put((typename T::E*)A.c[0] + (int64_t)m * A.ldc + n, v, A.N - n);
    }
}

// Joins the parts of the last round's tiles: eight blocks a tile, the same number of groups' tiles
// and of parts as the product found (`tiles` and `blocks` of its launch).  9 to 15 us.
template <typename P>
__global__ __launch_bounds__(256) void tail_join_kernel(const GroupArgs A, const int tiles, const int blocks)
{
    extern __shared__ int table_data[];
    const GroupTable table(table_data, A.groups);
    const int lane = threadIdx.x & 63;
    __shared__ int rows;
    if (threadIdx.x < 64) {
        const int total = fill_table<P::BM>(A, &table, lane, quotient(tiles, A.tiles_n));
        if (lane == 0) rows = total;
    }
    __syncthreads();
    const int all = __builtin_amdgcn_readfirstlane(rows) * A.tiles_n;
    const Tail tail(all, blocks, A.tail);
    const int slot = blockIdx.x >> 3;
    if (slot >= tail.tiles) return;
    Work w;
    locate<P>(A, table, lane, all - tail.tiles + slot, &w);
    constexpr int kChunks = P::BM * P::kCols / 8;
    for (int i = (blockIdx.x & 7) * 256 + threadIdx.x; i < kChunks; i += 2048) {
        const int r = i / (P::kCols / 8), c = i % (P::kCols / 8) * 8, m = w.m0 + r, n = w.n0 + c;
        if (m >= w.m_end || n >= A.N) continue;
        float v[8] = {};
        for (int s = 0; s < tail.parts; ++s) {
            float x[8];
            get(A.part + ((int64_t)s * tail.tiles + slot) * (P::BM * P::BN) + r * P::kCols + c, x, 8);
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] += x[k];
        }
        put((typename P::T::E*)A.c[0] + (int64_t)m * A.ldc + n, v, A.N - n);
    }
}

template <typename P>
hipError_t launch_group_tile(GroupArgs A, hipStream_t s)
{
    A.tiles_m = (A.M + P::BM - 1) / P::BM;
    A.tiles_n = (A.N + P::kCols - 1) / P::kCols;
    const int64_t one = P::GROUP == kRowGroups ? group_tiles(A.M, A.groups, P::BM) * A.tiles_n
                                               : (int64_t)A.tiles_m * A.tiles_n * A.batch, tiles = one * A.splits;
    if (tiles == 0) return hipSuccess;
    if (tiles > 0x7fffffff || (A.splits > 1 && !P::kSplit)) return hipErrorInvalidValue;
    // as many blocks as the compute units hold: with many groups the table leaves room for one
    const int table = GroupTable::bytes(P::GROUP, A.groups);
    constexpr int kBuffers = P::kStages * (P::BM + P::BN) * 128 + (P::kRowBytes ? 2 * P::BM * P::kRowBytes : 16) +
                             (P::EPI == kLossStats ? 8 * P::BM * P::WN : 8) + 64;
    const int64_t blocks = P::kBlocks > 1 && kBuffers + table > 163840 / 2 ? 1 : P::kBlocks;
    const int64_t grid = (std::min(tiles, 256 * blocks) + 7) / 8 * 8;
    if (!P::kTail || A.splits > 1 || one < grid) A.tail = 0;
    groups_kernel<P><<<(unsigned)grid, P::kThreads, table, s>>>(A, (int)one);
    hipError_t e = hipGetLastError();
    if constexpr (P::kTail)
        if (e == hipSuccess && A.tail > 1) {
            // not more than half of the blocks' tiles are shared out
            tail_join_kernel<P><<<(unsigned)(grid / 2 * 8), 256, table, s>>>(A, (int)one, (int)grid);
            return hipGetLastError();
        }
    if (e != hipSuccess || A.splits <= 1) return e;
    if constexpr (P::kSplit && P::GROUP == kRowGroups) {
        const int64_t waves = (int64_t)A.M * ((A.N + 511) / 512);
        rows_join_kernel<typename P::T, P::EPI><<<(unsigned)((waves + 3) / 4), 256, 0, s>>>(A);
        e = hipGetLastError();
    } else if constexpr (P::EPI == kWide) {
        const int64_t blocks = ((int64_t)A.batch * A.M * ((A.N + 7) / 8) + 255) / 256;
        groups_join_kernel<P><<<(unsigned)std::min<int64_t>(blocks, 8192), 256, 0, s>>>(A);
        e = hipGetLastError();
    }
    return e;
}

// Few rows: as skinny_kernel of arena_gemm.h, for 16 columns of C and a group that has rows
// (offsets null: one group of all), 16 of its rows at a time; C plain, gated or the
// statistics of a loss's logits.  Bound by the read of the weights: two experts of 4096 x
// 10944 in bfloat16 read 359 MB of gate and up weights in 68 us (5.3 TB/s).
template <typename T, int EPI, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void skinny_groups_kernel(const GroupArgs A)
{
    typedef typename T::E E;
    typedef typename T::V8 V8;
    constexpr bool DUAL = EPI == kGatedFwd;
    constexpr int NB = DUAL ? 2 : 1;
    __shared__ f32x4 part[WAVES][NB][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // the blockIdx.y-th group with rows
    int group = -1, lo = 0, hi = 0, left = blockIdx.y;
    if (A.offsets) {
        for (int g0 = 0; g0 < A.groups; g0 += 64) {
            int first, end;
            (void)tile_rows<1>(A, g0 + lane, &first, &end);
            uint64_t some = __ballot(end > first);
            const int n = __popcll(some);
            if (left >= n) {
                left -= n;
                continue;
            }
            for (; left > 0; --left) some &= some - 1;
            const int l = __ffsll((unsigned long long)some) - 1;
            group = g0 + l;
            lo = __builtin_amdgcn_readlane(first, l);
            hi = __builtin_amdgcn_readlane(end, l);
            break;
        }
        if (group < 0) return;
    } else {
        group = 0;
        hi = A.M;
    }
    const int n0 = blockIdx.x * 16, kc = (lane >> 4) * 8;
    const int row = min(n0 + (lane & 15), A.N - 1);
    const E* w[NB];
    w[0] = (const E*)A.b[0] + group * A.sb + (int64_t)row * A.ldb + kc;
    if (DUAL) w[NB - 1] = (const E*)A.b[1] + group * A.sb1 + (int64_t)row * A.ldb1 + kc;
    constexpr int U = 8 / NB;     // steps of 32 in flight
    const int steps = (A.K + 31) / 32, per = (steps + WAVES - 1) / WAVES;
    const int begin = wave * per * 32, end = min(A.K, begin + per * 32);
    for (int m0 = lo; m0 < hi; m0 += 16) {
        const E* x = (const E*)A.a[0] + (int64_t)min(m0 + (lane & 15), hi - 1) * A.lda + kc;
        f32x4 acc[NB];
#pragma unroll
        for (int b = 0; b < NB; ++b) acc[b] = f32x4{0, 0, 0, 0};
        int k = begin;
        for (; k + 32 * U <= end; k += 32 * U) {
            V8 wv[NB][U], xv[U];
#pragma unroll
            for (int i = 0; i < U; ++i) {
#pragma unroll
                for (int b = 0; b < NB; ++b) __builtin_memcpy(&wv[b][i], w[b] + k + 32 * i, 16);
                __builtin_memcpy(&xv[i], x + k + 32 * i, 16);
            }
#pragma unroll
            for (int i = 0; i < U; ++i)
#pragma unroll
                for (int b = 0; b < NB; ++b) acc[b] = T::mfma(wv[b][i], xv[i], acc[b]);
        }
        for (; k < end; k += 32) {
            const int rest = A.K - k - kc;
#pragma unroll
            for (int b = 0; b < NB; ++b) acc[b] = T::mfma(load_k<T>(w[b] + k, rest), load_k<T>(x + k, rest), acc[b]);
        }
#pragma unroll
        for (int b = 0; b < NB; ++b) part[wave][b][lane] = acc[b];
        __syncthreads();
        if (wave == 0) {
            const int m = m0 + (lane & 15), n = n0 + 4 * (lane >> 4);
            f32x4 v = part[0][0][lane], u = part[0][NB - 1][lane];
#pragma unroll
            for (int q = 1; q < WAVES; ++q) {
                v += part[q][0][lane];
                if (DUAL) u += part[q][NB - 1][lane];
            }
            float fv[4], fu[4];
            *(f32x4*)fv = v;
            *(f32x4*)fu = u;
            if constexpr (EPI == kGatedFwd) {
                if (m < hi && n < A.pad) gated_fwd_out<T, kGeluShort>(A, m, n, fv, fu);
            } else if constexpr (EPI == kLossStats) {
                const int64_t at = min(m, hi - 1);
                const int target = ((const int32_t*)A.target)[at << A.target_wide];       // its lower half
                const f32x4 one[1] = {v};
                const f32x2 e = row_stats<OneFragment>(A, one, m, n, target);
                if (lane < 16 && m < hi) ((f32x2*)A.stats)[(int64_t)blockIdx.x * A.M + m] = e;
            } else {
                if (m < hi && n < A.N) put((E*)A.c[0] + (int64_t)m * A.ldc + n, fv, A.N - n);
            }
        }
        __syncthreads();
    }
}

template <typename T, int EPI>
hipError_t launch_skinny_groups_of(const GroupArgs& A, hipStream_t s)
{
    const dim3 grid((A.N + 15) / 16, !A.offsets ? 1 : A.groups < A.M ? A.groups : A.M);
    skinny_groups_kernel<T, EPI, 8><<<grid, 512, 0, s>>>(A);
    return hipGetLastError();
}

template <typename T>
hipError_t launch_skinny_groups_t(const GroupArgs& A, Product what, hipStream_t s)
{
    switch (what) {
    case kRowsRows: return launch_skinny_groups_of<T, kPlain>(A, s);
    case kGateUp: return launch_skinny_groups_of<T, kGatedFwd>(A, s);
    case kLossLogits: return launch_skinny_groups_of<T, kLossStats>(A, s);
    default: return hipErrorInvalidValue;
    }
}

template <typename T, bool ATR, bool BTR, int EPI, int GROUP>
hipError_t launch_groups_of(const GroupArgs& A, int kind, hipStream_t s)
{
    if (A.any) {
        if (kind == kGroup128)
            return launch_group_tile<GroupTile<T, 128, 128, 2, 2, ATR, BTR, EPI, GROUP, false>>(A, s);
        if (kind == kGroup64x128)
            return launch_group_tile<GroupTile<T, 64, 128, 2, 2, ATR, BTR, EPI, GROUP, false>>(A, s);
        return hipErrorInvalidValue;
    }
    switch (kind) {
    case kGroup256: return launch_group_tile<GroupTile<T, 256, 256, 2, 4, ATR, BTR, EPI, GROUP, true>>(A, s);
    case kGroup128: return launch_group_tile<GroupTile<T, 128, 128, 2, 2, ATR, BTR, EPI, GROUP, true>>(A, s);
    case kGroup64x128: return launch_group_tile<GroupTile<T, 64, 128, 2, 2, ATR, BTR, EPI, GROUP, true>>(A, s);
    }
    return hipErrorInvalidValue;
}

template <typename T>
hipError_t launch_groups_t(const GroupArgs& A, Product what, int kind, hipStream_t s)
{
    switch (what) {
    case kRowsRows: return launch_groups_of<T, false, false, kPlain, kRowGroups>(A, kind, s);
    case kRowsCols: return launch_groups_of<T, false, true, kPlain, kRowGroups>(A, kind, s);
    case kColsCols: return launch_groups_of<T, true, true, kWide, kStepGroups>(A, kind, s);
    case kGateUp: return launch_groups_of<T, false, false, kGatedFwd, kRowGroups>(A, kind, s);
    case kGateUpBack: return launch_groups_of<T, false, true, kGatedBwd, kRowGroups>(A, kind, s);
    default: return hipErrorInvalidValue;
    }
}

template <typename T>
hipError_t launch_loss_t(const GroupArgs& A, Product what, int kind, hipStream_t s)
{
    switch (what) {
    case kLossLogits: return launch_groups_of<T, false, false, kLossStats, kOneGroup>(A, kind, s);
    case kLossGradient: return launch_groups_of<T, false, false, kLossGrad, kOneGroup>(A, kind, s);
    case kRowsCols: return launch_groups_of<T, false, true, kWide, kOneGroup>(A, kind, s);
    case kColsCols: return launch_groups_of<T, true, true, kWide, kOneGroup>(A, kind, s);
    default: return hipErrorInvalidValue;
    }
}

}  // namespace mm
}  // namespace arena
