// The router of a layer of experts, and tokens to experts and back.
//
//   route      of each token's logits the k largest, their softmax (over them or over
//              all), and the gradient of that
//   sort       where each choice's row lies when the choices are sorted by expert
//   dispatch   xs[row[t, j]] = x[t]
//   combine    y[t] = sum_j w[t, j] ys[row[t, j]], and its gradients
//
// Nothing here multiplies matrices: the moves are bound by memory, the router of many
// tokens by the passes over its lanes, small calls by the launch.
#include <hip/hip_runtime.h>

#include "arena_layer_internal.h"

namespace arena {
namespace {

typedef __bf16 bf16;
typedef _Float16 f16;

// ---------------------------------------------------------------- router

// Sums and maxima over groups of W neighbouring lanes, in every lane: within 16 by
// cross-lane operands, past that through the permute network.
template <int CTRL>
__device__ __forceinline__ uint32_t cross(uint32_t v)
{
    return __builtin_amdgcn_update_dpp(v, v, CTRL, 0xf, 0xf, false);
}

template <int W>
__device__ __forceinline__ uint32_t group_max(uint32_t v)
{
    v = max(v, cross<0xb1>(v));                   // lanes ^ 1
    v = max(v, cross<0x4e>(v));                   // lanes ^ 2
    v = max(v, cross<0x141>(v));                  // mirrored in 8
    if (W > 8) v = max(v, cross<0x140>(v));       // mirrored in 16
    if (W > 16) v = max(v, (uint32_t)__shfl_xor((int)v, 16, 64));
    if (W > 32) v = max(v, (uint32_t)__shfl_xor((int)v, 32, 64));
    return v;
}

template <int W>
__device__ __forceinline__ float group_sum(float v)
{
    v += __uint_as_float(cross<0xb1>(__float_as_uint(v)));
    v += __uint_as_float(cross<0x4e>(__float_as_uint(v)));
    v += __uint_as_float(cross<0x141>(__float_as_uint(v)));
    if (W > 8) v += __uint_as_float(cross<0x140>(__float_as_uint(v)));
    if (W > 16) v += __shfl_xor(v, 16, 64);
    if (W > 32) v += __shfl_xor(v, 32, 64);
    return v;
}

// Numbers as unsigned ones of the same order: NaN above everything, both zeros alike,
// -inf (an expert that is never chosen) 0.
__device__ __forceinline__ uint32_t key_of(float f)
{
    if (f != f) return 0xffffffffu;
    if (f == -INFINITY) return 0;
    const uint32_t u = __float_as_uint(f + 0.0f);
    return u >> 31 ? ~u : u | 0x80000000u;
}

__device__ __forceinline__ float value_of(uint32_t key)
{
    return __uint_as_float(key >> 31 ? key & 0x7fffffffu : ~key);
}

template <typename E, int N>
__device__ __forceinline__ void fetch(const E* p, int left, float (&v)[N], float past)
{
    if (left >= N) {
        E w[N];
        __builtin_memcpy(w, p, sizeof(w));
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = (float)w[i];
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = i < left ? (float)p[i] : past;
    }
}

template <typename E, int N>
__device__ __forceinline__ void store(E* p, int left, const float (&v)[N])
{
    if (left >= N) {
        E w[N];
#pragma unroll
        for (int i = 0; i < N; ++i) w[i] = (E)v[i];
        __builtin_memcpy(p, w, sizeof(w));
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < left) p[i] = (E)v[i];
    }
}

// A group of W lanes takes a token, each lane NV neighbouring experts in registers.  The
// largest key of the group is found k times: the first lane that holds it has the lowest
// index, and takes it out of its own.  Bound by that chain of k passes over the lanes: 16384
// tokens of 128 experts in float32, k = 8, 7.5 us (its 8.4 MB alone would take 2), one token 1.8.
template <typename E, int W, int NV>
__global__ __launch_bounds__(256) void route_kernel(const RouteArgs A)
{
    const int lane = threadIdx.x & 63, in = lane & (W - 1), base = lane & ~(W - 1);
    const int64_t t = (int64_t)blockIdx.x * (256 / W) + threadIdx.x / W;
    const bool there = t < A.tokens;
    float l[NV];
    const int e0 = in * NV;
    fetch((const E*)A.logits + (there ? t : 0) * A.ld_logits + e0, A.experts - e0, l, -INFINITY);
    uint32_t key[NV];
#pragma unroll
    for (int v = 0; v < NV; ++v) key[v] = key_of(l[v]);
    float first = 0.0f, mine = -INFINITY;
    int index = -1;
    for (int j = 0; j < A.k; ++j) {
        uint32_t most = key[0];
#pragma unroll
        for (int v = 1; v < NV; ++v) most = max(most, key[v]);
        const uint32_t top = group_max<W>(most);
        const uint64_t holders = __ballot(most == top && top != 0) >> base & (~0ull >> (64 - W));
        const int owner = holders ? __ffsll((unsigned long long)holders) - 1 : 0;
        int at = -1;
        if (holders && in == owner) {
#pragma unroll
            for (int v = NV - 1; v >= 0; --v) at = key[v] == top ? v : at;
#pragma unroll
            for (int v = 0; v < NV; ++v) key[v] = v == at ? 0 : key[v];
            at += e0;
        }
        at = __shfl(at, base + owner, 64);
        const float value = top ? value_of(top) : -INFINITY;
        if (j == 0 && top) first = value;
        if (in == j) {
            mine = value;
            index = at;
        }
    }
    // weights of -inf are 0 without an exponential of -inf - inf
    const float chosen = index >= 0 ? expf(mine - first) : 0.0f;
    float part = chosen;
    if (!A.normalise) {
        part = 0.0f;
#pragma unroll
        for (int v = 0; v < NV; ++v) part += l[v] == -INFINITY ? 0.0f : expf(l[v] - first);
    }
    const float total = group_sum<W>(part);
    if (!there || in >= A.k) return;
    ((int32_t*)A.index)[t * A.k + in] = index;
    A.weight[t * A.k + in] = index >= 0 ? A.scale * (chosen / total) : 0.0f;
}

// With q the softmax without the scale:  over the chosen, of a chosen logit
// q (s dw - sum_i q_i s dw_i); over all, of every logit -p sum_i p_i s dw_i, and of a
// chosen one p s dw more.  Choices that name an expert twice add up.  At the same size 7.0 us.
template <typename E, int W, int NV>
__global__ __launch_bounds__(256) void route_back_kernel(const RouteArgs A)
{
    const int lane = threadIdx.x & 63, in = lane & (W - 1), base = lane & ~(W - 1);
    const int64_t t = (int64_t)blockIdx.x * (256 / W) + threadIdx.x / W;
    const bool there = t < A.tokens;
    const E* row = (const E*)A.logits + (there ? t : 0) * A.ld_logits;
    const int e0 = in * NV;
    int index = -1;
    float dw = 0.0f, taken = -INFINITY;
    if (there && in < A.k) {
        index = ((const int32_t*)A.index)[t * A.k + in];
        if (index < 0 || index >= A.experts) index = -1;
    }
    if (index >= 0) {
        dw = A.scale * A.dweight[t * A.ld_dweight + in];
        taken = (float)row[index];
    }
    float l[NV], d[NV];
    uint32_t most = key_of(taken);
    if (!A.normalise) {
        fetch(row + e0, A.experts - e0, l, -INFINITY);
#pragma unroll
        for (int v = 0; v < NV; ++v) most = max(most, key_of(l[v]));
    }
    most = group_max<W>(most);
    const float first = most ? value_of(most) : 0.0f;
    const float e = index >= 0 && taken != -INFINITY ? expf(taken - first) : 0.0f;
    float part = e;
    if (!A.normalise) {
        part = 0.0f;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            l[v] = l[v] == -INFINITY ? 0.0f : expf(l[v] - first);
            part += l[v];
        }
    }
    const float total = group_sum<W>(part), inverse = total == 0.0f ? 0.0f : 1.0f / total;
    const float q = e * inverse, mean = group_sum<W>(index >= 0 ? q * dw : 0.0f);
    const float mine = index < 0 ? 0.0f : A.normalise ? q * (dw - mean) : q * dw;
#pragma unroll
    for (int v = 0; v < NV; ++v) d[v] = A.normalise ? 0.0f : -(l[v] * inverse) * mean;
    for (int j = 0; j < A.k; ++j) {
        const int at = __shfl(index, base + j, 64) - e0;
        const float more = __shfl(mine, base + j, 64);
#pragma unroll
        for (int v = 0; v < NV; ++v) d[v] += v == at ? more : 0.0f;
    }
    if (there) store((E*)A.dlogits + t * A.ld_dlogits + e0, A.experts - e0, d);
}

template <typename E, int W, int NV>
hipError_t launch_route_of(const RouteArgs& A, bool back, hipStream_t s)
{
    const int64_t blocks = (A.tokens + 256 / W - 1) / (256 / W);
    if (back) route_back_kernel<E, W, NV><<<(unsigned)blocks, 256, 0, s>>>(A);
    else route_kernel<E, W, NV><<<(unsigned)blocks, 256, 0, s>>>(A);
    return hipGetLastError();
}

// Lanes of a token: a power of two that holds its experts and its choices.
template <typename E>
hipError_t launch_route_t(const RouteArgs& A, bool back, hipStream_t s)
{
    const int n = A.experts > A.k ? A.experts : A.k;
    if (n <= 8) return launch_route_of<E, 8, 1>(A, back, s);
    if (n <= 16) return launch_route_of<E, 16, 1>(A, back, s);
    if (n <= 32) return launch_route_of<E, 16, 2>(A, back, s);
    if (n <= 64) return launch_route_of<E, 16, 4>(A, back, s);
    if (n <= 128) return launch_route_of<E, 16, 8>(A, back, s);
    if (n <= 256) return launch_route_of<E, 32, 8>(A, back, s);
    if (n <= 512) return launch_route_of<E, 64, 8>(A, back, s);
    return launch_route_of<E, 64, 16>(A, back, s);
}

hipError_t launch_route(const RouteArgs& A, int dtype, bool back, hipStream_t s)
{
    if (A.tokens == 0) return hipSuccess;
    switch (dtype) {
    case ARENA_F32: return launch_route_t<float>(A, back, s);
    case ARENA_BF16: return launch_route_t<bf16>(A, back, s);
    case ARENA_F16: return launch_route_t<f16>(A, back, s);
    }
    return hipErrorInvalidValue;
}

// ---------------------------------------------------------------- sort by expert

// The expert of choice i, or -1.
__device__ __forceinline__ int expert_of(const SortArgs& A, int64_t i, int64_t end)
{
    if (i >= end) return -1;
    const int64_t e = A.wide ? ((const int64_t*)A.index)[i] : ((const int32_t*)A.index)[i];
    return e >= 0 && e < A.experts ? (int)e : -1;
}

// How many choices of a block's share name each expert.
__device__ __forceinline__ void count_choices(const SortArgs& A, int64_t begin, int64_t end, int* hist)
{
    for (int e = threadIdx.x; e < A.experts; e += kSortThreads) hist[e] = 0;
    __syncthreads();
    for (int64_t i = begin + threadIdx.x; i < end; i += kSortThreads) {
        const int e = expert_of(A, i, end);
        if (e >= 0) atomicAdd(&hist[e], 1);
    }
    __syncthreads();
}

__global__ __launch_bounds__(kSortThreads) void sort_count_kernel(const SortArgs A)
{
    __shared__ int hist[kRouteMaxExperts];
    const int64_t begin = (int64_t)blockIdx.x * A.each, end = min(A.choices, begin + A.each);
    count_choices(A, begin, end, hist);
    for (int e = threadIdx.x; e < A.experts; e += kSortThreads) A.counts[(int64_t)blockIdx.x * A.experts + e] = hist[e];
}

// Rows of a block's choices, 1024 at a time: an expert's rows begin where those of the
// experts before end, within it those of the blocks before, of the chunks before, of the
// waves before and of the lanes before that chose it.  Counts are whole numbers, so
// nothing depends on the order in which they are added.  Bound by its barriers: 65536 choices of
// 64 experts 6.1 us and 5.0 for the counts, 74 of 8 experts 3.6 in one block.
__global__ __launch_bounds__(kSortThreads) void sort_place_kernel(const SortArgs A)
{
    constexpr int kWaves = kSortThreads / 64;
    __shared__ int next[kRouteMaxExperts];            // the expert's next row
    __shared__ int sums[kSortThreads], below[kSortThreads];
    __shared__ int waves[kWaves];
    __shared__ uint16_t each[kWaves][kRouteMaxExperts];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, E = A.experts;
    const int64_t begin = (int64_t)blockIdx.x * A.each, end = min(A.choices, begin + A.each);

    // all choices of expert `tid`, and those of the blocks before this one
    int all = 0, before = 0;
    if (A.blocks == 1) {
        count_choices(A, begin, end, next);
        if (tid < E) all = next[tid];
    } else {
        // several threads share an expert's column
        int width = 1;
        while (width < E) width *= 2;
        const int parts = kSortThreads / width, e = tid & (width - 1), part = tid / width;
        if (e < E)
#pragma unroll 4
            for (int b = part; b < A.blocks; b += parts) {
                const int n = A.counts[(int64_t)b * E + e];
                all += n;
                before += b < (int)blockIdx.x ? n : 0;
            }
        sums[tid] = all;
        below[tid] = before;
        __syncthreads();
        all = before = 0;
        if (tid < E)
            for (int p = 0; p < parts; ++p) {
                all += sums[p * width + tid];
                before += below[p * width + tid];
            }
    }
    // exclusive sums over the experts
    int sum = tid < E ? all : 0;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int w = __shfl_up(sum, d, 64);
        sum += lane >= d ? w : 0;
    }
    if (lane == 63) waves[wave] = sum;
    __syncthreads();
    int start = sum - all;
    for (int w = 0; w < wave; ++w) start += waves[w];
    if (tid < E) {
        next[tid] = start + before;
        if (blockIdx.x == 0) {
            A.offsets[tid] = start;
            if (tid == E - 1) A.offsets[E] = start + all;
        }
    }
    int bits = 0;
    while (1 << bits < E) ++bits;
    for (int64_t from = begin; from < end; from += kSortThreads) {
        __syncthreads();
        for (int e = tid; e < kWaves * E; e += kSortThreads) each[e / E][e % E] = 0;
        const int e = expert_of(A, from + tid, end);
        uint64_t same = __ballot(e >= 0);
        for (int b = 0; b < bits; ++b) {
            const uint64_t ones = __ballot(e >> b & 1);
            same &= e >> b & 1 ? ones : ~ones;
        }
        const int rank = __popcll(same & ((1ull << lane) - 1));
        __syncthreads();
        if (e >= 0 && rank == 0) each[wave][e] = (uint16_t)__popcll(same);
        __syncthreads();
        if (tid < E) {
            int n = 0;
            for (int w = 0; w < kWaves; ++w) {
                const int mine = each[w][tid];
                each[w][tid] = (uint16_t)n;          // at most 1024
                n += mine;
            }
            sums[tid] = next[tid];
            next[tid] += n;
        }
        __syncthreads();
        if (from + tid < end) A.row[from + tid] = e >= 0 ? sums[e] + each[wave][e] + rank : -1;
    }
}

// ---------------------------------------------------------------- moves

constexpr int kPieces = 2;            // 16-byte pieces of a row that a lane holds
constexpr int kBatch = 4;             // choices whose rows are read before the first is used

template <typename E>
struct Piece {
    static constexpr int n = 16 / sizeof(E);
};

// The first value of piece i of a row of `width` values, where it is one: the last
// piece ends with the row and takes up values of the piece before (`twice` of them), so
// that no piece is moved value by value.  Rows may start on any value.
template <typename E>
__device__ __forceinline__ bool piece_of(int i, int width, int* c, int* twice)
{
    constexpr int n = Piece<E>::n;
    *c = min(i * n, width - n);
    *twice = i * n - *c;
    return *twice < n && *c >= 0;
}

typedef uint32_t Bits __attribute__((ext_vector_type(4), aligned(2)));

template <typename E>
__device__ __forceinline__ void fetch_piece(const E* p, E (&w)[Piece<E>::n])
{
    const Bits v = __builtin_nontemporal_load((const Bits*)p);
    __builtin_memcpy(w, &v, 16);
}

// The rows of a token's choices from j on, -1 for those that are dropped or past the last.
__device__ __forceinline__ void rows_from(const MoveArgs& A, int64_t t, int j, int (&r)[kBatch])
{
#pragma unroll
    for (int q = 0; q < kBatch; ++q) {
        r[q] = j + q < A.k ? A.row[t * A.k + j + q] : -1;
        if (r[q] >= A.rows) r[q] = -1;
    }
}

// A wave's stretch of a token's row, copied to its choices' rows; first: its first piece.
template <typename E>
__device__ __forceinline__ void dispatch_row(const MoveArgs& A, int64_t t, int first, int lane)
{
    const E* x = (const E*)A.token + t * A.ld_token;
    int c[kPieces], twice;
    bool is[kPieces];
    Bits v[kPieces];
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
        is[i] = piece_of<E>(first + i * 64 + lane, A.model, &c[i], &twice);
        if (is[i]) v[i] = *(const Bits*)(x + c[i]);
    }
    for (int j = 0; j < A.k; ++j) {
        const int64_t r = A.row[t * A.k + j];
        if (r < 0 || r >= A.rows) continue;
        E* to = (E*)A.to_choice + r * A.ld_to_choice;
#pragma unroll
        for (int i = 0; i < kPieces; ++i)
            if (is[i]) *(Bits*)(to + c[i]) = v[i];
    }
}

// y = sum_j w_j ys[row_j], in 32 bits and in the order of j, rounded once.
template <typename E>
__device__ __forceinline__ void combine_row(const MoveArgs& A, int64_t t, int first, int lane)
{
    constexpr int n = Piece<E>::n;
    int c[kPieces], twice;
    bool is[kPieces];
    float sum[kPieces][n];
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
        is[i] = piece_of<E>(first + i * 64 + lane, A.model, &c[i], &twice);
#pragma unroll
        for (int q = 0; q < n; ++q) sum[i][q] = 0.0f;
    }
    for (int j = 0; j < A.k; j += kBatch) {
        int r[kBatch];
        rows_from(A, t, j, r);
        E raw[kBatch][kPieces][n];
#pragma unroll
        for (int b = 0; b < kBatch; ++b)
            if (r[b] >= 0) {
                const E* p = (const E*)A.choice + r[b] * A.ld_choice;
#pragma unroll
                for (int i = 0; i < kPieces; ++i)
                    if (is[i]) fetch_piece(p + c[i], raw[b][i]);
            }
#pragma unroll
        for (int b = 0; b < kBatch; ++b)
            if (r[b] >= 0) {
                const float w = A.weight ? A.weight[t * A.ld_weight + j + b] : 1.0f;
#pragma unroll
                for (int i = 0; i < kPieces; ++i)
#pragma unroll
                    for (int q = 0; q < n; ++q) sum[i][q] += w * (float)raw[b][i][q];
            }
    }
    E* y = (E*)A.to_token + t * A.ld_to_token;
#pragma unroll
    for (int i = 0; i < kPieces; ++i)
        if (is[i]) store(y + c[i], n, sum[i]);
}

// Rows of fewer values than a piece: a thread a value.
template <typename E, int WHAT>
__global__ __launch_bounds__(256) void narrow_kernel(const MoveArgs A)
{
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, t = i / A.model;
    if (t >= A.tokens) return;
    const int c = (int)(i - t * A.model);
    float sum = 0.0f;
    for (int j = 0; j < A.k; ++j) {
        const int64_t r = A.row[t * A.k + j];
        const bool there = r >= 0 && r < A.rows;
        const E* ys = (const E*)A.choice + r * A.ld_choice;
        E* to = (E*)A.to_choice + r * A.ld_to_choice;
        const E* x = (const E*)A.token + t * A.ld_token;
        if (WHAT == 0) {
            if (there) to[c] = x[c];
        } else if (WHAT == 1) {
            if (there) sum += (A.weight ? A.weight[t * A.ld_weight + j] : 1.0f) * (float)ys[c];
        } else {
            if (there) to[c] = (E)(A.weight[t * A.ld_weight + j] * (float)x[c]);
            if (c != 0) continue;
            float dot = 0.0f;
            for (int q = 0; there && q < A.model; ++q) dot += (float)x[q] * (float)ys[q];
            A.dweight[t * A.k + j] = dot;
        }
    }
    if (WHAT == 1) ((E*)A.to_token + t * A.ld_to_token)[c] = (E)sum;
}

// Waves take stretches of tokens in turn.  Bound by memory: 16384 x 4096 in bfloat16, k = 4,
// dispatch 131 us and combine 129 (671 MB each, 5.1 and 5.2 TB/s).
template <typename E, bool BACK>
__global__ __launch_bounds__(256) void move_kernel(const MoveArgs A, int stretches)
{
    const int lane = threadIdx.x & 63;
    const int64_t n = A.tokens * stretches, step = (int64_t)gridDim.x * 4;
    int64_t i = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    for (; i < n; i += step) {
        const int64_t t = stretches == 1 ? i : i / stretches;
        const int first = (int)(i - t * stretches) * (kPieces * 64);
        if (BACK) combine_row<E>(A, t, first, lane);
        else dispatch_row<E>(A, t, first, lane);
    }
}

// dys[row_j] = w_j dy and dw_j = <dy, ys[row_j]>: WAVES waves share a token's row, so that
// few long rows fill the card too.  At that size 238 us (1.21 GB, 5.1 TB/s).
template <typename E, int WAVES>
__global__ __launch_bounds__(256) void combine_back_kernel(const MoveArgs A)
{
    constexpr int n = Piece<E>::n, kEach = 4 / WAVES, kWide = WAVES * 64 * kPieces;
    __shared__ float dots[4][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), share = wave % WAVES;
    // a block's waves pass the barriers together, with or without a token
    for (int64_t t0 = (int64_t)blockIdx.x * kEach; t0 < A.tokens; t0 += (int64_t)gridDim.x * kEach) {
        const int64_t t = t0 + wave / WAVES;
        float mine = 0.0f;                  // of choice `lane`
        if (t < A.tokens) {
            const E* dy = (const E*)A.token + t * A.ld_token;
            for (int from = 0; from * n < A.model; from += kWide) {
                int c[kPieces], twice[kPieces];
                bool is[kPieces];
                float d[kPieces][n];
#pragma unroll
                for (int i = 0; i < kPieces; ++i) {
                    is[i] = piece_of<E>(from + (i * WAVES + share) * 64 + lane, A.model, &c[i], &twice[i]);
                    if (is[i]) fetch(dy + c[i], n, d[i], 0.0f);
                }
                for (int j = 0; j < A.k; j += kBatch) {
                    int r[kBatch];
                    rows_from(A, t, j, r);
                    E raw[kBatch][kPieces][n];
#pragma unroll
                    for (int b = 0; b < kBatch; ++b)
                        if (r[b] >= 0) {
                            const E* p = (const E*)A.choice + r[b] * A.ld_choice;
#pragma unroll
                            for (int i = 0; i < kPieces; ++i)
                                if (is[i]) fetch_piece(p + c[i], raw[b][i]);
                        }
#pragma unroll
                    for (int b = 0; b < kBatch; ++b)
                        if (r[b] >= 0) {
                            const float w = A.weight[t * A.ld_weight + j + b];
                            E* to = (E*)A.to_choice + r[b] * A.ld_to_choice;
                            float dot = 0.0f;
#pragma unroll
                            for (int i = 0; i < kPieces; ++i) {
                                if (!is[i]) continue;
                                float v[n];
#pragma unroll
                                for (int q = 0; q < n; ++q) {
                                    dot += q >= twice[i] ? d[i][q] * (float)raw[b][i][q] : 0.0f;
                                    v[q] = w * d[i][q];
                                }
                                store(to + c[i], n, v);
                            }
                            dot = group_sum<64>(dot);
                            if (lane == j + b) mine += dot;
                        }
                }
            }
        }
        if (WAVES > 1) {
            dots[wave][lane] = mine;
            __syncthreads();
            mine = 0.0f;
#pragma unroll
            for (int s = 0; s < WAVES; ++s) mine += dots[wave / WAVES * WAVES + s][lane];
            __syncthreads();
        }
        if (t < A.tokens && share == 0 && lane < A.k) A.dweight[t * A.k + lane] = mine;
    }
}

template <typename E, int WHAT>
hipError_t launch_narrow(const MoveArgs& A, hipStream_t s)
{
    const int64_t blocks = (A.tokens * A.model + 255) / 256;
    if (blocks > 0) narrow_kernel<E, WHAT><<<(unsigned)blocks, 256, 0, s>>>(A);
    return hipGetLastError();
}

template <typename E, bool BACK>
hipError_t launch_move(const MoveArgs& A, hipStream_t s)
{
    constexpr int wide = kPieces * 64 * Piece<E>::n;
    if (A.model < Piece<E>::n) return launch_narrow<E, BACK ? 1 : 0>(A, s);
    const int stretches = (A.model + wide - 1) / wide;
    const int64_t blocks = (A.tokens * stretches + 3) / 4;
    if (blocks == 0) return hipSuccess;
    move_kernel<E, BACK><<<(unsigned)(blocks < 1 << 20 ? blocks : 1 << 20), 256, 0, s>>>(A, stretches);
    return hipGetLastError();
}

template <typename E>
hipError_t launch_combine_back(const MoveArgs& A, hipStream_t s)
{
    if (A.tokens == 0) return hipSuccess;
    constexpr int wide = kPieces * 64 * Piece<E>::n;
    if (A.model < Piece<E>::n) return launch_narrow<E, 2>(A, s);
    const int waves = A.model <= wide ? 1 : A.model <= 2 * wide ? 2 : 4;
    const int64_t blocks = (A.tokens * waves + 3) / 4, grid = blocks < 1 << 20 ? blocks : 1 << 20;
    if (waves == 1) combine_back_kernel<E, 1><<<(unsigned)grid, 256, 0, s>>>(A);
    else if (waves == 2) combine_back_kernel<E, 2><<<(unsigned)grid, 256, 0, s>>>(A);
    else combine_back_kernel<E, 4><<<(unsigned)grid, 256, 0, s>>>(A);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_route_forward(const RouteArgs& A, int dtype, hipStream_t s) { return launch_route(A, dtype, false, s); }
hipError_t launch_route_backward(const RouteArgs& A, int dtype, hipStream_t s) { return launch_route(A, dtype, true, s); }

// One block up to 4096 choices; past that at most 128 blocks of whole chunks, whose
// counts every block reads.  One block and several, with the moves of 64 columns: 2048 choices of 8 to 512
// experts 18.1 and 21.0, 17.5 and 20.0, 19.9 and 21.9 us; 4096 choices 19.1 and 21.2, 20.1 and 20.5, of
// 512 experts 25.9 and 22.4; 8192 choices 25.5 and 22.3, 26.9 and 21.8, 39.4 and 23.3.
void sort_plan(int64_t choices, int* blocks, int* each)
{
    *blocks = 1;
    *each = (int)choices;
    if (choices <= 4096) return;
    const int64_t per = (choices + 127) / 128;
    *each = (int)((per + kSortThreads - 1) / kSortThreads * kSortThreads);
    *blocks = (int)((choices + *each - 1) / *each);
}

hipError_t launch_sort(const SortArgs& A, hipStream_t s)
{
    if (A.blocks > 1) {
        sort_count_kernel<<<A.blocks, kSortThreads, 0, s>>>(A);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    sort_place_kernel<<<A.blocks, kSortThreads, 0, s>>>(A);
    return hipGetLastError();
}

hipError_t launch_dispatch(const MoveArgs& A, int dtype, hipStream_t s)
{
    // bits are copied: 16-bit types alike
    return dtype == ARENA_F32 ? launch_move<float, false>(A, s) : launch_move<bf16, false>(A, s);
}

hipError_t launch_combine(const MoveArgs& A, int dtype, hipStream_t s)
{
    return dtype == ARENA_F32 ? launch_move<float, true>(A, s)
           : dtype == ARENA_BF16 ? launch_move<bf16, true>(A, s) : launch_move<f16, true>(A, s);
}

hipError_t launch_combine_backward(const MoveArgs& A, int dtype, hipStream_t s)
{
    return dtype == ARENA_F32 ? launch_combine_back<float>(A, s)
           : dtype == ARENA_BF16 ? launch_combine_back<bf16>(A, s) : launch_combine_back<f16>(A, s);
}

}  // namespace arena
