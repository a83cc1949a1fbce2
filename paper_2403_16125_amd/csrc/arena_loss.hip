// Cross entropy over a vocabulary: the passes beside the products (arena_gemm.h).
//
//   l = x w^T,  lse = log sum_v exp(l_v),  loss = lse - l_target
//   dl = dloss (exp(l - lse) - [v = target]),  dx = dl w,  dw = dl^T x
//
// The forward product leaves of each tile column and token the largest logit and the sum
// of exponentials beside it; the join here brings them to one.  Before the backward
// products a pass writes each token's record and copies x with zeros in the rows that the
// loss leaves out, so that nothing in such a row, infinities and NaN neither, reaches the
// weights' gradient.
#include <hip/hip_runtime.h>

#include "arena_layer_internal.h"

namespace arena {
namespace {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ int64_t target_of(const LossArgs& A, int64_t t)
{
    return A.target_wide ? ((const int64_t*)A.target)[t] : ((const int32_t*)A.target)[t];
}

// Two maxima with their sums become one; a maximum of -inf has a sum of 0 (or NaN).
__device__ __forceinline__ void merge(float* most, float* sum, float m, float s)
{
    const float top = fmaxf(*most, m), by = top == -INFINITY ? 0.0f : top;
    *sum = (*most == -INFINITY ? *sum : *sum * __expf(*most - by)) + (m == -INFINITY ? s : s * __expf(m - by));
    *most = top;
}

// ROWS tokens a block, its 1024 threads over them and the tile columns: reads of
// neighbouring tokens lie together.  Bound by their read: 8192 tokens of 512 tile columns 9.3 us
// (33 MB, 3.6 TB/s), one token of 8192 columns 5.4.
template <int ROWS>
__global__ __launch_bounds__(1024) void loss_join_kernel(const LossArgs A)
{
    constexpr int kParts = 1024 / ROWS;
    __shared__ f32x2 lds[1024];
    const int r = threadIdx.x % ROWS, part = threadIdx.x / ROWS;
    const int64_t t = (int64_t)blockIdx.x * ROWS + r;
    float most = -INFINITY, sum = 0.0f;
    if (t < A.tokens)
#pragma unroll 4
        for (int c = part; c < A.columns; c += kParts) {
            const f32x2 e = ((const f32x2*)A.stats)[(int64_t)c * A.tokens + t];
            merge(&most, &sum, e[0], e[1]);
        }
    lds[threadIdx.x] = f32x2{most, sum};
    for (int half = kParts / 2; half >= 1; half >>= 1) {
        __syncthreads();
        if (part < half) {
            const f32x2 e = lds[threadIdx.x + half * ROWS];
            merge(&most, &sum, e[0], e[1]);
            lds[threadIdx.x] = f32x2{most, sum};
        }
    }
    if (part != 0 || t >= A.tokens) return;
    const float lse = (most == -INFINITY ? 0.0f : most) + logf(sum);
    const int64_t target = target_of(A, t);
    float loss = 0.0f;
    // not lse - picked: of a target that has nearly all of the sum that would keep lse's rounding only
    if (target != A.ignore) loss = target >= 0 && target < A.vocabulary ? logf(sum) + (most - A.picked[t]) : NAN;
    if (A.loss) A.loss[t] = loss;
    A.lse[t] = lse;
}

// The power of two that brings the largest factor of a counted token to 2^10 .. 2^11:
// products of float16 then have entries of 6e-5 and more where probabilities are 6e-8
// and more of the largest's, and none past 65504.  One block, bound by latency: 777 tokens 4.7 us.
__global__ __launch_bounds__(1024) void loss_scale_kernel(const LossArgs A)
{
    __shared__ float lds[1024];
    float most = 0.0f;
    for (int64_t t = threadIdx.x; t < A.tokens; t += 1024)
        if (target_of(A, t) != A.ignore) most = fmaxf(most, fabsf(A.dloss[t * A.s_dloss]));
    lds[threadIdx.x] = most;
    for (int half = 512; half >= 1; half >>= 1) {
        __syncthreads();
        if ((int)threadIdx.x < half) lds[threadIdx.x] = fmaxf(lds[threadIdx.x], lds[threadIdx.x + half]);
    }
    if (threadIdx.x != 0) return;
    int up = 0;
    most = lds[0];
    if (most > 0.0f && most < INFINITY) {
        int power;
        (void)frexpf(most, &power);                     // most in 2^(power - 1) .. 2^power
        up = min(max(11 - power, -120), 120);
    }
    A.scale[0] = ldexpf(1.0f, up);
    A.scale[1] = ldexpf(1.0f, -up);
}

// A wave a token: its record, and its row of x.  Bound by memory: 8192 x 4096 23.7 us, 134 MB.
__global__ __launch_bounds__(256) void loss_rows_kernel(const LossArgs A)
{
    const int lane = threadIdx.x & 63;
    const int64_t t = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (t >= A.tokens) return;
    const int64_t target = target_of(A, t);
    const bool counted = target != A.ignore, inside = target >= 0 && target < A.vocabulary;
    if (lane == 0) {
        mm::LossRow row;
        row.lse = A.lse_in[t];
        // a target outside of the vocabulary is not passed over in silence
        row.factor = !inside ? NAN : A.dloss[t * A.s_dloss] * (A.scale ? A.scale[0] : 1.0f);
        row.target = !counted ? -1 : inside ? (int32_t)target : 0;
        row.unused = 0;
        A.rows[t] = row;
    }
    const uint16_t* from = (const uint16_t*)A.x + t * A.ld_x;
    uint16_t* to = (uint16_t*)A.x_to + t * A.ld_to;
    for (int c = lane * 8; c < A.ld_to; c += 512) {
        u32x4 v = {0, 0, 0, 0};
        if (counted) {
            if (c + 8 <= A.model) {
                __builtin_memcpy(&v, from + c, 16);
            } else {
                uint16_t h[8];
#pragma unroll
                for (int q = 0; q < 8; ++q) h[q] = c + q < A.model ? from[c + q] : 0;
                __builtin_memcpy(&v, h, 16);
            }
        }
        *(u32x4*)(to + c) = v;
        if (A.twice) *(u32x4*)(to + A.tokens * A.ld_to + c) = v;
    }
}

// Both halves of a gradient become one, rounded once.  Bound by its launch: 4.8 us for one token of 4096.
template <typename E>
__global__ __launch_bounds__(256) void loss_fold_kernel(const float* sum, E* dx, int64_t ld, int64_t tokens, int model)
{
    const int c = blockIdx.x * 256 + threadIdx.x;
    const int64_t t = blockIdx.y;
    if (c < model) dx[t * ld + c] = (E)(sum[t * model + c] + sum[(tokens + t) * model + c]);
}

}  // namespace

// Rows a block by how many blocks they make and how much of a line a row's reads share.  Whole
// forward passes of model 64, over 131072 entries, with 1, 8 and 32 rows: 17 tokens 18.7, 18.1 and
// 20.9 us, 1024 tokens 74, 67 and 67, 8192 tokens 488, 447 and 440; over 5000 entries 17 tokens
// 17.0, 17.5 and 18.0, 8192 tokens 70, 36 and 34.
hipError_t launch_loss_join(const LossArgs& A, hipStream_t s)
{
    if (A.tokens == 0) return hipSuccess;
    if (A.tokens >= 4096) loss_join_kernel<32><<<(unsigned)((A.tokens + 31) / 32), 1024, 0, s>>>(A);
    else if (A.tokens >= 64) loss_join_kernel<8><<<(unsigned)((A.tokens + 7) / 8), 1024, 0, s>>>(A);
    else loss_join_kernel<1><<<(unsigned)A.tokens, 1024, 0, s>>>(A);
    return hipGetLastError();
}

hipError_t launch_loss_rows(const LossArgs& A, hipStream_t s)
{
    if (A.tokens == 0) return hipSuccess;
    if (A.scale) {
        loss_scale_kernel<<<1, 1024, 0, s>>>(A);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    loss_rows_kernel<<<(unsigned)((A.tokens + 3) / 4), 256, 0, s>>>(A);
    return hipGetLastError();
}

hipError_t launch_loss_fold(const float* sum, void* dx, int64_t ld, int64_t tokens, int model, int dtype, hipStream_t s)
{
    const dim3 grid((unsigned)(model + 255) / 256, (unsigned)tokens);
    if (dtype == ARENA_BF16) loss_fold_kernel<<<grid, 256, 0, s>>>(sum, (__bf16*)dx, ld, tokens, model);
    else loss_fold_kernel<<<grid, 256, 0, s>>>(sum, (_Float16*)dx, ld, tokens, model);
    return hipGetLastError();
}

}  // namespace arena
