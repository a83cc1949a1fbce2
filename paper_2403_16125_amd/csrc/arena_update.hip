// Orthogonalised update: the passes over the gradient.
//
//   M' = mu M + G,  U = G + mu M' (Nesterov) or M',  X0 = U / (|U|_F + eps)
//
// The norm has to be known before X0 can be rounded, so U is formed twice: by
// the sum of squares (which stores M') and by the scaling.  Both are bound by
// memory, and small beside the products that follow: 10944 x 4096 in float32 with
// momentum 113 us (538 MB, 4.8 TB/s) and 90 us (538 MB, 6.0 TB/s, part of it from
// the cache) of 3300.
//
// X0 is held in float16 times 2^12.  Its entries are at most 1 in magnitude
// and about 1 / sqrt(rows cols) in size, and the products' operands keep 11
// bits that way where bfloat16 would keep 8, at the same rate; the scale lifts
// the small entries of X, X X^T and its polynomial out of float16's subnormals
// (magnitudes up to 15 are representable, which the host checks for the
// polynomial).
//
// What falls on small singular values grows by `a` in each step, the rounding of X
// with it, and a spectrum that decays leaves little beside it: with singular values
// of i^-2 (512 x 768, five steps of the usual polynomial) the result was off by 2.1e-2.  So
// what rounding takes off X is kept too (11 more bits, times 2^11), and the next step
// adds `a` times it, to first order what the polynomial makes of it there: 2.2e-3.
// The last two steps do without: little growth is left, and where singular values
// are large the polynomial makes less of it than a.  Costs 2 to 5 % of an update (10944
// x 4096: 3255 -> 3350 us).
#include "arena_layer_internal.h"

namespace arena {
namespace {

template <typename E>
__device__ __forceinline__ void fetch8(const E* p, int left, float* v)
{
    if (left >= 8) {
        E w[8];
        __builtin_memcpy(w, p, sizeof(w));
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = (float)w[i];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < left ? (float)p[i] : 0.0f;
    }
}

// U of eight neighbouring values; `m` holds M on entry, M' on return.
__device__ __forceinline__ void step8(const UpdateArgs& A, float* g, float* m)
{
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        m[i] = A.mu * m[i] + g[i];
        g[i] = A.nesterov ? g[i] + A.mu * m[i] : m[i];
    }
}

// Blocks of a matrix share its rows x chunks of 8; each leaves its sum of
// squares in double (squares of large gradients pass float's range).
template <typename E>
__global__ __launch_bounds__(256) void update_sum_kernel(const UpdateArgs A)
{
    __shared__ double lds[4];
    const int z = blockIdx.y, per = (A.cols + 7) / 8;
    const int64_t n = (int64_t)A.rows * per;
    double sum = 0.0;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
        const int64_t r = i / per;
        const int c = (int)(i % per) * 8, left = A.cols - c;
        float g[8];
        fetch8((const E*)A.grad + z * A.s_grad + r * A.ld_grad + c, left, g);
        if (A.momentum_out) {
            float m[8];
            fetch8(A.momentum + z * A.s_mom + r * A.ld_mom + c, left, m);
            step8(A, g, m);
            float* to = A.momentum_out + z * A.s_mom_out + r * A.ld_mom_out + c;
            if (left >= 8) {
                __builtin_memcpy(to, m, sizeof(m));
            } else {
#pragma unroll
                for (int q = 0; q < 8; ++q)
                    if (q < left) to[q] = m[q];
            }
        }
#pragma unroll
        for (int q = 0; q < 8; ++q) sum += (double)g[q] * (double)g[q];
    }
    for (int d = 32; d >= 1; d >>= 1) sum += __shfl_xor(sum, d, 64);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) A.part[z * A.blocks + blockIdx.x] = lds[0] + lds[1] + lds[2] + lds[3];
}

// X0 = 2^12 U / (|U| + eps), and what its rounding leaves; zero in the padding.
template <typename E>
__global__ __launch_bounds__(256) void update_scale_kernel(const UpdateArgs A)
{
    __shared__ double lds[4];
    const int z = blockIdx.y, per = A.ld_x / 8;
    double sum = threadIdx.x < A.blocks ? A.part[z * A.blocks + threadIdx.x] : 0.0;
    for (int d = 32; d >= 1; d >>= 1) sum += __shfl_xor(sum, d, 64);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = sum;
    __syncthreads();
    const double norm = sqrt(lds[0] + lds[1] + lds[2] + lds[3]) + (double)A.eps;
    // a matrix of zeros without eps stays zero; double, as 1 / norm may pass float's range
    const double scale = norm > 0.0 || norm != norm ? 4096.0 / norm : 0.0;
    const int64_t n = (int64_t)A.rows_p * per;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
        const int64_t r = i / per;
        const int c = (int)(i % per) * 8, left = r < A.rows ? A.cols - c : 0;
        float g[8];
        fetch8((const E*)A.grad + z * A.s_grad + r * A.ld_grad + c, left, g);
        if (A.momentum_out) {
            float m[8];
            fetch8(A.momentum_out + z * A.s_mom_out + r * A.ld_mom_out + c, left, m);
#pragma unroll
            for (int q = 0; q < 8; ++q) g[q] = A.nesterov ? g[q] + A.mu * m[q] : m[q];
        }
        const int64_t at = (z * (int64_t)A.rows_p + r) * A.ld_x + c;
        _Float16 h[8], rest[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            const float v = q < left ? (float)(g[q] * scale) : 0.0f;
            h[q] = (_Float16)v;
            rest[q] = (_Float16)((v - (float)h[q]) * 2048.0f);
        }
        __builtin_memcpy((_Float16*)A.x + at, h, sizeof(h));
        if (A.rest) __builtin_memcpy((_Float16*)A.rest + at, rest, sizeof(rest));
    }
}

}  // namespace

hipError_t launch_update_sum(const UpdateArgs& A, int dtype, hipStream_t s)
{
    const dim3 grid(A.blocks, A.batch);
    if (dtype == ARENA_F32) update_sum_kernel<float><<<grid, 256, 0, s>>>(A);
    else if (dtype == ARENA_BF16) update_sum_kernel<__bf16><<<grid, 256, 0, s>>>(A);
    else update_sum_kernel<_Float16><<<grid, 256, 0, s>>>(A);
    return hipGetLastError();
}

hipError_t launch_update_scale(const UpdateArgs& A, int dtype, hipStream_t s)
{
    const int64_t blocks = ((int64_t)A.rows_p * (A.ld_x / 8) + 255) / 256;
    const dim3 grid((unsigned)(blocks < 4096 ? blocks : 4096), A.batch);
    if (dtype == ARENA_F32) update_scale_kernel<float><<<grid, 256, 0, s>>>(A);
    else if (dtype == ARENA_BF16) update_scale_kernel<__bf16><<<grid, 256, 0, s>>>(A);
    else update_scale_kernel<_Float16><<<grid, 256, 0, s>>>(A);
    return hipGetLastError();
}

}  // namespace arena
