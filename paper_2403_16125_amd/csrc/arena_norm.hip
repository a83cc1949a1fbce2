// Norms around a block, fused with its gate and residual scale.
//
//   v = norm(y) w2 + b2      r = x + scale gate v      n = norm(r) w1 + b1
//   norm(z) = (z - mu) rs,   rs = 1 / sqrt(mean((z - mu)^2) + eps),  mu = mean(z) or 0
//
// and backwards, from the gradients dn and dr of n and r:
//   dR = dr + N(dn w1; rhat)              (the gradient of r, and of x)
//   dv = scale gate dR,  dy = N(dv w2; yhat),  dgate = sum of scale dR v
//   N(q; zhat) = rs (q - zhat mean(q zhat) - mean(q))   (the last term with a mean only)
//   dw1 = sum dn rhat, db1 = sum dn, dw2 = sum dv yhat, db2 = sum dv.
//
// Both passes are bound by memory: the forward reads x, y and writes r, n, the
// backward reads dn, dr, r, y and writes dx, dy, each once.  A row stays in
// the registers of its worker (one wave up to 512 values, 4 to 16 waves beyond),
// 8 neighbouring values a thread and load, so its means cost no second pass.
// All arithmetic is in 32 bits; values are rounded once, as they are stored.
//
// Column sums (gradients of weights, biases and gates) run down the rows of a
// worker in registers, go to memory once per worker and are joined by a second
// launch in the workers' order: the same inputs give the same bits.
#include "arena_layer_internal.h"

namespace arena {
namespace {

// Eight neighbouring values of a row.
template <typename E>
struct Eight {
    E v[8];
};

// `left` values lie inside the row; the others read as zero.  Rows may start
// on any value: the 16-byte accesses are unaligned where they do not.
template <typename E>
__device__ __forceinline__ Eight<E> get8(const void* base, int64_t at, int left)
{
    const E* p = (const E*)base + at;
    Eight<E> w;
    if (left >= 8) {
        __builtin_memcpy(&w, p, sizeof(w));
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) w.v[i] = i < left ? p[i] : (E)0.0f;
    }
    return w;
}

template <typename E>
__device__ __forceinline__ void put8(void* base, int64_t at, int left, const float* v)
{
    E* p = (E*)base + at;
    if (left >= 8) {
        Eight<E> w;
#pragma unroll
        for (int i = 0; i < 8; ++i) w.v[i] = (E)v[i];
        __builtin_memcpy(p, &w, sizeof(w));
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < left) p[i] = (E)v[i];
    }
}

// Sums of N values over the worker's threads, the same in each of them.
// `slot` alternates between calls, so one barrier a call is enough.
template <int WV, int N>
__device__ __forceinline__ void worker_sum(float (&v)[N], float (*lds)[WV][N], int& slot)
{
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int d = 32; d >= 1; d >>= 1) v[i] += __shfl_xor(v[i], d, 64);
    if (WV == 1) return;
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0)
#pragma unroll
        for (int i = 0; i < N; ++i) lds[slot][wave][i] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
        v[i] = lds[slot][0][i];
#pragma unroll
        for (int w = 1; w < WV; ++w) v[i] += lds[slot][w][i];
    }
    slot ^= 1;
}

template <int WV, int IT>
struct Row {
    static constexpr int kWorkers = WV == 1 ? 4 : 1;      // workers of a block
    static constexpr int kThreads = 64 * WV * kWorkers;
    static __device__ __forceinline__ int col(int it)
    {
        return (it * WV * 64 + (WV == 1 ? (threadIdx.x & 63) : threadIdx.x)) * 8;
    }
    static __device__ __forceinline__ int64_t worker()
    {
        return (int64_t)blockIdx.x * kWorkers + (WV == 1 ? threadIdx.x >> 6 : 0);
    }
};

// Mean (0 without one) and 1 / deviation of a row, the squares taken about the mean.
template <int WV, int IT>
__device__ __forceinline__ void moments(const float (&z)[IT][8], int width, bool layer, float eps,
                                        float (*lds)[WV][1], int& slot, float* mu, float* rs)
{
    float s[1] = {0.0f};
    float m = 0.0f;
    if (layer) {
#pragma unroll
        for (int it = 0; it < IT; ++it)
#pragma unroll
            for (int i = 0; i < 8; ++i) s[0] += z[it][i];
        worker_sum<WV, 1>(s, lds, slot);
        m = s[0] / width;
        s[0] = 0.0f;
    }
#pragma unroll
    for (int it = 0; it < IT; ++it) {
        const int left = width - Row<WV, IT>::col(it);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float d = i < left ? z[it][i] - m : 0.0f;
            s[0] += d * d;
        }
    }
    worker_sum<WV, 1>(s, lds, slot);
    *mu = m;
    *rs = 1.0f / sqrtf(s[0] / width + eps);
}

// One row a worker.  n is formed from the 32-bit r, not from the stored one.
template <typename TY, typename TX, int WV, int IT>
__global__ __launch_bounds__((Row<WV, IT>::kThreads)) void norm_forward_kernel(const NormArgs A)
{
    typedef Row<WV, IT> R;
    __shared__ float lds[2][WV][1];
    const int64_t t = R::worker();
    if (WV == 1 && t >= A.tokens) return;
    int slot = 0;
    float r[IT][8];
    float mu2 = 0.0f, rs2 = 0.0f, mu1 = 0.0f, rs1 = 0.0f;
#pragma unroll
    for (int it = 0; it < IT; ++it) {
        const Eight<TX> x = get8<TX>(A.x, t * A.ld_x + R::col(it), A.width - R::col(it));
#pragma unroll
        for (int i = 0; i < 8; ++i) r[it][i] = (float)x.v[i];
    }
    if (A.y) {
        float y[IT][8];
#pragma unroll
        for (int it = 0; it < IT; ++it) {
            const Eight<TY> w = get8<TY>(A.y, t * A.ld_y + R::col(it), A.width - R::col(it));
#pragma unroll
            for (int i = 0; i < 8; ++i) y[it][i] = (float)w.v[i];
        }
        moments<WV, IT>(y, A.width, A.layer, A.eps, lds, slot, &mu2, &rs2);
        const int64_t row = t / A.gate_rows;
#pragma unroll
        for (int it = 0; it < IT; ++it) {
            const int c = R::col(it), left = A.width - c;
            Eight<TY> w, b, g;
            if (A.w_post) w = get8<TY>(A.w_post, c, left);
            if (A.b_post) b = get8<TY>(A.b_post, c, left);
            if (A.gate) g = get8<TY>(A.gate, row * A.ld_gate + c, left);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float v = (y[it][i] - mu2) * rs2;
                if (A.w_post) v *= (float)w.v[i];
                if (A.b_post) v += (float)b.v[i];
                r[it][i] += A.scale * (A.gate ? (float)g.v[i] : 1.0f) * v;
                if (i >= left) r[it][i] = 0.0f;
            }
            put8<TX>(A.r, t * A.ld_r + c, left, r[it]);
        }
    }
    if (A.n) {
        moments<WV, IT>(r, A.width, A.layer, A.eps, lds, slot, &mu1, &rs1);
#pragma unroll
        for (int it = 0; it < IT; ++it) {
            const int c = R::col(it), left = A.width - c;
            Eight<TY> w, b;
            if (A.w_pre) w = get8<TY>(A.w_pre, c, left);
            if (A.b_pre) b = get8<TY>(A.b_pre, c, left);
            float n[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                n[i] = (r[it][i] - mu1) * rs1;
                if (A.w_pre) n[i] *= (float)w.v[i];
                if (A.b_pre) n[i] += (float)b.v[i];
            }
            put8<TY>(A.n, t * A.ld_n + c, left, n);
        }
    }
    if (A.stats && (WV == 1 ? (threadIdx.x & 63) == 0 : threadIdx.x == 0)) {
        float* s = A.stats + t * 4;
        s[0] = mu2;
        s[1] = rs2;
        s[2] = mu1;
        s[3] = rs1;
    }
}

// A worker goes down rows_each rows.
template <typename TY, typename TX, int WV, int IT, bool BIAS>
__global__ __launch_bounds__((Row<WV, IT>::kThreads)) void norm_backward_kernel(const NormArgs A)
{
    typedef Row<WV, IT> R;
    __shared__ float lds[2][WV][2];
    const int64_t me = R::worker();
    if (me >= A.workers) return;
    const int64_t t0 = me * A.rows_each, t1 = min(t0 + A.rows_each, A.tokens);
    int slot = 0;
    float s_w1[IT][8], s_w2[IT][8], s_g[IT][8], s_b1[BIAS ? IT : 1][8], s_b2[BIAS ? IT : 1][8];
#pragma unroll
    for (int it = 0; it < IT; ++it)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            s_w1[it][i] = s_w2[it][i] = s_g[it][i] = 0.0f;
            if (BIAS) s_b1[it][i] = s_b2[it][i] = 0.0f;
        }
    Eight<TY> w1[IT], w2[IT], gt[IT];
#pragma unroll
    for (int it = 0; it < IT; ++it) {
        const int c = R::col(it), left = A.width - c;
        if (A.w_pre) w1[it] = get8<TY>(A.w_pre, c, left);
        if (A.w_post) w2[it] = get8<TY>(A.w_post, c, left);
    }
    const float inv = 1.0f / A.width;
    const int64_t first = t0 / A.gate_rows;
    int64_t row = -1;
    // dgate of the gate row that ends here: to its place if the worker saw all of its tokens
    auto flush = [&]() {
        const bool whole = row * A.gate_rows >= t0 && min((row + 1) * A.gate_rows, A.tokens) <= t1;
#pragma unroll
        for (int it = 0; it < IT; ++it) {
            const int c = R::col(it), left = A.width - c;
            if (whole) {
                put8<TY>(A.dgate, row * A.width + c, left, s_g[it]);
            } else {
                put8<float>(A.part, (me * kNormSums + (row == first ? 4 : 5)) * A.width + c, left, s_g[it]);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) s_g[it][i] = 0.0f;
        }
    };
    for (int64_t t = t0; t < t1; ++t) {
        if (A.gate && t / A.gate_rows != row) {
            if (row >= 0 && A.dgate) flush();
            row = t / A.gate_rows;
#pragma unroll
            for (int it = 0; it < IT; ++it)
                gt[it] = get8<TY>(A.gate, row * A.ld_gate + R::col(it), A.width - R::col(it));
        }
        const float* st = A.stats + t * 4;
        const float mu2 = st[0], rs2 = st[1], mu1 = st[2], rs1 = st[3];
        float d[IT][8];            // gradient of r
        Eight<TX> res[IT];
        Eight<TY> dn[IT], y[IT];
#pragma unroll
        for (int it = 0; it < IT; ++it) {
            const int c = R::col(it), left = A.width - c;
            if (A.dn) {
                dn[it] = get8<TY>(A.dn, t * A.ld_dn + c, left);
                res[it] = get8<TX>(A.res, t * A.ld_res + c, left);
            }
            if (A.y) y[it] = get8<TY>(A.y, t * A.ld_y + c, left);
            Eight<TX> w;
            if (A.dr) w = get8<TX>(A.dr, t * A.ld_dr + c, left);
#pragma unroll
            for (int i = 0; i < 8; ++i) d[it][i] = A.dr ? (float)w.v[i] : 0.0f;
        }
        if (A.dn) {
            float m[2] = {0.0f, 0.0f};
#pragma unroll
            for (int it = 0; it < IT; ++it) {
                const int left = A.width - R::col(it);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float g = (float)dn[it].v[i], z = ((float)res[it].v[i] - mu1) * rs1;
                    const float q = A.w_pre ? g * (float)w1[it].v[i] : g;
                    if (i < left) {
                        m[0] += q * z;
                        m[1] += q;
                    }
                    s_w1[it][i] += g * z;
                    if (BIAS) s_b1[it][i] += g;
                }
            }
            worker_sum<WV, 2>(m, lds, slot);
            const float mz = m[0] * inv, mq = A.layer ? m[1] * inv : 0.0f;
#pragma unroll
            for (int it = 0; it < IT; ++it)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float g = (float)dn[it].v[i], z = ((float)res[it].v[i] - mu1) * rs1;
                    const float q = A.w_pre ? g * (float)w1[it].v[i] : g;
                    d[it][i] += rs1 * (q - z * mz - mq);
                }
        }
        if (A.dx)
#pragma unroll
            for (int it = 0; it < IT; ++it)
                put8<TX>(A.dx, t * A.ld_dx + R::col(it), A.width - R::col(it), d[it]);
        if (!A.y) continue;
        Eight<TY> b2[IT];
        if (BIAS && A.b_post)
#pragma unroll
            for (int it = 0; it < IT; ++it) b2[it] = get8<TY>(A.b_post, R::col(it), A.width - R::col(it));
        float m[2] = {0.0f, 0.0f};
#pragma unroll
        for (int it = 0; it < IT; ++it) {
            const int left = A.width - R::col(it);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float z = ((float)y[it].v[i] - mu2) * rs2;
                const float w = A.w_post ? (float)w2[it].v[i] : 1.0f;
                const float b = BIAS && A.b_post ? (float)b2[it].v[i] : 0.0f;
                const float sd = A.scale * d[it][i];
                s_g[it][i] += sd * (z * w + b);
                const float dv = A.gate ? sd * (float)gt[it].v[i] : sd;
                s_w2[it][i] += dv * z;
                if (BIAS) s_b2[it][i] += dv;
                const float q = dv * w;
                d[it][i] = q;
                if (i < left) {
                    m[0] += q * z;
                    m[1] += q;
                }
            }
        }
        worker_sum<WV, 2>(m, lds, slot);
        const float mz = m[0] * inv, mq = A.layer ? m[1] * inv : 0.0f;
        if (A.dy)
#pragma unroll
            for (int it = 0; it < IT; ++it) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float z = ((float)y[it].v[i] - mu2) * rs2;
                    d[it][i] = rs2 * (d[it][i] - z * mz - mq);
                }
                put8<TY>(A.dy, t * A.ld_dy + R::col(it), A.width - R::col(it), d[it]);
            }
    }
    if (A.dgate && row >= 0) flush();
#pragma unroll
    for (int it = 0; it < IT; ++it) {
        const int c = R::col(it), left = A.width - c;
        const int64_t at = me * kNormSums * A.width + c;
        if (A.dw_pre) put8<float>(A.part, at, left, s_w1[it]);
        if (BIAS && A.db_pre) put8<float>(A.part, at + A.width, left, s_b1[it]);
        if (A.dw_post) put8<float>(A.part, at + 2 * (int64_t)A.width, left, s_w2[it]);
        if (BIAS && A.db_post) put8<float>(A.part, at + 3 * (int64_t)A.width, left, s_b2[it]);
    }
}

// Joins the workers' column sums: blockIdx.y < 4 the weights and biases, above
// that the gate rows that several workers share.  64 columns a block, 16 waves
// over the workers.
template <typename TY>
__global__ __launch_bounds__(1024) void norm_join_kernel(const NormArgs A)
{
    __shared__ float lds[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int c = blockIdx.x * 64 + lane;
    TY* out;
    int64_t w0 = 0, w1 = A.workers, row = 0;
    if (blockIdx.y < 4) {
        void* const outs[4] = {A.dw_pre, A.db_pre, A.dw_post, A.db_post};
        out = (TY*)outs[blockIdx.y];
    } else {
        row = blockIdx.y - 4;
        const int64_t t0 = row * A.gate_rows, t1 = min(t0 + A.gate_rows, A.tokens);
        w0 = t0 / A.rows_each;
        w1 = (t1 - 1) / A.rows_each + 1;
        out = w1 - w0 > 1 ? (TY*)A.dgate + row * A.width : nullptr;      // one worker: already in place
        if (A.tokens == 0) {                                             // a sum over nothing
            w1 = w0;
            out = (TY*)A.dgate;
        }
    }
    if (!out) return;
    float s = 0.0f;
    if (c < A.width)
        for (int64_t w = w0 + wave; w < w1; w += 16) {
            const int which = blockIdx.y < 4 ? blockIdx.y : (w * A.rows_each / A.gate_rows == row ? 4 : 5);
            s += A.part[(w * kNormSums + which) * A.width + c];
        }
    lds[wave][lane] = s;
    __syncthreads();
    if (wave == 0 && c < A.width) {
        for (int w = 1; w < 16; ++w) s += lds[w][lane];
        out[c] = (TY)s;
    }
}

// Waves and chunks a thread by width.
int waves_of(int width) { return width <= 512 ? 1 : width <= 4096 ? 4 : width <= 8192 ? 8 : 16; }

template <typename TY, typename TX>
hipError_t forward(const NormArgs& A, hipStream_t s)
{
    const int64_t n = A.tokens;
    switch (waves_of(A.width)) {
    case 1: norm_forward_kernel<TY, TX, 1, 1><<<(unsigned)((n + 3) / 4), 256, 0, s>>>(A); break;
    case 4:
        if (A.width <= 2048) norm_forward_kernel<TY, TX, 4, 1><<<(unsigned)n, 256, 0, s>>>(A);
        else norm_forward_kernel<TY, TX, 4, 2><<<(unsigned)n, 256, 0, s>>>(A);
        break;
    case 8: norm_forward_kernel<TY, TX, 8, 2><<<(unsigned)n, 512, 0, s>>>(A); break;
    default: norm_forward_kernel<TY, TX, 16, 2><<<(unsigned)n, 1024, 0, s>>>(A); break;
    }
    return hipGetLastError();
}

template <typename TY, typename TX, bool BIAS>
hipError_t backward(const NormArgs& A, hipStream_t s)
{
    const unsigned n = (unsigned)A.workers;
    if (n) switch (waves_of(A.width)) {
    case 1: norm_backward_kernel<TY, TX, 1, 1, BIAS><<<(n + 3) / 4, 256, 0, s>>>(A); break;
    case 4:
        if (A.width <= 2048) norm_backward_kernel<TY, TX, 4, 1, BIAS><<<n, 256, 0, s>>>(A);
        else norm_backward_kernel<TY, TX, 4, 2, BIAS><<<n, 256, 0, s>>>(A);
        break;
    case 8: norm_backward_kernel<TY, TX, 8, 2, BIAS><<<n, 512, 0, s>>>(A); break;
    default: norm_backward_kernel<TY, TX, 16, 2, BIAS><<<n, 1024, 0, s>>>(A); break;
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    // rows_each is a multiple of gate_rows or less than it: only then gate rows are shared
    const int64_t rows = !A.dgate ? 0 : A.tokens == 0 ? 1
                         : A.gate_rows > A.rows_each ? (A.tokens + A.gate_rows - 1) / A.gate_rows : 0;
    norm_join_kernel<TY><<<dim3((A.width + 63) / 64, (unsigned)(4 + rows)), 1024, 0, s>>>(A);
    return hipGetLastError();
}

template <typename TY, typename TX>
hipError_t backward_any(const NormArgs& A, hipStream_t s)
{
    return A.b_post || A.db_post || A.db_pre ? backward<TY, TX, true>(A, s) : backward<TY, TX, false>(A, s);
}

}  // namespace

// Two blocks' worth of workers a compute unit: more would read ahead better but
// leave more sums to join.
void norm_plan(int64_t tokens, int64_t gate_rows, int width, int* workers, int* rows_each)
{
    const int64_t most = width <= 512 ? 2048 : 512;
    int64_t each = (tokens + most - 1) / most;
    if (each < 1) each = 1;
    if (gate_rows <= each) each = (each + gate_rows - 1) / gate_rows * gate_rows;
    *rows_each = (int)each;
    *workers = (int)((tokens + each - 1) / each);
}

hipError_t launch_norm_forward(const NormArgs& A, int dtype, int stream_dtype, hipStream_t s)
{
    if (dtype == ARENA_F32) return forward<float, float>(A, s);
    if (dtype == ARENA_BF16)
        return stream_dtype == ARENA_F32 ? forward<__bf16, float>(A, s) : forward<__bf16, __bf16>(A, s);
    return stream_dtype == ARENA_F32 ? forward<_Float16, float>(A, s) : forward<_Float16, _Float16>(A, s);
}

hipError_t launch_norm_backward(const NormArgs& A, int dtype, int stream_dtype, hipStream_t s)
{
    if (dtype == ARENA_F32) return backward_any<float, float>(A, s);
    if (dtype == ARENA_BF16)
        return stream_dtype == ARENA_F32 ? backward_any<__bf16, float>(A, s) : backward_any<__bf16, __bf16>(A, s);
    return stream_dtype == ARENA_F32 ? backward_any<_Float16, float>(A, s) : backward_any<_Float16, _Float16>(A, s);
}

}  // namespace arena
