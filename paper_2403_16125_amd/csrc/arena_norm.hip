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
// All arithmetic is in 32 bits; values are rounded once, as they are stored.  The
// backward reads the stored r, rounded where the stream has 16 bits, beside the
// statistics of the unrounded one: what a caller keeps of the forward pass.  Its error
// is then 2.4e-3 of a gradient in bfloat16 where a float stream has 1.7e-3.
// 16384 x 4096 in bfloat16: forward 110 to 123 us (0.54 GB at 4.4 to 4.9 TB/s),
// backward 175 to 195 us (0.81 GB at 4.1 to 4.6 TB/s) and 11 to 13 us for the
// joining of its column sums.  Of few rows the launches bound it: one row 3.6 us.
//
// Column sums (gradients of weights, biases and gates) run down the rows of a
// worker in registers, go to memory once per worker and are joined by a second
// launch in the workers' order: the same inputs give the same bits.
#include "arena_layer_internal.h"

namespace arena {
namespace {

template <typename E>
__device__ __forceinline__ float half_value(uint16_t h)
{
    E e;
    __builtin_memcpy(&e, &h, 2);
    return (float)e;
}
template <>
__device__ __forceinline__ float half_value<float>(uint16_t)
{
    return 0.0f;      // floats are taken whole
}

// Eight neighbouring values of a row as they lie in memory.
template <typename E>
struct Eight {
    static constexpr int kWords = sizeof(E) * 2;
    uint32_t w[kWords];
    __device__ __forceinline__ float operator[](int i) const
    {
        if (sizeof(E) == 4) return __uint_as_float(w[i]);
        const uint16_t h = (uint16_t)(w[i >> 1] >> (16 * (i & 1)));
        return half_value<E>(h);
    }
    // drops the first n (0 to 7) values; zeros follow the rest
    __device__ __forceinline__ void drop(int n)
    {
#pragma unroll
        for (int by = 4; by >= 1; by >>= 1) {
            const bool now = n & by;
            const int words = by * (int)sizeof(E) / 4;
#pragma unroll
            for (int i = 0; i < kWords; ++i) {
                const uint32_t next = i + 1 < kWords ? w[i + 1] : 0;
                const uint32_t moved = words == 0 ? w[i] >> 16 | next << 16 : i + words < kWords ? w[i + words] : 0;
                w[i] = now ? moved : w[i];
            }
        }
    }
};

// Thread k takes the columns 8 k .. 8 k + 7 of a row, or the row's last eight
// where it ends before: the first `lo` of those (8 where nothing is left) belong
// to the threads before and are computed with, but neither summed nor stored.  So
// a row's end costs the reads no branch: with a load for each of its values, which
// were waited for at once, 3001 x 1365 took 39 us backwards, so 28.
__device__ __forceinline__ int column_of(int k, int width) { return min(8 * k, width - 8); }
__device__ __forceinline__ int low_of(int k, int width) { return min(8 * k - column_of(k, width), 8); }

// The eight values from column c of the row that starts at `row` values from base
// (the same in all lanes, so it stays in scalar registers).  Rows may start on any
// value: the 16-byte accesses are unaligned where they do not.  In a row of less
// than eight values, which has one wave (WV), c is negative and the first `lo` are
// not read.
template <typename E, int WV>
__device__ __forceinline__ Eight<E> get8(const void* base, int64_t row, int c, int lo, int width)
{
    const char* p = (const char*)base + row * (int64_t)sizeof(E);
    Eight<E> w;
    if (WV > 1 || width >= 8) {
        __builtin_memcpy(w.w, p + (uint32_t)(c * (int)sizeof(E)), sizeof(w.w));
    } else {
        // values i < lo are not the row's
        auto half = [&](int i) -> uint32_t {
            return i >= lo * (int)(sizeof(E) / 2) ? *(const uint16_t*)(p + (uint32_t)(c * (int)sizeof(E) + 2 * i)) : 0;
        };
#pragma unroll
        for (int i = 0; i < Eight<E>::kWords; ++i) w.w[i] = half(2 * i) | half(2 * i + 1) << 16;
    }
    return w;
}

template <typename E>
__device__ __forceinline__ void put8(void* base, int64_t row, int c, int lo, const float* v)
{
    char* p = (char*)base + row * (int64_t)sizeof(E);
    E w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = (E)v[i];
    if (lo == 0) {
        __builtin_memcpy(p + (uint32_t)(c * (int)sizeof(E)), w, sizeof(w));
    } else {
        Eight<E> q;
        __builtin_memcpy(q.w, w, sizeof(w));
        q.drop(lo);
        uint32_t to = (uint32_t)((c + lo) * (int)sizeof(E));
#pragma unroll
        for (int by = 4; by >= 1; by >>= 1)
            if ((8 - lo) & by) {
                __builtin_memcpy(p + to, q.w, by * sizeof(E));
                to += by * sizeof(E);
                q.drop(by);
            }
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
        v[i] = lds[slot][threadIdx.x & (WV - 1)][i];
#pragma unroll
        for (int d = WV / 2; d >= 1; d >>= 1) v[i] += __shfl_xor(v[i], d, 64);
    }
    slot ^= 1;
}

template <int WV, int IT>
struct Row {
    static constexpr int kWorkers = WV == 1 ? 4 : 1;      // workers of a block
    static constexpr int kThreads = 64 * WV * kWorkers;
    static __device__ __forceinline__ int chunk(int it)
    {
        return it * WV * 64 + (WV == 1 ? (threadIdx.x & 63) : threadIdx.x);
    }
    static __device__ __forceinline__ int col(int it, int width) { return column_of(chunk(it), width); }
    static __device__ __forceinline__ int low(int it, int width) { return low_of(chunk(it), width); }
    static __device__ __forceinline__ int64_t worker()
    {
        return (int64_t)blockIdx.x * kWorkers + (WV == 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : 0);
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
            for (int i = 0; i < 8; ++i) s[0] += i < Row<WV, IT>::low(it, width) ? 0.0f : z[it][i];
        worker_sum<WV, 1>(s, lds, slot);
        m = s[0] / width;
        s[0] = 0.0f;
    }
#pragma unroll
    for (int it = 0; it < IT; ++it) {
        const int lo = Row<WV, IT>::low(it, width);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float d = i < lo ? 0.0f : z[it][i] - m;
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
    const int64_t t = A.first_token + R::worker();
    if (WV == 1 && t >= A.tokens) return;
    int slot = 0;
    float r[IT][8];
    float mu2 = 0.0f, rs2 = 0.0f, mu1 = 0.0f, rs1 = 0.0f;
#pragma unroll
    for (int it = 0; it < IT; ++it) {
        const Eight<TX> x = get8<TX, WV>(A.x, t * A.ld_x, R::col(it, A.width), R::low(it, A.width), A.width);
#pragma unroll
        for (int i = 0; i < 8; ++i) r[it][i] = x[i];
    }
    if (A.y) {
        float y[IT][8];
#pragma unroll
        for (int it = 0; it < IT; ++it) {
            const Eight<TY> w = get8<TY, WV>(A.y, t * A.ld_y, R::col(it, A.width), R::low(it, A.width), A.width);
#pragma unroll
            for (int i = 0; i < 8; ++i) y[it][i] = w[i];
        }
        moments<WV, IT>(y, A.width, A.layer, A.eps, lds, slot, &mu2, &rs2);
        const int64_t row = t / A.gate_rows;
#pragma unroll
        for (int it = 0; it < IT; ++it) {
            const int c = R::col(it, A.width), lo = R::low(it, A.width);
            Eight<TY> w, b, g;
            if (A.w_post) w = get8<TY, WV>(A.w_post, 0, c, lo, A.width);
            if (A.b_post) b = get8<TY, WV>(A.b_post, 0, c, lo, A.width);
            if (A.gate) g = get8<TY, WV>(A.gate, row * A.ld_gate, c, lo, A.width);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float v = (y[it][i] - mu2) * rs2;
                if (A.w_post) v *= w[i];
                if (A.b_post) v += b[i];
                r[it][i] += A.scale * (A.gate ? g[i] : 1.0f) * v;
                if (i < lo) r[it][i] = 0.0f;
            }
            put8<TX>(A.r, t * A.ld_r, c, lo, r[it]);
        }
    }
    if (A.n) {
        moments<WV, IT>(r, A.width, A.layer, A.eps, lds, slot, &mu1, &rs1);
#pragma unroll
        for (int it = 0; it < IT; ++it) {
            const int c = R::col(it, A.width), lo = R::low(it, A.width);
            Eight<TY> w, b;
            if (A.w_pre) w = get8<TY, WV>(A.w_pre, 0, c, lo, A.width);
            if (A.b_pre) b = get8<TY, WV>(A.b_pre, 0, c, lo, A.width);
            float n[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                n[i] = (r[it][i] - mu1) * rs1;
                if (A.w_pre) n[i] *= w[i];
                if (A.b_pre) n[i] += b[i];
            }
            put8<TY>(A.n, t * A.ld_n, c, lo, n);
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

// What the backward pass reads of a row.
template <typename TY, typename TX, int WV, int IT>
struct BackRow {
    Eight<TY> dn[IT], y[IT];
    Eight<TX> res[IT], dr[IT];
    float st[4];
    __device__ __forceinline__ void load(const NormArgs& A, int64_t t)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) st[i] = A.stats[t * 4 + i];
#pragma unroll
        for (int it = 0; it < IT; ++it) {
            const int c = Row<WV, IT>::col(it, A.width), lo = Row<WV, IT>::low(it, A.width);
            if (A.dn) {
                dn[it] = get8<TY, WV>(A.dn, t * A.ld_dn, c, lo, A.width);
                res[it] = get8<TX, WV>(A.res, t * A.ld_res, c, lo, A.width);
            }
            if (A.y) y[it] = get8<TY, WV>(A.y, t * A.ld_y, c, lo, A.width);
            if (A.dr) dr[it] = get8<TX, WV>(A.dr, t * A.ld_dr, c, lo, A.width);
        }
    }
};

// A worker goes down rows_each rows.  AHEAD: the next row's values are on their
// way while it works on one, and the weights stay in registers.  Otherwise it
// reads each value where it uses it, twice from a cache: with 16 waves there are
// 128 registers a thread, and two blocks of 8 waves on a compute unit need as few
// (16384 x 4096: 225 us with 135 registers and one block, 190 with 128, though 9 of
// them spill, with a float stream 16).  The form of 8 waves and 16 values a thread
// spills 14 to 17, of float32 values with biases 70.
// Past 8192 columns the column sums have no place either (a form that kept them
// spilled up to 1.3 KB a thread, 4096 x 12288 501 us; 289 so): the rows' means
// are left for norm_sums_kernel, which reads four of the six matrices once more.
template <typename TY, typename TX, int WV, int IT, bool BIAS>
__global__ __launch_bounds__((Row<WV, IT>::kThreads), (WV == 16 || (WV == 8 && IT == 1 && !BIAS && sizeof(TY) == 2) ? 4 : 2))
void norm_backward_kernel(const NormArgs A)
{
    typedef Row<WV, IT> R;
    constexpr bool AHEAD = IT == 1 && WV < 16, SUMS = IT == 1 || WV < 16;
    __shared__ float lds[2][WV][2];
    const int64_t me = R::worker();
    if (me >= A.workers) return;
    const int64_t t0 = me * A.rows_each, t1 = min(t0 + A.rows_each, A.tokens);
    int slot = 0;
    constexpr int SB = BIAS && SUMS ? IT : 1, SI = SUMS ? IT : 1;
    float s_w1[SI][8], s_w2[SI][8], s_g[SI][8], s_b1[SB][8], s_b2[SB][8];
    if (SUMS)
#pragma unroll
        for (int it = 0; it < SI; ++it)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                s_w1[it][i] = s_w2[it][i] = s_g[it][i] = 0.0f;
                if (BIAS) s_b1[it % SB][i] = s_b2[it % SB][i] = 0.0f;
            }
    const float inv = 1.0f / A.width;
    const int64_t first = t0 / A.gate_rows;
    int64_t row = -1;
    Eight<TY> w1[IT], w2[IT], gt[IT];
    auto read_w1 = [&](int it) { if (A.w_pre) w1[it] = get8<TY, WV>(A.w_pre, 0, R::col(it, A.width), R::low(it, A.width), A.width); };
    auto read_w2 = [&](int it) { if (A.w_post) w2[it] = get8<TY, WV>(A.w_post, 0, R::col(it, A.width), R::low(it, A.width), A.width); };
    auto read_gate = [&](int it) {
        if (A.gate) gt[it] = get8<TY, WV>(A.gate, row * A.ld_gate, R::col(it, A.width), R::low(it, A.width), A.width);
    };
    if (AHEAD)
#pragma unroll
        for (int it = 0; it < IT; ++it) {
            read_w1(it);
            read_w2(it);
        }
    // dgate of the gate row that ends here: to its place if the worker saw all of its tokens
    auto flush = [&]() {
        const bool whole = row * A.gate_rows >= t0 && min((row + 1) * A.gate_rows, A.tokens) <= t1;
#pragma unroll
        for (int it = 0; it < SI; ++it) {
            const int c = R::col(it, A.width), lo = R::low(it, A.width);
            if (whole) {
                put8<TY>(A.dgate, row * A.width, c, lo, s_g[it]);
            } else {
                put8<float>(A.part, (me * kNormSums + (row == first ? 4 : 5)) * A.width, c, lo, s_g[it]);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) s_g[it][i] = 0.0f;
        }
    };
    BackRow<TY, TX, WV, IT> now, ahead;
    if (AHEAD) ahead.load(A, t0);
    for (int64_t t = t0; t < t1; ++t) {
        if (A.gate && t / A.gate_rows != row) {
            if (SUMS && row >= 0 && A.dgate) flush();
            row = t / A.gate_rows;
            if (AHEAD)
#pragma unroll
                for (int it = 0; it < IT; ++it) read_gate(it);
        }
        if (AHEAD) {
            now = ahead;
            if (t + 1 < t1) ahead.load(A, t + 1);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) now.st[i] = A.stats[t * 4 + i];
        }
        const float mu2 = now.st[0], rs2 = now.st[1], mu1 = now.st[2], rs1 = now.st[3];
        auto read_n = [&](int it) {
            const int c = R::col(it, A.width), lo = R::low(it, A.width);
            if (AHEAD) return;
            now.dn[it] = get8<TY, WV>(A.dn, t * A.ld_dn, c, lo, A.width);
            now.res[it] = get8<TX, WV>(A.res, t * A.ld_res, c, lo, A.width);
            read_w1(it);
        };
        auto read_y = [&](int it) {
            if (AHEAD) return;
            now.y[it] = get8<TY, WV>(A.y, t * A.ld_y, R::col(it, A.width), R::low(it, A.width), A.width);
        };
        float d[IT][8];            // gradient of r
        float mz = 0.0f, mq = 0.0f;
        if (A.dn) {
            float m[2] = {0.0f, 0.0f};
#pragma unroll
            for (int it = 0; it < IT; ++it) {
                const int lo = R::low(it, A.width);
                read_n(it);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float g = now.dn[it][i], z = (now.res[it][i] - mu1) * rs1;
                    const float q = A.w_pre ? g * w1[it][i] : g;
                    if (i >= lo) {
                        m[0] += q * z;
                        m[1] += q;
                    }
                    if (SUMS) s_w1[it % SI][i] += g * z;
                    if (SUMS && BIAS) s_b1[it % SB][i] += g;
                }
            }
            worker_sum<WV, 2>(m, lds, slot);
            mz = m[0] * inv;
            mq = A.layer ? m[1] * inv : 0.0f;
        }
        if (!SUMS && threadIdx.x == 0) {
            A.means[t * 2] = mz;
            A.means[t * 2 + 1] = mq;
        }
#pragma unroll
        for (int it = 0; it < IT; ++it) {
            const int c = R::col(it, A.width), lo = R::low(it, A.width);
            if (!AHEAD && A.dr) now.dr[it] = get8<TX, WV>(A.dr, t * A.ld_dr, c, lo, A.width);
            if (A.dn) read_n(it);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                d[it][i] = A.dr ? now.dr[it][i] : 0.0f;
                if (A.dn) {
                    const float g = now.dn[it][i], z = (now.res[it][i] - mu1) * rs1;
                    const float q = A.w_pre ? g * w1[it][i] : g;
                    d[it][i] += rs1 * (q - z * mz - mq);
                }
            }
            if (A.dx && (SUMS || A.dx != A.dr)) put8<TX>(A.dx, t * A.ld_dx, c, lo, d[it]);
        }
        if (!A.y) continue;
        float m[2] = {0.0f, 0.0f};
#pragma unroll
        for (int it = 0; it < IT; ++it) {
            const int lo = R::low(it, A.width);
            Eight<TY> b2;
            if (SUMS && BIAS && A.b_post) b2 = get8<TY, WV>(A.b_post, 0, R::col(it, A.width), lo, A.width);
            read_y(it);
            if (!AHEAD) {
                read_w2(it);
                read_gate(it);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float z = (now.y[it][i] - mu2) * rs2;
                const float w = A.w_post ? w2[it][i] : 1.0f;
                const float b = SUMS && BIAS && A.b_post ? b2[i] : 0.0f;
                const float sd = A.scale * d[it][i];
                if (SUMS) s_g[it % SI][i] += sd * (z * w + b);
                const float dv = A.gate ? sd * gt[it][i] : sd;
                if (SUMS) s_w2[it % SI][i] += dv * z;
                if (SUMS && BIAS) s_b2[it % SB][i] += dv;
                const float q = dv * w;
                d[it][i] = q;
                if (i >= lo) {
                    m[0] += q * z;
                    m[1] += q;
                }
            }
        }
        worker_sum<WV, 2>(m, lds, slot);
        mz = m[0] * inv;
        mq = A.layer ? m[1] * inv : 0.0f;
        if (A.dy)
#pragma unroll
            for (int it = 0; it < IT; ++it) {
                read_y(it);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float z = (now.y[it][i] - mu2) * rs2;
                    d[it][i] = rs2 * (d[it][i] - z * mz - mq);
                }
                put8<TY>(A.dy, t * A.ld_dy, R::col(it, A.width), R::low(it, A.width), d[it]);
            }
    }
    if (!SUMS) return;
    if (A.dgate && row >= 0) flush();
#pragma unroll
    for (int it = 0; it < SI; ++it) {
        const int c = R::col(it, A.width), lo = R::low(it, A.width);
        const int64_t at = me * kNormSums * A.width;
        if (A.dw_pre) put8<float>(A.part, at, c, lo, s_w1[it]);
        if (BIAS && A.db_pre) put8<float>(A.part, at + A.width, c, lo, s_b1[it % SB]);
        if (A.dw_post) put8<float>(A.part, at + 2 * (int64_t)A.width, c, lo, s_w2[it]);
        if (BIAS && A.db_post) put8<float>(A.part, at + 3 * (int64_t)A.width, c, lo, s_b2[it % SB]);
    }
}

// The workers' column sums of wide rows, from the means of dn w_pre rhat (and of
// dn w_pre) that the rows' pass left: a thread owns 8 columns and goes down a
// worker's rows.  dx over dr is written here and not by the rows' pass: the sums
// take the gradient of r as it is before it is rounded, so they need dr.
template <typename TY, typename TX, bool BIAS>
__global__ __launch_bounds__(256) void norm_sums_kernel(const NormArgs A)
{
    const int c = column_of(blockIdx.x * 256 + threadIdx.x, A.width);
    const int lo = low_of(blockIdx.x * 256 + threadIdx.x, A.width);
    if (lo == 8) return;
    const int64_t me = blockIdx.y, t0 = me * A.rows_each, t1 = min(t0 + A.rows_each, A.tokens);
    float s_w1[8] = {}, s_w2[8] = {}, s_g[8] = {}, s_b1[8] = {}, s_b2[8] = {};
    Eight<TY> w1, w2, b2, gt;
    if (A.w_pre) w1 = get8<TY, 16>(A.w_pre, 0, c, lo, A.width);
    if (A.w_post) w2 = get8<TY, 16>(A.w_post, 0, c, lo, A.width);
    if (BIAS && A.b_post) b2 = get8<TY, 16>(A.b_post, 0, c, lo, A.width);
    const bool over = A.dx && A.dx == A.dr;
    const int64_t first = t0 / A.gate_rows;
    int64_t row = -1;
    auto flush = [&]() {
        const bool whole = row * A.gate_rows >= t0 && min((row + 1) * A.gate_rows, A.tokens) <= t1;
        if (whole) put8<TY>(A.dgate, row * A.width, c, lo, s_g);
        else put8<float>(A.part, (me * kNormSums + (row == first ? 4 : 5)) * A.width, c, lo, s_g);
#pragma unroll
        for (int i = 0; i < 8; ++i) s_g[i] = 0.0f;
    };
#pragma unroll 2
    for (int64_t t = t0; t < t1; ++t) {
        if (A.gate && t / A.gate_rows != row) {
            if (row >= 0 && A.dgate) flush();
            row = t / A.gate_rows;
            gt = get8<TY, 16>(A.gate, row * A.ld_gate, c, lo, A.width);
        }
        const float *st = A.stats + t * 4, *means = A.means + t * 2;
        const float mu2 = st[0], rs2 = st[1], mu1 = st[2], rs1 = st[3], mz = means[0], mq = means[1];
        Eight<TY> dn, y;
        Eight<TX> res, dr;
        if (A.dn) {
            dn = get8<TY, 16>(A.dn, t * A.ld_dn, c, lo, A.width);
            res = get8<TX, 16>(A.res, t * A.ld_res, c, lo, A.width);
        }
        if (A.y) y = get8<TY, 16>(A.y, t * A.ld_y, c, lo, A.width);
        if (A.dr) dr = get8<TX, 16>(A.dr, t * A.ld_dr, c, lo, A.width);
        float dx[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float d = A.dr ? dr[i] : 0.0f;
            if (A.dn) {
                const float g = dn[i], z = (res[i] - mu1) * rs1, q = A.w_pre ? g * w1[i] : g;
                d += rs1 * (q - z * mz - mq);
                s_w1[i] += g * z;
                if (BIAS) s_b1[i] += g;
            }
            dx[i] = d;
            if (!A.y) continue;
            const float z = (y[i] - mu2) * rs2, sd = A.scale * d;
            s_g[i] += sd * (z * (A.w_post ? w2[i] : 1.0f) + (BIAS && A.b_post ? b2[i] : 0.0f));
            const float dv = A.gate ? sd * gt[i] : sd;
            s_w2[i] += dv * z;
            if (BIAS) s_b2[i] += dv;
        }
        if (over) put8<TX>(A.dx, t * A.ld_dx, c, lo, dx);
    }
    if (A.dgate && row >= 0) flush();
    const int64_t at = me * kNormSums * A.width;
    if (A.dw_pre) put8<float>(A.part, at, c, lo, s_w1);
    if (BIAS && A.db_pre) put8<float>(A.part, at + A.width, c, lo, s_b1);
    if (A.dw_post) put8<float>(A.part, at + 2 * (int64_t)A.width, c, lo, s_w2);
    if (BIAS && A.db_post) put8<float>(A.part, at + 3 * (int64_t)A.width, c, lo, s_b2);
}

// Joins the workers' column sums: blockIdx.y < 4 the weights and biases, above
// that the gate rows that several workers share.  A block takes COLS columns,
// its threads share the workers: 16 columns where rows are narrow, so that
// enough blocks are at work (16384 x 512: 36 us with 64).
template <typename TY, int COLS>
__global__ __launch_bounds__(1024) void norm_join_kernel(const NormArgs A)
{
    constexpr int kShare = 1024 / COLS;
    __shared__ float lds[kShare][COLS];
    const int lane = threadIdx.x % COLS, part = threadIdx.x / COLS;
    const int c = blockIdx.x * COLS + lane;
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
#pragma unroll 8
        for (int64_t w = w0 + part; w < w1; w += kShare) {
            const int which = blockIdx.y < 4 ? blockIdx.y : (w * A.rows_each / A.gate_rows == row ? 4 : 5);
            s += A.part[(w * kNormSums + which) * A.width + c];
        }
    lds[part][lane] = s;
    for (int half = kShare / 2; half >= 1; half /= 2) {
        __syncthreads();
        if (part < half) lds[part][lane] += lds[part + half][lane];
    }
    if (part == 0 && c < A.width) out[c] = (TY)lds[0][lane];
}

// Waves of a worker by width, 8 values a thread up to 4096 columns.  Past that the
// forward takes 16 or 32 a thread; the backward 16 waves (of 8 or 16 values), or 8 of
// 16 values where two more sums or 32-bit values would not fit 128 registers
// (8192 x 8192 with biases: 560 us with 16 waves, 474 with 8; without 249 and 311).
int waves_of(int width) { return width <= 512 ? 1 : width <= 2048 ? 4 : 8; }

template <typename TY, typename TX>
hipError_t forward(const NormArgs& A, hipStream_t s)
{
    const int64_t n = A.tokens - A.first_token;
    switch (waves_of(A.width)) {
    case 1: norm_forward_kernel<TY, TX, 1, 1><<<(unsigned)((n + 3) / 4), 256, 0, s>>>(A); break;
    case 4: norm_forward_kernel<TY, TX, 4, 1><<<(unsigned)n, 256, 0, s>>>(A); break;
    default:
        if (A.width <= 4096) norm_forward_kernel<TY, TX, 8, 1><<<(unsigned)n, 512, 0, s>>>(A);
        else if (A.width <= 8192) norm_forward_kernel<TY, TX, 8, 2><<<(unsigned)n, 512, 0, s>>>(A);
        else norm_forward_kernel<TY, TX, 8, 4><<<(unsigned)n, 512, 0, s>>>(A);
    }
    return hipGetLastError();
}

template <typename TY, typename TX, bool BIAS>
hipError_t backward(const NormArgs& A, hipStream_t s)
{
    const unsigned n = (unsigned)A.workers;
    if (n) switch (waves_of(A.width)) {
    case 1: norm_backward_kernel<TY, TX, 1, 1, BIAS><<<(n + 3) / 4, 256, 0, s>>>(A); break;
    case 4: norm_backward_kernel<TY, TX, 4, 1, BIAS><<<n, 256, 0, s>>>(A); break;
    default:
        if (A.width <= 4096) norm_backward_kernel<TY, TX, 8, 1, BIAS><<<n, 512, 0, s>>>(A);
        else if (A.width > kNormSumsWidth) norm_backward_kernel<TY, TX, 16, 2, BIAS><<<n, 1024, 0, s>>>(A);
        else if constexpr (BIAS || sizeof(TY) == 4) norm_backward_kernel<TY, TX, 8, 2, BIAS><<<n, 512, 0, s>>>(A);
        else norm_backward_kernel<TY, TX, 16, 1, BIAS><<<n, 1024, 0, s>>>(A);
    }
    if (n && A.width > kNormSumsWidth)
        norm_sums_kernel<TY, TX, BIAS><<<dim3((A.width + 2047) / 2048, n), 256, 0, s>>>(A);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    // rows_each is a multiple of gate_rows or less than it: only then gate rows are shared
    const int64_t rows = !A.dgate ? 0 : A.tokens == 0 ? 1
                         : A.gate_rows > A.rows_each ? (A.tokens + A.gate_rows - 1) / A.gate_rows : 0;
    if (A.width <= 2048)
        norm_join_kernel<TY, 16><<<dim3((A.width + 15) / 16, (unsigned)(4 + rows)), 1024, 0, s>>>(A);
    else
        norm_join_kernel<TY, 64><<<dim3((A.width + 63) / 64, (unsigned)(4 + rows)), 1024, 0, s>>>(A);
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
    const int64_t most = width <= 512 ? 2048 : width <= kNormSumsWidth ? 512 : 256;
    int64_t each = (tokens + most - 1) / most;
    if (each < 1) each = 1;
    if (gate_rows <= each) each = (each + gate_rows - 1) / gate_rows * gate_rows;
    *rows_each = (int)each;
    *workers = (int)((tokens + each - 1) / each);
}

namespace {

hipError_t forward_any(const NormArgs& A, int dtype, int stream_dtype, hipStream_t s)
{
    if (dtype == ARENA_F32) return forward<float, float>(A, s);
    if (dtype == ARENA_BF16)
        return stream_dtype == ARENA_F32 ? forward<__bf16, float>(A, s) : forward<__bf16, __bf16>(A, s);
    return stream_dtype == ARENA_F32 ? forward<_Float16, float>(A, s) : forward<_Float16, _Float16>(A, s);
}

}  // namespace

hipError_t launch_norm_forward(const NormArgs& A, int dtype, int stream_dtype, hipStream_t s)
{
    // a launch holds less than 2^32 threads
    constexpr int64_t kMost = 1 << 22;
    NormArgs part = A;
    for (int64_t t = 0; t < A.tokens; t += kMost) {
        part.first_token = t;
        part.tokens = A.tokens - t < kMost ? A.tokens : t + kMost;
        const hipError_t e = forward_any(part, dtype, stream_dtype, s);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

hipError_t launch_norm_backward(const NormArgs& A, int dtype, int stream_dtype, hipStream_t s)
{
    if (dtype == ARENA_F32) return backward_any<float, float>(A, s);
    if (dtype == ARENA_BF16)
        return stream_dtype == ARENA_F32 ? backward_any<__bf16, float>(A, s) : backward_any<__bf16, __bf16>(A, s);
    return stream_dtype == ARENA_F32 ? backward_any<_Float16, float>(A, s) : backward_any<_Float16, _Float16>(A, s);
}

}  // namespace arena
