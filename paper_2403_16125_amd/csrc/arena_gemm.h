// Tiled matrix products on the matrix cores, with the epilogues of the layer
// operators.  C[m, n] = sum_k A(m, k) B(n, k), 16-bit operands, 32-bit sums.
//
// Each operand lies either with k contiguous (row m or n of ld elements) or
// with m or n contiguous (row k of ld elements), so the forward, data-gradient
// and weight-gradient products of a layer read the tensors as they are: no
// transposed copies.
//
// A block computes a BM x BN tile with WM x WN waves, 64 of k at a time, from
// two or four LDS buffers: while one is multiplied, the others are filled by
// direct global-to-LDS loads.  Those write 16 bytes per lane in lane order, so
// the bank swizzle sits on the global side (which chunk a lane fetches):
//   k contiguous: row r of 8 chunks; position p holds chunk p ^ (r & 7), and a
//     fragment read (16 rows, one chunk each) meets every bank once;
//   m or n contiguous: row k of R / 16 granules of 32 bytes; position q holds
//     granule q ^ f(k), f = (k & 3) | ((k >> 3) & 3) << 2, so the 16 rows that
//     one transposing read touches lie in different granules.
// The product is formed transposed (the B fragment is the first operand), so a
// lane holds four neighbouring columns of one row of C, and eight after a trip
// through LDS.
//
// Large products are bound by the matrix cores and the clock that the power
// leaves them (the plain ones issue products in 59 to 66 % of the compute units'
// cycles, those with gated epilogues in 49 to 57 %, the mirrored ones of an update
// in 51 to 55 %; LDS is busy for 20 to 34 %), and by each tile's start and end, since one
// block of 256 x 256 fits a compute unit.  8192 x 4096 x 10944 in bfloat16: 585 to 600 us (1220 to
// 1250 TFLOP/s), with two segments of k 1090 to 1110 us (1320 to 1350), with the
// gated forward epilogue on twice the columns 1230 to 1270 us (1160 to 1190), as
// a weight gradient 626 to 660 us.  Small ones are bound by latency: a block of
// 128 x 128 (64 x 64) takes 6 (3.5) us for its start, first loads and epilogue
// and 0.45 (0.28) us for a step of 64 of k, and operands that another kernel has
// just written cost up to twice that a step.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "arena_layer_internal.h"

namespace arena {
namespace mm {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

struct Bf16 {
    typedef __bf16 E;
    typedef __bf16 V8 __attribute__((ext_vector_type(8)));
    typedef __bf16 V4 __attribute__((ext_vector_type(4)));
    static __device__ __forceinline__ f32x4 mfma(V8 a, V8 b, f32x4 c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
    }
};

struct F16 {
    typedef _Float16 E;
    typedef _Float16 V8 __attribute__((ext_vector_type(8)));
    typedef _Float16 V4 __attribute__((ext_vector_type(4)));
    static __device__ __forceinline__ f32x4 mfma(V8 a, V8 b, f32x4 c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
    }
};

// act(z), and with it act'(z).  Reciprocals and exponentials are the hardware's.  An
// exponential of e is off by about |e| 2^-24 of itself (e^-80 by 2^-17), inside the 8
// or 11 bits that results keep.  The normal distribution function is erfc(-z / sqrt 2) / 2,
// exact to a few units for negative z too, where (1 + erf(z / sqrt 2)) / 2 cancels:
// 1e-3 of the value at -4, all of it below -5.4.
//
// kGeluShort is the same function in a fifth of the operations, without branches, for the
// experts' products, whose epilogues are a large share of their time.  With t = |z| the
// distribution function at -t is exp(-t^2 / 2) R(t), R half of the scaled complementary error
// function of t / sqrt 2: smooth, and in s = 1 / (1 + 0.3 t) a polynomial of degree 8 to 9e-8
// of itself for t up to 13.5, past which the exponential is below float's range (coefficients
// by a weighted least-squares fit with the weights moved to the largest errors).  The rounding
// of t^2, of -1 / (2 log 2) and of the exponential's argument is carried along.  With reciprocal and exponential
// rounded to nearest q is off by 4.0e-7 of itself at most on 260001 points (the roundings add up to 6.4e-7 at worst;
// a whole unit of either function makes it 7.5e-7).
__device__ __forceinline__ void normal_below(float t, float* q, float* e)
{
    const float s = __builtin_amdgcn_rcpf(__builtin_fmaf(0.3f, t, 1.0f)), c = -0.72134752044448170f;
    const float square = t * t, rest = __builtin_fmaf(t, t, -square);
    const float c_rest = -9.6298149e-9f;                 // -1 / (2 log 2) less c
    const float y = square * c, off = __builtin_fmaf(square, c_rest, __builtin_fmaf(rest, c, __builtin_fmaf(square, c, -y)));
    const float two = __builtin_amdgcn_exp2f(y);
    // past 2^127 the rest of the square is no number, and the exponential 0
    *e = y > -150.0f ? __builtin_fmaf(two, off * 0.69314718055994531f, two) : y == y ? 0.0f : y;
    float r = 0.03833426535129547f;
    r = __builtin_fmaf(r, s, -0.16895195841789246f);
    r = __builtin_fmaf(r, s, 0.22821730375289917f);
    r = __builtin_fmaf(r, s, -0.07599958777427673f);
    r = __builtin_fmaf(r, s, 0.1421850472688675f);
    r = __builtin_fmaf(r, s, 0.09483297914266586f);
    r = __builtin_fmaf(r, s, 0.12188205122947693f);
    r = __builtin_fmaf(r, s, 0.11949306726455688f);
    r = __builtin_fmaf(r, s, 6.852919796074275e-06f);
    *q = *e * r;
}

template <int ACT>
__device__ __forceinline__ float act_value(float z)
{
    if (ACT == kGeluShort) {
        float q, e;
        normal_below(__builtin_fabsf(z), &q, &e);
        return z * (z < 0.0f ? q : 1.0f - q);
    }
    if (ACT == kSilu) return z * __builtin_amdgcn_rcpf(1.0f + __expf(-z));
    if (ACT == kGelu) return 0.5f * z * erfcf(z * -0.70710678118654752f);
    return z > 0.0f ? z : (z == z ? 0.0f : z);
}

template <int ACT>
__device__ __forceinline__ void act_both(float z, float* v, float* d)
{
    if (ACT == kGeluShort) {
        float q, e;
        normal_below(__builtin_fabsf(z), &q, &e);
        const float c = z < 0.0f ? q : 1.0f - q;
        *v = z * c;
        *d = c + z * e * 0.39894228040143268f;
    } else if (ACT == kSilu) {
        const float s = __builtin_amdgcn_rcpf(1.0f + __expf(-z));
        *v = z * s;
        *d = s + *v * (1.0f - s);
    } else if (ACT == kGelu) {
        const float c = 0.5f * erfcf(z * -0.70710678118654752f);
        *v = z * c;
        *d = c + z * __expf(-0.5f * z * z) * 0.39894228040143268f;
    } else {
        *v = z > 0.0f ? z : (z == z ? 0.0f : z);
        *d = z > 0.0f ? 1.0f : (z == z ? 0.0f : z);
    }
}

__device__ const u32x4 g_zero_chunk = {0, 0, 0, 0};   // what a lane past the end of k fetches

typedef __attribute__((address_space(1))) const void GlobalVoid;
typedef __attribute__((address_space(3))) void LdsVoid;

__device__ __forceinline__ void load_to_lds(const char* src, char* dst)
{
    __builtin_amdgcn_global_load_lds((GlobalVoid*)src, (LdsVoid*)dst, 16, 0, 0);
}

// Which matrix and row a row of the B tile is.  In the gated forward product a
// wave's rows are gate features, then as many up features, so one wave holds
// both of a feature.
template <int W>        // rows of a wave
struct Dual {
    static __device__ __forceinline__ int row(int r) { return r / W * (W / 2) + r % (W / 2); }
    static __device__ __forceinline__ int up(int r) { return r / (W / 2) & 1; }
};

// One operand's share of a tile: R rows of C (or columns) x 64 of k.
template <typename P, int R, bool TR, bool DUAL>
struct Loader {
    static constexpr int kThreads = P::kThreads;
    static constexpr int kChunks = R * 8 / kThreads;
    static constexpr int kGran = R / 16;
    uint32_t off[kChunks];   // byte offset of this lane's chunk from the segment's base at step 0
    int64_t step;            // bytes from one step to the next
    int row0, ld;

    static __device__ __forceinline__ int k_of(int it, int tid)   // k of the chunk within the step
    {
        if (TR) return (it * kThreads + tid) / (R / 8);
        const int r = it * (kThreads / 8) + (tid >> 3);
        return ((tid & 7) ^ (r & 7)) * 8;
    }

    __device__ __forceinline__ void init(int tid, int first, int n, int64_t ld_)
    {
        ld = (int)ld_;
        row0 = first;
        step = TR ? ld_ * (2 * kBK) : 2 * kBK;
#pragma unroll
        for (int it = 0; it < kChunks; ++it) {
            if (TR) {
                const int c = it * kThreads + tid;
                const int k = c / (R / 8), pos = c % (R / 8);
                const int f = ((k & 3) | (((k >> 3) & 3) << 2)) & (kGran - 1);
                int col = first + (((pos >> 1) ^ f) << 4) + ((pos & 1) << 3);
                if (col >= n) col = 0;
                off[it] = (uint32_t)k * (uint32_t)(ld * 2) + (uint32_t)col * 2;
            } else {
                const int r = it * (kThreads / 8) + (tid >> 3);
                const int row = min(first + (DUAL ? Dual<P::BN / P::WN>::row(r) : r), n - 1) - first;
                off[it] = (uint32_t)row * (uint32_t)(ld * 2) + (uint32_t)(((tid & 7) ^ (r & 7)) << 4);
            }
        }
    }

    // base of step 0 of a segment
    __device__ __forceinline__ const char* base(const void* p, int64_t batch) const
    {
        const char* q = (const char*)p + 2 * batch;
        return TR ? q : q + 2 * (int64_t)row0 * ld;
    }

    // TAIL: lanes past the end of k (`left` of it remain) fetch zeros.
    template <bool TAIL>
    __device__ __forceinline__ void fetch(const char* p0, const char* p1, char* lds, int tid, int left) const
    {
        const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
#pragma unroll
        for (int it = 0; it < kChunks; ++it) {
            const char* p = p0;
            if (DUAL) p = Dual<P::BN / P::WN>::up(it * (kThreads / 8) + wave * 8) ? p1 : p0;
            const char* src = p + off[it];
            if (TAIL && k_of(it, tid) >= left) src = (const char*)&g_zero_chunk;
            load_to_lds(src, lds + (it * kThreads + wave * 64) * 16);
        }
    }
};

// A wave's fragment reader: 16 rows x 32 of k for one MFMA.
template <typename P, int R, bool TR>
struct Frags {
    typedef typename P::T::V8 V8;
    typedef typename P::T::V4 V4;
    int lo;      // byte address of fragment 0, first half of the step
    __device__ __forceinline__ void init(int lane, int row)
    {
        if (TR) {
            const int i = lane & 15, g = lane >> 4;
            const int f = ((i >> 2) | (g << 2)) & (R / 16 - 1);
            lo = (g * 8 + (i >> 2)) * (R * 2) + (((row >> 4) ^ f) << 5) + (i & 3) * 8;
        } else {
            const int r = row + (lane & 15);
            lo = r * 128 + (((lane >> 4) ^ (r & 7)) << 4);
        }
    }
    // fragment i (rows row + 16 i), half kk of the step
    __device__ __forceinline__ V8 get(const char* lds, int i, int kk) const
    {
        if (TR) {
            typedef __attribute__((address_space(3))) s16x4 LdsV;
            const char* p = lds + ((lo ^ (i << 5)) + kk * 32 * (R * 2));
            union { s16x4 s[2]; V8 v; } w;
            w.s[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsV*)p);
            w.s[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsV*)(p + 4 * (R * 2)));
            return w.v;
        }
        return *(const V8*)(lds + ((lo ^ (kk << 6)) + i * 2048));
    }
};

template <typename T_, int BM_, int BN_, int WM_, int WN_, int STAGES_, bool ATR_, bool BTR_, int EPI_>
struct Tile {
    typedef T_ T;
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_;
    static constexpr bool ATR = ATR_, BTR = BTR_, DUAL = EPI_ == kGatedFwd;
    static constexpr int EPI = EPI_;
    static constexpr int kThreads = 64 * WM * WN;
    static constexpr int kStages = STAGES_;
    // With few blocks on a compute unit a wave that issues its loads in a row
    // leaves the matrix cores idle (128 x 128, four buffers: 0.72 us a step, woven
    // between the products 0.54); with many, the others fill the gap and the
    // comparisons cost more than they bring (8192 x 4096 x 10944: 550 us, woven 582).
    static constexpr bool kWoven = STAGES_ > 2;
    // waves a SIMD, for the register limit: one block on a compute unit, or two by their LDS
    static constexpr int kWavesEach = kThreads / 256 * (kStages * (BM + BN) * 128 <= 81920 ? 2 : 1);
    static constexpr int FM = BM / WM / 16, FN = BN / WN / 16;
    static constexpr int kCols = DUAL ? BN / 2 : BN;     // columns of C of a tile
};

// C neighbouring values of a row, `left` of them inside the matrix.  Rows may
// start on any value: the wide accesses are unaligned where they do not.
template <typename E, int C>
__device__ __forceinline__ void put(E* p, const float (&v)[C], int left)
{
    if (left >= C) {
        E w[C];
#pragma unroll
        for (int r = 0; r < C; ++r) w[r] = (E)v[r];
        __builtin_memcpy(p, w, sizeof(w));
    } else {
        for (int r = 0; r < C; ++r)
            if (r < left) p[r] = (E)v[r];
    }
}

template <typename E, int C>
__device__ __forceinline__ void get(const E* p, float (&v)[C], int left)
{
    if (left >= C) {
        E w[C];
        __builtin_memcpy(w, p, sizeof(w));
#pragma unroll
        for (int r = 0; r < C; ++r) v[r] = (float)w[r];
    } else {
        for (int r = 0; r < C; ++r) v[r] = r < left ? (float)p[r] : 0.0f;
    }
}

// What an epilogue reads from memory for eight columns, apart from using it, so
// that several reads are in flight.
template <typename T, int EPI>
struct Side;

// plain: the added matrix, as it lies in memory (16-bit values in raw[0]).
template <typename T>
struct Side<T, kPlain> {
    u32x4 raw[2];
    __device__ __forceinline__ void load(const GemmArgs& A, int z, int m, int n)
    {
        if (A.beta == 0.0f) return;
        const char* p = (const char*)A.e[A.pairs ? z : 0];
        const int64_t from = (A.pairs ? 0 : z * A.se) + (int64_t)m * A.lde + n;
        const int left = A.N - n;
        if (A.out == kOutF32) {
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
struct Side<T, kGatedFwd> {
    __device__ __forceinline__ void load(const GemmArgs&, int, int, int) {}
};

// gated, backward: the heads and tails of the kept gate and up values.
template <typename T>
struct Side<T, kGatedBwd> {
    u32x4 gh, uh;
    u32x2 gt, ut;
    __device__ __forceinline__ void load(const GemmArgs& A, int, int m, int n)
    {
        const int64_t at = (int64_t)m * A.ldg + n, tails = 2 * (int64_t)A.M * A.ldg + at;
        gh = *(const u32x4*)((const uint16_t*)A.g + at);
        uh = *(const u32x4*)((const uint16_t*)A.u + at);
        gt = *(const u32x2*)((const uint8_t*)A.g + tails);
        ut = *(const u32x2*)((const uint8_t*)A.u + tails);
    }
    static __device__ __forceinline__ float value(u32x4 head, u32x2 tail, int r)
    {
        const uint32_t high = r & 1 ? 0x07060000 : 0x05040000;      // bytes: 0, the tail, the head's two
        return __uint_as_float(__builtin_amdgcn_perm(head[r >> 1], tail[r >> 2], high | (r & 3) << 8 | 0x0c));
    }
};

// Writes eight (or, of few rows, four) columns from n, those below N, of row m;
// z is the batch index.  Leaves the values written in v.
template <typename T, int C>
__device__ __forceinline__ void plain_out(const GemmArgs& A, int z, int m, int n, float (&v)[C],
                                          const Side<T, kPlain>& side)
{
    typedef typename T::E E;
    const int left = A.N - n;
    const int64_t at = (A.pairs ? 0 : z * A.sc) + (int64_t)m * A.ldc + n;
    void* c = A.c[A.pairs ? z : 0];
#pragma unroll
    for (int r = 0; r < C; ++r) v[r] *= A.alpha;
    if (A.beta != 0.0f)
#pragma unroll
        for (int r = 0; r < C; ++r) v[r] += A.beta * side.get(r, A.out == kOutF32);
    if (A.diag != 0.0f)
#pragma unroll
        for (int r = 0; r < C; ++r)
            if (m == n + r) v[r] -= A.diag;
    if (A.out == kOutF32) put((float*)c + at, v, left);
    else if (A.out == kOutBf16) put((__bf16*)c + at, v, left);
    else put((E*)c + at, v, left);
}

// Plain, with the part of the added matrix that its 16 bits left out: the next step's
// product takes C in 16 bits, and the rest goes on beside it.
template <typename T>
struct Side<T, kPlainRest> : Side<T, kPlain> {
    u32x4 rest;
    __device__ __forceinline__ void load(const GemmArgs& A, int z, int m, int n)
    {
        Side<T, kPlain>::load(A, z, m, n);
        rest = *(const u32x4*)((const typename T::E*)A.rest + z * A.se + (int64_t)m * A.lde + n);
    }
};

template <typename T>
__device__ __forceinline__ void plain_out(const GemmArgs& A, int z, int m, int n, float (&v)[8],
                                          const Side<T, kPlainRest>& side)
{
    typedef typename T::E E;
    E w[8], c[8];
    __builtin_memcpy(w, &side.rest, sizeof(w));
    const int64_t at = z * A.sc + (int64_t)m * A.ldc + n;
#pragma unroll
    for (int r = 0; r < 8; ++r) {
        v[r] = A.alpha * v[r] + A.beta * side.get(r, false) + A.rest_in * (float)w[r];
        c[r] = (E)v[r];
        w[r] = (E)((v[r] - (float)c[r]) * 2048.0f);
    }
    __builtin_memcpy((E*)A.c[0] + at, c, sizeof(c));
    if (A.rest_out) __builtin_memcpy((E*)A.rest + at, w, sizeof(w));
}

// Values kept for the backward pass: floats rounded to their upper 24 bits (to
// nearest, ties to even), 16 in a row of heads and 8 in a row of tails (all rows of
// heads, then all of tails).  In
// 16 bits they would cost the gradients two more roundings of the operands'
// size (1.8 times the error of one rounding of the result instead of 1.4); the
// tails are a sixth of the bytes that the pass writes here.
template <int C>
__device__ __forceinline__ void put24(void* p, const GemmArgs& A, int m, int n, const float (&v)[C])
{
    const int64_t at = (int64_t)m * A.ldg + n;
    uint32_t b[C], head[C / 2], tail[C / 4];
#pragma unroll
    for (int r = 0; r < C; ++r) {
        // a NaN of operands of 16 bits has nothing in the lower 8 that could carry
        b[r] = __float_as_uint(v[r]);
        b[r] += 127 + (b[r] >> 8 & 1);
    }
#pragma unroll
    for (int r = 0; r < C; r += 2) head[r / 2] = __builtin_amdgcn_perm(b[r + 1], b[r], 0x07060302);
#pragma unroll
    for (int r = 0; r < C; r += 4)
        tail[r / 4] = __builtin_amdgcn_perm(__builtin_amdgcn_perm(b[r + 3], b[r + 2], 0x0c0c0501),
                                            __builtin_amdgcn_perm(b[r + 1], b[r], 0x0c0c0501), 0x05040100);
    __builtin_memcpy((uint16_t*)p + at, head, sizeof(head));
    __builtin_memcpy((uint8_t*)p + 2 * (int64_t)A.M * A.ldg + at, tail, sizeof(tail));
}

// h = act(g) u from the 32-bit sums, rounded to 16 bits as the next product's
// operand.  n and pad are multiples of C's and of 8, so C columns are all
// inside pad.
template <typename T, int ACT, int C>
__device__ __forceinline__ void gated_fwd(const GemmArgs& A, int m, int n, float (&g)[C], float (&u)[C])
{
    typedef typename T::E E;
    float h[C];
    if (n + C > A.N) {
        // zeros past the last column: h is 0 there too
#pragma unroll
        for (int r = 0; r < C; ++r) {
            g[r] = n + r < A.N ? g[r] : 0.0f;
            u[r] = n + r < A.N ? u[r] : 0.0f;
        }
    }
#pragma unroll
    for (int r = 0; r < C; ++r) h[r] = act_value<ACT>(g[r]) * u[r];
    put((E*)A.c[0] + (int64_t)m * A.ldc + n, h, C);
    if (A.g) {
        put24(A.g, A, m, n, g);
        put24(A.u, A, m, n, u);
    }
}

template <typename T, int GELU = kGelu, int C>
__device__ __forceinline__ void gated_fwd_out(const GemmArgs& A, int m, int n, float (&g)[C], float (&u)[C])
{
    if (A.act == kSilu) gated_fwd<T, kSilu>(A, m, n, g, u);
    else if (A.act == kGelu) gated_fwd<T, GELU>(A, m, n, g, u);
    else gated_fwd<T, kRelu>(A, m, n, g, u);
}

// v = the gradient of h = act(g) u:  of g  v u act'(g),  of u  v act(g).
template <typename T, int ACT>
__device__ __forceinline__ void gated_bwd(const GemmArgs& A, int m, int n, const float (&v)[8],
                                              const Side<T, kGatedBwd>& side)
{
    typedef typename T::E E;
    float dg[8], du[8];
#pragma unroll
    for (int r = 0; r < 8; ++r) {
        float a, d;
        act_both<ACT>(side.value(side.gh, side.gt, r), &a, &d);
        du[r] = v[r] * a;
        dg[r] = v[r] * side.value(side.uh, side.ut, r) * d;
    }
    if (n + 8 > A.N)
#pragma unroll
        for (int r = 0; r < 8; ++r) {
            du[r] = n + r < A.N ? du[r] : 0.0f;
            dg[r] = n + r < A.N ? dg[r] : 0.0f;
        }
    put((E*)A.c[0] + (int64_t)m * A.ldc + n, dg, 8);
    put((E*)A.c[1] + (int64_t)m * A.ldc + n, du, 8);
}

template <typename T, int GELU = kGelu>
__device__ __forceinline__ void gated_bwd_out(const GemmArgs& A, int m, int n, const float (&v)[8],
                                              const Side<T, kGatedBwd>& side)
{
    if (A.act == kSilu) gated_bwd<T, kSilu>(A, m, n, v, side);
    else if (A.act == kGelu) gated_bwd<T, GELU>(A, m, n, v, side);
    else gated_bwd<T, kRelu>(A, m, n, v, side);
}

// Where the t-th tile of a launch lies; false if it is none (past the edge, or
// above the diagonal of a symmetric product).  Tiles of the product come in
// bands of 8 tile rows.
struct Place {
    int m0, n0, z;
    bool mirror;         // symmetric and off the diagonal: the transposed tile is written too
};

// a / b by a reciprocal, corrected: what comes before a block's first load is
// on the path of a short product.
__device__ __forceinline__ int quotient(int a, int b)
{
    int q = (int)((float)a * __builtin_amdgcn_rcpf((float)b)), r = a - q * b;
    while (r < 0) { --q; r += b; }
    while (r >= b) { ++q; r -= b; }
    return __builtin_amdgcn_readfirstlane(q);
}

template <typename P>
__device__ __forceinline__ bool place_of(const GemmArgs& A, int t, Place* at)
{
    const int sub = t & ((1 << 2 * A.ratio) - 1);
    int tile = A.first + (t >> 2 * A.ratio), tm, tn;
    at->z = 0;
    if (A.batch > 1) {
        const int tiles = A.sym ? A.tiles_m * (A.tiles_m + 1) / 2 : A.tiles_m * A.tiles_n;
        at->z = quotient(tile, tiles);
        tile -= at->z * tiles;
    }
    if (A.sym) {
        tm = (int)((__builtin_amdgcn_sqrtf(8.0f * tile + 1.0f) - 1.0f) * 0.5f);
        while (tm * (tm + 1) / 2 > tile) --tm;
        while ((tm + 1) * (tm + 2) / 2 <= tile) ++tm;
        tm = __builtin_amdgcn_readfirstlane(tm);
        tn = tile - tm * (tm + 1) / 2;
    } else {
        const int band = 8 * A.tiles_n, b = quotient(tile, band), in = tile - b * band;
        const int rows = min(8, A.tiles_m - b * 8);
        tn = quotient(in, rows);
        tm = b * 8 + in - tn * rows;
    }
    tm = (tm << A.ratio) + (sub >> A.ratio);
    tn = (tn << A.ratio) + (sub & ((1 << A.ratio) - 1));
    at->m0 = tm * P::BM;
    at->n0 = tn * P::kCols;
    at->mirror = A.sym && tm != tn;
    return at->m0 < A.M && at->n0 < A.N && !(A.sym && tm < tn);
}

// Blocks go to the 8 XCDs in turn, so each XCD gets a run of consecutive tiles:
// its L2 then holds the operands that they share.
__device__ __forceinline__ int tile_of(int bid, int n_blocks)
{
    const int per = n_blocks >> 3, more = n_blocks & 7;
    const int x = bid & 7, i = bid >> 3;
    return x * per + min(x, more) + i;
}

template <int N>
struct Int {
    static constexpr int value = N;
};

// Waits until at most N of the wave's global loads are in flight, and for all
// of its LDS reads.  (The compiler adds waits of its own, see Buffers.)
template <int N>
__device__ __forceinline__ void wait_loads()
{
    static_assert(N < 64, "the counter has six bits");
    __builtin_amdgcn_s_waitcnt((N & 15) | (N >> 4) << 14 | 7 << 4);
}

// The LDS buffers of a block: separate arrays, so that a fragment read can be told
// from the loads in flight.  Of two buffers the compiler does; of four, where it
// meets eight arrays, it waits for all loads before the reads of three steps in four:
// what is loaded two and three steps ahead is then only started earlier.
struct Buffers {
    char *a0, *a1, *b0, *b1, *a2, *a3, *b2, *b3;
};

#define ARENA_TILE_BUFFERS(P, name)                                                                        \
    constexpr int kMoreA = P::kStages > 2 ? P::BM * 128 : 16, kMoreB = P::kStages > 2 ? P::BN * 128 : 16;  \
    __shared__ __attribute__((aligned(16))) char sa0_[P::BM * 128];                                        \
    __shared__ __attribute__((aligned(16))) char sa1_[P::BM * 128];                                        \
    __shared__ __attribute__((aligned(16))) char sb0_[P::BN * 128];                                        \
    __shared__ __attribute__((aligned(16))) char sb1_[P::BN * 128];                                        \
    __shared__ __attribute__((aligned(16))) char sa2_[kMoreA];                                             \
    __shared__ __attribute__((aligned(16))) char sa3_[kMoreA];                                             \
    __shared__ __attribute__((aligned(16))) char sb2_[kMoreB];                                             \
    __shared__ __attribute__((aligned(16))) char sb3_[kMoreB];                                             \
    const Buffers name = {sa0_, sa1_, sb0_, sb1_, sa2_, sa3_, sb2_, sb3_}

// Tile t of a launch's n_tiles; part: which of the splits of k.
template <typename P>
__device__ __forceinline__ void tile_product(const GemmArgs& A, const int t, const int n_tiles, const int part,
                                             const Buffers& lds)
{
    typedef typename P::T T;
    char *const sa0 = lds.a0, *const sa1 = lds.a1, *const sb0 = lds.b0, *const sb1 = lds.b1;
    auto bufa = [&](int i) { return i == 0 ? lds.a0 : i == 1 ? lds.a1 : i == 2 ? lds.a2 : lds.a3; };
    auto bufb = [&](int i) { return i == 0 ? lds.b0 : i == 1 ? lds.b1 : i == 2 ? lds.b2 : lds.b3; };

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / P::WN, wn = wave % P::WN;
    Place at;
    if (!place_of<P>(A, t, &at)) return;
    const int zb = at.z, m0 = at.m0, n0 = at.n0;

    Loader<P, P::BM, P::ATR, false> la;
    Loader<P, P::BN, P::BTR, P::DUAL> lb;
    la.init(tid, m0, A.M, A.lda);
    lb.init(tid, n0, A.N, A.ldb);
    Frags<P, P::BM, P::ATR> fa;
    Frags<P, P::BN, P::BTR> fb;
    fa.init(lane, wm * (P::BM / P::WM));
    fb.init(lane, wn * (P::BN / P::WN));

    f32x4 acc[P::FM][P::FN];
#pragma unroll
    for (int i = 0; i < P::FM; ++i)
#pragma unroll
        for (int j = 0; j < P::FN; ++j) acc[i][j] = f32x4{0, 0, 0, 0};

    const int sps = (A.K + kBK - 1) / kBK;     // steps of a segment
    int s = 0, end = sps * A.nseg;
    if (A.splits > 1) {
        s = part * A.per;
        end = min(end, s + A.per);
    }
    const int64_t za = A.pairs ? 0 : zb * A.sa, zB = A.pairs ? 0 : zb * A.sb;
    const int sel = A.pairs ? zb : 0;

    auto where = [&](int step, const char** pa, const char** pb, const char** pb1, int* left) {
        int q = step, seg = sel;
        if (A.nseg == 2 && step >= sps) { q -= sps; seg = 1; }
        *pa = la.base(A.a[seg], za) + q * la.step;
        *pb = lb.base(A.b[seg], zB) + q * lb.step;
        *pb1 = P::DUAL ? lb.base(A.b[1], 0) + q * lb.step : *pb;
        *left = A.K - q * kBK;
    };
    // The loads of a step, of both operands (which = 3) or one of them.  Woven
    // between products they may not branch, so every lane compares its k with
    // the end; otherwise only the last step does.
    auto fetch = [&](int step, char* sa, char* sb, auto which) {
        const char *pa, *pb, *pb1;
        int left;
        where(step, &pa, &pb, &pb1, &left);
        if (P::kWoven || left < kBK) {
            if (which.value & 1) la.template fetch<true>(pa, pa, sa, tid, left);
            if (which.value & 2) lb.template fetch<true>(pb, pb1, sb, tid, left);
        } else {
            if (which.value & 1) la.template fetch<false>(pa, pa, sa, tid, left);
            if (which.value & 2) lb.template fetch<false>(pb, pb1, sb, tid, left);
        }
    };
    // What the epilogue reads from memory, in batches of pieces of 8 columns: the
    // first batch while the products run, each other while the one before is
    // finished.
    constexpr int RW = P::BM / P::WM, CW = P::BN / P::WN, kWaves = P::WM * P::WN;
    constexpr int kRows = RW < 64 ? RW : 64;                  // of a slice through LDS
    constexpr int kChunks = (P::DUAL ? CW / 2 : CW) / 8;      // pieces of a row
    constexpr int kPieces = kRows * kChunks / 64, kBatch = kPieces < 4 ? kPieces : 4, kAll = kPieces * (RW / kRows);
    const int mw = m0 + wm * RW, nw = n0 + wn * (P::DUAL ? CW / 2 : CW);
    Side<T, P::EPI> side[kBatch], next_side[kBatch];
    auto ask = [&](int at, Side<T, P::EPI>* to) {
        if (A.splits > 1 || at >= kAll) return;
#pragma unroll
        for (int q = 0; q < kBatch; ++q) {
            const int x = (at + q) * 64 + lane, m = mw + x / kChunks, n = nw + x % kChunks * 8;
            if (m < A.M && n < (P::EPI == kPlain ? A.N : A.pad)) to[q].load(A, zb, m, n);
        }
    };

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
    // Interleaves the fragment reads of a half step and its share of the loads
    // with the products of the half step before.
    auto weave = [&](auto n_loads) {
        constexpr int reads = P::FM * (P::ATR ? 2 : 1) + P::FN * (P::BTR ? 2 : 1), products = P::FM * P::FN;
        constexpr int loads = decltype(n_loads)::value, each = products / reads > 0 ? products / reads : 1;
#pragma unroll
        for (int i = 0; i < reads; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);          // an LDS read
            if (i < loads) __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);      // a load
            __builtin_amdgcn_sched_group_barrier(0x008, each, 0);       // products
        }
    };
    // One step, from buffer u.  At its barrier this step's loads have landed
    // (those of later steps may be in flight) and every wave holds its
    // fragments of the step before, so that one's buffer is free: the loads
    // kStages - 1 steps ahead start, and the second half of the step before is
    // multiplied while this step's first fragments are read.
    constexpr int kAhead = P::kStages - 1, kLoads = la.kChunks + lb.kChunks;
    auto turn = [&](int step, int u, bool first) {
        asm volatile("" ::: "memory");
        wait_loads<(kAhead - 1) * kLoads>();
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        char* const ta = bufa((u + kAhead) % P::kStages);
        char* const tb = bufb((u + kAhead) % P::kStages);
        // woven, past the end the last step is fetched again, into buffers that no step
        // reads; the epilogue waits for them
        const int next = P::kWoven ? min(step + kAhead, end - 1) : step + kAhead;
        if (!P::kWoven && next < end) fetch(next, ta, tb, Int<3>());
        __builtin_amdgcn_sched_barrier(0);
        if (P::kWoven) fetch(next, ta, tb, Int<1>());
        read(bufa(u), bufb(u), 0, fa0, fb0);
        if (!first) multiply(fa1, fb1);
        weave(Int<P::kWoven ? la.kChunks : 0>());
        __builtin_amdgcn_sched_barrier(0);
        if (P::kWoven) fetch(next, ta, tb, Int<2>());
        read(bufa(u), bufb(u), 1, fa1, fb1);
        multiply(fa0, fb0);
        weave(Int<P::kWoven ? lb.kChunks : 0>());
        __builtin_amdgcn_sched_barrier(0);
    };
    if (P::BM < 256) ask(0, side);
    if (s < end) {
#pragma unroll
        for (int u = 0; u < kAhead; ++u) fetch(min(s + u, end - 1), bufa(u), bufb(u), Int<3>());
        turn(s, 0, true);
        for (++s; s < end; s += P::kStages)
#pragma unroll
            for (int u = 0; u < P::kStages; ++u)
                if (s + u < end) turn(s + u, (u + 1) % P::kStages, false);
        multiply(fa1, fb1);
    }

    // Epilogue.  A lane holds row lane & 15 and columns 4 (lane >> 4) + 0..3 of
    // each fragment; through LDS (a slice of rows at a time, 16-byte pieces
    // swizzled by row) it gets 8 neighbouring columns, and the wave whole
    // stretches of rows.  The waves' quarters of the buffers lie in different
    // arrays or halves of them; a wave reads only what it wrote.
    static_assert(kRows * CW * 4 * (kWaves / 4) <= P::BM * 128 && kWaves % 4 == 0 && P::BM == P::BN,
                  "epilogue slices fit");
    char* const mine = (wave & 2 ? (wave & 1 ? sb1 : sb0) : (wave & 1 ? sa1 : sa0)) + (wave >> 2) * (kRows * CW * 4);
    auto piece = [&](int r, int c4) { return (f32x4*)(mine + (r * (CW / 4) + (c4 ^ (r & (CW / 4 - 1) & 15))) * 16); };
    const bool mirror = at.mirror && A.splits == 1;
    auto finish = [&](int x, const Side<T, P::EPI>& from) {
        const int r = x / kChunks % kRows, c = x % kChunks;
        const int m = mw + x / kChunks, n = nw + c * 8;
        float v[8], u[8];
        *(f32x4*)v = *piece(r, 2 * c);
        *(f32x4*)(v + 4) = *piece(r, 2 * c + 1);
        if (P::DUAL) {
            *(f32x4*)u = *piece(r, CW / 8 + 2 * c);
            *(f32x4*)(u + 4) = *piece(r, CW / 8 + 2 * c + 1);
        }
        if (m >= A.M || n >= (P::EPI == kPlain ? A.N : A.pad)) return;
        if (A.splits > 1) {
            float* to = A.part + ((int64_t)part * n_tiles + t) * (P::BM * P::BN) + (m - m0) * P::kCols + n - n0;
            put(to, v, 8);
            if (P::DUAL) put(to + P::BM * P::kCols, u, 8);
            return;
        }
        if constexpr (P::EPI == kGatedFwd) {
            gated_fwd_out<T>(A, m, n, v, u);
        } else if constexpr (P::EPI == kGatedBwd) {
            gated_bwd_out<T>(A, m, n, v, from);
        } else {
            plain_out<T>(A, zb, m, n, v, from);
            if (mirror) {
                *piece(r, 2 * c) = *(f32x4*)v;
                *piece(r, 2 * c + 1) = *(f32x4*)(v + 4);
            }
        }
    };
    // Loads into LDS may still be in flight here, and a wave's land in slices that
    // others write: each waits for its own before the barrier, which does not.
    asm volatile("" ::: "memory");
    wait_loads<0>();
    if (P::BM == 256) ask(0, side);      // no registers are left for it before
    __syncthreads();
#pragma unroll
    for (int h = 0; h < RW / kRows; ++h) {
#pragma unroll
        for (int i = 0; i < kRows / 16; ++i)
#pragma unroll
            for (int j = 0; j < P::FN; ++j)
                *piece(i * 16 + (lane & 15), j * 4 + (lane >> 4)) = acc[h * (kRows / 16) + i][j];
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll 1
        for (int y = 0; y < kPieces; y += kBatch) {
            const int at = h * kPieces + y;
            ask(at + kBatch, next_side);
#pragma unroll
            for (int q = 0; q < kBatch; ++q) finish((at + q) * 64 + lane, side[q]);
#pragma unroll
            for (int q = 0; q < kBatch; ++q) side[q] = next_side[q];
        }
        if (P::EPI == kPlain && mirror) {
            // the transposed tile: 8 rows of a column are 8 columns of its row
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll 1
            for (int x = lane; x < CW * (kRows / 8); x += 64) {
                const int c = x / (kRows / 8), r0 = x % (kRows / 8) * 8;
                const int m = mw + h * kRows + r0, n = nw + c;
                float v[8];
#pragma unroll
                for (int r = 0; r < 8; ++r) v[r] = ((const float*)piece(r0 + r, c >> 2))[c & 3];
                if (m < A.M && n < A.N)
                    put((typename T::E*)A.c[0] + zb * A.sc + (int64_t)n * A.ldc + m, v, A.M - m);
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
}

template <typename P>
__global__ __launch_bounds__(P::kThreads, P::kWavesEach) void gemm_kernel(const GemmArgs A)
{
    ARENA_TILE_BUFFERS(P, lds);
    tile_product<P>(A, tile_of(blockIdx.x, gridDim.x), gridDim.x, blockIdx.y, lds);
}

// Two independent products in one launch: blocks below n1 * A.splits belong to
// the first, the rest to the second.  Of medium sizes neither fills the compute
// units by itself.
template <typename P, typename Q>
__global__ __launch_bounds__(P::kThreads, P::kWavesEach) void pair_kernel(const GemmArgs A, int n1, const GemmArgs B,
                                                                          int n2)
{
    static_assert(P::BM == Q::BM && P::kThreads == Q::kThreads && P::kStages == Q::kStages, "one shape of tile");
    ARENA_TILE_BUFFERS(P, lds);
    const int first = n1 * A.splits, i = blockIdx.x;
    if (i < first) {
        const int part = quotient(i, n1);
        tile_product<P>(A, tile_of(i - part * n1, n1), n1, part, lds);
    } else {
        tile_product<Q>(B, tile_of(i - first, n2), n2, 0, lds);
    }
}

// Joins the parts of the tiles of a split product in their order and applies
// the epilogue.  A block takes 64 rows and up to 64 columns of a tile, a thread
// one or two pieces of eight columns.
template <typename P>
__global__ __launch_bounds__(256) void join_kernel(const GemmArgs A, int n_tiles)
{
    typedef typename P::T T;
    constexpr int CW = P::kCols < 64 ? P::kCols : 64, kChunks = CW / 8, kAcross = P::kCols / CW;
    constexpr int kEach = (P::BM / 64) * kAcross;         // blocks of a tile
    __shared__ float turned[P::EPI == kPlain ? 64 : 1][65];
    const int t = blockIdx.x / kEach, in = blockIdx.x % kEach;
    const int r0 = in / kAcross * 64, c0 = in % kAcross * CW;
    Place at;
    if (!place_of<P>(A, t, &at)) return;
    const int64_t each = (int64_t)n_tiles * (P::BM * P::BN);
    const float* part = A.part + (int64_t)t * (P::BM * P::BN);
#pragma unroll 1
    for (int x = threadIdx.x; x < 64 * kChunks; x += 256) {
        const int r = x / kChunks, c = x % kChunks * 8;
        const int m = at.m0 + r0 + r, n = at.n0 + c0 + c;
        const float* p = part + (r0 + r) * P::kCols + c0 + c;
        float v[8] = {}, u[8] = {};
        Side<T, P::EPI> side;
        if (m >= A.M || n >= (P::EPI == kPlain ? A.N : A.pad)) continue;
        side.load(A, at.z, m, n);
#pragma unroll 4
        for (int s = 0; s < A.splits; ++s) {
            float w[8];
            get(p + s * each, w, 8);
#pragma unroll
            for (int q = 0; q < 8; ++q) v[q] += w[q];
            if (!P::DUAL) continue;
            get(p + s * each + P::BM * P::kCols, w, 8);
#pragma unroll
            for (int q = 0; q < 8; ++q) u[q] += w[q];
        }
        if constexpr (P::EPI == kGatedFwd) gated_fwd_out<T>(A, m, n, v, u);
        else if constexpr (P::EPI == kGatedBwd) gated_bwd_out<T>(A, m, n, v, side);
        else plain_out<T>(A, at.z, m, n, v, side);
        if (P::EPI == kPlain && at.mirror)
#pragma unroll
            for (int q = 0; q < 8; ++q) turned[r][c + q] = v[q];
    }
    if (P::EPI != kPlain || !at.mirror) return;
    __syncthreads();
    for (int x = threadIdx.x; x < CW * 8; x += 256) {
        const int c = x / 8, r = x % 8 * 8;
        const int m = at.m0 + r0 + r, n = at.n0 + c0 + c;
        float v[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) v[q] = turned[P::EPI == kPlain ? r + q : 0][c];
        if (m < A.M && n < A.N)
            put((typename T::E*)A.c[0] + at.z * A.sc + (int64_t)n * A.ldc + m, v, A.M - m);
    }
}

// Few rows of A (tokens): nothing of B is used twice, so it goes from memory
// to registers and no LDS tile is filled.  A block takes 16 columns of C, its
// waves share k, and their sums meet in LDS in the waves' order.  Operands
// with k contiguous, any alignment.  Bound by the read of B: one token of 4096 x
// 10944 in bfloat16 reads 179 MB of gate and up weights in 37 us (4.8 TB/s) and
// 90 MB of down weights in 20 us (4.5 TB/s).
template <typename T>
__device__ __forceinline__ typename T::V8 load_k(const typename T::E* p, int left)
{
    typename T::V8 v;
    if (left >= 8) {
        __builtin_memcpy(&v, p, 16);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < left ? p[i] : (typename T::E)0.0f;
    }
    return v;
}

template <typename T, int NT, bool DUAL, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void skinny_kernel(const GemmArgs A)
{
    typedef typename T::E E;
    typedef typename T::V8 V8;
    constexpr int NB = DUAL ? 2 : 1;
    __shared__ f32x4 part[WAVES][NT * NB][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n0 = blockIdx.x * 16, kc = (lane >> 4) * 8;
    const int row = min(n0 + (lane & 15), A.N - 1);
    const E* w[NB];
    const E* x[NT];
    w[0] = (const E*)A.b[0] + (int64_t)row * A.ldb + kc;
    if (DUAL) w[NB - 1] = (const E*)A.b[1] + (int64_t)row * A.ldb1 + kc;
#pragma unroll
    for (int t = 0; t < NT; ++t)
        x[t] = (const E*)A.a[0] + (int64_t)min(t * 16 + (lane & 15), A.M - 1) * A.lda + kc;
    f32x4 acc[NB][NT];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int t = 0; t < NT; ++t) acc[b][t] = f32x4{0, 0, 0, 0};

    constexpr int U = 4;          // steps of 32 in flight
    const int steps = (A.K + 31) / 32, per = (steps + WAVES - 1) / WAVES;
    int k = wave * per * 32;
    const int end = min(A.K, k + per * 32);
    for (; k + 32 * U <= end; k += 32 * U) {
        V8 wv[NB][U], xv[NT][U];
#pragma unroll
        for (int i = 0; i < U; ++i) {
#pragma unroll
            for (int b = 0; b < NB; ++b) __builtin_memcpy(&wv[b][i], w[b] + k + 32 * i, 16);
#pragma unroll
            for (int t = 0; t < NT; ++t) __builtin_memcpy(&xv[t][i], x[t] + k + 32 * i, 16);
        }
#pragma unroll
        for (int i = 0; i < U; ++i)
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int t = 0; t < NT; ++t) acc[b][t] = T::mfma(wv[b][i], xv[t][i], acc[b][t]);
    }
    for (; k < end; k += 32) {
        const int left = A.K - k - kc;
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            const V8 wv = load_k<T>(w[b] + k, left);
#pragma unroll
            for (int t = 0; t < NT; ++t) acc[b][t] = T::mfma(wv, load_k<T>(x[t] + k, left), acc[b][t]);
        }
    }
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int t = 0; t < NT; ++t) part[wave][b * NT + t][lane] = acc[b][t];
    __syncthreads();
    for (int t = wave; t < NT; t += WAVES) {
        const int m = t * 16 + (lane & 15), n = n0 + 4 * (lane >> 4);
        f32x4 v = part[0][t][lane], u = part[0][(NB - 1) * NT + t][lane];
#pragma unroll
        for (int q = 1; q < WAVES; ++q) {
            v += part[q][t][lane];
            if (DUAL) u += part[q][(NB - 1) * NT + t][lane];
        }
        if (m >= A.M) continue;
        float fv[4], fu[4];
        *(f32x4*)fv = v;
        *(f32x4*)fu = u;
        if constexpr (DUAL) {
            if (n < A.pad) gated_fwd_out<T>(A, m, n, fv, fu);
        } else {
            if (n < A.N) plain_out<T>(A, 0, m, n, fv, Side<T, kPlain>());      // nothing is added here
        }
    }
}

template <typename P>
hipError_t launch_tile(const GemmArgs& A, int64_t n_tiles, hipStream_t s)
{
    if (n_tiles == 0) return hipSuccess;
    gemm_kernel<P><<<dim3((unsigned)n_tiles, A.splits), P::kThreads, 0, s>>>(A);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || A.splits == 1) return e;
    constexpr int kEach = (P::BM / 64) * (P::kCols < 64 ? 1 : P::kCols / 64);
    join_kernel<P><<<(unsigned)(n_tiles * kEach), 256, 0, s>>>(A, (int)n_tiles);
    return hipGetLastError();
}

template <typename T, bool ATR, bool BTR, int EPI>
hipError_t launch_kind(const GemmArgs& A, int kind, int64_t n_tiles, hipStream_t s)
{
    switch (kind) {
    case k256: return launch_tile<Tile<T, 256, 256, 2, 4, 2, ATR, BTR, EPI>>(A, n_tiles, s);
    case k128: return launch_tile<Tile<T, 128, 128, 2, 2, 2, ATR, BTR, EPI>>(A, n_tiles, s);
    case k128Deep: return launch_tile<Tile<T, 128, 128, 2, 2, 4, ATR, BTR, EPI>>(A, n_tiles, s);
    case k64: return launch_tile<Tile<T, 64, 64, 2, 2, 4, ATR, BTR, EPI>>(A, n_tiles, s);
    }
    return hipErrorInvalidValue;
}

template <typename T, bool ATR, bool BTR, int EPI>
hipError_t launch_layout(GemmArgs A, const Cut& cut, hipStream_t s)
{
    const int side = kTileSide[cut.main], cols = EPI == kGatedFwd ? side / 2 : side;
    A.tiles_m = (A.M + side - 1) / side;
    A.tiles_n = (A.N + cols - 1) / cols;
    const int64_t all = (A.sym ? (int64_t)A.tiles_m * (A.tiles_m + 1) / 2 : (int64_t)A.tiles_m * A.tiles_n) * A.batch;
    A.splits = 1;
    A.first = 0;
    A.ratio = 0;
    const hipError_t e = launch_kind<T, ATR, BTR, EPI>(A, cut.main, cut.first, s);
    if (e != hipSuccess || cut.first == all) return e;
    A.splits = cut.splits;
    A.per = cut.per;
    A.first = (int)cut.first;
    while (kTileSide[cut.tail] << A.ratio < side) ++A.ratio;
    return launch_kind<T, ATR, BTR, EPI>(A, cut.tail, (all - cut.first) << 2 * A.ratio, s);
}

// Both products on 128 x 128 tiles, k of the first in cut.splits parts.
template <typename T, int EPI>
hipError_t launch_pair_t(GemmArgs A, GemmArgs B, const Cut& cut, hipStream_t s)
{
    typedef Tile<T, 128, 128, 2, 2, 2, false, true, EPI> P;
    typedef Tile<T, 128, 128, 2, 2, 2, true, true, kPlain> Q;
    for (GemmArgs* g : {&A, &B}) {
        g->tiles_m = (g->M + 127) / 128;
        g->tiles_n = (g->N + 127) / 128;
        g->first = g->ratio = 0;
        g->splits = 1;
    }
    A.splits = cut.splits;
    A.per = cut.per;
    const int n1 = A.tiles_m * A.tiles_n * A.batch, n2 = B.tiles_m * B.tiles_n * B.batch;
    pair_kernel<P, Q><<<n1 * A.splits + n2, P::kThreads, 0, s>>>(A, n1, B, n2);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || A.splits == 1) return e;
    join_kernel<P><<<n1 * 4, 256, 0, s>>>(A, n1);
    return hipGetLastError();
}

template <typename T>
hipError_t launch_gemm_t(const GemmArgs& A, Product what, const Cut& cut, hipStream_t s)
{
    switch (what) {
    case kRowsRows: return launch_layout<T, false, false, kPlain>(A, cut, s);
    case kRowsCols: return launch_layout<T, false, true, kPlain>(A, cut, s);
    case kColsCols: return launch_layout<T, true, true, kPlain>(A, cut, s);
    case kGateUp: return launch_layout<T, false, false, kGatedFwd>(A, cut, s);
    case kGateUpBack: return launch_layout<T, false, true, kGatedBwd>(A, cut, s);
    default: return hipErrorInvalidValue;
    }
}

template <typename T>
hipError_t launch_pair_of(const GemmArgs& A, Product what, const GemmArgs& B, const Cut& cut, hipStream_t s)
{
    return what == kGateUpBack ? launch_pair_t<T, kGatedBwd>(A, B, cut, s) : launch_pair_t<T, kPlain>(A, B, cut, s);
}

template <typename T, bool DUAL, int WAVES>
hipError_t launch_skinny_n(const GemmArgs& A, hipStream_t s)
{
    const int blocks = (A.N + 15) / 16;
    if (A.M <= 16) skinny_kernel<T, 1, DUAL, WAVES><<<blocks, 64 * WAVES, 0, s>>>(A);
    else skinny_kernel<T, 2, DUAL, WAVES><<<blocks, 64 * WAVES, 0, s>>>(A);
    return hipGetLastError();
}

template <typename T>
hipError_t launch_skinny_t(const GemmArgs& A, bool dual, hipStream_t s)
{
    if (dual) return launch_skinny_n<T, true, 8>(A, s);
    // few columns: 16 waves a block, so that the compute units have enough to wait for
    return A.N <= 4096 ? launch_skinny_n<T, false, 16>(A, s) : launch_skinny_n<T, false, 8>(A, s);
}

}  // namespace mm
}  // namespace arena
