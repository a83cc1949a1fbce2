// The tiled and skinny products in bfloat16, and the launchers' dispatch by type.
#include "arena_gemm.h"

namespace arena {
namespace mm {

hipError_t launch_gemm_f16(const GemmArgs& A, Product what, const Cut& cut, hipStream_t s);
hipError_t launch_pair_f16(const GemmArgs& A, Product what, const GemmArgs& B, const Cut& cut, hipStream_t s);
hipError_t launch_skinny_f16(const GemmArgs& A, bool dual, hipStream_t s);

hipError_t launch_gemm(const GemmArgs& A, int dtype, Product what, const Cut& cut, hipStream_t s)
{
    return dtype == ARENA_BF16 ? launch_gemm_t<Bf16>(A, what, cut, s) : launch_gemm_f16(A, what, cut, s);
}

hipError_t launch_skinny(const GemmArgs& A, int dtype, bool dual, hipStream_t s)
{
    return dtype == ARENA_BF16 ? launch_skinny_t<Bf16>(A, dual, s) : launch_skinny_f16(A, dual, s);
}

hipError_t launch_pair(const GemmArgs& A, int dtype, Product what, const GemmArgs& B, const Cut& cut, hipStream_t s)
{
    return dtype == ARENA_BF16 ? launch_pair_of<Bf16>(A, what, B, cut, s) : launch_pair_f16(A, what, B, cut, s);
}

struct PackArgs {
    Pack p[kMaxPacks];
};

// Rows that do not start on 16 bytes: the reads are unaligned, the writes 16
// bytes a lane.  blockIdx.y: the matrix.
__global__ __launch_bounds__(256) void pack_kernel(const PackArgs A)
{
    const Pack p = A.p[blockIdx.y];
    const int per = (int)(p.ld_to / 8);
    const int64_t n = p.rows * per;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
        const int64_t r = i / per;
        const int c = (int)(i % per) * 8;
        const uint16_t* from = (const uint16_t*)p.from + r * p.ld_from + c;
        u32x4 v = {0, 0, 0, 0};
        if (c + 8 <= p.cols) {
            __builtin_memcpy(&v, from, 16);
        } else {
            uint32_t h[4] = {0, 0, 0, 0};
#pragma unroll
            for (int q = 0; q < 8; ++q)
                if (c + q < p.cols) h[q >> 1] |= (uint32_t)from[q] << (16 * (q & 1));
            v = u32x4{h[0], h[1], h[2], h[3]};
        }
        *(u32x4*)((uint16_t*)p.to + r * p.ld_to + c) = v;
    }
}

hipError_t launch_packs(const Pack* packs, int n, hipStream_t s)
{
    PackArgs A;
    int64_t most = 0;
    int k = 0;
    for (int i = 0; i < n && k < kMaxPacks; ++i) {
        const int64_t chunks = packs[i].rows * (packs[i].ld_to / 8);
        if (chunks == 0) continue;
        A.p[k++] = packs[i];
        most = chunks > most ? chunks : most;
    }
    if (k == 0) return hipSuccess;
    const int64_t blocks = (most + 255) / 256;
    pack_kernel<<<dim3((unsigned)(blocks < 2048 ? blocks : 2048), k), 256, 0, s>>>(A);
    return hipGetLastError();
}

}  // namespace mm
}  // namespace arena
