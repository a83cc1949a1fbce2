// The tiled and skinny products in bfloat16, and the launchers' dispatch by type.
#include "arena_gemm.h"

namespace arena {
namespace mm {

hipError_t launch_gemm_f16(const GemmArgs& A, Product what, const Cut& cut, hipStream_t s);
hipError_t launch_skinny_f16(const GemmArgs& A, bool dual, hipStream_t s);

hipError_t launch_gemm(const GemmArgs& A, int dtype, Product what, const Cut& cut, hipStream_t s)
{
    return dtype == ARENA_BF16 ? launch_gemm_t<Bf16>(A, what, cut, s) : launch_gemm_f16(A, what, cut, s);
}

hipError_t launch_skinny(const GemmArgs& A, int dtype, bool dual, hipStream_t s)
{
    return dtype == ARENA_BF16 ? launch_skinny_t<Bf16>(A, dual, s) : launch_skinny_f16(A, dual, s);
}

// A row of a matrix whose rows do not start on 16 bytes: the reads are
// unaligned, the writes 16 bytes a lane.
__global__ __launch_bounds__(256) void pack_kernel(const uint16_t* __restrict__ from, int64_t ld_from,
                                                   uint16_t* __restrict__ to, int64_t ld_to, int64_t rows, int cols)
{
    const int per = (int)(ld_to / 8);
    const int64_t n = rows * per;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
        const int64_t r = i / per;
        const int c = (int)(i % per) * 8;
        const uint16_t* p = from + r * ld_from + c;
        u32x4 v = {0, 0, 0, 0};
        if (c + 8 <= cols) {
            __builtin_memcpy(&v, p, 16);
        } else {
            uint32_t h[4] = {0, 0, 0, 0};
#pragma unroll
            for (int q = 0; q < 8; ++q)
                if (c + q < cols) h[q >> 1] |= (uint32_t)p[q] << (16 * (q & 1));
            v = u32x4{h[0], h[1], h[2], h[3]};
        }
        *(u32x4*)(to + r * ld_to + c) = v;
    }
}

hipError_t launch_pack(const void* from, int64_t ld_from, void* to, int64_t ld_to, int64_t rows, int64_t cols,
                       hipStream_t s)
{
    const int64_t blocks = (rows * (ld_to / 8) + 255) / 256;
    if (blocks == 0) return hipSuccess;
    pack_kernel<<<(unsigned)(blocks < 4096 ? blocks : 4096), 256, 0, s>>>((const uint16_t*)from, ld_from,
                                                                         (uint16_t*)to, ld_to, rows, (int)cols);
    return hipGetLastError();
}

}  // namespace mm
}  // namespace arena
