// The tiled and skinny products in float16.
#include "arena_gemm.h"

namespace arena {
namespace mm {

hipError_t launch_gemm_f16(const GemmArgs& A, Product what, const Cut& cut, hipStream_t s)
{
    if (what == kRowsRowsRest) return launch_layout<F16, false, false, kPlainRest>(A, cut, s);
    if (what == kRowsColsRest) return launch_layout<F16, false, true, kPlainRest>(A, cut, s);
    return launch_gemm_t<F16>(A, what, cut, s);
}

hipError_t launch_pair_f16(const GemmArgs& A, Product what, const GemmArgs& B, const Cut& cut, hipStream_t s)
{
    return launch_pair_of<F16>(A, what, B, cut, s);
}

hipError_t launch_skinny_f16(const GemmArgs& A, bool dual, hipStream_t s) { return launch_skinny_t<F16>(A, dual, s); }

}  // namespace mm
}  // namespace arena
