// The loss's tiled products in bfloat16, and the dispatch by type.
#include "arena_groups.h"

namespace arena {
namespace mm {

hipError_t launch_loss_f16(const GroupArgs& A, Product what, int kind, hipStream_t s);

hipError_t launch_loss(const GroupArgs& A, int dtype, Product what, int kind, hipStream_t s)
{
    return dtype == ARENA_BF16 ? launch_loss_t<Bf16>(A, what, kind, s) : launch_loss_f16(A, what, kind, s);
}

}  // namespace mm
}  // namespace arena
