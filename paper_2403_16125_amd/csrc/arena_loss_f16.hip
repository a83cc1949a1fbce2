// The loss's tiled products in float16.
#include "arena_groups.h"

namespace arena {
namespace mm {

hipError_t launch_loss_f16(const GroupArgs& A, Product what, int kind, hipStream_t s)
{
    return launch_loss_t<F16>(A, what, kind, s);
}

}  // namespace mm
}  // namespace arena
