// The experts' tiled products in float16.
#include "arena_groups.h"

namespace arena {
namespace mm {

hipError_t launch_groups_f16(const GroupArgs& A, Product what, int kind, hipStream_t s)
{
    return launch_groups_t<F16>(A, what, kind, s);
}

hipError_t launch_skinny_groups_f16(const GroupArgs& A, Product what, hipStream_t s)
{
    return launch_skinny_groups_t<F16>(A, what, s);
}

}  // namespace mm
}  // namespace arena
