// The experts' tiled products in bfloat16, and the dispatch by type.
#include "arena_groups.h"

namespace arena {
namespace mm {

hipError_t launch_groups_f16(const GroupArgs& A, Product what, int kind, hipStream_t s);
hipError_t launch_skinny_groups_f16(const GroupArgs& A, Product what, hipStream_t s);

hipError_t launch_groups(const GroupArgs& A, int dtype, Product what, int kind, hipStream_t s)
{
    return dtype == ARENA_BF16 ? launch_groups_t<Bf16>(A, what, kind, s) : launch_groups_f16(A, what, kind, s);
}

hipError_t launch_skinny_groups(const GroupArgs& A, int dtype, Product what, hipStream_t s)
{
    return dtype == ARENA_BF16 ? launch_skinny_groups_t<Bf16>(A, what, s) : launch_skinny_groups_f16(A, what, s);
}

}  // namespace mm
}  // namespace arena
