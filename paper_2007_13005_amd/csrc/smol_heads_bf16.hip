// smol_heads_bf16.hip -- rotation and norm of heads of type bf16.
#include "smol_heads_kernels.h"

int smol::launch_heads_bf16(const HeadArgs &a, const HeadForm &f, bool backward, unsigned grid,
                          void *s)
{
    return launch_heads<bf16>(a, f, backward, grid, s);
}
