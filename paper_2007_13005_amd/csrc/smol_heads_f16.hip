// smol_heads_f16.hip -- rotation and norm of heads of type f16.
#include "smol_heads_kernels.h"

int smol::launch_heads_f16(const HeadArgs &a, const HeadForm &f, bool backward, unsigned grid,
                          void *s)
{
    return launch_heads<f16>(a, f, backward, grid, s);
}
