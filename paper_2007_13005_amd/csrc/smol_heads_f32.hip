// smol_heads_f32.hip -- rotation and norm of heads of type float.
#include "smol_heads_kernels.h"

int smol::launch_heads_f32(const HeadArgs &a, const HeadForm &f, bool backward, unsigned grid,
                          void *s)
{
    return launch_heads<float>(a, f, backward, grid, s);
}
