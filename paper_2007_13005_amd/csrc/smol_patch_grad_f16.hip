// smol_patch_grad_f16.hip -- patch embedding with f16 weights, backward.
#include "smol_patch_kernels.h"

int smol::launch_patch_grad_f16(const PatchArgs &a, const SumArgs &b, int image_type, int mode,
                                int tile, void *stream)
{
    return launch_patch_grad<f16>(a, b, image_type, mode, tile, stream);
}
