// smol_patch_grad_f32.hip -- patch embedding with f32 weights, backward.
#include "smol_patch_kernels.h"

int smol::launch_patch_grad_f32(const PatchArgs &a, const SumArgs &b, int image_type, int mode,
                                int tile, void *stream)
{
    return launch_patch_grad<float>(a, b, image_type, mode, tile, stream);
}
