// smol_patch_grad_bf16.hip -- patch embedding with bf16 weights, backward.
#include "smol_patch_kernels.h"

int smol::launch_patch_grad_bf16(const PatchArgs &a, const SumArgs &b, int image_type, int mode,
                                int tile, void *stream)
{
    return launch_patch_grad<bf16>(a, b, image_type, mode, tile, stream);
}
