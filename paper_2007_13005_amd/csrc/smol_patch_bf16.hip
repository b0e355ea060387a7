// smol_patch_bf16.hip -- patch embedding with bf16 weights, forward.
#include "smol_patch_kernels.h"

int smol::launch_patch_bf16(const PatchArgs &a, int image_type, int mode, int tile, void *stream)
{
    return launch_patch<bf16>(a, image_type, mode, tile, stream);
}
