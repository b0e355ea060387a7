// smol_patch_f32.hip -- patch embedding with f32 weights, forward.
#include "smol_patch_kernels.h"

int smol::launch_patch_f32(const PatchArgs &a, int image_type, int mode, int tile, void *stream)
{
    return launch_patch<float>(a, image_type, mode, tile, stream);
}
