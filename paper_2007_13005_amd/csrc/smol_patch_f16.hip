// smol_patch_f16.hip -- patch embedding with f16 weights, forward.
#include "smol_patch_kernels.h"

int smol::launch_patch_f16(const PatchArgs &a, int image_type, int mode, int tile, void *stream)
{
    return launch_patch<f16>(a, image_type, mode, tile, stream);
}
