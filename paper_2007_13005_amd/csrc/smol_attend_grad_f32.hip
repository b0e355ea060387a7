// smol_attend_grad_f32.hip -- attention's gradients with matrices of type float.
#include "smol_attend_grad_kernels.h"

int smol::launch_attend_grad_f32(const AttendArgs &a, int kernel, int wide, unsigned grid, void *s)
{
    return launch_attend_grad<float>(a, kernel, wide, grid, s);
}
