// smol_attend_grad_f16.hip -- attention's gradients with matrices of type f16.
#include "smol_attend_grad_kernels.h"

int smol::launch_attend_grad_f16(const AttendArgs &a, int kernel, int wide, unsigned grid, void *s)
{
    return launch_attend_grad<f16>(a, kernel, wide, grid, s);
}
