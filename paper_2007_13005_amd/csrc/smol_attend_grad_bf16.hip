// smol_attend_grad_bf16.hip -- attention's gradients with matrices of type bf16.
#include "smol_attend_grad_kernels.h"

int smol::launch_attend_grad_bf16(const AttendArgs &a, int kernel, int wide, unsigned grid, void *s)
{
    return launch_attend_grad<bf16>(a, kernel, wide, grid, s);
}
