// smol_attend_f16.hip -- attention forward with matrices of type f16.
#include "smol_attend_kernels.h"

int smol::launch_attend_f16(const AttendArgs &a, int kernel, int wide, unsigned grid, void *s)
{
    return launch_attend<f16>(a, kernel, wide, grid, s);
}
