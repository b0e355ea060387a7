// smol_attend_f32.hip -- attention forward with matrices of type float.
#include "smol_attend_kernels.h"

int smol::launch_attend_f32(const AttendArgs &a, int kernel, int wide, unsigned grid, void *s)
{
    return launch_attend<float>(a, kernel, wide, grid, s);
}
