// smol_attend_bf16.hip -- attention forward with matrices of type bf16.
#include "smol_attend_kernels.h"

int smol::launch_attend_bf16(const AttendArgs &a, int kernel, int wide, unsigned grid, void *s)
{
    return launch_attend<bf16>(a, kernel, wide, grid, s);
}
