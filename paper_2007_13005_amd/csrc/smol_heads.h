// smol_heads.h -- arguments of the kernels that rotate and normalise heads
// (smol_heads_kernels.h), and their launchers, one file per type.
#ifndef SMOL_HEADS_H
#define SMOL_HEADS_H

#include <stdint.h>

#include "smol_tokens_device.h"

namespace smol {

// The queries or the keys; dy in the backward pass alone.
struct HeadSide {
    const void *dy, *x, *weight;
    void *out;
    int64_t dy_row, dy_head, x_row, x_head, out_row, out_head;
    int32_t heads;
    int32_t steps;  // of a block of rows: the wave's slots over its rows and heads
};

struct HeadArgs {
    HeadSide side[2];
    const void *positions;
    const double *freqs;
    float *part;  // backward: [workgroups][2][dim] sums of g xh
    int64_t items;  // parts of blocks of rows, one wave each
    int32_t rows, dim, half;  // half: rotated pairs
    int32_t wide;       // 64-bit positions
    int32_t weight_f32;
    int32_t units;      // pairs of chunks of a head
    int32_t lanes_log2; // lanes of a head
    int32_t rows_log2;  // rows of a block
    int32_t per;        // steps of an item
    int32_t parts;      // items of a block
    int32_t groups;     // backward: workgroups
    float eps, gain, sign;  // sign: -1 turns back
};

// V: elements of a chunk; K: units a lane.
struct HeadForm {
    int v, k;
    bool norm, interleaved;
};

int launch_heads_f32(const HeadArgs &a, const HeadForm &f, bool backward, unsigned grid, void *s);
int launch_heads_f16(const HeadArgs &a, const HeadForm &f, bool backward, unsigned grid, void *s);
int launch_heads_bf16(const HeadArgs &a, const HeadForm &f, bool backward, unsigned grid, void *s);

}  // namespace smol

#endif  // SMOL_HEADS_H
