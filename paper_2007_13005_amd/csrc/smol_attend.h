// smol_attend.h -- arguments of the attention kernels (smol_attend_kernels.h,
// smol_attend_grad_kernels.h), and their launchers, one file per type.
#ifndef SMOL_ATTEND_H
#define SMOL_ATTEND_H

#include <stdint.h>

#include "smol_tokens_device.h"

namespace smol {

// A matrix of heads: strides in elements.
struct HeadRows {
    const void *p;
    int64_t batch, row, head;
};

struct AttendArgs {
    HeadRows q, k, v, out, dout;  // out is written by the forward pass, read by the backward
    HeadRows dq, dk, dv;          // written
    HeadRows rest_in, lse_in;     // read by the backward pass (rest_in.p null: zeros)
    void *rest;
    float *lse;      // batch x queries x heads
    float *lse_delta;  // of each of these (backward): lse in base 2, and D
    float *part;   // sums of parts of the keys (forward, splits > 1), of the columns
                   // (gradients of keys)
    const int32_t *q_lengths, *k_lengths;
    int32_t queries, keys, heads, dim;
    int32_t columns;       // queries * group: pairs of a query and one of a key head's heads
    int32_t window, sinks; // window 0: none
    int32_t causal;
    int32_t direct_keys, direct_rows;  // k and v, q and dout go to LDS without registers
    int32_t tiles;         // of the columns
    int32_t pairs;         // batch * kv_heads
    int32_t splits;
    float scale, scale_log2, per_scale_log2;  // times log2 e; 1 / that
    // gradients of keys: tiles of keys that hold sinks, and columns of a part of
    // these and of the other tiles (as many parts: the two divisors)
    int32_t sink_tiles, sink_part, tile_part;
    uint32_t batch, delta_groups;  // rows that workgroups form D of
    uint32_t key_units;            // workgroups of a pair's keys: its first
    // pairs of a chunk, of the last one, and a chunk's workgroups
    Divisor chunk, chunk_last, chunk_groups;
    Divisor group, pair_div, kv_heads, tile_div, sink_div, split_div;
    Divisor heads_div, queries_div;
};

constexpr int kAttendKeys = 64;     // of a tile that four waves share
constexpr int kAttendColumns = 32;  // of a wave
constexpr int kAttendWaves = 4;     // of a workgroup
constexpr int kAttendFewKeys = 32;  // of a tile of one wave (few columns)
constexpr int kAttendSplits = 64;   // parts of the keys at most
constexpr int kAttendJoinParts = 16;  // that a wave joins
constexpr int kAttendJoinKeys = 4;  // of a workgroup that joins gradients of keys

// Lanes that form a row's D, eight values each.
constexpr int attend_delta_lanes(int wide) { return wide == 1 ? 4 : wide == 2 ? 8 : 16; }

// Kernels: the forward pass with the waves over columns, or over keys (few
// columns); the join of its splits; the sums D of the backward pass; its gradients;
// the join of the parts of those of keys.
enum { kAttendMany, kAttendFew, kAttendJoin, kAttendDelta, kAttendGrad, kAttendGradJoin };

// wide: values of a head in 32s, rounded up.
int launch_attend_f32(const AttendArgs &a, int kernel, int wide, unsigned grid, void *s);
int launch_attend_f16(const AttendArgs &a, int kernel, int wide, unsigned grid, void *s);
int launch_attend_bf16(const AttendArgs &a, int kernel, int wide, unsigned grid, void *s);
int launch_attend_grad_f32(const AttendArgs &a, int kernel, int wide, unsigned grid, void *s);
int launch_attend_grad_f16(const AttendArgs &a, int kernel, int wide, unsigned grid, void *s);
int launch_attend_grad_bf16(const AttendArgs &a, int kernel, int wide, unsigned grid, void *s);

}  // namespace smol

#endif  // SMOL_ATTEND_H
