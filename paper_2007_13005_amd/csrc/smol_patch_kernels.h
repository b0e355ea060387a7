// smol_patch_kernels.h -- the patch embedding's kernels as templates, for one
// type of the weight (instantiated by smol_patch_<type>.hip).
#ifndef SMOL_PATCH_KERNELS_H
#define SMOL_PATCH_KERNELS_H

#include "smol_internal.h"
#include "smol_patch.h"

namespace smol {
namespace {

// Forward: out[m][d] = sum_k patch[m][k] weight[d][k] + bias[d] + pos[t][d].
//
// The end of a wave's tile: row m0 + 16 j + lane % 16 has columns d0 + 32 i +
// 8 (lane / 16) .. + 7 in tiles (2 i, j) and (2 i + 1, j); bias and position
// are added, and the result rounded and written. Where all columns exist the
// positions of three rows are asked for together before any is used.
template <typename T, int FD, int FM>
__device__ __forceinline__ void finish(const PatchArgs &a, uint32_t m0, uint32_t d0, int lane,
                                       f32x4 (&sum)[FD][FM])
{
    constexpr int N = FD / 2, kRows = FM < 3 ? FM : 3;
    const uint32_t d1 = d0 + 8 * (lane >> 4);
    const auto sums_of = [&](int j, int k) {
        return __builtin_shufflevector(sum[2 * k][j], sum[2 * k + 1][j], 0, 1, 2, 3, 4, 5, 6, 7);
    };
    if (d0 + 16 * FD <= a.dim) {
        vec<T, 8> bias[N];
        if (a.bias)
#pragma unroll
            for (int k = 0; k < N; ++k)
                bias[k] = load<T, 8>((const T *)a.bias + d1 + 32 * k);
#pragma unroll
        for (int first = 0; first < FM; first += kRows) {
            vec<T, 8> pos[kRows][N];
            if (a.pos)
#pragma unroll
                for (int j = 0; j < kRows && first + j < FM; ++j) {
                    uint32_t m = m0 + 16 * (first + j) + (lane & 15);
                    m = m < a.rows ? m : a.rows - 1;
                    const uint32_t t = m - divide(m, a.tokens) * a.tokens.d;
#pragma unroll
                    for (int k = 0; k < N; ++k)
                        pos[j][k] = load<T, 8>((const T *)a.pos + (t * a.dim + d1 + 32 * k));
                }
            asm volatile("" ::: "memory");
#pragma unroll
            for (int j = 0; j < kRows && first + j < FM; ++j) {
                const uint32_t m = m0 + 16 * (first + j) + (lane & 15);
                if (m >= a.rows)
                    continue;
                const uint32_t i = divide(m, a.tokens), t = m - i * a.tokens.d;
                T *out = (T *)a.out + i * a.image_stride + t * a.row_stride + d1;
#pragma unroll
                for (int k = 0; k < N; ++k) {
                    vec<float, 8> v = sums_of(first + j, k);
                    if (a.bias)
                        v += to_f32<8, T>(bias[k]);
                    if (a.pos)
                        v += to_f32<8, T>(pos[j][k]);
                    store<T, 8>(out + 32 * k, from_f32<T, 8>(v));
                }
            }
        }
        return;
    }
#pragma unroll
    for (int j = 0; j < FM; ++j) {
        const uint32_t m = m0 + 16 * j + (lane & 15);
        if (m >= a.rows)
            continue;
        const uint32_t i = divide(m, a.tokens), t = m - i * a.tokens.d;
        T *out = (T *)a.out + i * a.image_stride + t * a.row_stride;
        const T *pos = (const T *)a.pos + (int64_t)t * a.dim;
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const vec<float, 8> v = sums_of(j, k);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint32_t d = d1 + 32 * k + e;
                if (d < a.dim)
                    out[d] = (T)(v[e] + (a.bias ? (float)((const T *)a.bias)[d] : 0.0f) +
                                 (a.pos ? (float)pos[d] : 0.0f));
            }
        }
    }
}

// Of a pair of 16-row operand tiles, the row (0 .. 31) that row r of tile h
// (0, 1) is: a lane's sums of the two tiles, rows 4 (lane / 16) .. + 3 of
// each, are then eight consecutive rows.
__device__ __forceinline__ int paired_row(int h, int r) { return 8 * (r >> 2) + 4 * h + (r & 3); }

// A workgroup of WD x WM waves makes tiles of 16 FD WD columns (weight rows)
// by 16 FM WM rows (patches) in steps of eight chunks (128 bytes) of the
// summed index. It goes through its tiles without a pause: the first steps of
// the next are on their way while one ends. Operands go from memory through registers into one of two
// LDS buffers: a load is issued a step before its data is stored, and the
// step after's load takes its registers. Stores, loads and the LDS reads that
// are needed next stand between the matrix instructions, a few at a time, and
// issue while the matrix unit is at work. Images are gathered (and rounded to
// the weight's type) on the way; no unfolded copy is made.
//
// A wave reads two chunks, one after the other, of 32 patches side by side:
// patches that are neighbours in the image are so in memory, run by run.
// Eight lanes read a weight row's step. In LDS chunk
// c of a row stands at slot c ^ (three bits of the row), so that rows read
// at once lie in different banks.
//
// 256 fp16 images of 224 x 224 in patches of 14 to 1024 bf16 columns, with
// positions: 122 us a call (647 TFLOP/s on the patches' values; the library's product
// of two ready matrices of these sizes takes 94 us and holds no gather, rounding,
// bias or positions). By stamps, before tiles followed each other without a
// pause: of a tile's 35 us the products took 25 (11 steps at 2.2 us: 1100
// TFLOP/s of the 1300 to 1400 that a large library product reaches), the end of
// the tile 6.8, which all units write at once, 2.7 without positions.
//
// Chunks round a run up: patches of 14 take 1.20 times their products, of 9
// 1.78, of 17 1.41; runs shorter than a chunk are loaded value by value. us of
// 64 fp16 images of 224 x 224 to 512 bf16 columns by the patch's side, forward /
// the weight's gradient: 4: 157 / 87, 5: 113 / 71, 7: 89 / 62, 8: 24 / 39, 9: 50
// / 45, 12: 25 / 34, 14: 22 / 33, 16: 19 / 30, 17: 46 / 40, 20: 28 / 35.
//
// fp32, 64 images, patches of 16 to 768 columns: 134 us where the products need
// 96: the matrix units are busy for 0.72 of the time (tiles of 64: the chain of
// loads, LDS and products of one tile is hidden by the other tiles of a unit
// but for its begin and end).
template <typename T, typename S, int WD, int WM, int FD, int FM, int Mode>
__global__ void __launch_bounds__(64 * WD * WM, 2) patch_kernel(PatchArgs a)
{
    constexpr int C = 16 / sizeof(T), kWaves = WD * WM, kThreads = 64 * kWaves;
    constexpr int kCols = 16 * FD * WD, kRows = 16 * FM * WM;
    constexpr int kLines = kRows * 8 / kThreads;  // loads a thread: patches, weight rows
    constexpr int kLoads = kCols * 8 / kThreads, kStride = kThreads / 8;
    typedef vec<T, C> Frag;
    __shared__ Frag patches[2][kRows * 8], weights[2][kCols * 8];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t slot = threadIdx.x & 7, line = threadIdx.x >> 3;
    const int pair = 2 * (wave & 3), line_p = (lane >> 1) + 32 * (wave >> 2);

    // Byte offsets of a tile's rows from its first (the host made sure that
    // they fit); rows past the last are read as the last, and not written.
    const S *images;
    const T *weight_base;
    uint32_t image[kLines], weight[kLoads];
    const auto tile_at = [&](uint32_t piece) {
        const uint32_t tile = piece_of(piece, a.tiles);
        const uint32_t tm = divide(tile, a.tiles_n), tn = tile - tm * a.tiles_n.d;
        return make_uint2(tm * kRows, tn * kCols);  // first row, first column
    };
    const auto rows_of = [&](uint32_t piece) {
        const uint2 tile = tile_at(piece);
        const int64_t first = patch_at(a, tile.x);
        images = (const S *)a.images + first;
        weight_base = (const T *)a.weight + (int64_t)tile.y * a.values;
#pragma unroll
        for (int i = 0; i < kLines; ++i) {
            const uint32_t m = tile.x + line_p + kWaves * 8 * i;
            image[i] = (uint32_t)(patch_at(a, m < a.rows ? m : a.rows - 1) - first) * sizeof(S);
        }
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const uint32_t d = tile.y + line + kStride * i;
            weight[i] = ((d < a.dim ? d : a.dim - 1) - tile.y) * a.values * sizeof(T);
        }
    };
    const auto place_p = [](int row, int c) { return row * 8 + (c ^ (row & 7)); };
    const auto place_w = [](int row, int c) {
        return row * 8 + (c ^ ((row & 3) | (row >> 1 & 4)));
    };
    // what is in flight is as it stands in memory: rounding and zeros wait
    // until it is stored
    vec<S, C> next_p[kLines];
    Frag next_w[kLoads];
    int32_t lead_p = 0, lead_w = 0, have = C;
    uint32_t at_p = 0, at_w = 0;
    Mask mask_p, mask_w;
    const auto place = [&](uint32_t step) {  // where a step's chunks are
        // both chunks of the wave: scalar work
        const Chunk<C> c0(a, step * 8 + pair), c1(a, step * 8 + pair + 1), c(a, step * 8 + slot);
        at_p = (lane & 1 ? c1.image : c0.image) * sizeof(S);
        lead_p = lane & 1 ? c1.lead : c0.lead;
        at_w = c.weight * sizeof(T);
        lead_w = c.lead;
        have = c0.have;
    };
    const auto fetch = [&](int i) {
        if (i < kLines)
            next_p[i] = load_chunk<S, C, Mode == kShort>(images, image[i] + at_p, have);
        else
            next_w[i - kLines] =
                load_chunk<T, C, Mode == kShort>(weight_base, weight[i - kLines] + at_w, have);
    };
    const auto stage = [&](int buffer, int i) {
        if (i < kLines) {
            const Frag p = rounded<T, S, C>(next_p[i]);
            patches[buffer][place_p(line_p + kWaves * 8 * i, pair + (lane & 1))] =
                Mode == kWhole ? p : masked(p, mask_p);
        } else {
            const Frag w = next_w[i - kLines];
            weights[buffer][place_w(line + kStride * (i - kLines), slot)] =
                Mode == kWhole ? w : masked(w, mask_w);
        }
    };
    f32x4 sum[FD][FM];
    const int row_w = wave % WD * 16 * FD, row_p = wave / WD * 16 * FM;
    const auto read_w = [&](int buffer, int k, int i) {
        return weights[buffer][place_w(row_w + 32 * (i >> 1) + paired_row(i & 1, lane & 15),
                                       4 * k + (lane >> 4))];
    };
    const auto read_p = [&](int buffer, int k, int j) {
        return patches[buffer][place_p(row_p + 16 * j + (lane & 15), 4 * k + (lane >> 4))];
    };
    // A step's products: 2 FM groups of FD, each behind the next reads, with
    // a part of the next steps' stores and loads after it.
    constexpr int kPieces = kLines + kLoads, kGroups = 2 * FM;
    const auto products = [&](int buffer) {
        Frag fw[2][FD], fp[2 * FM];
#pragma unroll
        for (int i = 0; i < FD; ++i)
            fw[0][i] = read_w(buffer, 0, i);
        fp[0] = read_p(buffer, 0, 0);
        fp[1] = read_p(buffer, 0, 1);
#pragma unroll
        for (int g = 0; g < 2 * FM; ++g) {
            if (g + 2 < 2 * FM)
                fp[g + 2] = read_p(buffer, (g + 2) / FM, (g + 2) % FM);
            if (g >= FM - FD && g < FM)
                fw[1][g - FM + FD] = read_w(buffer, 1, g - FM + FD);
            f32x4 *into[FD];
#pragma unroll
            for (int i = 0; i < FD; ++i)
                into[i] = &sum[i][g % FM];
            multiply<false>(into, fw[g / FM], fp[g]);
#pragma unroll
            for (int i = g * kPieces / kGroups; i < (g + 1) * kPieces / kGroups; ++i) {
                stage(buffer ^ 1, i);
                fetch(i);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    // Steps follow each other through all tiles of the workgroup; past the
    // last tile its last step is loaded again, and not used.
    const uint32_t steps = (a.chunks + 7) / 8;
    uint32_t ahead = blockIdx.x, ahead_step = 0;  // what is loaded next
    const auto advance = [&] {
        if (++ahead_step == steps) {
            if (ahead + gridDim.x < a.tiles) {
                ahead += gridDim.x;
                ahead_step = 0;
                rows_of(ahead);
            } else {
                --ahead_step;
            }
        }
        place(ahead_step);
    };
    rows_of(ahead);
    place(0);
#pragma unroll
    for (int i = 0; i < kPieces; ++i)
        fetch(i);
    mask_p = mask_of<C>(lead_p);
    mask_w = mask_of<C>(lead_w);
    advance();
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
        stage(0, i);
        fetch(i);
    }
    __syncthreads();
    int buffer = 0;
    for (uint32_t piece = blockIdx.x; piece < a.tiles; piece += gridDim.x) {
#pragma unroll
        for (int i = 0; i < FD; ++i)
#pragma unroll
            for (int j = 0; j < FM; ++j)
                sum[i][j] = (f32x4)0.0f;
        for (uint32_t step = 0; step < steps; ++step, buffer ^= 1) {
            mask_p = mask_of<C>(lead_p);
            mask_w = mask_of<C>(lead_w);
            advance();
            products(buffer);
            __syncthreads();
        }
        const uint2 tile = tile_at(piece);
        finish<T, FD, FM>(a, tile.x + row_p, tile.y + row_w, lane, sum);
    }
}

// Few rows: what counts is the time of one load. A workgroup of four waves
// makes 32 columns by 32 rows; the waves divide the summed index between
// them, load their operands straight into the matrix instruction's registers
// (kAhead steps of 64 bytes at once, no barrier), and add up at the end. One
// image of 224 x 224, 768 columns: 4.7 us (12 with tiles of 128).
template <typename T, typename S, int Mode>
__global__ void __launch_bounds__(256, 2) patch_small_kernel(PatchArgs a)
{
    constexpr int C = 16 / sizeof(T), kAhead = 6;
    typedef vec<T, C> Frag;
    __shared__ f32x4 sums[3][4][64];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t tile = piece_of(blockIdx.x, a.tiles);
    const uint32_t tm = divide(tile, a.tiles_n), tn = tile - tm * a.tiles_n.d;
    const uint32_t m0 = tm * 32, d0 = tn * 32;
    const S *image[2];
    const T *weight[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint32_t m = m0 + 16 * h + (lane & 15), d = d0 + paired_row(h, lane & 15);
        image[h] = (const S *)a.images + patch_at(a, m < a.rows ? m : a.rows - 1);
        weight[h] = (const T *)a.weight + (int64_t)(d < a.dim ? d : a.dim - 1) * a.values;
    }
    f32x4 sum[2][2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
            sum[i][j] = (f32x4)0.0f;
    const uint32_t steps = (a.chunks + 3) / 4;
    for (uint32_t first = wave; first < steps; first += 4 * kAhead) {
        vec<S, C> p[kAhead][2];
        Frag w[kAhead][2];
        int32_t lead[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            // steps past the last are zeros
            const Chunk<C> c(a, (first + 4 * k) * 4 + (lane >> 4));
            lead[k] = c.lead;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                p[k][h] = load_chunk<S, C, Mode == kShort>(image[h] + c.image, c.have);
                w[k][h] = load_chunk<T, C, Mode == kShort>(weight[h] + c.weight, c.have);
            }
        }
        asm volatile("" ::: "memory");  // all loads before the products
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const Mask mask = mask_of<C>(lead[k]);
            Frag fp[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                fp[h] = masked(rounded<T, S, C>(p[k][h]), mask);
                w[k][h] = masked(w[k][h], mask);
            }
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                f32x4 *const into[2] = {&sum[0][j], &sum[1][j]};
                multiply<false>(into, w[k], fp[j]);
            }
        }
    }
    if (wave > 0)
#pragma unroll
        for (int k = 0; k < 4; ++k)
            sums[wave - 1][k][lane] = sum[k >> 1][k & 1];
    __syncthreads();
    if (wave > 0)
        return;
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int w = 0; w < 3; ++w)
            sum[k >> 1][k & 1] += sums[w][k][lane];
    finish<T, 2, 2>(a, m0, d0, lane, sum);
}

template <typename T>
int launch_patch(const PatchArgs &a, int image_type, int mode, int tile, void *stream)
{
    with_image<T>(image_type, [&](auto s) {
        typedef decltype(s) S;
        // Large tiles: a workgroup for every compute unit goes through them
        // (256 images of 14-pixel patches to 1024 columns: 123 us, one tile a
        // workgroup 128; of 16-pixel patches to 768 columns 86 and 90). Tiles of
        // 128, of which the chip holds two a unit, are one a workgroup (the first
        // of these calls 171 us, 161 with two workgroups a unit that go through
        // them; a quarter of the second 30 and 29).
        const uint32_t cus = device_cus() > 0 ? device_cus() : 256;
        const dim3 grid(tile == 256 && a.tiles > cus ? cus : a.tiles);
        hipStream_t st = (hipStream_t)stream;
        const auto launch = [&](auto mode) {
            constexpr int M = mode.value;
            // no registers for the largest with short runs or wider pixels in
            // flight; fp32 products take long enough for tiles of 64
            if constexpr (M != kShort && sizeof(S) == 2 && sizeof(T) == 2) {
                if (tile == 256)
                    patch_kernel<T, S, 4, 2, 4, 8, M><<<grid, dim3(512), 0, st>>>(a);
            }
            if constexpr (sizeof(T) == 2) {
                if (tile == 128)
                    patch_kernel<T, S, 2, 2, 4, 4, M><<<grid, dim3(256), 0, st>>>(a);
            }
            if (tile == 64)
                patch_kernel<T, S, 2, 2, 2, 2, M><<<grid, dim3(256), 0, st>>>(a);
            else if (tile == 32)
                patch_small_kernel<T, S, M><<<grid, dim3(256), 0, st>>>(a);
        };
        if (mode == kWhole)
            launch(std::integral_constant<int, kWhole>{});
        else if (mode == kMasked)
            launch(std::integral_constant<int, kMasked>{});
        else
            launch(std::integral_constant<int, kShort>{});
    });
    return (int)hipGetLastError();
}

// Backward: part[s][d][q C + e] = sum over rows m of split s of grad_out[m][d]
// patch[m][chunk q, value e].
//
// The summed index is the row, which both operands have as their slow index.
// A step takes kRows rows of a tile's columns into LDS as they are; of 16-bit
// types the transposing LDS reads then give each lane four rows' values of
// one column, and fp32 operands are read a value a lane. A row's 16-byte
// chunks are moved by a swizzle that puts what is read, or written, at once
// into different banks.
template <typename T, int Cols>
struct GradTile {  // 16-bit types
    static constexpr int kRows = 64, kChunks = Cols / 8;
    // Pairs of chunks are moved by three bits of the row: reads take rows r,
    // r + 1, r + 2, r + 3 and the same + 8 of two chunks' columns, writes two
    // neighbouring rows' four chunks.
    static __device__ __forceinline__ int slot(int row, int chunk)
    {
        const int turn = (row & 1) << 2 | (row & 2) | ((row >> 2 ^ row >> 3) & 1);
        return row * kChunks + (chunk ^ (turn << 1 & (kChunks - 1)));
    }
    // Operands of N neighbouring tiles of 16 columns from col0 (a multiple of
    // 32) on: of tile i, rows 32 k + 8 (lane / 16) .. + 7 of its column lane %
    // 16, in two reads of four rows. Rows four further turn the chunk pairs'
    // lowest bit, so the second read of tile i has the place of the first of
    // tile i ^ 1, four rows on.
    template <int N>
    struct Reader {
        uint32_t at[N];
        __device__ __forceinline__ Reader(int col0, int lane)
        {
            const int row = 8 * (lane >> 4) + ((lane & 15) >> 2);
#pragma unroll
            for (int i = 0; i < N; ++i)
                at[i] = slot(row, (col0 + 16 * i + 4 * (lane & 3)) >> 3) * 16 + (lane & 1) * 8;
        }
        __device__ __forceinline__ vec<T, 8> read(const vec<T, 8> *tile, int k, int i) const
        {
            typedef short s16x4 __attribute__((ext_vector_type(4)));
            typedef __attribute__((address_space(3))) s16x4 Shared;
            s16x4 v[2];
#pragma unroll
            for (int h = 0; h < 2; ++h)
                v[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                    (Shared *)((const char *)tile + at[i ^ h] + (32 * k + 4 * h) * kChunks * 16));
            return __builtin_bit_cast(
                vec<T, 8>, __builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7));
        }
    };
};

template <int Cols>
struct GradTile<float, Cols> {
    static constexpr int kRows = 32, kChunks = Cols / 4;
    // 16 lanes read 64 bytes of a row, four rows at once
    static __device__ __forceinline__ int slot(int row, int chunk)
    {
        return row * kChunks + (chunk ^ (row << 2 & (kChunks - 1) & 28));
    }
    // of tile i, rows 16 k + 4 e + lane / 16, e = 0 .. 3, of its column lane % 16
    template <int N>
    struct Reader {
        int col0, lane;
        __device__ __forceinline__ Reader(int col0, int lane) : col0(col0), lane(lane) {}
        __device__ __forceinline__ vec<float, 4> read(const vec<float, 4> *tile, int k,
                                                      int i) const
        {
            const int col = col0 + 16 * i + (lane & 15);
            vec<float, 4> v;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                v[e] = ((const float *)(tile + slot(16 * k + 4 * e + (lane >> 4), col >> 2)))
                    [col & 3];
            return v;
        }
    };
};

// Loads, stores and products are arranged as in the forward pass: WD x WP
// waves, tiles of 16 FD WD columns of grad_out by 16 FP WP patch values. A
// thread loads one row of each operand a step, four chunks of it. The rows are
// split so that every compute unit has a tile; each split's tile is written once
// in fp32.
//
// 256 images of 224 x 224, patches of 16, 768 bf16 columns: 72 us (820
// TFLOP/s), 28 steps of 2.2 us, 3.3 before them and 4.4 for the tile. fp32, 16
// images of 203 x 331, patches of 20, 380 columns: 33 us; the matrix units are
// busy for 41 of 67 thousand cycles.
template <typename T, typename S, int WD, int WP, int FD, int FP, int Mode>
__global__ void __launch_bounds__(64 * WD * WP, 2) patch_grad_kernel(PatchArgs a, SumArgs b)
{
    if constexpr (WD * WP == 4) {
        // further workgroups, beside these, for the sums of grad_out's columns
        const uint32_t products = a.tiles * a.splits;
        if (blockIdx.x >= products) {
            sum_columns<T>(b, blockIdx.x - products);
            return;
        }
    }
    static_assert(FD * WD == FP * WP, "square tiles");
    constexpr int C = 16 / sizeof(T), kWaves = WD * WP, kThreads = 64 * kWaves;
    constexpr int kSide = 16 * FD * WD;
    typedef GradTile<T, kSide> Tile;
    constexpr int kRows = Tile::kRows, kChunks = Tile::kChunks;
    constexpr int kLoads = kRows * kChunks / kThreads;  // of each operand
    constexpr int kAcross = kThreads / kRows;           // threads of a grad_out row
    constexpr int kBands = kRows / 16;  // waves that read 16 patches each, side by side
    static_assert(kWaves % kBands == 0, "one row a thread");
    typedef vec<T, C> Frag;
    __shared__ Frag patches[2][kRows * kChunks], grads[2][kRows * kChunks];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // the tiles of a part of the rows are neighbours: they share its rows
    const uint32_t piece = piece_of(blockIdx.x, a.tiles * a.splits);
    const uint32_t split = piece / a.tiles, tile = piece - split * a.tiles;
    const uint32_t td = divide(tile, a.tiles_n), tq = tile - td * a.tiles_n.d;
    const uint32_t d0 = td * kSide, q0 = tq * kChunks;
    const uint32_t m_lo = split * a.split_rows;
    const uint32_t m_hi = a.rows - m_lo < a.split_rows ? a.rows : m_lo + a.split_rows;

    // Four lanes read four chunks of a patch, 16 patches side by side;
    // kAcross lanes read a row of grad_out. Values that a patch's chunk
    // repeats need no zeros here: their sums are not used. A chunk that passes
    // grad_out's columns is moved back, and what it repeats is not written.
    const int line_p = (lane >> 2) + 16 * (wave % kBands);
    const int line_g = threadIdx.x / kAcross;
    uint32_t image_at[kLoads];
    int32_t have = C;
    // rows of grad_out shorter than a chunk are left to the kernels of short runs
    const bool wide = Mode != kShort || a.dim >= (uint32_t)C;
    const auto slot_p = [&](int i) {
        return (lane & 3) + 4 * (wave / kBands + kWaves / kBands * i);
    };
    const auto slot_g = [&](int i) { return (int)(threadIdx.x % kAcross) + kAcross * i; };
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
        const Chunk<C> c(a, q0 + slot_p(i));
        image_at[i] = c.image;
        have = c.have;
    }
    const auto grad_at = [&](int i) {
        const uint32_t d = d0 + slot_g(i) * C;
        return d <= a.dim - C ? d : a.dim - C;
    };
    vec<S, C> next_p[kLoads];
    Frag next_g[kLoads];
    const S *image = nullptr;
    const T *grad = nullptr;
    // the present row's: whether the step in flight, and that being stored, have it
    bool live_p = false, live_g = false, store_p = false, store_g = false;
    const auto rows_of = [&](uint32_t m0) {
        const uint32_t mp = m0 + line_p, mg = m0 + line_g;
        live_p = mp < m_hi;
        live_g = mg < m_hi;
        image = (const S *)a.images + patch_at(a, live_p ? mp : m_lo);
        const uint32_t at = live_g ? mg : m_lo;
        const uint32_t im = divide(at, a.tokens), t = at - im * a.tokens.d;
        grad = (const T *)a.grad_out + im * a.image_stride + t * a.row_stride;
    };
    const auto fetch = [&](int i) {
        if (i < kLoads)
            next_p[i] = load_chunk<S, C, Mode == kShort>(image + image_at[i], have);
        else
            next_g[i - kLoads] = wide ? load<T, C>(grad + grad_at(i - kLoads))
                                      : load_chunk<T, C, true>(grad, a.dim);
    };
    const auto stage = [&](int buffer, int i) {  // rows past the part: zeros on both sides
        if (i < kLoads) {
            patches[buffer][Tile::slot(line_p, slot_p(i))] =
                store_p ? rounded<T, S, C>(next_p[i]) : (Frag)(T)0.0f;
        } else {
            grads[buffer][Tile::slot(line_g, slot_g(i - kLoads))] =
                store_g ? next_g[i - kLoads] : (Frag)(T)0.0f;
        }
    };
    f32x4 sum[FD][FP];  // [grad_out's columns][patch values]
#pragma unroll
    for (int i = 0; i < FD; ++i)
#pragma unroll
        for (int j = 0; j < FP; ++j)
            sum[i][j] = (f32x4)0.0f;
    const int col_g = wave % WD * 16 * FD, col_p = wave / WD * 16 * FP;
    constexpr int kPieces = 2 * kLoads, kGroups = 2 * FP;
    const typename Tile::template Reader<FD> reader_g(col_g, lane);
    const typename Tile::template Reader<FP> reader_p(col_p, lane);
    const auto products = [&](int buffer) {
        Frag fg[2][FD], fp[2 * FP];
#pragma unroll
        for (int i = 0; i < FD; ++i)
            fg[0][i] = reader_g.read(grads[buffer], 0, i);
        fp[0] = reader_p.read(patches[buffer], 0, 0);
#pragma unroll
        for (int g = 0; g < 2 * FP; ++g) {
            if (g + 1 < 2 * FP)
                fp[g + 1] = reader_p.read(patches[buffer], (g + 1) / FP, (g + 1) % FP);
            if (g >= FP - FD / 2 && g < FP) {
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    fg[1][2 * (g - FP + FD / 2) + h] =
                        reader_g.read(grads[buffer], 1, 2 * (g - FP + FD / 2) + h);
            }
            f32x4 *into[FD];
#pragma unroll
            for (int i = 0; i < FD; ++i)
                into[i] = &sum[i][g % FP];
            multiply<true>(into, fg[g / FP], fp[g]);
#pragma unroll
            for (int i = g * kPieces / kGroups; i < (g + 1) * kPieces / kGroups; ++i) {
                stage(buffer ^ 1, i);
                fetch(i);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    rows_of(m_lo);
#pragma unroll
    for (int i = 0; i < kPieces; ++i)
        fetch(i);
    store_p = live_p;
    store_g = live_g;
    rows_of(m_lo + kRows);
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
        stage(0, i);
        fetch(i);
    }
    __syncthreads();
    int buffer = 0;
    for (uint32_t m = m_lo; m < m_hi; m += kRows, buffer ^= 1) {
        store_p = live_p;
        store_g = live_g;
        rows_of(m + 2 * kRows);
        products(buffer);
        __syncthreads();
    }
    // A lane has four patch values of one column of grad_out: column col of
    // the tile is column d0 + col, or of a chunk moved back, counted from the
    // row's end.
    const uint32_t width = a.chunks * C;
    float *part = (float *)a.out + (int64_t)split * a.dim * width;
#pragma unroll
    for (int i = 0; i < FD; ++i) {
        const uint32_t col = col_g + 16 * i + (lane & 15);
        const uint32_t want = d0 + col / C * C;
        uint32_t d = d0 + col;
        if (wide && want > a.dim - C)  // in a chunk that was moved back
            d = want < a.dim ? a.dim - C + col % C : a.dim;
        if (d >= a.dim || (wide && d < want))
            continue;
#pragma unroll
        for (int j = 0; j < FP; ++j) {
            const uint32_t k = q0 * C + col_p + 16 * j + 4 * (lane >> 4);
            if (k < width)
                store<float, 4>(part + (int64_t)d * width + k, sum[i][j]);
        }
    }
}

template <typename T>
int launch_patch_grad(const PatchArgs &a, const SumArgs &b, int image_type, int mode, int tile,
                      void *stream)
{
    with_image<T>(image_type, [&](auto s) {
        typedef decltype(s) S;
        const dim3 grid(a.tiles * a.splits + b.groups);
        hipStream_t st = (hipStream_t)stream;
        const auto launch = [&](auto mode) {
            constexpr int M = mode.value;
            if constexpr (M == kWhole && sizeof(S) == 2 && sizeof(T) == 2) {
                if (tile == 256)
                    patch_grad_kernel<T, S, 4, 2, 4, 8, M><<<grid, dim3(512), 0, st>>>(a, b);
            }
            if (tile == 128)
                patch_grad_kernel<T, S, 2, 2, 4, 4, M><<<grid, dim3(256), 0, st>>>(a, b);
        };
        if (mode == kShort)
            launch(std::integral_constant<int, kShort>{});
        else
            launch(std::integral_constant<int, kWhole>{});
    });
    return (int)hipGetLastError();
}

}  // namespace
}  // namespace smol

#endif  // SMOL_PATCH_KERNELS_H
