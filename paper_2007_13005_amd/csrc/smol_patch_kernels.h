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
// positions of two rows are asked for together before any is used.
template <typename T, int FD, int FM>
__device__ __forceinline__ void finish(const PatchArgs &a, uint32_t m0, uint32_t d0, int lane,
                                       f32x4 (&sum)[FD][FM])
{
    constexpr int N = FD / 2;
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
        for (int first = 0; first < FM; first += 2) {
            T *out[2];
            vec<T, 8> pos[2][N];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                uint32_t m = m0 + 16 * (first + j) + (lane & 15);
                m = m < a.rows ? m : a.rows - 1;
                const uint32_t i = divide(m, a.tokens), t = m - i * a.tokens.d;
                out[j] = (T *)a.out + i * a.image_stride + t * a.row_stride + d1;
                if (a.pos)
#pragma unroll
                    for (int k = 0; k < N; ++k)
                        pos[j][k] = load<T, 8>((const T *)a.pos + (int64_t)t * a.dim + d1 + 32 * k);
            }
            asm volatile("" ::: "memory");
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                if (m0 + 16 * (first + j) + (lane & 15) >= a.rows)
                    continue;
#pragma unroll
                for (int k = 0; k < N; ++k) {
                    vec<float, 8> v = sums_of(first + j, k);
                    if (a.bias)
                        v += to_f32<8, T>(bias[k]);
                    if (a.pos)
                        v += to_f32<8, T>(pos[j][k]);
                    store<T, 8>(out[j] + 32 * k, from_f32<T, 8>(v));
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
    constexpr int kPieces = kLines + kLoads, kEvery = 2 * FM / kPieces;
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
#pragma unroll
            for (int i = 0; i < FD; ++i)
                sum[i][g % FM] = mma(fw[g / FM][i], fp[g], sum[i][g % FM]);
            if (g % kEvery == kEvery - 1) {
                stage(buffer ^ 1, g / kEvery);
                fetch(g / kEvery);
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
// (kAhead steps of 64 bytes at once, no barrier), and add up at the end.
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
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    sum[i][j] = mma(w[k][i], fp[j], sum[i][j]);
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
        // (256 images of 14-pixel patches to 1024 columns: 134 us, one tile a
        // workgroup 138). Of tiles of 128 the chip holds two a unit, and one
        // tile a workgroup is the faster (170 us, 177).
        const uint32_t cus = device_cus() > 0 ? device_cus() : 256;
        const dim3 grid(tile == 256 && a.tiles > cus ? cus : a.tiles);
        hipStream_t st = (hipStream_t)stream;
        const auto launch = [&](auto mode) {
            constexpr int M = mode.value;
            // no registers for the largest with short runs, wider pixels in
            // flight, or fp32 (whose products take long enough for a smaller)
            if constexpr (M != kShort && sizeof(S) == 2 && sizeof(T) == 2) {
                if (tile == 256)
                    patch_kernel<T, S, 4, 2, 4, 8, M><<<grid, dim3(512), 0, st>>>(a);
            }
            if (tile == 128)
                patch_kernel<T, S, 2, 2, 4, 4, M><<<grid, dim3(256), 0, st>>>(a);
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
// A step takes 64 rows (fp32: 32) of 32 F columns of each into LDS as they
// are; of 16-bit types the transposing LDS reads then give each lane four
// rows' values of one column, and fp32 operands are read a value a lane. A
// row's 16-byte chunks are moved by a swizzle of their 32-byte pairs that
// puts the rows read at once into different banks.
template <typename T, int F>
struct GradTile;

template <int F, typename T>
struct GradTile16 {
    static constexpr int kRows = 64, kCols = 32 * F, kChunks = kCols / 8;
    static __device__ __forceinline__ int slot(int row, int chunk)
    {
        const int pairs = kChunks / 2;
        const int turn = ((row & 7) ^ (row >> 1 & 4)) & (pairs - 1);
        return row * kChunks + ((((chunk >> 1) ^ turn) << 1) | (chunk & 1));
    }
    // rows 32 k + 8 (lane / 16) .. + 7 of column col0 + lane % 16
    static __device__ __forceinline__ vec<T, 8> read(const vec<T, 8> *tile, int k, int col0,
                                                     int lane)
    {
        typedef short s16x4 __attribute__((ext_vector_type(4)));
        typedef short s16x8 __attribute__((ext_vector_type(8)));
        typedef __attribute__((address_space(3))) s16x4 Shared;
        const int row = 32 * k + 8 * (lane >> 4) + ((lane & 15) >> 2);
        const int col = col0 + 4 * (lane & 3);
        s16x4 v[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const char *p = (const char *)(tile + slot(row + 4 * h, col >> 3)) + (col & 4) * 2;
            v[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Shared *)p);
        }
        return __builtin_bit_cast(vec<T, 8>, __builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5,
                                                                      6, 7));
    }
};
template <int F>
struct GradTile<f16, F> : GradTile16<F, f16> {};
template <int F>
struct GradTile<bf16, F> : GradTile16<F, bf16> {};

template <int F>
struct GradTile<float, F> {
    static constexpr int kRows = 32, kCols = 32 * F, kChunks = kCols / 4;
    // 16 lanes read 64 bytes of a row, four rows at once
    static __device__ __forceinline__ int slot(int row, int chunk)
    {
        return row * kChunks + (chunk ^ (row << 2 & (kChunks - 1)));
    }
    // rows 16 k + 4 e + lane / 16, e = 0 .. 3, of column col0 + lane % 16
    static __device__ __forceinline__ vec<float, 4> read(const vec<float, 4> *tile, int k,
                                                         int col0, int lane)
    {
        const int col = col0 + (lane & 15);
        vec<float, 4> v;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            v[e] = ((const float *)(tile + slot(16 * k + 4 * e + (lane >> 4), col >> 2)))[col & 3];
        return v;
    }
};

template <typename T, typename S, int F, int Mode>
__global__ void __launch_bounds__(256, F == 4 ? 2 : 4) patch_grad_kernel(PatchArgs a)
{
    typedef GradTile<T, F> Tile;
    constexpr int C = 16 / sizeof(T), kSide = 32 * F, kRows = Tile::kRows;
    constexpr int kLoads = kRows * Tile::kChunks / 256, kStride = 256 / Tile::kChunks;
    constexpr int kLines = kRows / 32, kSlots = Tile::kChunks / 8;
    typedef vec<T, C> Frag;
    __shared__ Frag patches[2][kRows * Tile::kChunks], grads[2][kRows * Tile::kChunks];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    // the tiles of a part of the rows are neighbours: they share its rows
    const uint32_t piece = piece_of(blockIdx.x, a.tiles * a.splits);
    const uint32_t split = piece / a.tiles, tile = piece - split * a.tiles;
    const uint32_t td = divide(tile, a.tiles_n), tq = tile - td * a.tiles_n.d;
    const uint32_t d0 = td * kSide, q0 = tq * Tile::kChunks;
    const uint32_t m_lo = split * a.split_rows;
    const uint32_t m_hi = a.rows - m_lo < a.split_rows ? a.rows : m_lo + a.split_rows;

    // This thread's loads: kLines patches of kSlots chunks, 32 patches side by
    // side; kLoads rows of one chunk of grad_out, whole lines of it. A chunk
    // that passes grad_out's columns is moved back, and what it repeats is
    // not written at the end.
    const uint32_t line_p = threadIdx.x & 31, slot_p = threadIdx.x >> 5;
    uint32_t image_at[kSlots];
    int32_t lead[kSlots], have = C;
#pragma unroll
    for (int k = 0; k < kSlots; ++k) {
        const Chunk<C> c(a, q0 + slot_p + 8 * k);
        image_at[k] = c.image;
        lead[k] = c.lead;
        have = c.have;
    }
    const uint32_t chunk = threadIdx.x % Tile::kChunks, line = threadIdx.x / Tile::kChunks;
    const uint32_t d = d0 + chunk * C;
    const bool wide = a.dim >= (uint32_t)C;
    const uint32_t d_at = !wide ? 0 : d <= a.dim - C ? d : a.dim - C;
    vec<S, C> next_p[kLines][kSlots];
    Frag next_g[kLoads];
    uint32_t fetched = 0;
    const auto fetch = [&](uint32_t m0) {
        fetched = m0;
#pragma unroll
        for (int i = 0; i < kLines; ++i) {
            const uint32_t m = m0 + line_p + 32 * i;
            const S *image = (const S *)a.images + patch_at(a, m < m_hi ? m : m_hi - 1);
#pragma unroll
            for (int k = 0; k < kSlots; ++k)
                next_p[i][k] = load_chunk<S, C, Mode == kShort>(image + image_at[k], have);
        }
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const uint32_t m = m0 + line + i * kStride;
            const uint32_t at = m < m_hi ? m : m_hi - 1;
            const uint32_t im = divide(at, a.tokens), t = at - im * a.tokens.d;
            const T *g = (const T *)a.grad_out + im * a.image_stride + t * a.row_stride + d_at;
            next_g[i] = wide ? load<T, C>(g) : load_chunk<T, C, true>(g, a.dim);
        }
    };
    const auto stage = [&](int buffer) {
        // rows past the part: zeros on both sides
#pragma unroll
        for (int k = 0; k < kSlots; ++k) {
            const Mask mask = mask_of<C>(lead[k]);
#pragma unroll
            for (int i = 0; i < kLines; ++i) {
                Frag p = rounded<T, S, C>(next_p[i][k]);
                if (Mode != kWhole)
                    p = masked(p, mask);
                if (fetched + line_p + 32 * i >= m_hi)
                    p = (Frag)(T)0.0f;
                patches[buffer][Tile::slot(line_p + 32 * i, slot_p + 8 * k)] = p;
            }
        }
#pragma unroll
        for (int i = 0; i < kLoads; ++i)
            grads[buffer][Tile::slot(line + i * kStride, chunk)] =
                fetched + line + i * kStride < m_hi ? next_g[i] : (Frag)(T)0.0f;
    };
    f32x4 sum[F][F];  // [grad_out's columns][patch values]
#pragma unroll
    for (int i = 0; i < F; ++i)
#pragma unroll
        for (int j = 0; j < F; ++j)
            sum[i][j] = (f32x4)0.0f;
    const int col_g = (wave & 1) * 16 * F, col_p = (wave >> 1) * 16 * F;
    fetch(m_lo);
    stage(0);
    __syncthreads();
    int buffer = 0;
    for (uint32_t m = m_lo; m < m_hi; m += kRows, buffer ^= 1) {
        const bool more = m_hi - m > kRows;
        if (more)
            fetch(m + kRows);
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            Frag fg[F], fp[F];
#pragma unroll
            for (int i = 0; i < F; ++i) {
                fg[i] = Tile::read(grads[buffer], k, col_g + 16 * i, lane);
                fp[i] = Tile::read(patches[buffer], k, col_p + 16 * i, lane);
            }
#pragma unroll
            for (int i = 0; i < F; ++i)
#pragma unroll
                for (int j = 0; j < F; ++j)
                    sum[i][j] = mma(fp[j], fg[i], sum[i][j]);
        }
        if (more)
            stage(buffer ^ 1);
        __syncthreads();
    }
    // a lane has four patch values of one column of grad_out. Column tile
    // chunks moved back end with the row: column col of the tile is column
    // d0 + col of grad_out, or of its chunk counted from the row's end.
    const uint32_t width = a.chunks * C;
    float *part = (float *)a.out + (int64_t)split * a.dim * width;
#pragma unroll
    for (int i = 0; i < F; ++i) {
        const uint32_t col = col_g + 16 * i + (lane & 15);
        const uint32_t want = d0 + col / C * C;
        uint32_t dd = d0 + col;
        if (wide && want > a.dim - C)  // in a chunk that was moved back
            dd = want < a.dim ? a.dim - C + col % C : a.dim;
        if (dd >= a.dim || (wide && dd < want))
            continue;
#pragma unroll
        for (int j = 0; j < F; ++j) {
            const uint32_t k = q0 * C + col_p + 16 * j + 4 * (lane >> 4);
            if (k < width)
                store<float, 4>(part + (int64_t)dd * width + k, sum[i][j]);
        }
    }
}

template <typename T>
int launch_patch_grad(const PatchArgs &a, int image_type, int mode, int tile, void *stream)
{
    with_image<T>(image_type, [&](auto s) {
        typedef decltype(s) S;
        const dim3 grid(a.tiles * a.splits), block(256);
        hipStream_t st = (hipStream_t)stream;
        const auto launch = [&](auto f) {
            constexpr int F = f.value;
            if (mode == kWhole)
                patch_grad_kernel<T, S, F, kWhole><<<grid, block, 0, st>>>(a);
            else if (mode == kMasked)
                patch_grad_kernel<T, S, F, kMasked><<<grid, block, 0, st>>>(a);
            else
                patch_grad_kernel<T, S, F, kShort><<<grid, block, 0, st>>>(a);
        };
        if (tile == 4)
            launch(std::integral_constant<int, 4>{});
        else
            launch(std::integral_constant<int, 2>{});
    });
    return (int)hipGetLastError();
}

}  // namespace
}  // namespace smol

#endif  // SMOL_PATCH_KERNELS_H
