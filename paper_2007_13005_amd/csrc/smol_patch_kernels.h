// smol_patch_kernels.h -- the patch embedding's kernels as templates, for one
// type of the weight (instantiated by smol_patch_<type>.hip).
#ifndef SMOL_PATCH_KERNELS_H
#define SMOL_PATCH_KERNELS_H

#include "smol_patch.h"

namespace smol {
namespace {

// Forward: out[m][d] = sum_k patch[m][k] weight[d][k] + bias[d] + pos[t][d].
//
// A workgroup of four waves makes a tile of 32 F x 32 F outputs, two waves
// each way, in steps of eight chunks (128 bytes of a patch). The step after
// next's operands are loaded into registers while the present one is
// multiplied out of LDS: images are gathered (and rounded to the weight's
// type) on the way, so no unfolded copy of them is made. A chunk c of row r
// stands at slot c ^ (r & 7) of its row, so the 16 rows that a wave reads at
// once are spread over the banks.
template <typename T, typename S, int F, int Mode>
__global__ void __launch_bounds__(256, F == 4 ? 2 : 4) patch_kernel(PatchArgs a)
{
    constexpr int C = 16 / sizeof(T), kSide = 32 * F;
    typedef vec<T, C> Frag;
    __shared__ Frag patches[2][kSide * 8], weights[2][kSide * 8];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint32_t tile = piece_of(blockIdx.x, a.tiles);
    const uint32_t tm = divide(tile, a.tiles_n), tn = tile - tm * a.tiles_n.d;
    const uint32_t m0 = tm * kSide, d0 = tn * kSide;
    const uint32_t slot = threadIdx.x & 7, line = threadIdx.x >> 3;

    // rows past the last are read as the last, and not written
    const S *image[F];
    const T *weight[F];
#pragma unroll
    for (int i = 0; i < F; ++i) {
        const uint32_t m = m0 + line + 32 * i, d = d0 + line + 32 * i;
        image[i] = (const S *)a.images + patch_at(a, m < a.rows ? m : a.rows - 1);
        weight[i] = (const T *)a.weight + (int64_t)(d < a.dim ? d : a.dim - 1) * a.values;
    }
    Frag next_p[F], next_w[F];
    const auto fetch = [&](uint32_t step) {
        const Chunk<C> c(a, step * 8 + slot);
#pragma unroll
        for (int i = 0; i < F; ++i) {
            next_p[i] = load_chunk<S, T, C, Mode == kShort>(image[i] + c.image, c.have);
            next_w[i] = load_chunk<T, T, C, Mode == kShort>(weight[i] + c.weight, c.have);
            if (Mode != kWhole) {
                next_p[i] = masked<T, C>(next_p[i], c.lead);
                next_w[i] = masked<T, C>(next_w[i], c.lead);
            }
        }
    };
    const auto stage = [&](int buffer) {
#pragma unroll
        for (int i = 0; i < F; ++i) {
            const uint32_t to = (line + 32 * i) * 8 + (slot ^ (line & 7));
            patches[buffer][to] = next_p[i];
            weights[buffer][to] = next_w[i];
        }
    };
    f32x4 sum[F][F];  // [weight rows][patches]
#pragma unroll
    for (int i = 0; i < F; ++i)
#pragma unroll
        for (int j = 0; j < F; ++j)
            sum[i][j] = (f32x4)0.0f;
    const int row_w = (wave & 1) * 16 * F + (lane & 15), row_p = (wave >> 1) * 16 * F + (lane & 15);
    const uint32_t steps = (a.chunks + 7) / 8;
    fetch(0);
    stage(0);
    __syncthreads();
    for (uint32_t step = 0; step < steps; ++step) {
        const int buffer = step & 1;
        if (step + 1 < steps)
            fetch(step + 1);
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int at = (4 * k + (lane >> 4)) ^ (lane & 7);
            Frag fw[F], fp[F];
#pragma unroll
            for (int i = 0; i < F; ++i) {
                fw[i] = weights[buffer][(row_w + 16 * i) * 8 + at];
                fp[i] = patches[buffer][(row_p + 16 * i) * 8 + at];
            }
#pragma unroll
            for (int i = 0; i < F; ++i)
#pragma unroll
                for (int j = 0; j < F; ++j)
                    sum[i][j] = mma(fw[i], fp[j], sum[i][j]);
        }
        if (step + 1 < steps)
            stage(buffer ^ 1);
        __syncthreads();
    }
#pragma unroll
    for (int j = 0; j < F; ++j) {
        const uint32_t m = m0 + row_p + 16 * j;
        if (m >= a.rows)
            continue;
        const uint32_t i = divide(m, a.tokens), t = m - i * a.tokens.d;
        T *out = (T *)a.out + i * a.image_stride + t * a.row_stride;
        const T *pos = a.pos ? (const T *)a.pos + (int64_t)t * a.dim : nullptr;
#pragma unroll
        for (int k = 0; k < F; ++k) {
            const uint32_t d = d0 + (wave & 1) * 16 * F + 16 * k + 4 * (lane >> 4);
            f32x4 v = sum[k][j];
            if (d + 4 <= a.dim) {
                if (a.bias)
                    v += to_f32<4, T>(load<T, 4>((const T *)a.bias + d));
                if (pos)
                    v += to_f32<4, T>(load<T, 4>(pos + d));
                store<T, 4>(out + d, from_f32<T, 4>(v));
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (d + e < a.dim) {
                        float y = v[e];
                        if (a.bias)
                            y += (float)((const T *)a.bias)[d + e];
                        if (pos)
                            y += (float)pos[d + e];
                        out[d + e] = (T)y;
                    }
            }
        }
    }
}

template <typename T>
int launch_patch(const PatchArgs &a, int image_type, int mode, int tile, void *stream)
{
    with_image<T>(image_type, [&](auto s) {
        typedef decltype(s) S;
        const dim3 grid(a.tiles), block(256);
        hipStream_t st = (hipStream_t)stream;
        const auto launch = [&](auto f) {
            constexpr int F = f.value;
            if (mode == kWhole)
                patch_kernel<T, S, F, kWhole><<<grid, block, 0, st>>>(a);
            else if (mode == kMasked)
                patch_kernel<T, S, F, kMasked><<<grid, block, 0, st>>>(a);
            else
                patch_kernel<T, S, F, kShort><<<grid, block, 0, st>>>(a);
        };
        if (tile == 4)
            launch(std::integral_constant<int, 4>{});
        else if (tile == 2)
            launch(std::integral_constant<int, 2>{});
        else
            launch(std::integral_constant<int, 1>{});
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
        const int turn = ((row & 3) | (row >> 1 & 4)) & (pairs - 1);
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
        return row * kChunks + (chunk ^ ((row & 3) << 2 & (kChunks - 1)));
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
    typedef vec<T, C> Frag;
    __shared__ Frag patches[2][kRows * Tile::kChunks], grads[2][kRows * Tile::kChunks];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    // the tiles of a part of the rows are neighbours: they share its rows
    const uint32_t piece = piece_of(blockIdx.x, a.tiles * a.splits);
    const uint32_t split = piece / a.tiles, tile = piece - split * a.tiles;
    const uint32_t td = divide(tile, a.tiles_n), tq = tile - td * a.tiles_n.d;
    const uint32_t d0 = td * kSide, q0 = tq * Tile::kChunks;
    const int chunk = threadIdx.x % Tile::kChunks, line = threadIdx.x / Tile::kChunks;

    const uint32_t m_lo = split * a.split_rows;
    const uint32_t m_hi = a.rows - m_lo < a.split_rows ? a.rows : m_lo + a.split_rows;
    // this thread's chunk of the patches, and of grad_out's columns: a chunk
    // that passes the columns is moved back, what it repeats is not written
    const Chunk<C> c(a, q0 + chunk);
    const uint32_t d = d0 + chunk * C;
    const bool wide = a.dim >= (uint32_t)C;
    const uint32_t d_at = !wide ? 0 : d <= a.dim - C ? d : a.dim - C;
    const int32_t d_have = wide ? C : a.dim;
    (void)d_have;
    Frag next_p[kLoads], next_g[kLoads];
    const auto fetch = [&](uint32_t m0) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const uint32_t m = m0 + line + i * kStride;
            const uint32_t at = m < m_hi ? m : m_hi - 1;
            const S *image = (const S *)a.images + patch_at(a, at) + c.image;
            next_p[i] = load_chunk<S, T, C, Mode == kShort>(image, c.have);
            if (Mode != kWhole)
                next_p[i] = masked<T, C>(next_p[i], c.lead);
            const uint32_t im = divide(at, a.tokens), t = at - im * a.tokens.d;
            const T *g = (const T *)a.grad_out + im * a.image_stride + t * a.row_stride + d_at;
            next_g[i] = wide ? load<T, C>(g) : load_chunk<T, T, C, true>(g, d_have);
            if (m >= m_hi) {  // rows past the part: zeros on both sides
                next_p[i] = (Frag)(T)0.0f;
                next_g[i] = (Frag)(T)0.0f;
            }
        }
    };
    const auto stage = [&](int buffer) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int to = Tile::slot(line + i * kStride, chunk);
            patches[buffer][to] = next_p[i];
            grads[buffer][to] = next_g[i];
        }
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
