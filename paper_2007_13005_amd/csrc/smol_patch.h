// smol_patch.h -- what the patch embedding's forward and backward kernels
// share: where a patch's values stand in the image, and their loads.
//
// A patch is `runs` runs of `length` consecutive image elements (NCHW: one
// per channel and patch row, `patch` long; NHWC: one per patch row, patch *
// channels long), and a weight row is the same runs one after the other. The
// kernels take runs in chunks of 16 bytes of the weight's type; a run's last
// chunk is moved back to end with the run, and the values that it repeats
// count as zeros ("lead" of them). So no load passes a run, whatever its
// length, and a matrix product over chunks is one over the values.
#ifndef SMOL_PATCH_H
#define SMOL_PATCH_H

#include <type_traits>

#include "smol_tokens.h"
#include "smol_tokens_device.h"

namespace smol {

struct PatchArgs {
    const void *images, *weight, *bias, *pos;
    void *out;              // forward: rows; backward: partial products
    const void *grad_out;
    int64_t image_stride, row_stride;  // of out or grad_out
    int64_t image_size;     // elements of an image
    uint32_t rows, dim;     // n * tokens; columns
    uint32_t values;        // of a patch: runs * length
    uint32_t length;        // of a run
    uint32_t chunks;        // of a patch
    uint32_t step_y, step_x;      // elements from a patch to the next
    uint32_t plane, pitch;        // from a channel, and a run, to the next
    Divisor tokens, across, per_run, per_channel;  // tokens of an image and
                            // across it; chunks of a run; runs of a channel
    uint32_t tiles;  // of the output; tiles_n of them side by side
    Divisor tiles_n;
    uint32_t splits, split_rows;  // backward: parts of the rows, rows a part
};

// Where image row m's patch (m = image * tokens + token) begins.
__device__ __forceinline__ int64_t patch_at(const PatchArgs &a, uint32_t m)
{
    const uint32_t i = divide(m, a.tokens), t = m - i * a.tokens.d;
    const uint32_t ty = divide(t, a.across), tx = t - ty * a.across.d;
    return i * a.image_size + (int64_t)ty * a.step_y + tx * a.step_x;
}

// Chunk q of a patch for elements of which C make a chunk: its place in the
// patch, in the weight row, and how many of its first values are not its own
// (C for a chunk past the patch).
template <int C>
struct Chunk {
    uint32_t image, weight;
    int32_t lead;
    int32_t have;  // values from `image` on that the run has (C unless the run is shorter)
    __device__ __forceinline__ Chunk(const PatchArgs &a, uint32_t q)
    {
        const bool past = q >= a.chunks;
        q = past ? a.chunks - 1 : q;
        const uint32_t r = divide(q, a.per_run), j = (q - r * a.per_run.d) * C;
        const uint32_t back = a.length >= C ? a.length - C : 0;
        const uint32_t at = j < back ? j : back;
        const uint32_t ch = divide(r, a.per_channel);
        image = ch * a.plane + (r - ch * a.per_channel.d) * a.pitch + at;
        weight = r * a.length + at;
        lead = past ? C : j - at;
        have = a.length < C ? a.length : C;
    }
};

// Sets a chunk's first `lead` values to zero.
struct Mask {
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
    u32x4 keep;
};
template <int C>
__device__ __forceinline__ Mask mask_of(int32_t lead)
{
    Mask m;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        if (C == 4)
            m.keep[w] = w >= lead ? ~0u : 0u;
        else
            m.keep[w] = (2 * w >= lead ? 0xffffu : 0u) | (2 * w + 1 >= lead ? 0xffff0000u : 0u);
    }
    return m;
}
template <typename V>
__device__ __forceinline__ V masked(V v, const Mask &m)
{
    return __builtin_bit_cast(V, __builtin_bit_cast(Mask::u32x4, v) & m.keep);
}

// C elements from p; Short: only the first `have` exist. The second form takes
// an offset in bytes below 2^32 from a base that the wave shares.
template <typename S, int C, bool Short>
__device__ __forceinline__ vec<S, C> load_chunk(const S *p, int32_t have)
{
    if (!Short)
        return load<S, C>(p);
    vec<S, C> v;
#pragma unroll
    for (int e = 0; e < C; ++e)
        v[e] = e < have ? p[e] : (S)0.0f;
    return v;
}

template <typename S, int C, bool Short>
__device__ __forceinline__ vec<S, C> load_chunk(const void *base, uint32_t bytes, int32_t have)
{
    return load_chunk<S, C, Short>((const S *)((const char *)base + bytes), have);
}

// To the weight's type.
template <typename T, typename S, int C>
__device__ __forceinline__ vec<T, C> rounded(vec<S, C> v)
{
    if constexpr (std::is_same<S, T>::value)
        return v;
    else
        return from_f32<T, C>(to_f32<C, S>(v));
}

typedef float f32x4 __attribute__((ext_vector_type(4)));

// The products of N first operands with one second operand, or the other way
// round (Swap), each added to a 16 x 16 tile in fp32. A lane has 16 bytes of
// each operand, of one of its 16 rows; the four quarters of the wave hold
// different values of the summed index. Lane l of a result has rows 4 (l / 16)
// .. + 3 of the first operand, column l % 16 of the second.
template <bool Swap, int N, typename V>
__device__ __forceinline__ void multiply(f32x4 *const (&sum)[N], const V (&many)[N], const V &one)
{
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const V a = Swap ? one : many[i], b = Swap ? many[i] : one;
        if constexpr (std::is_same<V, vec<f16, 8>>::value)
            *sum[i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, *sum[i], 0, 0, 0);
        else if constexpr (std::is_same<V, vec<bf16, 8>>::value)
            *sum[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, *sum[i], 0, 0, 0);
    }
    if constexpr (std::is_same<V, vec<float, 4>>::value) {
        // the N tiles in turn: an instruction does not wait for the last
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int i = 0; i < N; ++i)
                *sum[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(
                    Swap ? one[e] : many[i][e], Swap ? many[i][e] : one[e], *sum[i], 0, 0, 0);
    }
}

// Workgroup b's piece of work of `count`: workgroups are dealt out to the
// chip's eight dies in turn, and neighbouring pieces share operands, so each
// die takes a contiguous range of them (its L2 then holds the shared rows).
__device__ __forceinline__ uint32_t piece_of(uint32_t b, uint32_t count)
{
    const uint32_t die = b & 7, each = count >> 3, more = count & 7;
    return die * each + (die < more ? die : more) + (b >> 3);
}

// Column sums of grad_out over the images of a part, for every token: eight
// columns a thread, 256 threads a workgroup. sums[part][token][column]. 256
// images of 196 tokens, 768 bf16 columns: 15 us, 5.1 TB/s.
struct SumArgs {
    const void *grad_out;
    float *sums;
    int64_t image_stride, row_stride;
    uint32_t n, tokens, dim, part_images;
    Divisor columns;   // groups of columns in a row
    Divisor per_part;  // workgroups of a part
    uint32_t groups;   // of all parts (0: no sums wanted)
};

template <typename T, int V>
__device__ __forceinline__ void sum_columns_of(const SumArgs &a, uint32_t group)
{
    const uint32_t part = divide(group, a.per_part);
    const uint32_t e = (group - part * a.per_part.d) * 256 + threadIdx.x;
    const uint32_t t = divide(e, a.columns), col = (e - t * a.columns.d) * V;
    if (t >= a.tokens)
        return;
    const uint32_t at = col <= a.dim - V ? col : a.dim - V;
    const uint32_t lo = part * a.part_images;
    const uint32_t hi = a.n - lo < a.part_images ? a.n : lo + a.part_images;
    const T *p = (const T *)a.grad_out + (int64_t)t * a.row_stride + at;
    vec<float, V> sum = (vec<float, V>)0.0f;
#pragma unroll 8
    for (uint32_t i = lo; i < hi; ++i)
        sum += to_f32<V, T>(load<T, V>(p + i * a.image_stride));
    // columns of a group moved back are written twice, alike
    store<float, V>(a.sums + ((int64_t)part * a.tokens + t) * a.dim + at, sum);
}

template <typename T>
__device__ __forceinline__ void sum_columns(const SumArgs &a, uint32_t group)
{
    if (a.dim >= 8)
        sum_columns_of<T, 8>(a, group);
    else
        sum_columns_of<T, 1>(a, group);
}

// How a patch's runs meet the chunks: whole runs of whole chunks and a whole
// number of K steps; chunks that repeat values or are past the patch; runs
// shorter than a chunk.
enum { kWhole, kMasked, kShort };

// Calls f with the image's element type; a type of the weight takes fp32 and
// fp16 images, and bf16 ones if it is bf16 itself.
template <typename T, typename F>
auto with_image(int type, F f)
{
    if constexpr (std::is_same<T, bf16>::value)
        if (type == SMOL_ELEM_BF16)
            return f(bf16{});
    return type == SMOL_ELEM_F32 ? f(float{}) : f(f16{});
}

// Launchers, one file per type of the weight (smol_patch_<type>.hip). tile:
// index of a tile shape. Return a hipError_t as int.
int launch_patch_f32(const PatchArgs &a, int image_type, int mode, int tile, void *stream);
int launch_patch_f16(const PatchArgs &a, int image_type, int mode, int tile, void *stream);
int launch_patch_bf16(const PatchArgs &a, int image_type, int mode, int tile, void *stream);
int launch_patch_grad_f32(const PatchArgs &a, const SumArgs &b, int image_type, int mode, int tile,
                          void *stream);
int launch_patch_grad_f16(const PatchArgs &a, const SumArgs &b, int image_type, int mode, int tile,
                          void *stream);
int launch_patch_grad_bf16(const PatchArgs &a, const SumArgs &b, int image_type, int mode, int tile,
                          void *stream);

}  // namespace smol

#endif  // SMOL_PATCH_H
