// smol_patch.hip -- patch embedding and its backward pass (smol_patch_embed,
// smol_patch_embed_backward): argument checks, the choice of tiles, and the
// backward pass's column sums and joins. The matrix products are in
// smol_patch_kernels.h.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "smol.h"
#include "smol_internal.h"
#include "smol_patch.h"

namespace smol {
namespace {

// Column sums alone, beside products of 256-wide tiles (whose workgroups leave
// no room for others).
template <typename T>
__global__ void __launch_bounds__(256) patch_sum_kernel(SumArgs a)
{
    sum_columns<T>(a, blockIdx.x);
}

// Joins: the first workgroups add the splits of the weight's gradient, the
// next the parts of the positions', the last the bias's (over parts and
// tokens; 8 columns a workgroup, 32 threads a column). 28 splits of 768 x 768:
// 15 us, 4.6 TB/s.
struct JoinArgs {
    PatchArgs patch;
    const float *part, *sums;
    void *weight, *pos, *bias;
    uint32_t tokens, parts;
    uint32_t weight_groups, pos_groups;
    Divisor chunks;
    int32_t accumulate;
};

template <typename P, int C>
__global__ void __launch_bounds__(256) patch_join_kernel(JoinArgs a)
{
    const uint32_t dim = a.patch.dim;
    if (blockIdx.x < a.weight_groups) {
        const uint32_t e = blockIdx.x * 256 + threadIdx.x;
        const uint32_t d = divide(e, a.chunks), q = e - d * a.chunks.d;
        if (d >= dim)
            return;
        const Chunk<C> c(a.patch, q);
        const int64_t width = (int64_t)a.patch.chunks * C;
        const float *p = a.part + d * width + q * C;
        vec<float, C> sum = (vec<float, C>)0.0f;
#pragma unroll 4
        for (uint32_t s = 0; s < a.patch.splits; ++s)
            sum += load<float, C>(p + s * dim * width);
        P *out = (P *)a.weight + (int64_t)d * a.patch.values + c.weight;
#pragma unroll
        for (int k = 0; k < C; ++k)
            if (k >= c.lead && k < c.have)
                out[k] = (P)(a.accumulate ? (float)out[k] + sum[k] : sum[k]);
        return;
    }
    if (blockIdx.x < a.weight_groups + a.pos_groups) {
        const uint32_t e = (blockIdx.x - a.weight_groups) * 256 + threadIdx.x;
        const uint32_t count = a.tokens * dim;
        if (e >= count)
            return;
        float sum = 0.0f;
#pragma unroll 8
        for (uint32_t s = 0; s < a.parts; ++s)
            sum += a.sums[(int64_t)s * count + e];
        P *out = (P *)a.pos + e;
        *out = (P)(a.accumulate ? (float)*out + sum : sum);
        return;
    }
    __shared__ float rows[32][9];
    const uint32_t d = (blockIdx.x - a.weight_groups - a.pos_groups) * 8 + (threadIdx.x & 7);
    const uint32_t q = threadIdx.x >> 3;
    float sum = 0.0f;
    if (d < dim)
#pragma unroll 8
        for (uint32_t r = q; r < a.parts * a.tokens; r += 32)
            sum += a.sums[(int64_t)r * dim + d];
    rows[q][threadIdx.x & 7] = sum;
    __syncthreads();
    if (q != 0 || d >= dim)
        return;
    for (int k = 1; k < 32; ++k)
        sum += rows[k][threadIdx.x];
    P *out = (P *)a.bias + d;
    *out = (P)(a.accumulate ? (float)*out + sum : sum);
}

// What a shape amounts to.
struct Plan {
    PatchArgs a;  // without pointers, strides and tiles
    uint32_t tokens;
    int mode;
};

int plan_of(const smol_patch_shape &s, Plan *plan)
{
    if (s.n < 0 || s.channels < 1 || s.height < 1 || s.width < 1 || s.patch < 1 || s.dim < 1)
        return set_error(SMOL_ERR_INVALID_ARG, "a size of the shape is out of range");
    if (s.layout != SMOL_LAYOUT_NCHW && s.layout != SMOL_LAYOUT_NHWC)
        return set_error(SMOL_ERR_INVALID_ARG, "layout %d unknown", s.layout);
    if (s.type < SMOL_ELEM_F32 || s.type > SMOL_ELEM_BF16)
        return set_error(SMOL_ERR_INVALID_ARG, "type %d unknown", s.type);
    if (s.image_type < SMOL_ELEM_F32 || s.image_type > SMOL_ELEM_BF16 ||
        (s.image_type == SMOL_ELEM_BF16 && s.type != SMOL_ELEM_BF16))
        return set_error(SMOL_ERR_INVALID_ARG, "image_type %d does not go with type %d",
                         s.image_type, s.type);
    for (int32_t r : s.reserved)
        if (r)
            return set_error(SMOL_ERR_INVALID_ARG, "reserved fields are not zero");
    const bool sides = s.height <= SMOL_MAX_DIM && s.width <= SMOL_MAX_DIM &&
                       s.patch <= SMOL_MAX_PATCH && s.channels <= SMOL_MAX_PATCH_VALUES &&
                       s.dim <= SMOL_MAX_PATCH_DIM;  // no product below overflows
    const int64_t values = sides ? (int64_t)s.channels * s.patch * s.patch : 0;
    const int64_t image = sides ? (int64_t)s.channels * s.height * s.width : 0;
    const int64_t th = s.height / s.patch, tw = s.width / s.patch;
    if (!sides || values > SMOL_MAX_PATCH_VALUES || values * s.dim >= INT32_MAX ||
        image >= INT32_MAX || th * tw * s.n > SMOL_MAX_ROWS || th * tw * s.dim >= INT32_MAX)
        return set_error(SMOL_ERR_UNSUPPORTED,
                         "%d images of %d x %d x %d, patches of %d, %d columns: beyond the limits",
                         s.n, s.channels, s.height, s.width, s.patch, s.dim);
    const bool nhwc = s.layout == SMOL_LAYOUT_NHWC;
    const int C = 16 / elem_size(s.type);
    PatchArgs &a = plan->a;
    a = PatchArgs{};
    plan->tokens = (uint32_t)(th * tw);
    a.image_size = image;
    a.rows = (uint32_t)(th * tw * s.n);
    a.dim = (uint32_t)s.dim;
    a.values = (uint32_t)values;
    a.length = (uint32_t)(nhwc ? s.patch * s.channels : s.patch);
    const uint32_t per_run = (a.length + C - 1) / C;
    a.chunks = per_run * (a.values / a.length);
    a.step_x = a.length;
    a.pitch = (uint32_t)(nhwc ? s.width * s.channels : s.width);
    a.step_y = (uint32_t)s.patch * a.pitch;
    a.plane = (uint32_t)s.height * (uint32_t)s.width;
    a.tokens = make_divisor(plan->tokens ? plan->tokens : 1);
    a.across = make_divisor(tw ? (uint32_t)tw : 1);
    a.per_run = make_divisor(per_run);
    // channels-last runs belong to no channel
    a.per_channel = make_divisor(nhwc ? SMOL_MAX_PATCH_VALUES : (uint32_t)s.patch);
    plan->mode = a.length < (uint32_t)C           ? kShort
                 : a.length % C || a.chunks % 8 ? kMasked
                                                : kWhole;
    return SMOL_OK;
}

void set_tiles(PatchArgs *a, uint32_t rows, uint32_t cols)
{
    a->tiles = rows * cols;
    a->tiles_n = make_divisor(cols);
}

uint32_t ceil_div(uint32_t n, uint32_t d) { return (n + d - 1) / d; }

// The tile side of a forward call: the least of the times that the sides take
// for patches of 768 values. Measured, us, for 224 x 224 images to 768 columns, sides 32 / 64 / 128 / 256:
//   fp16, images   1: 4.7 / 8.0 / 12.3 / 23.9     8: 12.5 / 10.1 / 13.0 / 25.6
//                 16: 22.2 / 13.0 / 13.8 / 26.6  32: 38.0 / 19.2 / 18.9 / 27.1
//                 64: 68.2 / 32.5 / 29.9 / 28.4  96: 101 / 45.3 / 35.7 / 30.5
//                128: 133 / 60.1 / 46.4 / 53.4
//   fp32, images   1: 10.4 / 21.5 / 57.4   4: 19.8 / 23.3 / 57.8
//                 16: 53.4 / 48.8 / 60.1  64: 175 / 138 / 155 (128: not used)
// (32, 64: several tiles a compute unit at once; 128: two, one for the first
// 256; 256: one). For patches of 14 to 1024 columns the side taken (*) was the
// fastest, for fewer values, where a tile's begin and end weigh more, sometimes
// the second:
//   p 14, 1024 columns,  1 image 4.7* / 10.3 / 15.4 / 27.2
//                       16: 28.4 / 20.2 / 17.2* / 28.7  64: 94.9 / 62.2 / 40.1 / 32.4*
//   p  9, 512 columns,   1: 10.6* / 7.8 / 12.8 / 24.6   64: 293 / 80.9 / 52.6* / 46.6
//   p  8, 384 columns,   1: 6.1* / 4.4 / 6.8 / 13.4     16: 37.4 / 9.9 / 10.0* / 14.9
//   p  4, 768 columns,   1: 56.7 / 10.3 / 11.2*          4: 194 / 28.8* / 24.5
//   fp32, p 8, 384 columns, 4: 15.1* / 11.4             16: 44.6 / 23.8*
// Rows of a tile from 64 on must lie within 2^32 bytes.
int forward_tile(const smol_patch_shape &s, const Plan &plan)
{
    const PatchArgs &a = plan.a;
    const auto tiles = [&](uint32_t side) {
        return (double)ceil_div(a.rows, side) * ceil_div(a.dim, side);
    };
    const auto rounds = [](double n, double at_once) {
        const double r = n / at_once;
        return (double)(int64_t)r < r ? (double)(int64_t)r + 1 : r;
    };
    const double cus = device_cus() > 0 ? device_cus() : 256;
    const int64_t span = (int64_t)(256 / plan.tokens + 2) * a.image_size * elem_size(s.image_type);
    if (span > UINT32_MAX)
        return 32;
    const auto more = [](double x, double y) { return x > y ? x : y; };
    if (s.type == SMOL_ELEM_F32)
        return 5 + tiles(32) / 53 <= more(22, 18 + tiles(64) / 19.6) ? 32 : 64;
    const bool large = plan.mode != kShort && elem_size(s.image_type) == 2;
    const double us[4] = {4 + tiles(32) / 140, more(8.2, 6.5 + tiles(64) / 88),
                          tiles(128) <= cus ? 13 : 3 + 16 * rounds(tiles(128), 2 * cus),
                          large ? 1 + 25 * rounds(tiles(256), cus) : 1e30};
    int best = 0;
    for (int k = 1; k < 4; ++k)
        if (us[k] < us[best])
            best = k;
    return 32 << best;
}

// The backward pass's parts. A part of the rows costs its partial products a
// write and a read, so there are only as many as fill the chip.
struct GradPlan {
    int tile;
    uint32_t parts, part_images;
    int64_t sums, bytes;  // offset of the column sums; workspace bytes
};

GradPlan grad_plan(const smol_patch_shape &s, Plan *plan)
{
    PatchArgs &a = plan->a;
    const int C = 16 / elem_size(s.type), rows_a_step = C * 8;
    const uint32_t width = a.chunks * C;
    GradPlan g;
    const uint32_t steps = ceil_div(a.rows, rows_a_step);
    if (s.dim < C)
        plan->mode = kShort;
    const bool large = plan->mode != kShort && elem_size(s.image_type) == 2 && C == 8;
    // Large tiles where each compute unit has 20 of their steps or more: us of
    // fp16 images of 224 x 224 in patches of 16 to 768 bf16 columns, sides 128 /
    // 256: 1 image 15 / 26, 16: 25 / 35, 64: 41 / 48, 128: 60 / 66, 192: 81 / 82,
    // 256: 102 / 99; to 256 columns, 512 images: 90 / 96; patches of 14 to 1024
    // columns, 64: 53 / 57, 96: 69 / 72, 128: 89 / 86, 192: 125 / 114; of 8 to 384
    // columns, 128: 62 / 73. (256 units: the workspace's size, which a host
    // without the device may ask for, depends on this choice.)
    const uint64_t large_steps =
        (uint64_t)ceil_div(a.dim, 256) * ceil_div(width, 256) * ceil_div(a.rows, 64);
    g.tile = large && large_steps >= 20 * 256 ? 256 : 128;
    const uint32_t at_once = g.tile == 256 || C == 4 ? 256 : 512;
    set_tiles(&a, ceil_div(a.dim, g.tile), ceil_div(width, g.tile));
    uint32_t splits = a.tiles < at_once ? at_once / a.tiles : 1;
    if (splits > ceil_div(steps, 4))
        splits = ceil_div(steps, 4);
    a.split_rows = splits ? ceil_div(steps, splits) * rows_a_step : rows_a_step;
    a.splits = ceil_div(a.rows, a.split_rows);
    const uint32_t V = a.dim >= 8 ? 8 : 1, threads = plan->tokens * ceil_div(a.dim, V);
    uint32_t parts = threads ? ceil_div(2048 * 64, threads) : 0;
    // a part's sums are written and read again: eight images at least
    if (parts > ceil_div((uint32_t)s.n, 8))
        parts = ceil_div((uint32_t)s.n, 8);
    g.part_images = parts ? ceil_div((uint32_t)s.n, parts) : 1;
    g.parts = parts ? ceil_div((uint32_t)s.n, g.part_images) : 0;
    g.sums = ((int64_t)a.splits * a.dim * width * 4 + 15) / 16 * 16;
    g.bytes = g.sums + (int64_t)g.parts * plan->tokens * a.dim * 4 + 16;
    return g;
}

int check_tensor(const char *name, const void *p, int type)
{
    if (!p || (uintptr_t)p % elem_size(type))
        return set_error(SMOL_ERR_INVALID_ARG, "%s is NULL or not aligned to its elements", name);
    return SMOL_OK;
}

// Strides of n images' rows; written rows may not overlap.
int check_strides(const char *name, int64_t image_stride, int64_t row_stride, int64_t n,
                  int64_t tokens, int64_t dim, bool written)
{
    const int64_t most = INT64_MAX / 16 / (n * tokens);
    bool ok = image_stride >= 0 && row_stride >= 0 && image_stride <= most && row_stride <= most;
    if (ok && written) {
        const int64_t span_rows = (tokens - 1) * row_stride + dim;
        const int64_t span_images = (n - 1) * image_stride + dim;
        const bool rows_apart = tokens == 1 || row_stride >= dim;
        const bool images_apart = n == 1 || image_stride >= dim;
        ok = rows_apart && images_apart &&
             (n == 1 || tokens == 1 || image_stride >= span_rows || row_stride >= span_images);
    }
    if (!ok)
        return set_error(SMOL_ERR_INVALID_ARG, "%s: strides %lld, %lld out of range", name,
                         (long long)image_stride, (long long)row_stride);
    return SMOL_OK;
}

}  // namespace
}  // namespace smol

extern "C" int smol_patch_embed(const smol_patch_args *p, void *stream)
{
    using namespace smol;
    clear_error();
    if (!p)
        return set_error(SMOL_ERR_INVALID_ARG, "args is NULL");
    const smol_patch_shape &s = p->shape;
    Plan plan;
    int st = plan_of(s, &plan);
    if (st != SMOL_OK)
        return st;
    PatchArgs &a = plan.a;
    if (a.rows == 0)
        return SMOL_OK;
    if ((st = check_tensor("images", p->images, s.image_type)) != SMOL_OK ||
        (st = check_tensor("weight", p->weight, s.type)) != SMOL_OK ||
        (p->bias && (st = check_tensor("bias", p->bias, s.type)) != SMOL_OK) ||
        (p->pos && (st = check_tensor("pos", p->pos, s.type)) != SMOL_OK) ||
        (st = check_tensor("out", p->out, s.type)) != SMOL_OK ||
        (st = check_strides("out", p->image_stride, p->row_stride, s.n, plan.tokens, s.dim,
                            true)) != SMOL_OK)
        return st;
    a.images = p->images;
    a.weight = p->weight;
    a.bias = p->bias;
    a.pos = p->pos;
    a.out = p->out;
    a.image_stride = p->image_stride;
    a.row_stride = p->row_stride;
    const int tile = forward_tile(s, plan);
    if ((int64_t)ceil_div(a.rows, tile) * ceil_div(a.dim, tile) >= 1 << 24)
        return set_error(SMOL_ERR_UNSUPPORTED, "%u rows of %u columns: too many for a launch",
                         a.rows, a.dim);
    set_tiles(&a, ceil_div(a.rows, tile), ceil_div(a.dim, tile));
    const int e = (s.type == SMOL_ELEM_F32   ? launch_patch_f32
                   : s.type == SMOL_ELEM_F16 ? launch_patch_f16
                                             : launch_patch_bf16)(a, s.image_type, plan.mode, tile,
                                                                  stream);
    if (e != hipSuccess)
        return set_error(SMOL_ERR_HIP, "patch embedding launch: %s",
                         hipGetErrorString((hipError_t)e));
    return SMOL_OK;
}

extern "C" int64_t smol_patch_workspace_bytes(const smol_patch_shape *shape)
{
    using namespace smol;
    Plan plan;
    if (!shape || plan_of(*shape, &plan) != SMOL_OK)
        return 0;
    return grad_plan(*shape, &plan).bytes;
}

extern "C" int smol_patch_embed_backward(const smol_patch_grad_args *p, void *stream)
{
    using namespace smol;
    clear_error();
    if (!p)
        return set_error(SMOL_ERR_INVALID_ARG, "args is NULL");
    const smol_patch_shape &s = p->shape;
    Plan plan;
    int st = plan_of(s, &plan);
    if (st != SMOL_OK)
        return st;
    if (p->grad_type != SMOL_ELEM_F32 && p->grad_type != s.type)
        return set_error(SMOL_ERR_INVALID_ARG, "grad_type %d is neither fp32 nor the type",
                         p->grad_type);
    if (p->accumulate != 0 && p->accumulate != 1)
        return set_error(SMOL_ERR_INVALID_ARG, "accumulate %d is neither 0 nor 1", p->accumulate);
    PatchArgs &a = plan.a;
    if (a.rows > 0 &&
        ((st = check_tensor("grad_out", p->grad_out, s.type)) != SMOL_OK ||
         (st = check_strides("grad_out", p->image_stride, p->row_stride, s.n, plan.tokens, s.dim,
                             false)) != SMOL_OK ||
         (p->grad_weight && (st = check_tensor("images", p->images, s.image_type)) != SMOL_OK)))
        return st;
    if ((p->grad_weight &&
         (st = check_tensor("grad_weight", p->grad_weight, p->grad_type)) != SMOL_OK) ||
        (p->grad_bias && (st = check_tensor("grad_bias", p->grad_bias, p->grad_type)) != SMOL_OK) ||
        (p->grad_pos && (st = check_tensor("grad_pos", p->grad_pos, p->grad_type)) != SMOL_OK))
        return st;
    const GradPlan g = grad_plan(s, &plan);
    if (!p->workspace || (uintptr_t)p->workspace % 16 || p->workspace_bytes < g.bytes)
        return set_error(SMOL_ERR_INVALID_ARG,
                         "workspace must be 16-byte aligned and hold %lld bytes",
                         (long long)g.bytes);
    if (!p->grad_weight && !p->grad_bias && !p->grad_pos)
        return SMOL_OK;
    // The join's workgroups; of 256 threads a launch takes less than 2^24. (Of
    // the products' tiles and the sums' parts the limits allow fewer.)
    const uint32_t weight_groups =
        p->grad_weight ? (uint32_t)(((int64_t)a.dim * a.chunks + 255) / 256) : 0;
    const uint32_t pos_groups = p->grad_pos ? ceil_div(plan.tokens * a.dim, 256) : 0;
    const uint32_t join_groups =
        weight_groups + pos_groups + (p->grad_bias ? ceil_div(a.dim, 8) : 0);
    if (join_groups >= 1 << 24)
        return set_error(SMOL_ERR_UNSUPPORTED,
                         "gradients of %lld and %lld values: too many for a launch",
                         (long long)a.dim * a.values, (long long)plan.tokens * a.dim);
    hipStream_t hs = (hipStream_t)stream;
    float *part = (float *)p->workspace, *sums = (float *)((char *)p->workspace + g.sums);
    a.images = p->images;
    a.grad_out = p->grad_out;
    a.out = part;
    a.image_stride = p->image_stride;
    a.row_stride = p->row_stride;
    SumArgs b = {};
    if ((p->grad_bias || p->grad_pos) && g.parts > 0) {
        b.grad_out = p->grad_out;
        b.sums = sums;
        b.image_stride = p->image_stride;
        b.row_stride = p->row_stride;
        b.n = (uint32_t)s.n;
        b.tokens = plan.tokens;
        b.dim = a.dim;
        b.part_images = g.part_images;
        b.columns = make_divisor(ceil_div(a.dim, a.dim >= 8 ? 8 : 1));
        b.per_part = make_divisor(ceil_div(plan.tokens * b.columns.d, 256));
        b.groups = b.per_part.d * g.parts;
    }
    const bool beside = p->grad_weight && g.tile == 128;
    int e = hipSuccess;
    if (p->grad_weight && a.rows > 0)
        e = (s.type == SMOL_ELEM_F32   ? launch_patch_grad_f32
             : s.type == SMOL_ELEM_F16 ? launch_patch_grad_f16
                                       : launch_patch_grad_bf16)(a, beside ? b : SumArgs{},
                                                                 s.image_type, plan.mode, g.tile,
                                                                 stream);
    if (e == hipSuccess && b.groups > 0 && !beside) {
        with_type(s.type, [&](auto t) {
            hipLaunchKernelGGL((patch_sum_kernel<decltype(t)>), dim3(b.groups), dim3(256), 0, hs,
                               b);
        });
        e = hipGetLastError();
    }
    if (e == hipSuccess) {
        JoinArgs j;
        j.patch = a;
        j.part = part;
        j.sums = sums;
        j.weight = p->grad_weight;
        j.pos = p->grad_pos;
        j.bias = p->grad_bias;
        j.tokens = plan.tokens;
        j.parts = g.parts;
        j.chunks = make_divisor(a.chunks);
        j.accumulate = p->accumulate;
        j.weight_groups = weight_groups;
        j.pos_groups = pos_groups;
        const dim3 grid(join_groups);
        if (grid.x > 0)
            with_type(p->grad_type, [&](auto t) {
                typedef decltype(t) P;
                if (elem_size(s.type) == 4)
                    hipLaunchKernelGGL((patch_join_kernel<P, 4>), grid, dim3(256), 0, hs, j);
                else
                    hipLaunchKernelGGL((patch_join_kernel<P, 8>), grid, dim3(256), 0, hs, j);
            });
        e = hipGetLastError();
    }
    if (e != hipSuccess)
        return set_error(SMOL_ERR_HIP, "patch embedding backward launch: %s",
                         hipGetErrorString((hipError_t)e));
    return SMOL_OK;
}
