// smol_heads.hip -- rotation by positions and norms of heads: checks, the form
// of the kernels, launches (smol_rotate, smol_rotate_backward, smol_head_norm,
// smol_head_norm_backward, smol_rotary_frequencies).
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "smol.h"
#include "smol_attention.h"
#include "smol_heads.h"
#include "smol_internal.h"

namespace smol {
namespace {

// Joins the workgroups' sums in order: 16 columns a workgroup, 64 threads a
// column each taking every 64th workgroup's, eight loads at once (all there are:
// 512 workgroups), then four threads a column, then one.
template <typename P>
__global__ void __launch_bounds__(1024) head_join_kernel(const float *sums, P *q, P *k,
                                                         int32_t dim, int32_t groups,
                                                         int32_t accumulate)
{
    constexpr int kAhead = 8;
    const int32_t c = blockIdx.x * 16 + (threadIdx.x & 15), first = threadIdx.x >> 4;
    __shared__ float part[64][17];
    float s = 0.0f;
    if (c < 2 * dim)
        for (int32_t g = first; g < groups; g += 64 * kAhead) {
            float x[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const int32_t at = g + 64 * u;
                x[u] = sums[(int64_t)(at < groups ? at : first) * 2 * dim + c];
            }
            asm volatile("" ::: "memory");
#pragma unroll
            for (int u = 0; u < kAhead; ++u)
                s += g + 64 * u < groups ? x[u] : 0.0f;
        }
    part[first][threadIdx.x & 15] = s;
    __syncthreads();
    if (first >= 4)
        return;
    // (one wave from here on)
    s = 0.0f;
#pragma unroll
    for (int t = 0; t < 16; ++t)
        s += part[first * 16 + t][threadIdx.x & 15];
    const float s1 = __shfl_down(s, 16), s2 = __shfl_down(s, 32), s3 = __shfl_down(s, 48);
    if (first != 0 || c >= 2 * dim)
        return;
    s = s + s1 + s2 + s3;
    P *out = c < dim ? q : k;
    if (!out)
        return;
    out += c < dim ? c : c - dim;
    *out = (P)(accumulate ? (float)*out + s : s);
}

constexpr int kWaves = 4;             // of a workgroup (kHeadWaves)
constexpr int64_t kFewItems = 8192;   // waves that the chip holds at once
// of the backward pass, whose waves' angles, weights and sums serve more heads so
// (2048 rows of 32 and 8 heads of 128 bf16 values: 27 us with 8192 waves, 19)
constexpr int64_t kFewGradItems = 2048;
constexpr int kGradGroups = 512;      // workgroups of the backward pass at most

int floor_log2(int v)
{
    int l = 0;
    while (v >> (l + 1))
        ++l;
    return l;
}

// Chunks, lanes, rows and parts for heads of this width.
void plan(HeadArgs *a, HeadForm *f, int type, int64_t few = kFewItems)
{
    const int dim = a->dim, half = a->half, rot = 2 * half;
    // the widest chunk of 16 bytes or less of which every run is whole: the
    // halves and what follows them, or the head
    int v = type == SMOL_ELEM_F32 ? 4 : 8;
    const auto whole = [&](int n) {
        return f->interleaved && half ? rot % n == 0 && dim % n == 0
                                      : half % n == 0 && (dim - rot) % n == 0;
    };
    while (v > 1 && !whole(v))
        v >>= 1;
    f->v = v;
    const int chunks = dim / v, turning = f->interleaved ? 0 : half / v;
    a->units = turning + (chunks - 2 * turning + 1) / 2;
    f->k = a->units > 64 ? 2 : 1;
    int log2 = 0;
    while ((f->k << log2) < a->units)
        ++log2;
    a->lanes_log2 = log2;
    const int slots = 64 >> log2;
    const int heads = a->side[0].heads > a->side[1].heads ? a->side[0].heads : a->side[1].heads;
    // rows that fill the slots, as far as there are rows to spread over the chip
    int rows = heads < slots ? slots / heads : 1;
    while (rows > 1 && (int64_t)a->rows / rows < kFewItems)
        rows >>= 1;
    a->rows_log2 = floor_log2(rows);
    int steps = 0;
    for (HeadSide &s : a->side) {
        s.steps = (int)((((int64_t)s.heads << a->rows_log2) + slots - 1) / slots);
        steps += s.steps;
    }
    const int64_t blocks = ((int64_t)a->rows + (1 << a->rows_log2) - 1) >> a->rows_log2;
    // a wave takes all of a block's steps, so that angles and weights are formed
    // once, unless there would be too few waves
    int64_t per = blocks * steps / few;
    per = per < 1 ? 1 : per < steps ? per : steps;
    a->per = (int)per;
    a->parts = (int)((steps + per - 1) / per);
    a->items = blocks * a->parts;
}

int launch(const HeadArgs &a, const HeadForm &f, int type, bool backward, int64_t grid, void *s)
{
    const auto f_of = type == SMOL_ELEM_F32   ? launch_heads_f32
                      : type == SMOL_ELEM_F16 ? launch_heads_f16
                                              : launch_heads_bf16;
    return f_of(a, f, backward, (unsigned)grid, s);
}

// Strides of rows and heads; least: the smallest stride between two heads of a
// matrix that is written (its dim), 0 for one that is read.
int check_heads(const char *name, const void *p, int64_t rows, int32_t heads, int32_t dim,
                int64_t row_stride, int64_t head_stride, bool written, int type)
{
    if (!p)
        return set_error(SMOL_ERR_INVALID_ARG, "%s is NULL", name);
    if ((uintptr_t)p % elem_size(type))
        return set_error(SMOL_ERR_INVALID_ARG, "%s is not aligned to its elements", name);
    const int64_t least = written ? dim : 0, most = INT64_MAX / 16;
    if (heads > 1 && (head_stride < least || head_stride > most / heads))
        return set_error(SMOL_ERR_INVALID_ARG, "%s: head stride %lld out of range", name,
                         (long long)head_stride);
    if (rows > 1 && (row_stride < least || row_stride > most / rows))
        return set_error(SMOL_ERR_INVALID_ARG, "%s: row stride %lld out of range", name,
                         (long long)row_stride);
    if (written && rows > 1 && heads > 1) {
        // heads within rows, or rows within heads
        const int64_t row = (heads - 1) * head_stride + dim, head = (rows - 1) * row_stride + dim;
        if (row_stride < row && head_stride < head)
            return set_error(SMOL_ERR_INVALID_ARG, "%s: rows overlap", name);
    }
    return SMOL_OK;
}

// An output that stands where an input does has its strides.
int check_in_place(const void *out, int64_t out_row, int64_t out_head, const void *in,
                   int64_t in_row, int64_t in_head, int64_t rows, int32_t heads)
{
    if (out == in && ((rows > 1 && out_row != in_row) || (heads > 1 && out_head != in_head)))
        return set_error(SMOL_ERR_INVALID_ARG, "strides of a call in place differ");
    return SMOL_OK;
}

int check_sizes(int64_t rows, int32_t dim, int32_t rot, int32_t type, int32_t positions_type,
                int32_t interleaved)
{
    if (rows < 0 || dim < 1)
        return set_error(SMOL_ERR_INVALID_ARG, "rows %lld or dim %d out of range",
                         (long long)rows, dim);
    if (type < SMOL_ELEM_F32 || type > SMOL_ELEM_BF16)
        return set_error(SMOL_ERR_INVALID_ARG, "type %d unknown", type);
    if (positions_type != SMOL_IDS_I32 && positions_type != SMOL_IDS_I64)
        return set_error(SMOL_ERR_INVALID_ARG, "positions_type %d unknown", positions_type);
    if (interleaved != 0 && interleaved != 1)
        return set_error(SMOL_ERR_INVALID_ARG, "interleaved %d is neither 0 nor 1", interleaved);
    if (rot < 0 || rot > dim || rot % 2)
        return set_error(SMOL_ERR_INVALID_ARG, "rot %d is odd or not within 0 .. dim %d", rot,
                         dim);
    if (rows > SMOL_MAX_ROWS || dim > SMOL_MAX_HEAD_DIM)
        return set_error(SMOL_ERR_UNSUPPORTED, "rows %lld beyond %d or dim %d beyond %d",
                         (long long)rows, SMOL_MAX_ROWS, dim, SMOL_MAX_HEAD_DIM);
    return SMOL_OK;
}

int check_head_count(const char *name, int32_t heads)
{
    if (heads < 0)
        return set_error(SMOL_ERR_INVALID_ARG, "%s: %d heads", name, heads);
    if (heads > SMOL_MAX_HEADS)
        return set_error(SMOL_ERR_UNSUPPORTED, "%s: %d heads beyond %d", name, heads,
                         SMOL_MAX_HEADS);
    return SMOL_OK;
}

int check_angles(const void *positions, int32_t positions_type, const double *freqs, float gain)
{
    if (!positions || (uintptr_t)positions % (positions_type == SMOL_IDS_I64 ? 8 : 4))
        return set_error(SMOL_ERR_INVALID_ARG, "positions is NULL or not aligned");
    if (!freqs || (uintptr_t)freqs % 8)
        return set_error(SMOL_ERR_INVALID_ARG, "freqs is NULL or not aligned");
    if (!isfinite(gain))
        return set_error(SMOL_ERR_INVALID_ARG, "gain is not finite");
    return SMOL_OK;
}

int check_small_vector(const char *name, const void *p, int type)
{
    if ((uintptr_t)p % elem_size(type))
        return set_error(SMOL_ERR_INVALID_ARG, "%s is not aligned to its elements", name);
    return SMOL_OK;
}

int rotate(const smol_rotate_args *p, bool backward, void *stream)
{
    clear_error();
    if (!p)
        return set_error(SMOL_ERR_INVALID_ARG, "args is NULL");
    int st = check_sizes(p->rows, p->dim, p->rot, p->type, p->positions_type, p->interleaved);
    if (st != SMOL_OK || (st = check_head_count("x", p->heads)) != SMOL_OK)
        return st;
    if (p->rot < 2 || p->heads < 1)
        return set_error(SMOL_ERR_INVALID_ARG, "rot %d or heads %d out of range", p->rot,
                         p->heads);
    if (p->reserved)
        return set_error(SMOL_ERR_INVALID_ARG, "reserved field is not zero");
    if (!isfinite(p->gain))
        return set_error(SMOL_ERR_INVALID_ARG, "gain is not finite");
    if (p->rows == 0)
        return SMOL_OK;
    if ((st = check_angles(p->positions, p->positions_type, p->freqs, p->gain)) != SMOL_OK ||
        (st = check_heads("x", p->x, p->rows, p->heads, p->dim, p->x_row_stride,
                          p->x_head_stride, false, p->type)) != SMOL_OK ||
        (st = check_heads("out", p->out, p->rows, p->heads, p->dim, p->out_row_stride,
                          p->out_head_stride, true, p->type)) != SMOL_OK ||
        (st = check_in_place(p->out, p->out_row_stride, p->out_head_stride, p->x,
                             p->x_row_stride, p->x_head_stride, p->rows, p->heads)) != SMOL_OK)
        return st;
    HeadArgs a = {};
    HeadForm f = {};
    a.side[0].x = p->x;
    a.side[0].out = p->out;
    a.side[0].x_row = p->x_row_stride;
    a.side[0].x_head = p->x_head_stride;
    a.side[0].out_row = p->out_row_stride;
    a.side[0].out_head = p->out_head_stride;
    a.side[0].heads = p->heads;
    a.positions = p->positions;
    a.freqs = p->freqs;
    a.rows = (int32_t)p->rows;
    a.dim = p->dim;
    a.half = p->rot / 2;
    a.wide = p->positions_type == SMOL_IDS_I64;
    a.gain = p->gain;
    a.sign = backward ? -1.0f : 1.0f;
    f.interleaved = p->interleaved;
    plan(&a, &f, p->type);
    const int64_t groups = (a.items + kWaves - 1) / kWaves;
    const int e = launch(a, f, p->type, false, groups < 1 << 20 ? groups : 1 << 20, stream);
    if (e != hipSuccess)
        return set_error(SMOL_ERR_HIP, "rotation launch: %s", hipGetErrorString((hipError_t)e));
    return SMOL_OK;
}

int check_shape(const smol_head_shape &s, int32_t q_heads, int32_t k_heads)
{
    int st = check_sizes(s.rows, s.dim, s.rot, s.type, s.positions_type, s.interleaved);
    if (st != SMOL_OK || (st = check_head_count("q", q_heads)) != SMOL_OK ||
        (st = check_head_count("k", k_heads)) != SMOL_OK)
        return st;
    if (s.weight_type != SMOL_ELEM_F32 && s.weight_type != s.type)
        return set_error(SMOL_ERR_INVALID_ARG, "weight_type %d is neither fp32 nor the type",
                         s.weight_type);
    if (!(s.eps >= 0.0f) || isinf(s.eps))
        return set_error(SMOL_ERR_INVALID_ARG, "eps is negative or not finite");
    if (s.reserved[0] || s.reserved[1])
        return set_error(SMOL_ERR_INVALID_ARG, "reserved fields are not zero");
    if (s.rot && !isfinite(s.gain))
        return set_error(SMOL_ERR_INVALID_ARG, "gain is not finite");
    if (s.rot && s.rows > 0 && q_heads + k_heads > 0)
        return check_angles(s.positions, s.positions_type, s.freqs, s.gain);
    return SMOL_OK;
}

void fill_shape(HeadArgs *a, HeadForm *f, const smol_head_shape &s)
{
    a->positions = s.positions;
    a->freqs = s.freqs;
    a->rows = (int32_t)s.rows;
    a->dim = s.dim;
    a->half = s.rot / 2;
    a->wide = s.positions_type == SMOL_IDS_I64;
    a->weight_f32 = s.weight_type == SMOL_ELEM_F32;
    a->eps = s.eps;
    a->gain = s.gain;
    f->norm = true;
    f->interleaved = s.interleaved && s.rot;
}

int64_t grad_groups(int64_t rows, int32_t q_heads, int32_t k_heads)
{
    if (q_heads + k_heads == 0)
        return 0;
    // a wave takes a row's heads or fewer of them; no more workgroups than heads
    const int64_t heads = rows * (q_heads + k_heads);
    return heads < kGradGroups ? heads : kGradGroups;
}

}  // namespace
}  // namespace smol

extern "C" int smol_rotary_frequencies(const smol_rotary_plan *p, double *freqs, float *gain)
{
    using namespace smol;
    clear_error();
    if (!p || !freqs || !gain)
        return set_error(SMOL_ERR_INVALID_ARG, "plan, freqs or gain is NULL");
    if (p->dim < 2 || p->dim % 2)
        return set_error(SMOL_ERR_INVALID_ARG, "dim %d is odd or below 2", p->dim);
    if (p->dim > SMOL_MAX_HEAD_DIM)
        return set_error(SMOL_ERR_UNSUPPORTED, "dim %d beyond %d", p->dim, SMOL_MAX_HEAD_DIM);
    if (!(p->base > 0.0) || !isfinite(p->base))
        return set_error(SMOL_ERR_INVALID_ARG, "base is not positive and finite");
    if (p->scaling < SMOL_ROTARY_NONE || p->scaling > SMOL_ROTARY_PARTS)
        return set_error(SMOL_ERR_INVALID_ARG, "scaling %d unknown", p->scaling);
    if (p->scaling != SMOL_ROTARY_NONE && (!(p->factor >= 1.0) || !isfinite(p->factor)))
        return set_error(SMOL_ERR_INVALID_ARG, "factor is below 1 or not finite");
    const bool parts = p->scaling == SMOL_ROTARY_PARTS;
    if (parts && (!(p->length > 0.0) || !isfinite(p->length) || !(p->low < p->high) ||
                  !isfinite(p->low) || !isfinite(p->high)))
        return set_error(SMOL_ERR_INVALID_ARG, "length is not positive, or low not below high");
    double base = p->base;
    if (p->scaling == SMOL_ROTARY_BASE && p->dim > 2)
        base *= pow(p->factor, (double)p->dim / (p->dim - 2));
    for (int i = 0; i < p->dim / 2; ++i) {
        double f = pow(base, -2.0 * i / p->dim);
        if (p->scaling == SMOL_ROTARY_LINEAR)
            f /= p->factor;
        if (parts) {
            const double turns = f * p->length / 6.283185307179586477;
            const double at = (turns - p->low) / (p->high - p->low);
            const double keep = at < 0.0 ? 0.0 : at > 1.0 ? 1.0 : at;
            f = f * keep + f / p->factor * (1.0 - keep);
        }
        freqs[i] = f;
    }
    *gain = parts ? (float)(0.1 * log(p->factor) + 1.0) : 1.0f;
    return SMOL_OK;
}

extern "C" int smol_rotate(const smol_rotate_args *p, void *stream)
{
    return smol::rotate(p, false, stream);
}

extern "C" int smol_rotate_backward(const smol_rotate_args *p, void *stream)
{
    return smol::rotate(p, true, stream);
}

extern "C" int smol_head_norm(const smol_head_norm_args *p, void *stream)
{
    using namespace smol;
    clear_error();
    if (!p)
        return set_error(SMOL_ERR_INVALID_ARG, "args is NULL");
    const smol_head_shape &s = p->shape;
    int st = check_shape(s, p->q.heads, p->k.heads);
    if (st != SMOL_OK)
        return st;
    HeadArgs a = {};
    HeadForm f = {};
    for (int k = 0; k < 2; ++k) {
        const smol_head_side &in = k ? p->k : p->q;
        const char *names[2][3] = {{"q", "q's out", "q's weight"}, {"k", "k's out", "k's weight"}};
        if (in.reserved)
            return set_error(SMOL_ERR_INVALID_ARG, "reserved field is not zero");
        if (in.heads == 0 || s.rows == 0)
            continue;
        if ((st = check_heads(names[k][0], in.x, s.rows, in.heads, s.dim, in.x_row_stride,
                              in.x_head_stride, false, s.type)) != SMOL_OK ||
            (st = check_heads(names[k][1], in.out, s.rows, in.heads, s.dim, in.out_row_stride,
                              in.out_head_stride, true, s.type)) != SMOL_OK ||
            (st = check_in_place(in.out, in.out_row_stride, in.out_head_stride, in.x,
                                 in.x_row_stride, in.x_head_stride, s.rows, in.heads)) !=
                SMOL_OK ||
            (st = check_small_vector(names[k][2], in.weight, s.weight_type)) != SMOL_OK)
            return st;
        HeadSide &to = a.side[k];
        to.x = in.x;
        to.out = in.out;
        to.weight = in.weight;
        to.x_row = in.x_row_stride;
        to.x_head = in.x_head_stride;
        to.out_row = in.out_row_stride;
        to.out_head = in.out_head_stride;
        to.heads = in.heads;
    }
    if (s.rows == 0 || p->q.heads + p->k.heads == 0)
        return SMOL_OK;
    if (p->q.heads && p->k.heads &&
        (p->q.out == p->k.out || p->q.out == p->k.x || p->k.out == p->q.x))
        return set_error(SMOL_ERR_INVALID_ARG, "an output of q stands where one of k does");
    fill_shape(&a, &f, s);
    a.sign = 1.0f;
    plan(&a, &f, s.type);
    const int64_t groups = (a.items + kWaves - 1) / kWaves;
    const int e = launch(a, f, s.type, false, groups < 1 << 20 ? groups : 1 << 20, stream);
    if (e != hipSuccess)
        return set_error(SMOL_ERR_HIP, "head norm launch: %s", hipGetErrorString((hipError_t)e));
    return SMOL_OK;
}

extern "C" int64_t smol_head_norm_workspace_bytes(int64_t rows, int32_t q_heads, int32_t k_heads,
                                                  int32_t dim)
{
    using namespace smol;
    if (rows < 0 || rows > SMOL_MAX_ROWS || dim < 1 || dim > SMOL_MAX_HEAD_DIM || q_heads < 0 ||
        q_heads > SMOL_MAX_HEADS || k_heads < 0 || k_heads > SMOL_MAX_HEADS)
        return 0;
    return grad_groups(rows, q_heads, k_heads) * 2 * dim * 4 + 16;
}

extern "C" int smol_head_norm_backward(const smol_head_norm_grad_args *p, void *stream)
{
    using namespace smol;
    clear_error();
    if (!p)
        return set_error(SMOL_ERR_INVALID_ARG, "args is NULL");
    const smol_head_shape &s = p->shape;
    int st = check_shape(s, p->q.heads, p->k.heads);
    if (st != SMOL_OK)
        return st;
    if (p->accumulate != 0 && p->accumulate != 1)
        return set_error(SMOL_ERR_INVALID_ARG, "accumulate %d is neither 0 nor 1", p->accumulate);
    if (p->reserved)
        return set_error(SMOL_ERR_INVALID_ARG, "reserved field is not zero");
    HeadArgs a = {};
    HeadForm f = {};
    for (int k = 0; k < 2; ++k) {
        const smol_head_grad_side &in = k ? p->k : p->q;
        const char *names[2][5] = {
            {"q's grad_out", "q", "q's grad_x", "q's weight", "q's grad_weight"},
            {"k's grad_out", "k", "k's grad_x", "k's weight", "k's grad_weight"}};
        if (in.reserved)
            return set_error(SMOL_ERR_INVALID_ARG, "reserved field is not zero");
        if ((st = check_small_vector(names[k][4], in.grad_weight, s.weight_type)) != SMOL_OK)
            return st;
        if (in.heads == 0 || s.rows == 0)
            continue;
        if ((st = check_heads(names[k][0], in.grad_out, s.rows, in.heads, s.dim,
                              in.grad_out_row_stride, in.grad_out_head_stride, false, s.type)) !=
                SMOL_OK ||
            (st = check_heads(names[k][1], in.x, s.rows, in.heads, s.dim, in.x_row_stride,
                              in.x_head_stride, false, s.type)) != SMOL_OK ||
            (st = check_heads(names[k][2], in.grad_x, s.rows, in.heads, s.dim,
                              in.grad_x_row_stride, in.grad_x_head_stride, true, s.type)) !=
                SMOL_OK ||
            (st = check_in_place(in.grad_x, in.grad_x_row_stride, in.grad_x_head_stride, in.x,
                                 in.x_row_stride, in.x_head_stride, s.rows, in.heads)) !=
                SMOL_OK ||
            (st = check_in_place(in.grad_x, in.grad_x_row_stride, in.grad_x_head_stride,
                                 in.grad_out, in.grad_out_row_stride, in.grad_out_head_stride,
                                 s.rows, in.heads)) != SMOL_OK ||
            (st = check_small_vector(names[k][3], in.weight, s.weight_type)) != SMOL_OK)
            return st;
        HeadSide &to = a.side[k];
        to.dy = in.grad_out;
        to.x = in.x;
        to.out = in.grad_x;
        to.weight = in.weight;
        to.dy_row = in.grad_out_row_stride;
        to.dy_head = in.grad_out_head_stride;
        to.x_row = in.x_row_stride;
        to.x_head = in.x_head_stride;
        to.out_row = in.grad_x_row_stride;
        to.out_head = in.grad_x_head_stride;
        to.heads = in.heads;
    }
    const int64_t need = smol_head_norm_workspace_bytes(s.rows, p->q.heads, p->k.heads, s.dim);
    if (!p->workspace || (uintptr_t)p->workspace % 16 || p->workspace_bytes < need)
        return set_error(SMOL_ERR_INVALID_ARG,
                         "workspace must be 16-byte aligned and hold %lld bytes",
                         (long long)need);
    const auto &q = p->q, &k = p->k;
    if ((q.grad_weight && q.grad_weight == k.grad_weight) ||
        (s.rows > 0 && q.heads && k.heads &&
         (q.grad_x == k.grad_x || q.grad_x == k.x || q.grad_x == k.grad_out ||
          k.grad_x == q.x || k.grad_x == q.grad_out)))
        return set_error(SMOL_ERR_INVALID_ARG, "a gradient of q stands where one of k does");
    a.part = (float *)p->workspace;
    int e = hipSuccess;
    if (s.rows > 0 && p->q.heads + p->k.heads > 0) {
        fill_shape(&a, &f, s);
        a.sign = -1.0f;
        plan(&a, &f, s.type, kFewGradItems);
        const int64_t groups = (a.items + kWaves - 1) / kWaves;
        a.groups = (int32_t)(groups < kGradGroups ? groups : kGradGroups);
        e = launch(a, f, s.type, true, a.groups, stream);
    }
    if (e == hipSuccess && (p->q.grad_weight || p->k.grad_weight)) {
        with_type(s.weight_type, [&](auto t) {
            typedef decltype(t) P;
            hipLaunchKernelGGL((head_join_kernel<P>), dim3((2 * s.dim + 15) / 16), dim3(1024), 0,
                               (hipStream_t)stream, a.part, (P *)p->q.grad_weight,
                               (P *)p->k.grad_weight, s.dim, a.groups, p->accumulate);
        });
        e = (int)hipGetLastError();
    }
    if (e != hipSuccess)
        return set_error(SMOL_ERR_HIP, "head norm backward launch: %s",
                         hipGetErrorString((hipError_t)e));
    return SMOL_OK;
}
