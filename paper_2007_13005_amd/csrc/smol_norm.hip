// smol_norm.hip -- layer norm and its backward pass (smol_layer_norm,
// smol_layer_norm_backward).
//
// A row stays in the registers of W waves between its one read and its one
// write: E elements a lane, columns in chunks of 16 bytes a lane. Mean and
// variance are formed wave by wave (the variance from differences to the
// wave's own mean) and joined over the waves by
//   n = n1 + n2, mean = mean1 + (mean2 - mean1) n2 / n,
//   M2 = M2_1 + M2_2 + (mean2 - mean1)^2 n1 n2 / n,
// which needs one exchange through LDS and no difference of squares.
// Both directions are bound by memory: about 1.5 operations a byte.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "smol.h"
#include "smol_internal.h"
#include "smol_tokens.h"
#include "smol_tokens_device.h"

namespace smol {
namespace {

struct NormArgs {
    const void *x, *residual, *weight, *bias;
    void *out, *sum;
    float *mean, *rstd;
    int64_t x_stride, residual_stride, out_stride, sum_stride;
    int32_t rows, dim;
    int32_t weight_f32;
    float eps;
};

// The columns of a lane. Chunk c of a row starts at column (c * W * 64 +
// thread) * V; a chunk that would pass the row's end is moved back to end
// with it (its first elements are then another lane's, "lead" of them), one
// that starts past it has no elements. dim >= V.
template <int V, int C, int W>
struct Columns {
    int32_t at[C], lead[C];
    __device__ __forceinline__ Columns(int32_t dim, int32_t thread)
    {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int32_t col = (c * W * 64 + thread) * V;
            at[c] = col <= dim - V ? col : dim - V;
            lead[c] = col < dim ? col - at[c] : V;
        }
    }
};

template <typename T, int V>
__device__ __forceinline__ vec<float, V> weights_at(const void *p, int32_t f32, int32_t at,
                                                    float none)
{
    if (!p)
        return (vec<float, V>)none;
    if (f32)
        return load<float, V>((const float *)p + at);
    return to_f32<V, T>(load<T, V>((const T *)p + at));
}

// W waves a row; a workgroup of R * W waves takes R rows at a time, and the
// weights stay in registers over its rows. Bound by memory: 50432 rows of 1024
// bf16 values with a residual sum, 81 us, 5.1 TB/s (what a large copy reaches);
// one row of 4096 fp16 values 2.8 us. Up to 1024 columns a wave has one row, so
// narrow rows leave lanes and loads idle: 65536 rows of bf16 values without a
// residual, columns 512: 27 us, 5.0 TB/s, 256: 18.7, 3.6, 128: 17.5, 1.9, 64:
// 17.3, 1.0.
template <typename T, int V, int C, int W, int R>
__global__ void __launch_bounds__(64 * W * R) norm_kernel(NormArgs a)
{
    const int32_t thread = threadIdx.x % (64 * W), wave = (threadIdx.x >> 6) % W;
    const int32_t slot = __builtin_amdgcn_readfirstlane(threadIdx.x / (64 * W));
    const Columns<V, C, W> col(a.dim, thread);
    __shared__ float part[2][R][W][2];
    const float inv = 1.0f / (float)a.dim;
    vec<float, V> w[C], b[C];
#pragma unroll
    for (int c = 0; c < C; ++c) {
        w[c] = weights_at<T, V>(a.weight, a.weight_f32, col.at[c], 1.0f);
        b[c] = weights_at<T, V>(a.bias, a.weight_f32, col.at[c], 0.0f);
    }
    // elements of this wave's columns
    int32_t count = 0;
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int32_t first = (c * W + wave) * 64 * V, left = a.dim - first;
        count += left < 0 ? 0 : left < 64 * V ? left : 64 * V;
    }
    int32_t flip = 0;
    // every wave of a workgroup makes the same number of turns (barriers)
    for (int32_t r0 = blockIdx.x * R; r0 < a.rows; r0 += gridDim.x * R, flip ^= 1) {
        const int32_t row = r0 + slot;
        const bool live = R == 1 || row < a.rows;
        vec<T, V> x[C];
        if (live) {
            const T *px = (const T *)a.x + row * a.x_stride;
#pragma unroll
            for (int c = 0; c < C; ++c)
                x[c] = load<T, V>(px + col.at[c]);
            if (a.residual) {
                const T *pr = (const T *)a.residual + row * a.residual_stride;
                vec<T, V> r[C];
#pragma unroll
                for (int c = 0; c < C; ++c)
                    r[c] = load<T, V>(pr + col.at[c]);
#pragma unroll
                for (int c = 0; c < C; ++c)
                    x[c] = from_f32<T, V>(to_f32<V, T>(x[c]) + to_f32<V, T>(r[c]));
            }
        } else {
#pragma unroll
            for (int c = 0; c < C; ++c)
                x[c] = (vec<T, V>)(T)0.0f;
        }
        vec<float, V> z[C];
        float sum = 0.0f;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            z[c] = to_f32<V, T>(x[c]);
#pragma unroll
            for (int e = 0; e < V; ++e)
                sum += e >= col.lead[c] ? z[c][e] : 0.0f;
        }
        sum = wave_sum(sum);
        float mean = sum * (W == 1 ? inv : count ? 1.0f / (float)count : 0.0f);
        float m2 = 0.0f;
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float d = z[c][e] - mean;
                m2 = e >= col.lead[c] ? fmaf(d, d, m2) : m2;
            }
        m2 = wave_sum(m2);
        if (W > 1) {
            if ((threadIdx.x & 63) == 0) {
                part[flip][slot][wave][0] = mean;
                part[flip][slot][wave][1] = m2;
            }
            __syncthreads();
            mean = part[flip][slot][0][0];
            m2 = part[flip][slot][0][1];
            float n1 = (float)(a.dim < 64 * V ? a.dim : 64 * V);
#pragma unroll
            for (int c = 1; c < C; ++c) {
                const int32_t left = a.dim - c * W * 64 * V;
                n1 += (float)(left < 0 ? 0 : left < 64 * V ? left : 64 * V);
            }
#pragma unroll
            for (int k = 1; k < W; ++k) {
                int32_t nk = 0;
#pragma unroll
                for (int c = 0; c < C; ++c) {
                    const int32_t left = a.dim - (c * W + k) * 64 * V;
                    nk += left < 0 ? 0 : left < 64 * V ? left : 64 * V;
                }
                const float n2 = (float)nk, n = n1 + n2;
                const float d = part[flip][slot][k][0] - mean, f = n2 / n;
                mean = fmaf(d, f, mean);
                m2 += part[flip][slot][k][1] + d * d * (n1 * f);
                n1 = n;
            }
        }
        const float rstd = 1.0f / sqrtf(m2 * inv + a.eps);
        if (!live)
            continue;
        if (a.sum) {
            T *ps = (T *)a.sum + row * a.sum_stride;
#pragma unroll
            for (int c = 0; c < C; ++c)
                if (col.lead[c] < V)
                    store<T, V>(ps + col.at[c], x[c]);
        }
        T *po = (T *)a.out + row * a.out_stride;
#pragma unroll
        for (int c = 0; c < C; ++c)
            if (col.lead[c] < V) {
                vec<float, V> y;
#pragma unroll
                for (int e = 0; e < V; ++e)
                    y[e] = fmaf((z[c][e] - mean) * rstd, w[c][e], b[c][e]);
                store<T, V>(po + col.at[c], from_f32<T, V>(y));
            }
        if (thread == 0) {
            if (a.mean)
                a.mean[row] = mean;
            if (a.rstd)
                a.rstd[row] = rstd;
        }
    }
}

struct NormGradArgs {
    const void *dy, *h, *dsum, *weight;
    const float *mean, *rstd;
    void *dx, *dw, *db;
    float *part;  // [workgroups][2][dim]: sums of dy xh, of dy
    int64_t dy_stride, h_stride, dsum_stride, dx_stride;
    int32_t rows, dim;
    int32_t weight_f32, weight_type;
    int32_t groups, accumulate;
};

// Backward: rows as in the forward pass; the sums over rows of dy xh and dy stay
// in registers until the workgroup's last row, so that the weights' gradients
// cost one row of sums a workgroup and no second reading. 50432 rows of 1024
// bf16 values with a gradient past the norm: 79 us, 5.2 TB/s. Narrow rows,
// 65536 of bf16 values, columns 512: 48 us, 4.2 TB/s, 256: 36, 2.8, 128: 34, 1.5,
// 64: 33, 0.8.
template <typename T, int V, int C, int W, int R>
__global__ void __launch_bounds__(64 * W * R) norm_grad_kernel(NormGradArgs a)
{
    const int32_t thread = threadIdx.x % (64 * W), wave = (threadIdx.x >> 6) % W;
    const int32_t slot = __builtin_amdgcn_readfirstlane(threadIdx.x / (64 * W));
    const Columns<V, C, W> col(a.dim, thread);
    __shared__ float part[2][R][W][2];
    const float inv = 1.0f / (float)a.dim;
    vec<float, V> w[C], dw[C], db[C];
#pragma unroll
    for (int c = 0; c < C; ++c) {
        w[c] = weights_at<T, V>(a.weight, a.weight_f32, col.at[c], 1.0f);
        dw[c] = db[c] = (vec<float, V>)0.0f;
    }
    int32_t flip = 0;
    for (int32_t r0 = blockIdx.x * R; r0 < a.rows; r0 += gridDim.x * R, flip ^= 1) {
        const int32_t row = r0 + slot;
        const bool live = R == 1 || row < a.rows;
        if (W == 1 && !live)
            break;
        const int32_t at = live ? row : a.rows - 1;  // past the last row: read, not used
        vec<T, V> dy[C], h[C], ds[C];
        const T *pd = (const T *)a.dy + at * a.dy_stride;
        const T *ph = (const T *)a.h + at * a.h_stride;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            dy[c] = load<T, V>(pd + col.at[c]);
            h[c] = load<T, V>(ph + col.at[c]);
        }
        if (a.dsum) {
            const T *ps = (const T *)a.dsum + at * a.dsum_stride;
#pragma unroll
            for (int c = 0; c < C; ++c)
                ds[c] = load<T, V>(ps + col.at[c]);
        }
        const float mean = a.mean[at], rstd = a.rstd[at];
        float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const bool own = live && e >= col.lead[c];
                const float d = own ? (float)dy[c][e] : 0.0f;
                const float xh = own ? ((float)h[c][e] - mean) * rstd : 0.0f;
                const float g = d * w[c][e];
                s1 += own ? g : 0.0f;
                s2 = own ? fmaf(g, xh, s2) : s2;
                dw[c][e] = fmaf(d, xh, dw[c][e]);
                db[c][e] += d;
            }
        s1 = wave_sum(s1);
        s2 = wave_sum(s2);
        if (W > 1) {
            if ((threadIdx.x & 63) == 0) {
                part[flip][slot][wave][0] = s1;
                part[flip][slot][wave][1] = s2;
            }
            __syncthreads();
            s1 = s2 = 0.0f;
#pragma unroll
            for (int k = 0; k < W; ++k) {
                s1 += part[flip][slot][k][0];
                s2 += part[flip][slot][k][1];
            }
        }
        s1 *= inv;
        s2 *= inv;
        T *px = (T *)a.dx + at * a.dx_stride;
#pragma unroll
        for (int c = 0; c < C; ++c)
            if (live && col.lead[c] < V) {
                vec<float, V> v;
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float xh = ((float)h[c][e] - mean) * rstd;
                    v[e] = rstd * ((float)dy[c][e] * w[c][e] - s1 - xh * s2);
                    if (a.dsum)
                        v[e] += (float)ds[c][e];
                }
                store<T, V>(px + col.at[c], from_f32<T, V>(v));
            }
    }
    // the workgroup's sums: slot 0 adds the other slots' in order
    float *out = a.part + (int64_t)blockIdx.x * 2 * a.dim;
    if (R > 1) {
        __shared__ float rows[R > 1 ? (R - 1) * W * 64 * C * V : 1];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            __syncthreads();
            if (slot > 0)
#pragma unroll
                for (int c = 0; c < C; ++c)
#pragma unroll
                    for (int e = 0; e < V; ++e)
                        rows[(((slot - 1) * C + c) * V + e) * W * 64 + thread] =
                            k ? db[c][e] : dw[c][e];
            __syncthreads();
            if (slot == 0)
#pragma unroll
                for (int c = 0; c < C; ++c)
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        float v = k ? db[c][e] : dw[c][e];
#pragma unroll
                        for (int s = 0; s < R - 1; ++s)
                            v += rows[((s * C + c) * V + e) * W * 64 + thread];
                        if (k)
                            db[c][e] = v;
                        else
                            dw[c][e] = v;
                    }
        }
    }
    if (slot == 0)
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int e = 0; e < V; ++e)
                if (e >= col.lead[c]) {
                    out[col.at[c] + e] = dw[c][e];
                    out[a.dim + col.at[c] + e] = db[c][e];
                }
}

// Joins the workgroups' sums, in order: 16 columns a workgroup, 16 threads a
// column each taking every 16th workgroup's sums (512 workgroups, 1024
// columns: 5 us; 12 us with the loads one after the other).
template <typename P>
__global__ void __launch_bounds__(256) norm_join_kernel(NormGradArgs a)
{
    const int32_t c = blockIdx.x * 16 + (threadIdx.x & 15), q = threadIdx.x >> 4;
    __shared__ float part[16][17];
    float s = 0.0f;
    if (c < 2 * a.dim) {
        constexpr int kAhead = 8;
        const float *p = a.part + c;
        for (int32_t g = q; g < a.groups; g += 16 * kAhead) {
            float x[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const int32_t at = g + 16 * u;
                x[u] = p[(int64_t)(at < a.groups ? at : q) * 2 * a.dim];
            }
            asm volatile("" ::: "memory");  // eight loads at once
#pragma unroll
            for (int u = 0; u < kAhead; ++u)
                s += g + 16 * u < a.groups ? x[u] : 0.0f;
        }
    }
    part[q][threadIdx.x & 15] = s;
    __syncthreads();
    if (q != 0 || c >= 2 * a.dim)
        return;
    for (int k = 1; k < 16; ++k)
        s += part[k][threadIdx.x];
    P *out = (P *)(c < a.dim ? a.dw : a.db);
    if (!out)
        return;
    out += c < a.dim ? c : c - a.dim;
    *out = (P)(a.accumulate ? (float)*out + s : s);
}

// Workgroups of the backward pass at most: two a compute unit keep memory busy,
// and each adds a row of sums to the join.
constexpr int kGradGroups = 512;

// f<T, V, C, W, R>: the kernel of a row's width. Rows narrower than a chunk
// have one element a lane.
template <typename T, typename F>
void with_shape(int dim, F f)
{
    constexpr int V = 16 / sizeof(T);
    if (dim < V)
        f(std::integral_constant<int, 1>{}, std::integral_constant<int, 1>{},
          std::integral_constant<int, 1>{}, std::integral_constant<int, 4>{});
    else if (dim <= 512)
        f(std::integral_constant<int, V>{}, std::integral_constant<int, 8 / V>{},
          std::integral_constant<int, 1>{}, std::integral_constant<int, 4>{});
#define SMOL_SHAPE(W, R)                                                                         \
    f(std::integral_constant<int, V>{}, std::integral_constant<int, 16 / V>{},                  \
      std::integral_constant<int, W>{}, std::integral_constant<int, R>{})
    else if (dim <= 1024) SMOL_SHAPE(1, 4);
    else if (dim <= 2048) SMOL_SHAPE(2, 2);
    else if (dim <= 4096) SMOL_SHAPE(4, 1);
    else SMOL_SHAPE(8, 1);
#undef SMOL_SHAPE
}

int rows_per_group(int dim) { return dim <= 1024 ? 4 : dim <= 2048 ? 2 : 1; }

int64_t grad_groups(int64_t rows, int dim)
{
    const int64_t g = (rows + rows_per_group(dim) - 1) / rows_per_group(dim);
    return g < kGradGroups ? g : kGradGroups;
}

int check_common(int64_t rows, int32_t dim, int32_t type, int32_t weight_type)
{
    if (rows < 0 || dim < 1)
        return set_error(SMOL_ERR_INVALID_ARG, "rows %lld or dim %d out of range",
                         (long long)rows, dim);
    if (type < SMOL_ELEM_F32 || type > SMOL_ELEM_BF16)
        return set_error(SMOL_ERR_INVALID_ARG, "type %d unknown", type);
    if (weight_type != SMOL_ELEM_F32 && weight_type != type)
        return set_error(SMOL_ERR_INVALID_ARG, "weight_type %d is neither fp32 nor the type",
                         weight_type);
    if (rows > SMOL_MAX_ROWS || dim > SMOL_MAX_NORM_DIM)
        return set_error(SMOL_ERR_UNSUPPORTED, "rows %lld beyond %d or dim %d beyond %d",
                         (long long)rows, SMOL_MAX_ROWS, dim, SMOL_MAX_NORM_DIM);
    return SMOL_OK;
}

// least: the smallest row stride, the width for a matrix that is written.
int check_matrix(const char *name, const void *p, int64_t stride, int64_t rows, int64_t least,
                 int type)
{
    if (!p)
        return set_error(SMOL_ERR_INVALID_ARG, "%s is NULL", name);
    if ((uintptr_t)p % elem_size(type))
        return set_error(SMOL_ERR_INVALID_ARG, "%s is not aligned to its elements", name);
    // one row has no next row for its stride to reach
    if (rows > 1 && (stride < least || stride > INT64_MAX / 8 / rows))
        return set_error(SMOL_ERR_INVALID_ARG, "%s: row stride %lld out of range", name,
                         (long long)stride);
    return SMOL_OK;
}

int check_vector(const char *name, const void *p, int type)
{
    if ((uintptr_t)p % elem_size(type))
        return set_error(SMOL_ERR_INVALID_ARG, "%s is not aligned to its elements", name);
    return SMOL_OK;
}

}  // namespace
}  // namespace smol

extern "C" int smol_layer_norm(const smol_norm_args *p, void *stream)
{
    using namespace smol;
    clear_error();
    if (!p)
        return set_error(SMOL_ERR_INVALID_ARG, "args is NULL");
    int st = check_common(p->rows, p->dim, p->type, p->weight_type);
    if (st != SMOL_OK)
        return st;
    if (p->reserved[0] || p->reserved[1])
        return set_error(SMOL_ERR_INVALID_ARG, "reserved fields are not zero");
    if (!(p->eps >= 0.0f) || isinf(p->eps))
        return set_error(SMOL_ERR_INVALID_ARG, "eps is negative or not finite");
    if (p->rows == 0)
        return SMOL_OK;
    if ((st = check_matrix("x", p->x, p->x_stride, p->rows, 0, p->type)) != SMOL_OK ||
        (st = check_matrix("out", p->out, p->out_stride, p->rows, p->dim, p->type)) != SMOL_OK ||
        (p->residual && (st = check_matrix("residual", p->residual, p->residual_stride, p->rows,
                                           0, p->type)) != SMOL_OK) ||
        (p->sum && (st = check_matrix("sum", p->sum, p->sum_stride, p->rows, p->dim, p->type)) !=
                       SMOL_OK) ||
        (st = check_vector("weight", p->weight, p->weight_type)) != SMOL_OK ||
        (st = check_vector("bias", p->bias, p->weight_type)) != SMOL_OK ||
        (st = check_vector("mean", p->mean, SMOL_ELEM_F32)) != SMOL_OK ||
        (st = check_vector("rstd", p->rstd, SMOL_ELEM_F32)) != SMOL_OK)
        return st;
    if (p->sum && p->sum == p->out)
        return set_error(SMOL_ERR_INVALID_ARG, "sum and out are the same matrix");
    NormArgs a;
    a.x = p->x;
    a.residual = p->residual;
    a.weight = p->weight;
    a.bias = p->bias;
    a.out = p->out;
    a.sum = p->sum;
    a.mean = p->mean;
    a.rstd = p->rstd;
    a.x_stride = p->x_stride;
    a.residual_stride = p->residual_stride;
    a.out_stride = p->out_stride;
    a.sum_stride = p->sum_stride;
    a.rows = (int32_t)p->rows;
    a.dim = p->dim;
    a.weight_f32 = p->weight_type == SMOL_ELEM_F32;
    a.eps = p->eps;
    const int R = rows_per_group(p->dim);
    int64_t grid = (p->rows + R - 1) / R;
    if (grid > 2048)
        grid = 2048;
    with_type(p->type, [&](auto t) {
        typedef decltype(t) T;
        with_shape<T>(p->dim, [&](auto v, auto c, auto w, auto r) {
            hipLaunchKernelGGL((norm_kernel<T, v.value, c.value, w.value, r.value>),
                               dim3((unsigned)grid), dim3(64 * w.value * r.value), 0,
                               (hipStream_t)stream, a);
        });
    });
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess)
        return set_error(SMOL_ERR_HIP, "layer norm launch: %s", hipGetErrorString(e));
    return SMOL_OK;
}

extern "C" int64_t smol_norm_workspace_bytes(int64_t rows, int32_t dim)
{
    using namespace smol;
    if (rows < 0 || rows > SMOL_MAX_ROWS || dim < 1 || dim > SMOL_MAX_NORM_DIM)
        return 0;
    return (grad_groups(rows, dim) * 2 * dim * 4 + 15) / 16 * 16 + 16;
}

extern "C" int smol_layer_norm_backward(const smol_norm_grad_args *p, void *stream)
{
    using namespace smol;
    clear_error();
    if (!p)
        return set_error(SMOL_ERR_INVALID_ARG, "args is NULL");
    int st = check_common(p->rows, p->dim, p->type, p->weight_type);
    if (st != SMOL_OK)
        return st;
    if (p->accumulate != 0 && p->accumulate != 1)
        return set_error(SMOL_ERR_INVALID_ARG, "accumulate %d is neither 0 nor 1", p->accumulate);
    if (p->rows > 0 &&
        ((st = check_matrix("grad_out", p->grad_out, p->grad_stride, p->rows, 0, p->type)) !=
             SMOL_OK ||
         (st = check_matrix("h", p->h, p->h_stride, p->rows, 0, p->type)) != SMOL_OK ||
         (st = check_matrix("grad_x", p->grad_x, p->x_stride, p->rows, p->dim, p->type)) !=
             SMOL_OK ||
         (p->grad_sum && (st = check_matrix("grad_sum", p->grad_sum, p->sum_stride, p->rows, 0,
                                            p->type)) != SMOL_OK) ||
         (st = check_matrix("mean", p->mean, 0, 1, 0, SMOL_ELEM_F32)) != SMOL_OK ||
         (st = check_matrix("rstd", p->rstd, 0, 1, 0, SMOL_ELEM_F32)) != SMOL_OK))
        return st;
    if ((st = check_vector("weight", p->weight, p->weight_type)) != SMOL_OK ||
        (st = check_vector("grad_weight", p->grad_weight, p->weight_type)) != SMOL_OK ||
        (st = check_vector("grad_bias", p->grad_bias, p->weight_type)) != SMOL_OK)
        return st;
    if (!p->workspace || (uintptr_t)p->workspace % 16 ||
        p->workspace_bytes < smol_norm_workspace_bytes(p->rows, p->dim))
        return set_error(SMOL_ERR_INVALID_ARG,
                         "workspace must be 16-byte aligned and hold %lld bytes",
                         (long long)smol_norm_workspace_bytes(p->rows, p->dim));
    NormGradArgs a;
    a.dy = p->grad_out;
    a.h = p->h;
    a.dsum = p->grad_sum;
    a.weight = p->weight;
    a.mean = p->mean;
    a.rstd = p->rstd;
    a.dx = p->grad_x;
    a.dw = p->grad_weight;
    a.db = p->grad_bias;
    a.part = (float *)p->workspace;
    a.dy_stride = p->grad_stride;
    a.h_stride = p->h_stride;
    a.dsum_stride = p->sum_stride;
    a.dx_stride = p->x_stride;
    a.rows = (int32_t)p->rows;
    a.dim = p->dim;
    a.weight_f32 = p->weight_type == SMOL_ELEM_F32;
    a.groups = (int32_t)grad_groups(p->rows, p->dim);
    a.accumulate = p->accumulate;
    hipStream_t s = (hipStream_t)stream;
    if (a.groups > 0)
        with_type(p->type, [&](auto t) {
            typedef decltype(t) T;
            with_shape<T>(p->dim, [&](auto v, auto c, auto w, auto r) {
                hipLaunchKernelGGL((norm_grad_kernel<T, v.value, c.value, w.value, r.value>),
                                   dim3((unsigned)a.groups), dim3(64 * w.value * r.value), 0, s,
                                   a);
            });
        });
    hipError_t e = hipGetLastError();
    if (e == hipSuccess && (a.dw || a.db)) {
        with_type(p->weight_type, [&](auto t) {
            hipLaunchKernelGGL((norm_join_kernel<decltype(t)>), dim3((2 * a.dim + 15) / 16),
                               dim3(256), 0, s, a);
        });
        e = hipGetLastError();
    }
    if (e != hipSuccess)
        return set_error(SMOL_ERR_HIP, "layer norm backward launch: %s", hipGetErrorString(e));
    return SMOL_OK;
}
