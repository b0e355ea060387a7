// smol_heads_kernels.h -- rotation by positions and norm of heads, as
// templates for one type (instantiated by smol_heads_<type>.hip).
//
// A head's values are chunks of V elements, taken in units of two: the chunks
// of the two halves that turn together (or neighbouring chunks, interleaved,
// where a chunk holds whole pairs), so that a rotation needs no other lane's
// values. G lanes, a power of two, hold a head, K units each; the wave's 64 / G
// slots take the rows and heads of a block of R rows in turn, and since R
// divides the slots, a lane keeps its row and its columns for the whole block:
// cosines and sines are computed once for a row and pair, over the wave's
// lanes, passed through LDS, and stay in registers for all heads.
//
// The angle's turns, p f / 2 pi, are formed and reduced to -0.5 .. 0.5 in fp64
// (32 bits would lose the angle of far positions: at 2^20 they resolve 1/16
// radian); cosine and sine of the reduced angle are fp32.
#ifndef SMOL_HEADS_KERNELS_H
#define SMOL_HEADS_KERNELS_H

#include <hip/hip_runtime.h>
#include <math.h>

#include <type_traits>

#include "smol_heads.h"

namespace smol {
namespace {

constexpr int kHeadWaves = 4;

// Pairs of a block at most: R rows of `half` of them. A lane's K units hold K V
// pairs, G lanes a head, and R <= 64 / G.
template <int V, int K>
constexpr int kHeadPairs = 64 * V * K;

// The sum over the 2^log2 neighbouring lanes of a head, the same bits in each:
// with every partner the sum of the other half, as far as the group goes.
__device__ __forceinline__ float head_sum(float x, int log2)
{
#define SMOL_DPP_ADD(ctrl)                                                                       \
    x += __builtin_bit_cast(                                                                     \
        float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), ctrl, 0xf, 0xf, true))
    if (log2 > 0)
        SMOL_DPP_ADD(0xb1);  // quad_perm 1, 0, 3, 2
    if (log2 > 1)
        SMOL_DPP_ADD(0x4e);  // quad_perm 2, 3, 0, 1
    if (log2 > 2)
        SMOL_DPP_ADD(0x141);  // row_half_mirror: the other four of eight
    if (log2 > 3)
        SMOL_DPP_ADD(0x140);  // row_mirror: the other eight of sixteen
#undef SMOL_DPP_ADD
    if (log2 > 4)
        x += __shfl_xor(x, 16);
    if (log2 > 5)
        x += __shfl_xor(x, 32);
    return x;
}

// A lane's columns.
template <int V, int K, bool Inter>
struct Units {
    int32_t a[K], b[K];       // first columns of the two chunks
    bool live[K], both[K];    // the unit, and its second chunk, exist
    bool turn_a[K], turn_b[K];
    int32_t pair[K];          // the first rotated pair
    __device__ __forceinline__ Units(const HeadArgs &h, int sub)
    {
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int32_t u = sub + (k << h.lanes_log2);
            live[k] = u < h.units;
            const int32_t at = live[k] ? u : 0;
            const int32_t halves = Inter ? 0 : h.half / V;
            const bool pairs = at < halves;  // the chunks turn together
            const int32_t beside = (Inter ? 0 : 2 * h.half) + 2 * (at - halves) * V;
            const int32_t first = pairs ? at * V : beside;
            const int32_t second = pairs ? h.half + at * V : beside + V;
            a[k] = first;
            pair[k] = pairs ? first : first >> 1;
            turn_a[k] = Inter ? first < 2 * h.half : pairs;
            turn_b[k] = Inter ? second < 2 * h.half : pairs;
            both[k] = live[k] && second < h.dim;
            b[k] = second < h.dim ? second : first;
        }
    }
};

// Cosines and sines of the lane's pairs, V a unit.
template <int V, int K, bool Inter>
struct Angles {
    float c[K][V], s[K][V];
    // The table of a block's pairs, [row][pair], by the wave's lanes in turn.
    static __device__ __forceinline__ void tabulate(const HeadArgs &h, int32_t row0, int lane,
                                                    float2 *table)
    {
        const int32_t rows = 1 << h.rows_log2, count = h.half << h.rows_log2;
        for (int32_t t = lane; t < count; t += 64) {
            const int32_t r = t & (rows - 1), p = t >> h.rows_log2;
            const int32_t row = row0 + r < h.rows ? row0 + r : h.rows - 1;
            const double at = h.wide ? (double)((const int64_t *)h.positions)[row]
                                     : (double)((const int32_t *)h.positions)[row];
            double turns = at * h.freqs[p] * 0.15915494309189533577;
            turns -= rint(turns);
            float sn, cs;
            sincospif(2.0f * (float)turns, &sn, &cs);
            table[r * h.half + p] = make_float2(cs * h.gain, sn * (h.gain * h.sign));
        }
        asm volatile("" ::: "memory");  // other lanes read what this one writes
    }
    __device__ __forceinline__ void take(const HeadArgs &h, const Units<V, K, Inter> &u, int32_t r,
                                         const float2 *table)
    {
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const int32_t p = u.pair[k] + e;
                const float2 v = table[p < h.half ? r * h.half + p : 0];
                c[k][e] = v.x;
                s[k][e] = v.y;
            }
        asm volatile("" ::: "memory");  // the next block writes the table again
    }
    // Turns unit k's values; what does not turn stays as it is, whatever its
    // neighbours hold.
    __device__ __forceinline__ void turn(const Units<V, K, Inter> &u, int k, vec<float, V> &a,
                                         vec<float, V> &b) const
    {
        const vec<float, V> x = a, y = b;
        if (!Inter || V == 1) {
#pragma unroll
            for (int e = 0; e < V; ++e) {
                a[e] = u.turn_a[k] ? x[e] * c[k][e] - y[e] * s[k][e] : x[e];
                b[e] = u.turn_a[k] ? y[e] * c[k][e] + x[e] * s[k][e] : y[e];
            }
            return;
        }
#pragma unroll
        for (int e = 0; e + 1 < V; e += 2) {
            const int p = e / 2, q = V / 2 + e / 2;
            a[e] = u.turn_a[k] ? x[e] * c[k][p] - x[e + 1] * s[k][p] : x[e];
            a[e + 1] = u.turn_a[k] ? x[e + 1] * c[k][p] + x[e] * s[k][p] : x[e + 1];
            b[e] = u.turn_b[k] ? y[e] * c[k][q] - y[e + 1] * s[k][q] : y[e];
            b[e + 1] = u.turn_b[k] ? y[e + 1] * c[k][q] + y[e] * s[k][q] : y[e + 1];
        }
    }
};

template <typename T, int V>
__device__ __forceinline__ vec<float, V> head_weights(const HeadArgs &h, const void *p, int32_t at)
{
    if (!p)
        return (vec<float, V>)1.0f;
    if (h.weight_f32)
        return load<float, V>((const float *)p + at);
    return to_f32<V, T>(load<T, V>((const T *)p + at));
}

template <int V>
__device__ __forceinline__ float squares(vec<float, V> x)
{
    float s = 0.0f;
#pragma unroll
    for (int e = 0; e < V; ++e)
        s = fmaf(x[e], x[e], s);
    return s;
}

// A wave's place in its work.
struct HeadPlace {
    int32_t row0, row, slot, slots, first, last;  // steps [first, last) of both sides
    bool row_live;
    __device__ __forceinline__ HeadPlace(const HeadArgs &h, int64_t item, int lane)
    {
        int32_t block = (int32_t)item, part = 0;
        if (h.parts > 1) {
            block = (int32_t)((uint32_t)item / (uint32_t)h.parts);
            part = (int32_t)item - block * h.parts;
        }
        slots = 64 >> h.lanes_log2;
        slot = lane >> h.lanes_log2;
        row0 = block << h.rows_log2;
        row = row0 + (slot & ((1 << h.rows_log2) - 1));
        row_live = row < h.rows;
        row = row_live ? row : h.rows - 1;
        first = part * h.per;
        last = first + h.per;
    }
};

// Forward, and the rotation's gradient. Bound by memory: 32768 rows of 16 heads of 128
// bf16 values turned, 269 MB, in 50 us (5.3 TB/s); 32 and 8 heads normalised and
// turned, 671 MB, in 125 (5.4). One row's call is the launch: 3.8 us.
template <typename T, int V, int K, bool Norm, bool Inter>
__global__ void __launch_bounds__(64 * kHeadWaves) head_kernel(HeadArgs h)
{
    __shared__ float2 tables[kHeadWaves][kHeadPairs<V, K>];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Units<V, K, Inter> u(h, lane & ((1 << h.lanes_log2) - 1));
    const float inv = 1.0f / (float)h.dim;
    for (int64_t item = (int64_t)blockIdx.x * kHeadWaves + wave; item < h.items;
         item += (int64_t)gridDim.x * kHeadWaves) {
        const HeadPlace at(h, item, lane);
        Angles<V, K, Inter> angles;
        if (h.half) {
            angles.tabulate(h, at.row0, lane, tables[wave]);
            angles.take(h, u, at.row - at.row0, tables[wave]);
        }
        int32_t before = 0;
#pragma unroll 1
        for (int sd = 0; sd < 2; ++sd) {
            const HeadSide &side = h.side[sd];
            const int32_t lo = at.first > before ? at.first - before : 0;
            const int32_t hi = at.last - before < side.steps ? at.last - before : side.steps;
            before += side.steps;
            if (lo >= hi)
                continue;
            vec<float, V> wa[K], wb[K];
            if (Norm)
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    wa[k] = head_weights<T, V>(h, side.weight, u.a[k]);
                    wb[k] = head_weights<T, V>(h, side.weight, u.b[k]);
                }
            const auto head_of = [&](int32_t s) {
                return (s * at.slots + at.slot) >> h.rows_log2;
            };
            vec<T, V> na[K], nb[K];
            const auto fetch = [&](int32_t s) {
                const int32_t head = head_of(s);
                const T *p = (const T *)side.x + at.row * side.x_row +
                             (head < side.heads ? head : side.heads - 1) * side.x_head;
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    na[k] = load<T, V>(p + u.a[k]);
                    nb[k] = load<T, V>(p + u.b[k]);
                }
            };
            fetch(lo);
            for (int32_t s = lo; s < hi; ++s) {
                vec<float, V> a[K], b[K];
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    a[k] = to_f32<V, T>(na[k]);
                    b[k] = to_f32<V, T>(nb[k]);
                }
                if (s + 1 < hi)  // each head is read before any of it is written
                    fetch(s + 1);
                if (Norm) {
                    float sum = 0.0f;
#pragma unroll
                    for (int k = 0; k < K; ++k) {
                        sum += u.live[k] ? squares<V>(a[k]) : 0.0f;
                        sum += u.both[k] ? squares<V>(b[k]) : 0.0f;
                    }
                    const float r =
                        1.0f / sqrtf(head_sum(sum, h.lanes_log2) * inv + h.eps);
#pragma unroll
                    for (int k = 0; k < K; ++k) {
                        a[k] = a[k] * r * wa[k];
                        b[k] = b[k] * r * wb[k];
                    }
                }
                if (h.half)
#pragma unroll
                    for (int k = 0; k < K; ++k)
                        angles.turn(u, k, a[k], b[k]);
                const int32_t head = head_of(s);
                if (!at.row_live || head >= side.heads)
                    continue;
                T *p = (T *)side.out + at.row * side.out_row + head * side.out_head;
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    if (u.live[k])
                        store<T, V>(p + u.a[k], from_f32<T, V>(a[k]));
                    if (u.both[k])
                        store<T, V>(p + u.b[k], from_f32<T, V>(b[k]));
                }
            }
        }
    }
}

// Backward of the norm: the sums over rows and heads of g xh stay in registers
// until the workgroup's last row. Bound by memory: 32768 rows of 32 and 8 heads of 128
// bf16 values, 1007 MB, in 193 us (5.2 TB/s); a call of a few rows is its two launches
// (331 x 3 rows of 5 and 5 heads of 72 in fp32: 8.5 us and the join's 2).
template <typename T, int V, int K, bool Inter>
__global__ void __launch_bounds__(64 * kHeadWaves) head_grad_kernel(HeadArgs h)
{
    __shared__ float2 tables[kHeadWaves][kHeadPairs<V, K>];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Units<V, K, Inter> u(h, lane & ((1 << h.lanes_log2) - 1));
    const float inv = 1.0f / (float)h.dim;
    vec<float, V> dwa[2][K], dwb[2][K];
#pragma unroll
    for (int sd = 0; sd < 2; ++sd)
#pragma unroll
        for (int k = 0; k < K; ++k)
            dwa[sd][k] = dwb[sd][k] = (vec<float, V>)0.0f;
    for (int64_t item = (int64_t)blockIdx.x * kHeadWaves + wave; item < h.items;
         item += (int64_t)gridDim.x * kHeadWaves) {
        const HeadPlace at(h, item, lane);
        Angles<V, K, Inter> angles;
        if (h.half) {
            angles.tabulate(h, at.row0, lane, tables[wave]);
            angles.take(h, u, at.row - at.row0, tables[wave]);
        }
        int32_t before = 0;
#pragma unroll
        for (int sd = 0; sd < 2; ++sd) {
            const HeadSide &side = h.side[sd];
            const int32_t lo = at.first > before ? at.first - before : 0;
            const int32_t hi = at.last - before < side.steps ? at.last - before : side.steps;
            before += side.steps;
            if (lo >= hi)
                continue;
            vec<float, V> wa[K], wb[K];
#pragma unroll
            for (int k = 0; k < K; ++k) {
                wa[k] = head_weights<T, V>(h, side.weight, u.a[k]);
                wb[k] = head_weights<T, V>(h, side.weight, u.b[k]);
            }
            const auto head_of = [&](int32_t s) {
                return (s * at.slots + at.slot) >> h.rows_log2;
            };
            vec<T, V> nxa[K], nxb[K], nda[K], ndb[K];
            const auto fetch = [&](int32_t s) {
                const int32_t of = head_of(s), head = of < side.heads ? of : side.heads - 1;
                const T *px = (const T *)side.x + at.row * side.x_row + head * side.x_head;
                const T *pd = (const T *)side.dy + at.row * side.dy_row + head * side.dy_head;
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    nxa[k] = load<T, V>(px + u.a[k]);
                    nxb[k] = load<T, V>(px + u.b[k]);
                    nda[k] = load<T, V>(pd + u.a[k]);
                    ndb[k] = load<T, V>(pd + u.b[k]);
                }
            };
            fetch(lo);
            for (int32_t s = lo; s < hi; ++s) {
                vec<float, V> xa[K], xb[K], ga[K], gb[K];
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    xa[k] = to_f32<V, T>(nxa[k]);
                    xb[k] = to_f32<V, T>(nxb[k]);
                    ga[k] = to_f32<V, T>(nda[k]);
                    gb[k] = to_f32<V, T>(ndb[k]);
                }
                if (s + 1 < hi)
                    fetch(s + 1);
                const int32_t head = head_of(s);
                const bool live = at.row_live && head < side.heads;
                float xx = 0.0f, ux = 0.0f;
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    if (h.half)
                        angles.turn(u, k, ga[k], gb[k]);
                    xx += u.live[k] ? squares<V>(xa[k]) : 0.0f;
                    xx += u.both[k] ? squares<V>(xb[k]) : 0.0f;
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        ux = u.live[k] ? fmaf(ga[k][e] * wa[k][e], xa[k][e], ux) : ux;
                        ux = u.both[k] ? fmaf(gb[k][e] * wb[k][e], xb[k][e], ux) : ux;
                    }
                }
                const float r = 1.0f / sqrtf(head_sum(xx, h.lanes_log2) * inv + h.eps);
                // mean(u xh), xh = x r
                const float along = head_sum(ux, h.lanes_log2) * r * inv;
                if (!live)
                    continue;
                T *p = (T *)side.out + at.row * side.out_row + head * side.out_head;
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    vec<float, V> da, db;
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        const float ha = xa[k][e] * r, hb = xb[k][e] * r;
                        da[e] = r * (ga[k][e] * wa[k][e] - ha * along);
                        db[e] = r * (gb[k][e] * wb[k][e] - hb * along);
                        dwa[sd][k][e] = fmaf(ga[k][e], ha, dwa[sd][k][e]);
                        dwb[sd][k][e] = fmaf(gb[k][e], hb, dwb[sd][k][e]);
                    }
                    if (u.live[k])
                        store<T, V>(p + u.a[k], from_f32<T, V>(da));
                    if (u.both[k])
                        store<T, V>(p + u.b[k], from_f32<T, V>(db));
                }
            }
        }
    }
    // the workgroup's sums: over the wave's slots, then its waves, in order
    float *sums = (float *)tables[wave];  // dim <= 2 * kHeadPairs
    float *out = h.part + (int64_t)blockIdx.x * 2 * h.dim;
#pragma unroll
    for (int sd = 0; sd < 2; ++sd) {
        for (int step = 1 << h.lanes_log2; step < 64; step <<= 1)
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    dwa[sd][k][e] += __shfl_xor(dwa[sd][k][e], step);
                    dwb[sd][k][e] += __shfl_xor(dwb[sd][k][e], step);
                }
        __syncthreads();
        if (lane >> h.lanes_log2 == 0)
#pragma unroll
            for (int k = 0; k < K; ++k) {
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    if (u.live[k])
                        sums[u.a[k] + e] = dwa[sd][k][e];
                    if (u.both[k])
                        sums[u.b[k] + e] = dwb[sd][k][e];
                }
            }
        __syncthreads();
        for (int c = threadIdx.x; c < h.dim; c += 64 * kHeadWaves) {
            float v = 0.0f;
#pragma unroll
            for (int w = 0; w < kHeadWaves; ++w)
                v += ((const float *)tables[w])[c];
            out[sd * h.dim + c] = v;
        }
    }
}

template <typename T>
int launch_heads(const HeadArgs &a, const HeadForm &f, bool backward, unsigned grid, void *s)
{
    const auto form = [&](auto v, auto k) {
        const auto order = [&](auto inter) {
            const dim3 g(grid), b(64 * kHeadWaves);
            hipStream_t st = (hipStream_t)s;
            constexpr int V = decltype(v)::value, K = decltype(k)::value;
            constexpr bool I = decltype(inter)::value;
            if (backward)
                hipLaunchKernelGGL((head_grad_kernel<T, V, K, I>), g, b, 0, st, a);
            else if (f.norm)
                hipLaunchKernelGGL((head_kernel<T, V, K, true, I>), g, b, 0, st, a);
            else
                hipLaunchKernelGGL((head_kernel<T, V, K, false, I>), g, b, 0, st, a);
        };
        if (f.interleaved)
            order(std::true_type{});
        else
            order(std::false_type{});
    };
    typedef std::integral_constant<int, 1> One;
    if (f.v == 8) {
        if constexpr (sizeof(T) == 2)
            form(std::integral_constant<int, 8>{}, One{});
    } else if (f.v == 4)
        form(std::integral_constant<int, 4>{}, One{});
    else if (f.v == 2)
        form(std::integral_constant<int, 2>{}, One{});
    else if (f.k == 1)
        form(One{}, One{});
    else
        form(One{}, std::integral_constant<int, 2>{});
    return (int)hipGetLastError();
}

}  // namespace
}  // namespace smol

#endif  // SMOL_HEADS_KERNELS_H
