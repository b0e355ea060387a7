// smol_attend_grad_kernels.h -- attention's gradients, as templates for one type
// (instantiated by smol_attend_grad_<type>.hip).
//
// With p = exp(s - lse) formed again from the forward pass's lse and D =
// grad_out . (out + rest) a row, d = p (grad_out v^T - D):
//   grad_q = scale d k,  grad_k = scale d^T q,  grad_v = p^T grad_out.
// Two kernels, each with its sums in registers and no atomics: one over columns
// (five products of scores, two of them for what it keeps: s, grad_out v^T, d k),
// which also writes D; one over keys (s, grad_out v^T, p^T grad_out, d^T q). The
// scores are formed twice, seven products for the five that one kernel with
// joined partial sums would need.
//
// p and d are rounded to the type as operands. fp16 has few exponents: there
// both are carried times 2^6 (a weight of 2^-20 is then still a normal number);
// d past 2^10 overflows, and its row is summed again as below.
//
// What a query does not see has p and d zero, by selection. Sums that are not
// finite in the end are formed again over what is seen alone (smol_attend_kernels.h).
#ifndef SMOL_ATTEND_GRAD_KERNELS_H
#define SMOL_ATTEND_GRAD_KERNELS_H

#include "smol_attend_device.h"

namespace smol {
namespace {

template <typename T>
constexpr float kCarry = std::is_same<T, f16>::value ? 6.0f : 0.0f;  // log2

template <typename T>
constexpr float kCarried = std::is_same<T, f16>::value ? 1.0f / 64.0f : 1.0f;

// Writes a result [values x rows]: the lane's row at p, times f; zeros for a row
// that has no pair (its sums may hold 0 times a NaN).
template <typename T, int N>
__device__ __forceinline__ void write_row(T *p, const f32x16 (&sum)[N], float f, bool none,
                                          int32_t dim, int lane)
{
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int32_t d = 32 * n + 8 * g + 4 * (lane >> 5);
            if (d >= dim)
                continue;
            vec<float, 4> y;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                y[e] = none ? 0.0f : sum[n][4 * g + e] * f;
            store<T, 4>(p + d, from_f32<T, 4>(y));
        }
}

// The weight of one pair and its d, over the wave.
struct PairOf {
    float p, d;
    __device__ __forceinline__ PairOf(const AttendArgs &a, const Spread &q, const Spread &dy,
                                      const Spread &k, const Spread &v, float lse2, float delta)
    {
        // not 0: an infinity counts however small its weight
        p = fmaxf(exp2_of(fmaf(dot(q, k), a.scale_log2, -lse2)), 1.0e-37f);
        d = p * (dot(dy, v) - delta);
    }
};

// Gradients of queries: four waves of 32 columns over shared tiles of 64 keys.
template <typename T, int N>
__global__ void __launch_bounds__(64 * kAttendWaves, sizeof(T) == 2 ? 2 : 1)
    attend_grad_q_kernel(AttendArgs a)
{
    constexpr int kThreads = 64 * kAttendWaves, kKeys = kAttendKeys;
    typedef LdsRows<T, N> Rows;
    constexpr int kBytes = kKeys * Rows::kStride;
    __shared__ __attribute__((aligned(512))) char lds[2][2 * kBytes];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t turn = divide(blockIdx.x, a.pair_div);
    const uint32_t pair = blockIdx.x - turn * a.pair_div.d;
    const uint32_t tile = a.causal ? a.tiles - 1 - turn : turn;
    const Sequence s(a, pair);
    const int32_t c0 = tile * (kAttendWaves * 32), mine = c0 + wave * 32;
    const Column c_first(a, s, c0), c_last(a, s, c0 + kAttendWaves * 32 - 1);
    const Walk<kKeys> walk(a, s, c_first.i, c_last.i);
    const Column c(a, s, mine + (lane & 31));
    const int64_t at = ((int64_t)s.b * a.queries + c.i) * a.heads + c.head;
    const int32_t last = c.exists ? s.last(a, c.i) : -1, first = s.first(a, c.i);
    const Column lo(a, s, mine), hi(a, s, mine + 31);
    const int32_t last_max =
        lo.i < s.q_length ? s.last(a, hi.i < s.q_length ? hi.i : s.q_length - 1) : -1;
    const int32_t last_min = mine + 31 < a.columns && hi.i < s.q_length ? s.last(a, lo.i) : -1;
    const int32_t first_min = s.first(a, lo.i), first_max = s.first(a, hi.i);
    vec<T, 8> q[2 * N], dy[2 * N];
    const T *qp = s.rows<T>(a.q, c.head) + c.i * a.q.row;
    const T *dyp = s.rows<T>(a.dout, c.head) + c.i * a.dout.row;
    row_operands<T, N>(qp, a.dim, lane, q);
    row_operands<T, N>(dyp, a.dim, lane, dy);
    float delta = 0.0f;
    {
        const T *op = s.rows<T>(a.out, c.head) + c.i * a.out.row;
        const T *rp = a.rest_in ? (const T *)a.rest_in + at * a.dim : nullptr;
#pragma unroll
        for (int t = 0; t < 2 * N; ++t) {
            const int32_t d = 16 * t + 8 * (lane >> 5);
            if (d >= a.dim)
                continue;
            vec<float, 8> y = to_f32<8, T>(load<T, 8>(op + d));
            if (rp)
                y += to_f32<8, T>(load<T, 8>(rp + d));
#pragma unroll
            for (int e = 0; e < 8; ++e)
                delta = fmaf((float)dy[t][e], y[e], delta);
        }
        delta = both_halves(delta, [](float u, float v) { return u + v; });
    }
    const float lse2 = last < 0 ? 0.0f : a.lse[at] * kLog2e;
    if (c.exists && lane < 32)
        a.delta[at] = delta;
    f32x16 sum[N];
#pragma unroll
    for (int n = 0; n < N; ++n)
        sum[n] = (f32x16)0.0f;
    const T *kp = s.rows<T>(a.k, s.kv), *vp = s.rows<T>(a.v, s.kv);
    Mover<T, N, kKeys, kThreads> k(a.dim, threadIdx.x), v(a.dim, threadIdx.x);
    const auto fetch = [&](int32_t n) {
        const int32_t j0 = walk.tile(n) * kKeys;
        k.fetch(kp, a.k.row, j0, s.k_length);
        v.fetch(vp, a.v.row, j0, s.k_length);
    };
    if (walk.count)
        fetch(0);
    const int row_at0 = Rows::row_at(lane), column_at0 = Rows::column_at(lane);
    for (int32_t n = 0; n < walk.count; ++n) {
        char *keys = lds[n & 1], *values = keys + kBytes;
        k.put(keys);
        v.put(values);
        __syncthreads();  // a tile is written again two turns on
        if (n + 1 < walk.count)
            fetch(n + 1);
        const int32_t j0 = walk.tile(n) * kKeys;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int32_t k0 = j0 + 32 * h, k1 = k0 + 31;
            if (k0 > last_max || (k1 < first_min && k0 >= a.sinks))
                continue;
            const int row_at = fresh(row_at0), column_at = fresh(column_at0);
            f32x16 x = (f32x16)0.0f, y = (f32x16)0.0f;
#pragma unroll
            for (int t = 0; t < 2 * N; ++t) {
                multiply<T>(x, Rows::row(keys, row_at, 32 * h, t), q[t]);
                multiply<T>(y, Rows::row(values, row_at, 32 * h, t), dy[t]);
            }
            const bool whole = k1 <= last_min && (k0 >= first_max || k1 < a.sinks);
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const float p = exp2_of(fmaf(x[e], a.scale_log2, kCarry<T> - lse2));
                x[e] = p * (y[e] - delta);
            }
            if (!whole)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int32_t j = k0 + 8 * (e >> 2) + 4 * (lane >> 5) + (e & 3);
                    x[e] = sees(j, last, first, a.sinks) ? x[e] : 0.0f;
                }
#pragma unroll
            for (int g = 0; g < 2; ++g) {
                const vec<T, 8> w = operand<T>(x, g);
#pragma unroll
                for (int n2 = 0; n2 < N; ++n2)
                    multiply<T>(sum[n2], Rows::column(keys, column_at, 32 * h + 16 * g, n2), w);
            }
        }
    }
    const bool bad = any_not_finite(sum) && last >= 0 && fabsf(lse2) < INFINITY &&
                     fabsf(delta) < INFINITY;
    uint64_t which = __ballot(bad);
    which = (which | which >> 32) & 0xffffffffu;
    while (which) {
        const int col = __builtin_ctzll(which);
        which &= which - 1;
        const int32_t to = __builtin_amdgcn_readlane(last, col);
        const int32_t from = __builtin_amdgcn_readlane(first, col);
        const float l2 = __shfl(lse2, col), dl = __shfl(delta, col);
        const Column cc(a, s, mine + col);
        const Spread qs = Spread::of(s.rows<T>(a.q, cc.head) + cc.i * a.q.row, a.dim, lane);
        const Spread ds = Spread::of(s.rows<T>(a.dout, cc.head) + cc.i * a.dout.row, a.dim, lane);
        Spread y = {0.0f, 0.0f};
        for (int32_t n = 0; n < walk.count && !settled(y, a.dim, lane); ++n) {
            const int32_t j0 = walk.tile(n) * kKeys;
            for (int32_t j = j0; j < j0 + kKeys && j <= to; ++j) {
                if (!sees(j, to, from, a.sinks))
                    continue;
                const Spread ks = Spread::of(kp + j * a.k.row, a.dim, lane);
                const Spread vs = Spread::of(vp + j * a.v.row, a.dim, lane);
                const PairOf w(a, qs, ds, ks, vs, l2, dl);
                y.x = fmaf(w.d, ks.x, y.x);
                y.y = fmaf(w.d, ks.y, y.y);
            }
        }
        y.x *= 1.0f / kCarried<T>;
        y.y *= 1.0f / kCarried<T>;
        set_column(sum, y, col, lane);
    }
    if (c.exists)
        write_row<T, N>((T *)s.rows<T>(a.dq, c.head) + c.i * a.dq.row, sum,
                        a.scale * kCarried<T>, last < 0, a.dim, lane);
}

// The queries that see any of keys j0 .. j1, and their columns.
struct KeySpan {
    int32_t begin, end;  // columns
    __device__ __forceinline__ KeySpan(const AttendArgs &a, const Sequence &s, int32_t j0,
                                       int32_t j1)
    {
        int32_t i0 = 0, i1 = s.q_length - 1;
        if (a.causal) {
            i0 = j0 - s.shift > 0 ? j0 - s.shift : 0;
            // position p sees down to p - window + 1 (a window is less than the keys)
            if (a.window && j0 >= a.sinks && j1 + a.window - 1 - s.shift < i1)
                i1 = j1 + a.window - 1 - s.shift;
        }
        const bool some = j0 < s.k_length && i0 <= i1;
        begin = some ? i0 * (int32_t)a.group.d : 0;
        end = some ? (i1 + 1) * (int32_t)a.group.d : 0;
    }
};

// A workgroup's keys and part of their columns. Tiles that hold sinks come first:
// all later queries see them, so they have most columns, and parts of their own
// size.
struct KeyTask {
    uint32_t pair, tile, part;
    bool whole;  // the only part
    int32_t begin, end;
    __device__ __forceinline__ KeyTask(const AttendArgs &a)
    {
        const uint32_t unit = divide(blockIdx.x, a.pair_div);
        pair = blockIdx.x - unit * a.pair_div.d;
        const uint32_t first = a.sink_tiles * a.sink_div.d;
        if (unit < first) {
            tile = divide(unit, a.sink_div);
            part = unit - tile * a.sink_div.d;
            whole = a.sink_div.d == 1;
        } else {
            const uint32_t n = divide(unit - first, a.tile_div);
            tile = a.sink_tiles + n;
            part = unit - first - n * a.tile_div.d;
            whole = a.tile_div.d == 1;
        }
    }
    __device__ __forceinline__ int32_t size(const AttendArgs &a) const
    {
        return tile < (uint32_t)a.sink_tiles ? a.sink_part : a.tile_part;
    }
};

// Gradients of keys and values: four waves of 32 keys each over shared tiles of
// 32 columns, the columns (queries and heads) that read these keys or a part of
// them. Keys stay in registers and values in LDS, which leaves room for two waves
// a SIMD.
template <typename T, int N>
__global__ void __launch_bounds__(64 * kAttendWaves, sizeof(T) == 2 ? 2 : 1)
    attend_grad_k_kernel(AttendArgs a)
{
    constexpr int kThreads = 64 * kAttendWaves, kCols = 32, kKeys = kAttendWaves * 32;
    typedef LdsRows<T, N> Rows;
    typedef typename Rows::Chunk Chunk;
    constexpr int kBytes = kCols * Rows::kStride;
    __shared__ __attribute__((aligned(512))) char lds[2][2 * kBytes];
    __shared__ __attribute__((aligned(512))) char values[kKeys * Rows::kStride];
    __shared__ __attribute__((aligned(16))) float lses[2][kCols], deltas[2][kCols];
    __shared__ __attribute__((aligned(16))) int32_t lasts[2][kCols], firsts[2][kCols];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const KeyTask task(a);
    const Sequence s(a, task.pair);
    const int32_t j0 = task.tile * kKeys, mine = j0 + wave * 32, j = mine + (lane & 31);
    const int32_t group = (int32_t)a.group.d, head0 = s.kv * group;
    const KeySpan span(a, s, j0, j0 + kKeys - 1);
    int32_t c_begin = span.begin, c_end = span.end;
    if (!task.whole) {
        const int32_t size = task.size(a);
        const int64_t from = (int64_t)c_begin + (int64_t)task.part * size;
        c_begin = from < c_end ? (int32_t)from : c_end;
        c_end = c_end - c_begin < size ? c_end : c_begin + size;
        if (c_begin >= c_end)
            return;  // the join knows that this part is empty
    }
    f32x16 dk[N], dv[N];
#pragma unroll
    for (int n = 0; n < N; ++n)
        dk[n] = dv[n] = (f32x16)0.0f;
    const T *kp = s.rows<T>(a.k, s.kv), *vp = s.rows<T>(a.v, s.kv);
    vec<T, 8> k[2 * N];
    if (c_begin < c_end) {
        row_operands<T, N>(kp + (j < a.keys ? j : a.keys - 1) * a.k.row, a.dim, lane, k);
        Mover<T, N, kKeys, kThreads> v(a.dim, threadIdx.x);
        v.fetch(vp, a.v.row, j0, s.k_length);
        v.put(values);
    }
    // what the thread moves: chunk m_c of rows m_r, m_r + kPass, ..., and of the
    // first 32 threads one column's numbers
    constexpr int kSlots = Mover<T, N, kKeys, kThreads>::kSlots, kPass = kThreads / kSlots;
    constexpr int kMoved = kPass < kCols ? kCols / kPass : 1;
    const int m_r = threadIdx.x / kSlots, m_c = threadIdx.x % kSlots;
    const bool m_some = m_c * Rows::kEach < a.dim && m_r < kCols;
    const T *qp = s.rows<T>(a.q, head0) + m_c * Rows::kEach;
    const T *dp = s.rows<T>(a.dout, head0) + m_c * Rows::kEach;
    const int64_t stat0 = (int64_t)s.b * a.queries * a.heads + head0;
    Chunk mq[kMoved], md[kMoved];
    float m_lse = 0.0f, m_delta = 0.0f;
    int32_t m_last = -1, m_first = 0;
    const auto fetch = [&](int32_t c0) {
#pragma unroll
        for (int n = 0; n < kMoved; ++n) {
            const int32_t c = c0 + m_r + n * kPass, i = (int32_t)divide(c, a.group);
            const int32_t g = c - i * group;
            mq[n] = md[n] = (Chunk)(T)0.0f;
            if (m_some && c < c_end) {
                mq[n] = load<T, Rows::kEach>(qp + (i * a.q.row + g * a.q.head));
                md[n] = load<T, Rows::kEach>(dp + (i * a.dout.row + g * a.dout.head));
            }
        }
        if (threadIdx.x < kCols) {
            const int32_t c = c0 + threadIdx.x, i = (int32_t)divide(c, a.group);
            m_last = c < c_end ? s.last(a, i) : -1;
            m_first = s.first(a, i);
            m_lse = m_delta = 0.0f;
            if (m_last >= 0) {
                const int64_t row = stat0 + (int64_t)i * a.heads + c - i * group;
                m_lse = a.lse[row] * kLog2e;
                m_delta = a.delta[row];
            }
        }
    };
    const auto put = [&](int buffer) {
        char *to = lds[buffer];
        if (m_c < Rows::kChunks && m_r < kCols)
#pragma unroll
            for (int n = 0; n < kMoved; ++n) {
                Rows::put(to, m_r + n * kPass, m_c, mq[n]);
                Rows::put(to + kBytes, m_r + n * kPass, m_c, md[n]);
            }
        if (threadIdx.x < kCols) {
            lses[buffer][threadIdx.x] = m_lse;
            deltas[buffer][threadIdx.x] = m_delta;
            lasts[buffer][threadIdx.x] = m_last;
            firsts[buffer][threadIdx.x] = m_first;
        }
    };
    if (c_begin < c_end)
        fetch(c_begin);
    const int row_at0 = Rows::row_at(lane), column_at0 = Rows::column_at(lane);
    int buffer = 0;
    for (int32_t c0 = c_begin; c0 < c_end; c0 += kCols, buffer ^= 1) {
        put(buffer);
        __syncthreads();  // a tile is written again two turns on
        if (c0 + kCols < c_end)
            fetch(c0 + kCols);
        // the wave's keys against the tile's first and last query
        const int32_t end = c0 + kCols < c_end ? c0 + kCols : c_end;
        const int32_t ia = (int32_t)divide(c0, a.group), ib = (int32_t)divide(end - 1, a.group);
        const int32_t mine1 = mine + 31;
        if (mine > s.last(a, ib) || (mine1 < s.first(a, ia) && mine >= a.sinks))
            continue;
        const bool whole = c0 + kCols <= c_end && mine1 <= s.last(a, ia) &&
                           (mine >= s.first(a, ib) || mine1 < a.sinks);
        const char *qs = lds[buffer], *dys = qs + kBytes;
        const int row_at = fresh(row_at0), column_at = fresh(column_at0);
        f32x16 x = (f32x16)0.0f, y = (f32x16)0.0f;
#pragma unroll
        for (int t = 0; t < 2 * N; ++t) {
            multiply<T>(x, Rows::row(qs, row_at, 0, t), k[t]);
            multiply<T>(y, Rows::row(dys, row_at, 0, t), Rows::row(values, row_at, wave * 32, t));
        }
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int r = 8 * g + 4 * (lane >> 5);
            const f32x4 l4 = *(const f32x4 *)&lses[buffer][r];
            const f32x4 d4 = *(const f32x4 *)&deltas[buffer][r];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float p = exp2_of(fmaf(x[4 * g + e], a.scale_log2, kCarry<T> - l4[e]));
                x[4 * g + e] = p;
                y[4 * g + e] = p * (y[4 * g + e] - d4[e]);
            }
            if (!whole) {
                typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
                const i32x4 last = *(const i32x4 *)&lasts[buffer][r];
                const i32x4 first = *(const i32x4 *)&firsts[buffer][r];
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (!sees(j, last[e], first[e], a.sinks))
                        x[4 * g + e] = y[4 * g + e] = 0.0f;
            }
        }
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            const vec<T, 8> p = operand<T>(x, g), d = operand<T>(y, g);
#pragma unroll
            for (int n = 0; n < N; ++n) {
                multiply<T>(dv[n], Rows::column(dys, column_at, 16 * g, n), p);
                multiply<T>(dk[n], Rows::column(qs, column_at, 16 * g, n), d);
            }
        }
    }
    const bool bad = (any_not_finite(dk) || any_not_finite(dv)) && j < s.k_length;
    uint64_t which = __ballot(bad);
    which = (which | which >> 32) & 0xffffffffu;
    while (which) {
        const int col = __builtin_ctzll(which);
        which &= which - 1;
        const int32_t key = mine + col;
        const Spread ks = Spread::of(kp + key * a.k.row, a.dim, lane);
        const Spread vs = Spread::of(vp + key * a.v.row, a.dim, lane);
        Spread gk = {0.0f, 0.0f}, gv = {0.0f, 0.0f};
        for (int32_t at = c_begin; at < c_end; ++at) {
            const Column c(a, s, at);
            if (!sees(key, s.last(a, c.i), s.first(a, c.i), a.sinks))
                continue;
            const int64_t row = ((int64_t)s.b * a.queries + c.i) * a.heads + c.head;
            const Spread qs = Spread::of(s.rows<T>(a.q, c.head) + c.i * a.q.row, a.dim, lane);
            const Spread ds =
                Spread::of(s.rows<T>(a.dout, c.head) + c.i * a.dout.row, a.dim, lane);
            const PairOf w(a, qs, ds, ks, vs, a.lse[row] * kLog2e, a.delta[row]);
            gk.x = fmaf(w.d, qs.x, gk.x);
            gk.y = fmaf(w.d, qs.y, gk.y);
            gv.x = fmaf(w.p, ds.x, gv.x);
            gv.y = fmaf(w.p, ds.y, gv.y);
            if (settled(gk, a.dim, lane) && settled(gv, a.dim, lane))
                break;
        }
        constexpr float up = 1.0f / kCarried<T>;
        set_column(dk, Spread{gk.x * up, gk.y * up}, col, lane);
        set_column(dv, Spread{gv.x * up, gv.y * up}, col, lane);
    }
    const bool none = j >= s.k_length;
    const float fk = a.scale * kCarried<T>, fv = kCarried<T>;
    if (!task.whole) {
        float *p = a.part + ((int64_t)blockIdx.x * 2 * kKeys + wave * 32 + (lane & 31)) * (N * 32);
        write_row<float, N>(p, dk, fk, none, N * 32, lane);
        write_row<float, N>(p + kKeys * (N * 32), dv, fv, none, N * 32, lane);
        return;
    }
    if (j >= a.keys)
        return;
    write_row<T, N>((T *)s.rows<T>(a.dk, s.kv) + j * a.dk.row, dk, fk, none, a.dim, lane);
    write_row<T, N>((T *)s.rows<T>(a.dv, s.kv) + j * a.dv.row, dv, fv, none, a.dim, lane);
}

// Joins the parts of the keys' gradients, in order: four keys a workgroup, four
// values a thread.
template <typename T, int N>
__global__ void __launch_bounds__(64 * kAttendWaves) attend_grad_join_kernel(AttendArgs a)
{
    constexpr int kKeys = kAttendWaves * 32, kFours = N * 8, kRows = kAttendJoinKeys;
    static_assert(kRows * kFours * 2 <= 64 * kAttendWaves, "a thread for each four values");
    const uint32_t unit = divide(blockIdx.x, a.pair_div);
    const uint32_t pair = blockIdx.x - unit * a.pair_div.d;
    const uint32_t tile = unit / (kKeys / kRows), row0 = unit % (kKeys / kRows) * kRows;
    const Sequence s(a, pair);
    const KeySpan span(a, s, tile * kKeys, tile * kKeys + kKeys - 1);
    const bool sink = tile < (uint32_t)a.sink_tiles;
    const int32_t size = sink ? a.sink_part : a.tile_part;
    const int32_t parts = (int32_t)(((int64_t)span.end - span.begin + size - 1) / size);
    // the first part's place among the workgroups' sums
    const int64_t first = sink ? (int64_t)tile * a.sink_div.d
                               : (int64_t)a.sink_tiles * a.sink_div.d +
                                     (int64_t)(tile - a.sink_tiles) * a.tile_div.d;
    const int matrix = threadIdx.x & 1, at = threadIdx.x >> 1;
    const int row = row0 + at / kFours, d = at % kFours * 4;
    const int32_t j = tile * kKeys + row;
    if (at >= kRows * kFours || j >= a.keys || d >= a.dim)
        return;
    const int64_t step = (int64_t)a.pairs * 2 * kKeys * (N * 32);
    const float *p = a.part + first * step +
                     (((int64_t)pair * 2 + matrix) * kKeys + row) * (N * 32) + d;
    f32x4 y = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
    for (int32_t k = 0; k < parts; ++k)
        y += *(const f32x4 *)(p + k * step);
    const HeadRows &to = matrix ? a.dv : a.dk;
    store<T, 4>((T *)s.rows<T>(to, s.kv) + j * to.row + d, from_f32<T, 4>(y));
}

template <typename T>
int launch_attend_grad(const AttendArgs &a, int kernel, int wide, unsigned grid, void *s)
{
    const auto with = [&](auto n) {
        constexpr int N = decltype(n)::value;
        const dim3 g(grid), b(64 * kAttendWaves);
        hipStream_t st = (hipStream_t)s;
        if (kernel == kAttendGradQ)
            hipLaunchKernelGGL((attend_grad_q_kernel<T, N>), g, b, 0, st, a);
        else if (kernel == kAttendGradK)
            hipLaunchKernelGGL((attend_grad_k_kernel<T, N>), g, b, 0, st, a);
        else
            hipLaunchKernelGGL((attend_grad_join_kernel<T, N>), g, b, 0, st, a);
    };
    if (wide == 1)
        with(std::integral_constant<int, 1>{});
    else if (wide == 2)
        with(std::integral_constant<int, 2>{});
    else if (wide == 3)
        with(std::integral_constant<int, 3>{});
    else
        with(std::integral_constant<int, 4>{});
    return (int)hipGetLastError();
}

}  // namespace
}  // namespace smol

#endif  // SMOL_ATTEND_GRAD_KERNELS_H
