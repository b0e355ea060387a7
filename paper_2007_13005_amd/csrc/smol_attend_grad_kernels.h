// smol_attend_grad_kernels.h -- attention's gradients, as templates for one type
// (instantiated by smol_attend_grad_<type>.hip).
//
// With p = exp(s - lse) formed again from the forward pass's lse and D =
// grad_out . (out + rest) a row, d = p (grad_out v^T - D):
//   grad_q = scale d k,  grad_k = scale d^T q,  grad_v = p^T grad_out.
// After a small kernel that forms D, one launch whose workgroups take either 128
// columns (products s, grad_out v^T, d k) or 128 keys (s, grad_out v^T,
// p^T grad_out, d^T q), each with its sums in registers and no atomics. s and
// grad_out v^T are formed twice: seven products for the five that are needed, but no
// sums in memory (those of the columns would be written and read once for every
// 128 keys). In two launches, each waiting for the other's last workgroups, 4 ragged
// sequences of 4096 rows, 16 heads of 128 over 4, a window of 1024, bf16, took 428
// us for 401, 5906 rows of 8 heads of 96 350 for 290.
//
// p and d are rounded to the type as operands. fp16 has few exponents: there
// both are carried times 2^6 (a weight of 2^-20 is then still a normal number).
//
// What a query does not see has a score of minus infinity, so p and d are zero.
// Where it holds a NaN or an infinity they may not be, and d past 2^10 overflows as
// carried. So a workgroup some of whose sums are not finite in the end, though lse
// and D are, forms them once more: with zeros for p and d of pairs that are not seen
// and for what is not finite in the products' other operands, which is added where it
// is seen; and with d carried by less where it grows past fp16, as a running maximum
// would. 2048 rows, 16 heads of 128 over 4, causal, fp16: 146 us, with a NaN in a query
// 210, with d past 2^10 everywhere 375.
#ifndef SMOL_ATTEND_GRAD_KERNELS_H
#define SMOL_ATTEND_GRAD_KERNELS_H

#include "smol_attend_device.h"

namespace smol {
namespace {

template <typename T>
constexpr float kCarry = std::is_same<T, f16>::value ? 6.0f : 0.0f;  // log2

template <typename T>
constexpr float kCarried = std::is_same<T, f16>::value ? 1.0f / 64.0f : 1.0f;

// fp16: by what the lane's d are carried beside p's 2^6, a power of two so that the
// largest of them stays below 2^15. Sums change with it.
template <typename T, int N>
__device__ __forceinline__ void carry_less(f32x16 &d, f32x16 (&sum)[N], float &carry)
{
    if constexpr (std::is_same<T, f16>::value) {
        float top = 0.0f;
#pragma unroll
        for (int e = 0; e < 16; ++e)
            top = fmaxf(top, fabsf(d[e]));
        top = both_halves(top, [](float u, float v) { return fmaxf(u, v); });
        if (__any(top * carry >= 0x1p15f && top < INFINITY)) {
            // top is below 2^exponent, at least half of it
            const float to = top < INFINITY
                                 ? fminf(carry, ldexpf(1.0f, 15 - __builtin_amdgcn_frexp_expf(top)))
                                 : carry;
            const float f = to / carry;
            carry = to;
#pragma unroll
            for (int n = 0; n < N; ++n)
                sum[n] *= f;
        }
        d *= carry;
    }
}

// D of every row of queries that exists, beside its lse (which may lie at strides of
// its own): a group of lanes a row, eight values a lane. Bound by memory (the ragged
// sequences above: 138 MB in 31 us).
template <typename T, int N>
__global__ void __launch_bounds__(64 * kAttendWaves) attend_delta_kernel(AttendArgs a)
{
    constexpr int kLanes = attend_delta_lanes(N);
    const int32_t d = threadIdx.x % kLanes * 8;
    for (uint32_t block = blockIdx.x; block < a.delta_groups; block += gridDim.x) {
        const uint32_t r = block * (64 * kAttendWaves / kLanes) + threadIdx.x / kLanes;
        const uint32_t row = divide(r, a.heads_div), b = divide(row, a.queries_div);
        const int32_t head = r - row * a.heads_div.d, i = row - b * a.queries_div.d;
        const bool some = b < a.batch;
        const bool exists = some && (!a.q_lengths || i < a.q_lengths[b]);
        float delta = 0.0f;
        if (exists && d < a.dim) {
            const auto at = [&](const HeadRows &m) {
                return (const T *)m.p + b * m.batch + i * m.row + head * m.head + d;
            };
            vec<float, 8> y = to_f32<8, T>(load<T, 8>(at(a.out)));
            const vec<float, 8> dy = to_f32<8, T>(load<T, 8>(at(a.dout)));
            if (a.rest_in.p)
                y += to_f32<8, T>(load<T, 8>(at(a.rest_in)));
#pragma unroll
            for (int e = 0; e < 8; ++e)
                delta = fmaf(dy[e], y[e], delta);
        }
#pragma unroll
        for (int step = 1; step < kLanes; step <<= 1)
            delta += __shfl_xor(delta, step);
        if (some && d == 0 && exists) {
            const float lse = *((const float *)a.lse_in.p + b * a.lse_in.batch +
                                i * a.lse_in.row + head * a.lse_in.head);
            *((float2 *)a.lse_delta + r) = make_float2(lse * kLog2e, delta);
        }
    }
}

// A row's lse in base 2, and its D.
__device__ __forceinline__ float2 lse_delta(const AttendArgs &a, int64_t row)
{
    return *((const float2 *)a.lse_delta + row);
}

// Gradients of queries: four waves of 32 columns over shared tiles of 64 keys. Both
// halves' scores and grad_out v^T come before the first half's d k, so that the
// exponentials and differences of one stand between the products of the other.
template <typename T, int N>
struct GradQ {
    static constexpr int kKeys = kAttendKeys;
    typedef LdsRows<T, N> Rows;
    static constexpr int kBytes = kKeys * Rows::kStride;
    static constexpr int kLds = 4 * kBytes;
    static __device__ __forceinline__ void run(const AttendArgs &a, uint32_t pair, uint32_t turn,
                                               char *lds);
};

template <typename T, int N>
__device__ __forceinline__ void GradQ<T, N>::run(const AttendArgs &a, uint32_t pair, uint32_t turn,
                                                 char *lds)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t tile = a.causal ? a.tiles - 1 - turn : turn;
    const Sequence s(a, pair);
    const int32_t c0 = tile * (kAttendWaves * 32), mine = c0 + wave * 32;
    const Column c_first(a, s, c0), c_last(a, s, c0 + kAttendWaves * 32 - 1);
    const Walk<kKeys> walk(a, s, c_first.i, c_last.i);
    const Column c(a, s, mine + (lane & 31));
    const int64_t at = ((int64_t)s.b * a.queries + c.i) * a.heads + c.head;
    Sight sight;
    sight.start(a, s, mine, c);
    vec<T, 8> q[2 * N], dy[2 * N];
    const T *qp = s.rows<T>(a.q, c.head) + c.i * a.q.row;
    const T *dyp = s.rows<T>(a.dout, c.head) + c.i * a.dout.row;
    row_operands<T, N>(qp, a.dim, lane, q);
    row_operands<T, N>(dyp, a.dim, lane, dy);
    const float2 stat = sight.last < 0 ? make_float2(0.0f, 0.0f) : lse_delta(a, at);
    const float minus_lse = kCarry<T> - stat.x, delta = stat.y;
    f32x16 sum[N];
#pragma unroll
    for (int n = 0; n < N; ++n)
        sum[n] = (f32x16)0.0f;
    const T *kp = s.rows<T>(a.k, s.kv), *vp = s.rows<T>(a.v, s.kv);
    typedef RowMover<T, N, kKeys, kAttendWaves> Moves;
    const Moves k_moves(a.k.row, a.dim, wave, lane), v_moves(a.v.row, a.dim, wave, lane);
    const auto fetch = [&](int32_t n) {
        const int32_t j0 = walk.tile(n) * kKeys;
        char *to = lds + (n & 1) * (2 * kBytes);
        k_moves.fetch(kp, a.k.row, a.direct_keys, a.dim, to, wave, lane, j0, s.k_length);
        v_moves.fetch(vp, a.v.row, a.direct_keys, a.dim, to + kBytes, wave, lane, j0, s.k_length);
    };
    if (walk.count)
        fetch(0);
    const int row_at0 = Rows::row_at(lane), column_at0 = Rows::column_at(lane);
    for (int32_t n = 0; n < walk.count; ++n) {
        // tile n is there, for all waves; the other buffer's tile has been used by all
        loads_done();
        __syncthreads();
        if (n + 1 < walk.count)
            fetch(n + 1);
        const int32_t j0 = walk.tile(n) * kKeys;
        if (!sight.any(a, j0, j0 + kKeys - 1))
            continue;
        const int at_keys = (n & 1) * (2 * kBytes);
        const int row_at = fresh(row_at0 + at_keys), column_at = fresh(column_at0 + at_keys);
        // operands in the order of their products, kAhead read before they are used;
        // of each 32 keys: scores, grad_out v^T, then (after the second 32 keys') d k
        constexpr int kAhead = 4, kHalf = 2 * N;
        vec<T, 8> ahead[kAhead];
        const auto read = [&](int k) {
            const int part = k / kHalf, t = k % kHalf;
            if (part < 4)
                ahead[k % kAhead] =
                    Rows::row(lds + (part & 1) * kBytes, row_at, (part >> 1) * 32, t);
            else if (part < 6)
                ahead[k % kAhead] =
                    Rows::column(lds, column_at, (part - 4) * 32 + t / N * 16, t % N);
        };
        // scores start from minus infinity where a key is not seen, which leaves
        // weights of zero
        f32x16 x[2] = {(f32x16)0.0f, (f32x16)0.0f}, y[2] = {(f32x16)0.0f, (f32x16)0.0f};
        vec<T, 8> d[4];
#pragma unroll
        for (int h = 0; h < 2; ++h)
            sight.hide<true>(a, x[h], j0 + 32 * h, lane, -INFINITY);
        const auto weigh = [&](int h, int k) {
#pragma unroll
            for (int e = 16 * k / kHalf; e < 16 * (k + 1) / kHalf; ++e)
                x[h][e] = here(exp2_of(fmaf(x[h][e], a.scale_log2, minus_lse)));
        };
        const auto differ = [&](int h, int k) {
#pragma unroll
            for (int e = 16 * k / kHalf; e < 16 * (k + 1) / kHalf; ++e)
                x[h][e] = here(x[h][e] * (y[h][e] - delta));
        };
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
            read(k);
        in_order();
#pragma unroll
        for (int part = 0; part < 6; ++part) {
#pragma unroll
            for (int k = 0; k < kHalf; ++k) {
                const vec<T, 8> next = ahead[(part * kHalf + k) % kAhead];
                if (part == 0 || part == 2)
                    multiply<T>(x[part >> 1], next, q[k]);
                else if (part < 4)
                    multiply<T>(y[part >> 1], next, dy[k]);
                else
                    multiply<T>(sum[k % N], next, d[2 * (part - 4) + k / N]);
                read(part * kHalf + k + kAhead);
                if (part == 1 || part == 3)
                    weigh(part >> 1, k);
                else if (part == 2 || part == 4)
                    differ((part >> 1) - 1, k);
                in_order();
            }
            if (part == 2 || part == 4) {
                d[part - 2] = operand<T>(x[(part >> 1) - 1], 0);
                d[part - 1] = operand<T>(x[(part >> 1) - 1], 1);
            }
        }
    }
    // written, and formed and written once more if need be (as in
    // smol_attend_kernels.h)
    float carry = 1.0f;
    const bool bad = any_not_finite(sum) && sight.last >= 0 && fabsf(minus_lse) < INFINITY &&
                     fabsf(delta) < INFINITY;
    const auto write = [&](const AttendArgs &late) {
        if (c.exists)
            write_row<T, N>((T *)s.rows<T>(late.dq, c.head) + c.i * late.dq.row, nullptr, sum,
                            late.scale * kCarried<T> / carry, sight.last < 0, late.dim, lane);
    };
    write(args_again());
    // (told in the buffer that the last tile is not in)
    if (!any_wave((int *)(lds + (walk.count & 1) * (2 * kBytes)), __any(bad), wave, lane))
        return;
    const AttendArgs &late = args_again();
    __syncthreads();  // before tiles take its place
#pragma unroll
    for (int n = 0; n < N; ++n)
        sum[n] = (f32x16)0.0f;
    fetch(0);
#pragma unroll 1
    for (int32_t n = 0; n < walk.count; ++n) {
        loads_done();
        __syncthreads();
        if (n + 1 < walk.count)
            fetch(n + 1);
        const int l = fresh(lane), row_at = Rows::row_at(l), column_at = Rows::column_at(l);
#pragma unroll 1
        for (int h = 0; h < 2; ++h) {
            const int32_t j0 = walk.tile(n) * kKeys + 32 * h;
            if (!sight.any(late, j0, j0 + 31))
                continue;
            const char *keys = lds + (n & 1) * (2 * kBytes) + 32 * h * Rows::kStride;
            f32x16 x = (f32x16)0.0f, y = (f32x16)0.0f;
#pragma unroll
            for (int k = 0; k < 2 * N; ++k) {
                multiply<T>(x, Rows::row(keys, row_at, 0, k), q[k]);
                multiply<T>(y, Rows::row(keys + kBytes, row_at, 0, k), dy[k]);
                in_order();
            }
#pragma unroll
            for (int e = 0; e < 16; ++e)
                x[e] = exp2_of(fmaf(x[e], late.scale_log2, minus_lse)) * (y[e] - delta);
            sight.hide<true>(late, x, j0, l, 0.0f);
            carry_less<T, N>(x, sum, carry);
            in_order();
            bool some = false;
#pragma unroll
            for (int g = 0; g < 2; ++g) {
                const vec<T, 8> d = operand<T>(x, g);
#pragma unroll
                for (int k = 0; k < N; ++k) {
                    multiply<T>(
                        sum[k], finite_of<T>(Rows::column(keys, column_at, 16 * g, k), some),
                        d);
                    in_order();
                }
            }
            // a key that is not finite: its weight is zero, or lse is not finite
            if (some)
                add_not_finite<true, T, N>(sum, keys, late.dim, sight.last >= 0, l, [&](int r) {
                    return sees(j0 + r, sight.last, sight.first, late.sinks);
                });
        }
    }
    write(args_again());
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
    uint32_t tile, part;
    __device__ __forceinline__ KeyTask(const AttendArgs &a, uint32_t unit)
    {
        const uint32_t first = a.sink_tiles * a.sink_div.d;
        if (unit < first) {
            tile = divide(unit, a.sink_div);
            part = unit - tile * a.sink_div.d;
        } else {
            const uint32_t n = divide(unit - first, a.tile_div);
            tile = a.sink_tiles + n;
            part = unit - first - n * a.tile_div.d;
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
// a SIMD. Of 241 us by itself for the sequences above, 25 are waits for tiles, 12 for
// the barrier, 19 for LDS reads.
template <typename T, int N>
struct GradK {
    static constexpr int kCols = 32, kKeys = kAttendWaves * 32;
    typedef LdsRows<T, N> Rows;
    static constexpr int kBytes = kCols * Rows::kStride;
    // one column's numbers, of two tiles
    struct Stats {
        float lses[2][kCols], deltas[2][kCols];
        int32_t lasts[2][kCols], firsts[2][kCols];
    };
    static constexpr int kValues = 4 * kBytes, kStats = kValues + kKeys * Rows::kStride;
    static constexpr int kLds = kStats + sizeof(Stats);
    static __device__ __forceinline__ void run(const AttendArgs &a, uint32_t pair, uint32_t unit,
                                               char *lds);
};

template <typename T, int N>
__device__ __forceinline__ void GradK<T, N>::run(const AttendArgs &a, uint32_t pair, uint32_t unit,
                                                 char *lds)
{
    char *values = lds + kValues;
    Stats &stats = *(Stats *)(lds + kStats);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const KeyTask task(a, unit);
    const Sequence s(a, pair);
    const int32_t j0 = task.tile * kKeys, mine = j0 + wave * 32, j = mine + (lane & 31);
    const int32_t group = (int32_t)a.group.d, head0 = s.kv * group;
    const KeySpan span(a, s, j0, j0 + kKeys - 1);
    int32_t c_begin = span.begin, c_end = span.end;
    const int32_t size = task.size(a);
    const bool whole = c_end - c_begin <= size;  // one part, which may be empty
    if (task.part) {
        const int64_t from = (int64_t)c_begin + (int64_t)task.part * size;
        if (from >= c_end)
            return;  // the join knows that there is no such part
        c_begin = (int32_t)from;
    }
    c_end = c_end - c_begin < size ? c_end : c_begin + size;
    f32x16 dk[N], dv[N];
#pragma unroll
    for (int n = 0; n < N; ++n)
        dk[n] = dv[n] = (f32x16)0.0f;
    const T *kp = s.rows<T>(a.k, s.kv), *vp = s.rows<T>(a.v, s.kv);
    vec<T, 8> k_rows[2 * N];
    if (c_begin < c_end) {
        row_operands<T, N>(kp + (j < a.keys ? j : a.keys - 1) * a.k.row, a.dim, lane,
                           k_rows);
        RowMover<T, N, kKeys, kAttendWaves>(a.v.row, a.dim, wave, lane)
            .fetch(vp, a.v.row, a.direct_keys, a.dim, values, wave, lane, j0, s.k_length);
    }
    const T *qp = s.rows<T>(a.q, head0), *dp = s.rows<T>(a.dout, head0);
    const int64_t stat0 = (int64_t)s.b * a.queries * a.heads + head0;
    // of the first 32 lanes one column's numbers
    float m_lse = 0.0f, m_delta = 0.0f;
    int32_t m_last = -1, m_first = 0;
    // offsets of the thread's chunks from the tile's first query: the same for all
    // tiles where these begin with whole queries
    typedef Share<T, N, kCols, kAttendWaves> Mine;
    const bool whole_queries = kCols % group == 0;
    uint32_t q_offset[Mine::kCount], d_offset[Mine::kCount];
    const auto place = [&](int32_t c0) {
        const int32_t i0 = (int32_t)divide(c0, a.group);
#pragma unroll
        for (int n = 0; n < Mine::kCount; ++n) {
            const int32_t c = c0 + Mine::row(n, wave, lane), i = (int32_t)divide(c, a.group);
            const uint32_t at = Mine::at(n, wave, lane), g = c - i * group;
            const bool some = at < (uint32_t)a.dim;
            q_offset[n] = some ? ((uint32_t)(i - i0) * (uint32_t)a.q.row + g * (uint32_t)a.q.head +
                                  at) * (uint32_t)sizeof(T)
                               : kNoChunk;
            d_offset[n] = some ? ((uint32_t)(i - i0) * (uint32_t)a.dout.row +
                                  g * (uint32_t)a.dout.head + at) * (uint32_t)sizeof(T)
                               : kNoChunk;
        }
    };
    const auto fetch = [&](int32_t c0, int buffer) {
        char *to = lds + buffer * (2 * kBytes);
        if (a.direct_rows) {
            const int32_t i0 = (int32_t)divide(c0, a.group);
            if (!whole_queries)
                place(c0);
#pragma unroll
            for (int n = 0; n < Mine::kCount; ++n) {
                const bool some = c0 + Mine::row(n, wave, lane) < c_end;
                if (!Mine::has(n, wave))
                    break;
                load_to_lds(qp + i0 * a.q.row, 0x80000000u, some ? q_offset[n] : kNoChunk,
                            to + Mine::first(n, wave) * 16);
                load_to_lds(dp + i0 * a.dout.row, 0x80000000u, some ? d_offset[n] : kNoChunk,
                            to + kBytes + Mine::first(n, wave) * 16);
            }
        } else {
            const int l = fresh(lane);
#pragma unroll
            for (int n = 0; n < Mine::kCount; ++n) {
                if (!Mine::has(n, wave))
                    break;
                typedef typename Rows::Chunk Chunk;
                const int32_t c = c0 + Mine::row(n, wave, l), i = (int32_t)divide(c, a.group);
                const int32_t g = c - i * group, at = Mine::at(n, wave, l);
                Chunk v = (Chunk)(T)0.0f, w = v;
                if (c < c_end && at < a.dim) {
                    v = load<T, Rows::kEach>(qp + i * a.q.row + g * a.q.head + at);
                    w = load<T, Rows::kEach>(dp + i * a.dout.row + g * a.dout.head + at);
                }
                char *here = to + (Mine::first(n, wave) + l) * 16;
                *(Chunk *)here = v;
                *(Chunk *)(here + kBytes) = w;
            }
        }
        if (wave == 0 && lane < kCols) {
            const int32_t c = c0 + fresh(lane), i = (int32_t)divide(c, a.group);
            m_last = c < c_end ? s.last(a, i) : -1;
            m_first = s.first(a, i);
            m_lse = m_delta = 0.0f;  // what the scores' and the products' sums start from
            if (m_last >= 0) {
                const int64_t row = stat0 + (int64_t)i * a.heads + c - i * group;
                const float2 stat = lse_delta(a, row);
                m_lse = (kCarry<T> - stat.x) * a.per_scale_log2;
                m_delta = -stat.y;
            }
        }
    };
    const auto tell = [&](int buffer) {
        if (wave == 0 && lane < kCols) {
            stats.lses[buffer][lane] = m_lse;
            stats.deltas[buffer][lane] = m_delta;
            stats.lasts[buffer][lane] = m_last;
            stats.firsts[buffer][lane] = m_first;
        }
    };
    if (c_begin < c_end) {
        place(c_begin);
        fetch(c_begin, 0);
    }
    const int row_at0 = Rows::row_at(lane), column_at0 = Rows::column_at(lane);
    int buffer = 0;
    for (int32_t c0 = c_begin; c0 < c_end; c0 += kCols, buffer ^= 1) {
        tell(buffer);
        // the tile is there, for all waves; the other buffer's tile has been used by all
        loads_done();
        __syncthreads();
        if (c0 + kCols < c_end)
            fetch(c0 + kCols, buffer ^ 1);
        // the wave's keys (those that exist) against the tile's first and last query;
        // columns past the last are zeros
        const int32_t end = c0 + kCols < c_end ? c0 + kCols : c_end;
        const int32_t ia = (int32_t)divide(c0, a.group), ib = (int32_t)divide(end - 1, a.group);
        const int32_t mine1 = mine + 31 < s.k_length ? mine + 31 : s.k_length - 1;
        if (mine > s.last(a, ib) || (mine1 < s.first(a, ia) && mine >= a.sinks))
            continue;
        const bool whole =
            mine1 <= s.last(a, ia) && (mine >= s.first(a, ib) || mine1 < a.sinks);
        const int row_at = fresh(row_at0 + buffer * (2 * kBytes));
        const int column_at = fresh(column_at0 + buffer * (2 * kBytes));
        const int value_at = fresh(row_at0 + wave * (32 * Rows::kStride));
        // products take turns with what is made of the scores, operands read kAhead
        // before they are used: scores; grad_out v^T beside the weights p; p^T grad_out
        // beside d; d^T q. The sums start from minus lse and minus D; where a key is not
        // seen from minus infinity, which leaves weights of zero.
        constexpr int kAhead = 3, kHalf = 2 * N;
        vec<T, 8> ahead[kAhead], ahead_v[2];
        const auto read = [&](int k) {
            const int part = k / kHalf, t = k % kHalf;
            if (part < 2)
                ahead[k % kAhead] = Rows::row(lds + part * kBytes, row_at, 0, t);
            else if (part < 4)
                ahead[k % kAhead] = Rows::column(lds + (3 - part) * kBytes, column_at,
                                                 t / N * 16, t % N);
        };
        const auto read_v = [&](int t) {
            if (t < kHalf)
                ahead_v[t % 2] = Rows::row(values, value_at, 0, t);
        };
        f32x16 x, y;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int r = 8 * g + 4 * (lane >> 5);
            const f32x4 l4 = *(const f32x4 *)&stats.lses[buffer][r];
            const f32x4 d4 = *(const f32x4 *)&stats.deltas[buffer][r];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                x[4 * g + e] = l4[e];
                y[4 * g + e] = d4[e];
            }
            if (!whole) {
                typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
                const i32x4 last = *(const i32x4 *)&stats.lasts[buffer][r];
                const i32x4 first = *(const i32x4 *)&stats.firsts[buffer][r];
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    x[4 * g + e] = sees(j, last[e], first[e], a.sinks) ? x[4 * g + e] : -INFINITY;
            }
        }
        vec<T, 8> p[2], d[2];
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
            read(k);
        in_order();
#pragma unroll
        for (int part = 0; part < 4; ++part) {
#pragma unroll
            for (int k = 0; k < kHalf; ++k) {
                const vec<T, 8> next = ahead[(part * kHalf + k) % kAhead];
                if (part == 0)
                    multiply<T>(x, next, k_rows[k]);
                else if (part == 1)
                    multiply<T>(y, next, ahead_v[k % 2]);
                else if (part == 2)
                    multiply<T>(dv[k % N], next, p[k / N]);
                else
                    multiply<T>(dk[k % N], next, d[k / N]);
                read(part * kHalf + k + kAhead);
                if (part == 1)
                    read_v(k + 2);
#pragma unroll
                for (int e = 16 * k / kHalf; e < 16 * (k + 1) / kHalf; ++e) {
                    if (part == 1)
                        x[e] = here(exp2_of(x[e] * a.scale_log2));
                    else if (part == 2)
                        y[e] = here(x[e] * y[e]);
                }
                in_order();
            }
            if (part == 0) {
                read_v(0);
                read_v(1);
            }
            if (part == 1) {
                p[0] = operand<T>(x, 0);
                p[1] = operand<T>(x, 1);
            } else if (part == 2) {
                d[0] = operand<T>(y, 0);
                d[1] = operand<T>(y, 1);
            }
        }
    }
    // written, and formed and written once more if need be
    float carry = 1.0f;
    const bool none = j >= s.k_length;
    const bool bad = (any_not_finite(dk) || any_not_finite(dv)) && !none;
    const auto write = [&](const AttendArgs &late) {
        const int l = fresh(lane);
        const int32_t j1 = fresh(j);
        const float fk = late.scale * kCarried<T> / carry, fv = kCarried<T>;
        if (!whole) {
            const Place at(late, blockIdx.x);
            const int64_t place = (int64_t)at.unit * late.pairs + at.pair;
            float *p = late.part + (place * 2 * kKeys + wave * 32 + (l & 31)) * (N * 32);
            write_row<float, N>(p, nullptr, dk, fk, none, N * 32, l);
            write_row<float, N>(p + kKeys * (N * 32), nullptr, dv, fv, none, N * 32, l);
        } else if (j1 < late.keys) {
            write_row<T, N>((T *)s.rows<T>(late.dk, s.kv) + j1 * late.dk.row, nullptr, dk, fk,
                            none, late.dim, l);
            write_row<T, N>((T *)s.rows<T>(late.dv, s.kv) + j1 * late.dv.row, nullptr, dv, fv,
                            none, late.dim, l);
        }
    };
    write(args_again());
    // (told in the buffer that the last tile is not in)
    if (!any_wave((int *)(lds + buffer * (2 * kBytes)), __any(bad), wave, lane))
        return;
    const AttendArgs &late = args_again();
    __syncthreads();  // before tiles take its place
#pragma unroll
    for (int n = 0; n < N; ++n)
        dk[n] = dv[n] = (f32x16)0.0f;
    fetch(c_begin, 0);
    buffer = 0;
#pragma unroll 1
    for (int32_t c0 = c_begin; c0 < c_end; c0 += kCols, buffer ^= 1) {
        tell(buffer);
        loads_done();
        __syncthreads();
        if (c0 + kCols < c_end)
            fetch(c0 + kCols, buffer ^ 1);
        const int32_t end = c0 + kCols < c_end ? c0 + kCols : c_end;
        if (mine > s.last(late, (int32_t)divide(end - 1, late.group)))
            continue;
        const int l = fresh(lane), row_at = Rows::row_at(l), column_at = Rows::column_at(l);
        const char *rows = lds + buffer * (2 * kBytes), *grads = rows + kBytes;
        f32x16 x, y;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const int r = 8 * (e >> 2) + 4 * (l >> 5) + (e & 3);
            x[e] = stats.lses[buffer][r];
            y[e] = stats.deltas[buffer][r];
        }
#pragma unroll
        for (int k = 0; k < 2 * N; ++k) {
            multiply<T>(x, Rows::row(rows, row_at, 0, k), k_rows[k]);
            multiply<T>(y, Rows::row(grads, row_at, 0, k),
                        Rows::row(values, row_at + wave * (32 * Rows::kStride), 0, k));
            in_order();
        }
        const auto seen = [&](int r) {
            return sees(j, stats.lasts[buffer][r], stats.firsts[buffer][r], late.sinks);
        };
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const bool some = seen(8 * (e >> 2) + 4 * (l >> 5) + (e & 3));
            x[e] = some ? exp2_of(x[e] * late.scale_log2) : 0.0f;
            y[e] = some ? x[e] * y[e] : 0.0f;
        }
        carry_less<T, N>(y, dk, carry);
        in_order();
        bool some_grads = false, some_rows = false;
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            const vec<T, 8> p = operand<T>(x, g), d = operand<T>(y, g);
#pragma unroll
            for (int k = 0; k < N; ++k) {
                const vec<T, 8> of_grads = Rows::column(grads, column_at, 16 * g, k);
                const vec<T, 8> of_rows = Rows::column(rows, column_at, 16 * g, k);
                multiply<T>(dv[k], finite_of<T>(of_grads, some_grads), p);
                multiply<T>(dk[k], finite_of<T>(of_rows, some_rows), d);
                in_order();
            }
        }
        // (a query that is not finite has no finite weight)
        if (some_grads)
            add_not_finite<false, T, N>(dv, grads, late.dim, j < s.k_length, l, seen);
        if (some_rows)
            add_not_finite<true, T, N>(dk, rows, late.dim, j < s.k_length, l, seen);
    }
    write(args_again());
}

// Workgroups of keys, then those of queries, which are shorter: either's last run
// beside the other's (queries first: 431 us for 397). Bound by the matrix
// instructions and what they wait for: the ragged sequences take 377 us, seven
// products at a library's rate would take 208. 64 images of 197 rows of 12
// heads of 64 in fp16, 74 us: 197 rows fill 77 % of two tiles of 128. (Either reads the
// arguments for itself: read for both at the start they do not fit the registers.)
template <typename T, int N>
__global__ void __launch_bounds__(64 * kAttendWaves, sizeof(T) == 2 ? 2 : 1)
    attend_grad_kernel(AttendArgs a)
{
    typedef GradK<T, N> Keys;
    typedef GradQ<T, N> Queries;
    __shared__ __attribute__((aligned(
        512))) char lds[Keys::kLds > Queries::kLds ? Keys::kLds : Queries::kLds];
    const Place at(a, blockIdx.x);
    if (at.unit < a.key_units)
        Keys::run(a, at.pair, at.unit, lds);
    else
        Queries::run(args_again(), at.pair, at.unit - a.key_units, lds);
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
    if (parts <= 1)
        return;  // written whole
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
        if (kernel == kAttendDelta)
            hipLaunchKernelGGL((attend_delta_kernel<T, N>), g, b, 0, st, a);
        else if (kernel == kAttendGrad)
            hipLaunchKernelGGL((attend_grad_kernel<T, N>), g, b, 0, st, a);
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
