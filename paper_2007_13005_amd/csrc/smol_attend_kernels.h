// smol_attend_kernels.h -- attention forward, as templates for one type
// (instantiated by smol_attend_<type>.hip).
//
// One pass over the keys with the running maximum m and sum l of a softmax in
// base 2: weights 2^(s - m) are rounded to the type and multiplied with the
// values in fp32; a maximum that grows scales what was summed before. m is a
// whole number and may stay up to 8 behind the maximum (weights up to 256), so
// most tiles scale nothing, and scaling sums rounds nothing.
//
// fp16 has few exponents: there m is 7 less, so weights are carried times 2^7 (up to
// 2^15), in l too. A weight below 2^-32 of the largest is then zero, so that n keys
// lose at most n 2^-32 of a row's weight (2^-25 without: a key of e^18 times the weight
// of each of 8192 others left them none of their 2^-13).
//
// What a query does not see takes no part: its score is set to minus infinity
// before the maximum. A weight of 0 times a NaN or an infinity among the values
// would still spoil the sums (of a tile that other queries see). So where a
// column's sums are not finite in the end, though its weights are, the waves that
// share its tiles sum once more, with zeros for such values in the products, and add
// the values themselves to the columns that see them.
#ifndef SMOL_ATTEND_KERNELS_H
#define SMOL_ATTEND_KERNELS_H

#include "smol_attend_device.h"

namespace smol {
namespace {

constexpr float kBehind = 8.0f;

// log2 of what weights are carried by.
template <typename T>
constexpr float kWeightCarry = std::is_same<T, f16>::value ? 7.0f : 0.0f;

// The same where sums are formed again, which may be because they neared fp32's end: the
// maximum is never behind and weights are 2^-24 at most, so that as many of them as
// there can be, times the largest value, stay within it (fp16's sums cannot pass it).
template <typename T>
constexpr float kCarefulCarry = std::is_same<T, f16>::value ? 7.0f : -24.0f;

// lse in base e, of a maximum m and sum l of weights. l of weights carried far down is
// taken up first, so that the logarithm's integer is added exactly.
__device__ __forceinline__ float lse_of(float m, float l)
{
    const bool down = l < 0x1p-6f;
    return ((down ? m - 24.0f : m) + __builtin_amdgcn_logf(down ? l * 0x1p24f : l)) * kLn2;
}

// One wave's 32 columns: scores, weights and sums.
template <typename T, int N>
struct Columns {
    vec<T, 8> q[2 * N];
    f32x16 sum[N];   // [values x columns]
    float m, l;      // l: of this half of the wave
    Sight sight;

    __device__ __forceinline__ void start(const AttendArgs &a, const Sequence &s, int32_t c0,
                                          int lane)
    {
        const Column c(a, s, c0 + (lane & 31));
        row_operands<T, N>(s.rows<T>(a.q, c.head) + c.i * a.q.row, a.dim, lane, q);
        sight.start(a, s, c0, c);
        clear();
    }
    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int n = 0; n < N; ++n)
            sum[n] = (f32x16)0.0f;
        m = kLowest;
        l = 0.0f;
    }
    // Scores x of 32 keys from j0 on (register rows): what is not seen leaves, and
    // the maximum follows. True (and f) where what was summed, and weights formed
    // before, are to be scaled by f. The maximum is kept as a whole number, so f is a
    // power of two and scaling rounds nothing but fp16 weights that come below 2^-14.
    template <bool Careful = false>
    __device__ __forceinline__ bool look(const AttendArgs &a, f32x16 &x, int32_t j0, int lane,
                                         float *f)
    {
        constexpr float carry = Careful ? kCarefulCarry<T> : kWeightCarry<T>;
        sight.hide<false>(a, x, j0, lane, -INFINITY);
        float top = -INFINITY;
#pragma unroll
        for (int e = 0; e < 16; ++e)
            top = fmaxf(top, x[e]);
        top = both_halves(top, [](float u, float v) { return fmaxf(u, v); }) * a.scale_log2;
        if (!__any(top > m + (Careful ? carry : kBehind + carry)))
            return false;
        const float to = fmaxf(m, ceilf(top) - carry);
        *f = exp2_of(m - to);
        m = to;
        l *= *f;
#pragma unroll
        for (int n = 0; n < N; ++n)
            sum[n] *= *f;
        return true;
    }
    // Weights of elements from .. to - 1.
    __device__ __forceinline__ void weigh(const AttendArgs &a, f32x16 &x, int from, int to)
    {
#pragma unroll
        for (int e = 0; e < 16; ++e)
            if (e >= from && e < to) {
                x[e] = here(exp2_of(fmaf(x[e], a.scale_log2, -m)));
                l += x[e];
            }
    }
    // Whether a column's sums alone are not finite, spoiled by what it does not see
    // perhaps, or past 2^112 and so perhaps not in what joins waves and parts (256 of
    // them): over the wave, the same in each lane.
    __device__ __forceinline__ bool spoiled() const
    {
        const float all = both_halves(l, [](float u, float v) { return u + v; });
        return __any(any_not_finite(sum, 0x1p16f) && fabsf(all) < INFINITY && sight.last >= 0);
    }
    // Scores, weights and sums of 32 keys from j0 on, whose values stand at `values` in
    // LDS; keys(k) gives the operands of their scores. What is not finite among the
    // values takes no part in the products, and is added where it is seen.
    template <typename Keys>
    __device__ __forceinline__ void carefully(const AttendArgs &a, Keys keys, const char *values,
                                              int32_t j0, int lane)
    {
        typedef LdsRows<T, N> Rows;
        lane = fresh(lane);  // (no address of these is kept through the loops)
        const int value_at = Rows::column_at(lane);
        f32x16 x = (f32x16)0.0f;
        float f;
#pragma unroll
        for (int k = 0; k < 2 * N; ++k)
            multiply<T>(x, keys(k), q[k]);
        in_order();
        look<true>(a, x, j0, lane, &f);
        weigh(a, x, 0, 16);
        in_order();
        bool some = false;
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            const vec<T, 8> w = operand<T>(x, g);
#pragma unroll
            for (int n = 0; n < N; ++n) {
                multiply<T>(sum[n], finite_of<T>(Rows::column(values, value_at, 16 * g, n), some),
                            w);
                in_order();
            }
        }
        if (some)
            add_not_finite<false, T, N>(sum, values, a.dim, sight.last >= 0, lane, [&](int r) {
                return sees(j0 + r, sight.last, sight.first, a.sinks);
            });
    }
    // Rows of out, rest and lse; or, of a part of the keys, sums, m and l.
    __device__ __forceinline__ void finish(const AttendArgs &a, const Sequence &s, int32_t c0,
                                           uint32_t pair, uint32_t split, int lane)
    {
        l = both_halves(l, [](float u, float v) { return u + v; });
        lane = fresh(lane);
        const int32_t at = c0 + (lane & 31);
        if (at >= a.columns)
            return;
        if (a.splits > 1) {
            const int64_t row = ((int64_t)split * a.pairs + pair) * a.columns + at;
            float *p = a.part + row * (N * 32);
#pragma unroll
            for (int n = 0; n < N; ++n)
#pragma unroll
                for (int g = 0; g < 4; ++g)
                    *(f32x4 *)(p + 32 * n + 8 * g + 4 * (lane >> 5)) =
                        f32x4{sum[n][4 * g], sum[n][4 * g + 1], sum[n][4 * g + 2],
                              sum[n][4 * g + 3]};
            if (lane < 32) {
                float *ml = a.part + (int64_t)a.splits * a.pairs * a.columns * (N * 32) + 2 * row;
                ml[0] = m;
                ml[1] = l;
            }
            return;
        }
        const Column c(a, s, at);
        T *out = (T *)s.rows<T>(a.out, c.head) + c.i * a.out.row;
        const int64_t row = ((int64_t)s.b * a.queries + c.i) * a.heads + c.head;
        write_row<T, N>(out, a.rest ? (T *)a.rest + row * a.dim : nullptr, sum, 1.0f / l,
                        sight.last < 0, a.dim, lane);
        if (a.lse && lane < 32)
            a.lse[row] = sight.last < 0 ? -INFINITY : lse_of(m, l);
    }
};

// Which work a workgroup has: a pair of a sequence and a key head (the fastest
// index: neighbours on a die's L2 share keys), a tile of columns, a part of the
// keys. Causal tiles run from the last, which has most keys.
struct Task {
    uint32_t pair, tile, split;
    __device__ __forceinline__ Task(const AttendArgs &a)
    {
        const Place at(a, blockIdx.x);
        pair = at.pair;
        split = divide(at.unit, a.tile_div);
        tile = at.unit - split * a.tile_div.d;
        if (a.causal)
            tile = a.tiles - 1 - tile;
    }
};

// Four waves of 32 columns each over shared tiles of 64 keys.
//
// Bound by the matrix instructions with the exponentials beside them: each 32 x 32
// scores need d / 8 instructions for both products, and 16 exponentials a lane. So a
// wave's tile of 64 keys is two halves, and one half's exponentials stand between the
// other's products; operands are read from LDS a few instructions ahead; the next
// tile is on its way to LDS while this one is used.
// 8192 tokens, 32 heads of 128 over 8, a window of 2048, bf16: 272 to 282 us by the card,
// 855 to 886 TFLOP/s of the scores that are seen (products alone 138, with the softmax
// 209, with LDS reads 233). Three buffers of tiles instead of two left too little LDS: 64
// images of 197 rows and 16 heads of 64 took 42 us for 38. Up to 64 values a head four
// waves a SIMD fit (these images 38 -> 36 us, and 33 since pairs come in chunks).
template <typename T, int N>
__global__ void __launch_bounds__(64 * kAttendWaves, sizeof(T) == 4 ? 1 : N <= 2 ? 4 : 2)
    attend_kernel(AttendArgs a)
{
    constexpr int kKeys = kAttendKeys;
    typedef LdsRows<T, N> Rows;
    constexpr int kBytes = kKeys * Rows::kStride;
    __shared__ __attribute__((aligned(512))) char lds[2][2 * kBytes];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Task task(a);
    const Sequence s(a, task.pair);
    const int32_t c0 = task.tile * (kAttendWaves * 32), mine = c0 + wave * 32;
    const Column c_first(a, s, c0), c_last(a, s, c0 + kAttendWaves * 32 - 1);
    const Walk<kKeys> walk(a, s, c_first.i, c_last.i);
    const int32_t lo = (int32_t)divide(walk.count * task.split, a.split_div);
    const int32_t hi = (int32_t)divide(walk.count * (task.split + 1), a.split_div);
    Columns<T, N> cols;
    cols.start(a, s, mine, lane);
    const T *kp = s.rows<T>(a.k, s.kv), *vp = s.rows<T>(a.v, s.kv);
    typedef RowMover<T, N, kKeys, kAttendWaves> Moves;
    const Moves k_moves(a.k.row, a.dim, wave, lane), v_moves(a.v.row, a.dim, wave, lane);
    const auto fetch = [&](int32_t n) {
        const int32_t j0 = walk.tile(n) * kKeys;
        char *to = lds[(n - lo) & 1];
        k_moves.fetch(kp, a.k.row, a.direct_keys, a.dim, to, wave, lane, j0, s.k_length);
        v_moves.fetch(vp, a.v.row, a.direct_keys, a.dim, to + kBytes, wave, lane, j0, s.k_length);
    };
    if (lo < hi)
        fetch(lo);
    const int key_at0 = Rows::row_at(lane), value_at0 = Rows::column_at(lane);
    for (int32_t n = lo; n < hi; ++n) {
        // tile n is there, for all waves; the other buffer's tile has been used by all
        loads_done();
        __syncthreads();
        if (n + 1 < hi)
            fetch(n + 1);
        const int32_t j0 = walk.tile(n) * kKeys;
        if (!cols.sight.any(a, j0, j0 + kKeys - 1))
            continue;
        const int key_at = fresh(key_at0 + (n - lo & 1) * (2 * kBytes));
        const int value_at = fresh(value_at0 + (n - lo & 1) * (2 * kBytes) + kBytes);
        if (!cols.sight.any(a, j0 + 32, j0 + kKeys - 1)) {
            // the tile's first 32 keys alone (the last of 197 keys: 5 of them)
            f32x16 x = (f32x16)0.0f;
            float f;
#pragma unroll
            for (int k = 0; k < 2 * N; ++k)
                multiply<T>(x, Rows::row(lds[0], key_at, 0, k), cols.q[k]);
            cols.look(a, x, j0, lane, &f);
            cols.weigh(a, x, 0, 16);
#pragma unroll
            for (int k = 0; k < 2 * N; ++k)
                multiply<T>(cols.sum[k % N], Rows::column(lds[0], value_at, k / N * 16, k % N),
                            operand<T>(x, k / N));
            continue;
        }
        // operands in the order of their products, kAhead read before they are used:
        // scores of the first 32 keys, of the second, values with the first 32 keys'
        // weights, with the second's
        constexpr int kAhead = 4, kHalf = 2 * N;
        vec<T, 8> ahead[kAhead];
        const auto read = [&](int k) {
            if (k < 2 * kHalf)
                ahead[k % kAhead] = Rows::row(lds[0], key_at, k / kHalf * 32, k % kHalf);
            else if (k < 4 * kHalf)
                ahead[k % kAhead] =
                    Rows::column(lds[0], value_at, (k - 2 * kHalf) / N * 16, (k - 2 * kHalf) % N);
        };
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
            read(k);
        in_order();
        f32x16 x[2] = {(f32x16)0.0f, (f32x16)0.0f};
        vec<T, 8> w[4];
        float f;
#pragma unroll
        for (int k = 0; k < kHalf; ++k) {
            multiply<T>(x[0], ahead[k % kAhead], cols.q[k]);
            read(k + kAhead);
            in_order();
        }
        cols.look(a, x[0], j0, lane, &f);
        // from here on products and exponentials take turns, so that both units work
#pragma unroll
        for (int k = 0; k < kHalf; ++k) {
            multiply<T>(x[1], ahead[(kHalf + k) % kAhead], cols.q[k]);
            read(kHalf + k + kAhead);
            cols.weigh(a, x[0], 16 * k / kHalf, 16 * (k + 1) / kHalf);
            in_order();
        }
        w[0] = operand<T>(x[0], 0);
        w[1] = operand<T>(x[0], 1);
        if (cols.look(a, x[1], j0 + 32, lane, &f)) {
            w[0] = from_f32<T, 8>(to_f32<8, T>(w[0]) * f);
            w[1] = from_f32<T, 8>(to_f32<8, T>(w[1]) * f);
        }
#pragma unroll
        for (int k = 0; k < kHalf; ++k) {
            multiply<T>(cols.sum[k % N], ahead[(2 * kHalf + k) % kAhead], w[k / N]);
            read(2 * kHalf + k + kAhead);
            cols.weigh(a, x[1], 16 * k / kHalf, 16 * (k + 1) / kHalf);
            in_order();
        }
        w[2] = operand<T>(x[1], 0);
        w[3] = operand<T>(x[1], 1);
#pragma unroll
        for (int k = 0; k < kHalf; ++k) {
            multiply<T>(cols.sum[k % N], ahead[(3 * kHalf + k) % kAhead], w[2 + k / N]);
            read(3 * kHalf + k + kAhead);
            in_order();
        }
    }
    const AttendArgs &late = args_again();
    // What there is is written before the waves tell each other, so that none waits with
    // it (gradients of 2 x 148 rows: 19.6 us if it does, 18.7), and once more if need be.
    // Told in the buffer that the last tile is not in: four bytes of LDS more than two
    // buffers, 64 KB for heads of 128, cost a tenth (4096 tokens, 16 heads of 128 over
    // 4, bf16, 98 us -> 110).
    for (bool again = false;; again = true) {
        const bool spoiled = cols.spoiled();
        cols.finish(late, s, mine, task.pair, task.split, lane);
        if (again || !any_wave((int *)lds[(hi - lo) & 1], spoiled, wave, lane))
            return;
        __syncthreads();  // before tiles take its place
        cols.clear();
        fetch(lo);
#pragma unroll 1
        for (int32_t n = lo; n < hi; ++n) {
            loads_done();
            __syncthreads();
            if (n + 1 < hi)
                fetch(n + 1);
            const char *tile = lds[(n - lo) & 1];
            const int32_t j0 = walk.tile(n) * kKeys;
#pragma unroll 1
            for (int h = 0; h < 2; ++h)
                if (cols.sight.any(late, j0 + 32 * h, j0 + 32 * h + 31))
                    cols.carefully(
                        late,
                        [&](int k) {
                            return Rows::row(tile, Rows::row_at(fresh(lane)), 32 * h, k);
                        },
                        tile + kBytes + 32 * h * Rows::kStride, j0 + 32 * h, lane);
        }
    }
}

// 32 columns a workgroup: its four waves take tiles of 32 keys in turn, each
// with its own piece of LDS and no barrier, and join their sums at the end.
//
// For single tokens: bound by reading the cache. Keys go from memory to the
// registers of their product, values through LDS, both a tile ahead: one token over
// 32768 keys of 8 heads of 128 in fp16, 134 MB, 26 us and the join's 3 (5.1 TB/s;
// the kernel above, whose other waves would have no column, takes the same there and
// twice as long in fp32: 4 tokens over 3000 keys 83 us for 42).
template <typename T, int N>
__global__ void __launch_bounds__(64 * kAttendWaves, sizeof(T) == 2 ? 2 : 1)
    attend_few_kernel(AttendArgs a)
{
    constexpr int kKeys = kAttendFewKeys;
    typedef LdsRows<T, N> Rows;
    constexpr int kBytes = kKeys * Rows::kStride;
    static_assert(kAttendWaves * 2 * kBytes >= 2 * 64 * N * 16 * 4, "room for two waves' sums");
    __shared__ __attribute__((aligned(512))) char lds[kAttendWaves * 2 * kBytes];
    __shared__ float tops[kAttendWaves][32], sums[kAttendWaves][32];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Task task(a);
    const Sequence s(a, task.pair);
    const int32_t c0 = task.tile * 32;
    const Column c_first(a, s, c0), c_last(a, s, c0 + 31);
    const Walk<kKeys> walk(a, s, c_first.i, c_last.i);
    const int32_t lo = (int32_t)divide(walk.count * task.split, a.split_div);
    const int32_t hi = (int32_t)divide(walk.count * (task.split + 1), a.split_div);
    Columns<T, N> cols;
    cols.start(a, s, c0, lane);
    const T *kp = s.rows<T>(a.k, s.kv), *vp = s.rows<T>(a.v, s.kv);
    char *values = lds + wave * (2 * kBytes);
    vec<T, 8> k[2 * N];
    const RowMover<T, N, kKeys, 1> moves(a.v.row, a.dim, 0, lane);
    // (the keys' registers are asked for first: they are used first)
    const auto fetch = [&](int32_t n, int buffer) {
        const int32_t j0 = walk.tile(n) * kKeys, j = j0 + (lane & 31);
        row_operands<T, N>(kp + (j < s.k_length ? j : s.k_length - 1) * a.k.row, a.dim, lane, k);
        moves.fetch(vp, a.v.row, a.direct_keys, a.dim, values + buffer * kBytes, 0, lane, j0,
                    s.k_length);
    };
    const int32_t own = lo + wave;
    if (own < hi)
        fetch(own, 0);
    const int value_at0 = Rows::column_at(lane);
    int buffer = 0;
    for (int32_t n = own; n < hi; n += kAttendWaves, buffer ^= 1) {
        const int32_t j0 = walk.tile(n) * kKeys;
        const int value_at = fresh(value_at0 + buffer * kBytes);
        f32x16 x[1] = {(f32x16)0.0f};
#pragma unroll
        for (int t = 0; t < 2 * N; ++t)
            multiply<T>(x[0], k[t], cols.q[t]);
        loads_done();
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // reads of the other buffer
        if (n + kAttendWaves < hi)
            fetch(n + kAttendWaves, buffer ^ 1);
        float f;
        cols.look(a, x[0], j0, lane, &f);
        cols.weigh(a, x[0], 0, 16);
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            const vec<T, 8> w = operand<T>(x[0], g);
#pragma unroll
            for (int n2 = 0; n2 < N; ++n2)
                multiply<T>(cols.sum[n2], Rows::column(values, value_at, 16 * g, n2), w);
        }
    }
    const AttendArgs &late = args_again();
    if (cols.spoiled()) {
        cols.clear();
        fetch(own, 0);
#pragma unroll 1
        for (int32_t n = own; n < hi; n += kAttendWaves) {
            loads_done();
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            cols.carefully(late, [&](int t) { return k[t]; }, values, walk.tile(n) * kKeys, lane);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // before the tile is replaced
            if (n + kAttendWaves < hi)
                fetch(n + kAttendWaves, 0);
        }
    }
    loads_done();
    // the waves' sums at one maximum, then waves 2 and 3 into 0 and 1, 1 into 0:
    // of those that had a tile
    const int32_t busy = hi - lo;
    const float half = both_halves(cols.l, [](float u, float v) { return u + v; });
    if (lane < 32) {
        tops[wave][lane] = cols.m;
        sums[wave][lane] = half;
    }
    __syncthreads();
    float top = tops[0][lane & 31], total = 0.0f;
#pragma unroll
    for (int w = 1; w < kAttendWaves; ++w)
        top = fmaxf(top, tops[w][lane & 31]);
#pragma unroll
    for (int w = 0; w < kAttendWaves; ++w)
        total += sums[w][lane & 31] * exp2_of(tops[w][lane & 31] - top);
    const float f = exp2_of(cols.m - top);
#pragma unroll
    for (int n = 0; n < N; ++n)
        cols.sum[n] *= f;
    cols.m = top;
    float *room = (float *)lds;
#pragma unroll
    for (int step = 2; step >= 1; step >>= 1) {
        if (busy <= step)
            continue;
        if (wave >= step && wave < 2 * step)
#pragma unroll
            for (int n = 0; n < N; ++n)
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    room[((wave - step) * N * 16 + n * 16 + e) * 64 + lane] = cols.sum[n][e];
        __syncthreads();
        if (wave < step)
#pragma unroll
            for (int n = 0; n < N; ++n)
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    cols.sum[n][e] += room[(wave * N * 16 + n * 16 + e) * 64 + lane];
        __syncthreads();
    }
    if (wave != 0)
        return;
    cols.l = lane < 32 ? total : 0.0f;  // finish adds the halves
    cols.finish(late, s, c0, task.pair, task.split, lane);
}

// Joins the parts of the keys: a wave a column, all its parts' loads at once; past
// 16 parts a workgroup a column, each wave a quarter of the parts in order, then
// the four waves' sums in order.
template <typename T, int N>
__global__ void __launch_bounds__(64 * kAttendWaves) attend_join_kernel(AttendArgs a)
{
    constexpr int kParts = kAttendJoinParts;
    static_assert(kAttendSplits <= kParts * kAttendWaves, "parts that the waves hold");
    __shared__ Spread quarter[kAttendWaves][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const bool alone = a.splits <= kParts;
    const uint32_t at = alone ? blockIdx.x * kAttendWaves + wave : blockIdx.x;
    const uint32_t rows = (uint32_t)a.pairs * (uint32_t)a.columns;  // of a part
    if (at >= rows)
        return;
    const uint32_t pair = at / (uint32_t)a.columns;
    const Sequence s(a, pair);
    const Column c(a, s, (int32_t)(at - pair * (uint32_t)a.columns));
    const int per = alone ? a.splits : (a.splits + kAttendWaves - 1) / kAttendWaves;
    const int first = alone ? 0 : wave * per;
    const float *p = a.part + ((int64_t)first * rows + at) * (N * 32);
    Spread x[kParts];
#pragma unroll
    for (int k = 0; k < kParts; ++k) {
        const bool own = k < per && first + k < a.splits;
        const float *from = p + (int64_t)k * rows * (N * 32);
        x[k].x = own && lane < N * 32 ? from[lane] : 0.0f;
        x[k].y = own && lane + 64 < N * 32 ? from[lane + 64] : 0.0f;
    }
    const float *ml = a.part + (int64_t)a.splits * rows * (N * 32) + 2 * (int64_t)at;
    const bool own = lane < a.splits;  // splits <= 64
    const float m = own ? ml[2 * (int64_t)lane * rows] : kLowest;
    const float l = own ? ml[2 * (int64_t)lane * rows + 1] : 0.0f;
    float top = m;
#pragma unroll
    for (int step = 32; step; step >>= 1)
        top = fmaxf(top, __shfl_xor(top, step));
    const float f = exp2_of(m - top);
    const float total = wave_sum(l * f);
    Spread y = {0.0f, 0.0f};
#pragma unroll
    for (int k = 0; k < kParts; ++k)
        if (k < per) {
            const float w = __shfl(f, (first + k) & 63);
            y.x = fmaf(w, x[k].x, y.x);
            y.y = fmaf(w, x[k].y, y.y);
        }
    if (!alone) {
        quarter[wave][lane] = y;
        __syncthreads();
        if (wave != 0)
            return;
#pragma unroll
        for (int w = 1; w < kAttendWaves; ++w) {
            y.x += quarter[w][lane].x;
            y.y += quarter[w][lane].y;
        }
    }
    const bool none = s.last(a, c.i) < 0;
    const float inv = 1.0f / total;
    T *out = (T *)s.rows<T>(a.out, c.head) + c.i * a.out.row;
    const int64_t row = ((int64_t)s.b * a.queries + c.i) * a.heads + c.head;
    const auto write = [&](int32_t d, float v) {
        if (d >= a.dim)
            return;
        v = none ? 0.0f : v * inv;
        const T z = (T)v;
        out[d] = z;
        if (a.rest)
            ((T *)a.rest)[row * a.dim + d] = (T)(v - (float)z);
    };
    write(lane, y.x);
    if (N > 2)
        write(lane + 64, y.y);
    if (a.lse && lane == 0)
        a.lse[row] = none ? -INFINITY : lse_of(top, total);
}

template <typename T>
int launch_attend(const AttendArgs &a, int kernel, int wide, unsigned grid, void *s)
{
    const auto with = [&](auto n) {
        constexpr int N = decltype(n)::value;
        const dim3 g(grid), b(64 * kAttendWaves);
        hipStream_t st = (hipStream_t)s;
        if (kernel == kAttendMany)
            hipLaunchKernelGGL((attend_kernel<T, N>), g, b, 0, st, a);
        else if (kernel == kAttendFew)
            hipLaunchKernelGGL((attend_few_kernel<T, N>), g, b, 0, st, a);
        else
            hipLaunchKernelGGL((attend_join_kernel<T, N>), g, b, 0, st, a);
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

#endif  // SMOL_ATTEND_KERNELS_H
