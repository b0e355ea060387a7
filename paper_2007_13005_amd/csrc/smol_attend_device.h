// smol_attend_device.h -- what the attention kernels share: operands of the
// matrix instructions and their tiles in LDS, which keys a query sees, and the
// walk over the tiles that have any.
//
// Columns. The `group` query heads that read one key head are taken together:
// column c of a sequence and key head is query c / group and the group's head
// c % group, so single tokens of grouped heads fill a tile's columns, and keys
// are read once for all of them.
//
// Operands. All products are 32 x 32 x 16 (fp32: eight of 32 x 32 x 2). A lane
// holds eight values of the summed index for one row of an operand (lane %
// 32); which values is free as long as both operands agree. Lane l of a result
// has column l % 32 and, in register 4 g + r, row 8 g + 4 (l / 32) + r. So with
// scores formed as (keys x columns), a lane's eight registers 8 s .. 8 s + 7 hold
// keys 16 s + {0 .. 3, 8 .. 11} + 4 (l / 32) of its own column: the second
// operand of the next product, as they are, if its first operand takes the
// keys in that order. Row statistics are sums over a lane's registers and one
// exchange with the other half of the wave.
#ifndef SMOL_ATTEND_DEVICE_H
#define SMOL_ATTEND_DEVICE_H

#include <hip/hip_runtime.h>
#include <math.h>

#include <type_traits>

#include "smol_attend.h"

namespace smol {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr float kLowest = -3.0e38f;  // below every finite maximum of scores
constexpr float kLn2 = 0.693147180559945309f;
constexpr float kLog2e = 1.44269504088896341f;

__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }

template <typename T>
__device__ __forceinline__ void multiply(f32x16 &sum, vec<T, 8> a, vec<T, 8> b)
{
    if constexpr (std::is_same<T, f16>::value)
        sum = __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, sum, 0, 0, 0);
    else if constexpr (std::is_same<T, bf16>::value)
        sum = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, sum, 0, 0, 0);
    else
#pragma unroll
        for (int e = 0; e < 8; ++e)
            sum = __builtin_amdgcn_mfma_f32_32x32x2f32(a[e], b[e], sum, 0, 0, 0);
}

// Eight neighbouring registers of a result as an operand.
template <typename T>
__device__ __forceinline__ vec<T, 8> operand(const f32x16 &x, int s)
{
    vec<float, 8> v;
#pragma unroll
    for (int e = 0; e < 8; ++e)
        v[e] = x[8 * s + e];
    return from_f32<T, 8>(v);
}

// x of both halves of the wave joined by f.
template <typename F>
__device__ __forceinline__ float both_halves(float x, F f)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, x),
                                                    __builtin_bit_cast(uint32_t, x), false, false);
    return f(__builtin_bit_cast(float, (uint32_t)r[0]), __builtin_bit_cast(float, (uint32_t)r[1]));
}

// x as if it were new: what is computed from it is not kept over a loop's turns
// (a dozen addresses would take the registers of operands).
__device__ __forceinline__ int fresh(int x)
{
    asm volatile("" : "+v"(x));
    return x;
}

// The same for a value that the wave shares.
__device__ __forceinline__ int64_t fresh_scalar(int64_t x)
{
    asm volatile("" : "+s"(x));
    return x;
}

// The kernel's arguments (its only parameter) read again: those that its end alone
// needs would else take scalar registers through its loop.
__device__ __forceinline__ const AttendArgs &args_again()
{
    auto p = (const __attribute__((address_space(4))) AttendArgs *)
        __builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(p));
    return *(const AttendArgs *)p;
}

// Nothing moves past this: the compiler keeps the order that is written.
__device__ __forceinline__ void in_order() { __builtin_amdgcn_sched_barrier(0); }

// x is formed here and not where it is first used.
__device__ __forceinline__ float here(float x)
{
    asm volatile("" : "+v"(x));
    return x;
}

// Rows of N * 32 values in LDS, one after the other, in chunks of 16 bytes whose
// places within a row are turned by the row (an exclusive or), so that both kinds
// of reads spread over the 256 bytes of the banks: a row operand's 16 neighbouring
// lanes read one chunk of 16 rows; a transposing read takes 64 bytes of four rows.
// (Padding alone, 16 or 32 bytes a row, left a quarter to a half of the LDS cycles
// to conflicts.) Tiles begin at a multiple of 512 bytes.
template <typename T, int N>
struct LdsRows {
    static constexpr int kStride = N * 32 * (int)sizeof(T);
    static constexpr int kChunks = kStride / 16;
    static constexpr int kEach = 16 / (int)sizeof(T);
    // the bytes within a row that turn: all of 256, of half a bank line, of 64
    static constexpr int kTurned = kStride % 256 == 0 ? 0xf0 : kStride % 128 == 0 ? 0x70 : 0x30;
    typedef vec<T, kEach> Chunk;

    static __device__ __forceinline__ int turn(int row)
    {
        const int high = kTurned == 0xf0 ? (row & 3) << 2 : kTurned == 0x70 ? (row & 2) << 1 : 0;
        return high | (row >> 2 & 3);
    }
    static __device__ __forceinline__ int place(int row, int chunk)
    {
        return row * kStride + ((chunk ^ turn(row)) << 4);
    }
    // `bytes` further in a row
    static __device__ __forceinline__ int along(int at, int bytes)
    {
        return (at ^ (bytes & kTurned)) + (bytes & ~kTurned);
    }
    // Row operand: of row row0 + lane % 32, values 16 t + 8 (lane / 32) .. + 7; row0
    // a multiple of 32.
    static __device__ __forceinline__ int row_at(int lane)
    {
        return place(lane & 31, (lane >> 5) * 8 * (int)sizeof(T) / 16);
    }
    static __device__ __forceinline__ vec<T, 8> row(const char *tile, int at, int row0, int t)
    {
        const int p = along(at, t * 16 * (int)sizeof(T));
        tile += row0 * kStride;
        if constexpr (sizeof(T) == 2) {
            return *(const vec<T, 8> *)(tile + p);
        } else {
            const f32x4 a = *(const f32x4 *)(tile + p), b = *(const f32x4 *)(tile + (p ^ 16));
            return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
        }
    }
    // Column operand: of column 32 n + lane % 32, rows row0 + {0 .. 3, 8 .. 11} +
    // 4 (lane / 32); row0 a multiple of 16.
    static __device__ __forceinline__ int column_at(int lane)
    {
        const int row = (lane >> 5) * 4;
        if (sizeof(T) == 4)
            return place(row, (lane & 31) >> 2) + (lane & 3) * 4;
        return place(row + ((lane & 15) >> 2), (lane >> 4 & 1) * 2 + (lane >> 1 & 1)) +
               (lane & 1) * 8;
    }
    static __device__ __forceinline__ vec<T, 8> column(const char *tile, int at, int row0, int n)
    {
        const int p = along(at, n * 32 * (int)sizeof(T));
        // eight rows further the turn's second bit is the other
        const int q = p ^ 32;
        tile += row0 * kStride;
        const char *further = tile + 8 * kStride;
        if constexpr (sizeof(T) == 2) {
            // 16 lanes give the places of four rows by 16 columns and get a column each
            typedef short s16x4 __attribute__((ext_vector_type(4)));
            typedef __attribute__((address_space(3))) s16x4 Shared;
            const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Shared *)(tile + p));
            const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Shared *)(further + q));
            return __builtin_bit_cast(vec<T, 8>,
                                      __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
        } else {
            vec<T, 8> v;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int step = turn(e) << 4;  // e < 4
                v[e] = *(const float *)(tile + e * kStride + (p ^ step));
                v[e + 4] = *(const float *)(further + e * kStride + (q ^ step));
            }
            return v;
        }
    }
};

// A sequence and one of its key heads.
struct Sequence {
    int32_t b, kv, q_length, k_length, shift;  // query i stands at shift + i
    __device__ __forceinline__ Sequence(const AttendArgs &a, uint32_t pair)
    {
        b = (int32_t)divide(pair, a.kv_heads);
        kv = (int32_t)(pair - b * a.kv_heads.d);
        // (the same in all lanes, which the compiler need not see through args_again)
        q_length = __builtin_amdgcn_readfirstlane(a.q_lengths ? a.q_lengths[b] : a.queries);
        k_length = __builtin_amdgcn_readfirstlane(a.k_lengths ? a.k_lengths[b] : a.keys);
        q_length = q_length < 0 ? 0 : q_length < a.queries ? q_length : a.queries;
        k_length = k_length < 0 ? 0 : k_length < a.keys ? k_length : a.keys;
        shift = k_length - q_length;
    }
    // The last and first key that query i sees, sinks aside; last < 0: none.
    __device__ __forceinline__ int32_t last(const AttendArgs &a, int32_t i) const
    {
        return i >= q_length ? -1 : a.causal ? shift + i : k_length - 1;
    }
    __device__ __forceinline__ int32_t first(const AttendArgs &a, int32_t i) const
    {
        const int32_t lo = a.window ? shift + i - a.window + 1 : 0;
        return lo > 0 ? lo : 0;
    }
    template <typename T>
    __device__ __forceinline__ const T *rows(const HeadRows &m, int32_t head) const
    {
        return (const T *)m.p + b * m.batch + head * m.head;
    }
};

// A workgroup's sequence and key head (a pair), and which of the pair's workgroups it
// is. Pairs come in chunks whose workgroups run at the same time, so that what a
// pair's share is read from memory once; within a chunk all pairs' first workgroups
// come first, those of a pair a multiple of 8 apart and so on one XCD with one L2.
struct Place {
    uint32_t pair, unit;
    __device__ __forceinline__ Place(const AttendArgs &a, uint32_t block)
    {
        const uint32_t n = divide(block, a.chunk_groups), p0 = n * a.chunk.d;
        block -= n * a.chunk_groups.d;
        const bool whole = p0 + a.chunk.d <= (uint32_t)a.pairs;
        const Divisor pairs = {whole ? a.chunk.d : a.chunk_last.d,
                               whole ? a.chunk.m : a.chunk_last.m,
                               whole ? a.chunk.s : a.chunk_last.s};
        unit = divide(block, pairs);
        pair = p0 + block - unit * pairs.d;
    }
};

__device__ __forceinline__ bool sees(int32_t j, int32_t last, int32_t first, int32_t sinks)
{
    return j <= last && (j >= first || j < sinks);
}

// Column c's query and head. c past the last: the last.
struct Column {
    int32_t i, head;
    bool exists;
    __device__ __forceinline__ Column(const AttendArgs &a, const Sequence &s, int32_t c)
    {
        exists = c < a.columns;
        c = exists ? c : a.columns - 1;
        i = (int32_t)divide((uint32_t)c, a.group);
        head = s.kv * (int32_t)a.group.d + c - i * (int32_t)a.group.d;
    }
};

// What 32 columns from c0 on see, as a wave has to know it for a tile of keys.
// Columns that do not exist, or see nothing, count for neither: whatever comes of
// them is not kept.
struct Sight {
    int32_t last, first;  // of the lane's column
    int32_t last_min, last_max, first_min, first_max;  // over the columns
    __device__ __forceinline__ void start(const AttendArgs &a, const Sequence &s, int32_t c0,
                                          const Column &c)
    {
        last = c.exists ? s.last(a, c.i) : -1;
        first = s.first(a, c.i);
        const Column lo(a, s, c0), hi(a, s, c0 + 31);
        const int32_t end = hi.i < s.q_length ? hi.i : s.q_length - 1;
        last_max = lo.i < s.q_length ? s.last(a, end) : -1;
        last_min = s.last(a, lo.i) > 0 ? s.last(a, lo.i) : 0;
        first_min = s.first(a, lo.i);
        first_max = s.first(a, end);
    }
    // Whether any column sees a key of j0 .. j1.
    __device__ __forceinline__ bool any(const AttendArgs &a, int32_t j0, int32_t j1) const
    {
        return j0 <= last_max && (j1 >= first_min || j0 < a.sinks);
    }
    // x[e] for keys j0 + 8 (e / 4) + 4 (lane / 32) + e % 4, e = 0 .. 15: `hidden` where the
    // lane's column does not see the key. Ends: tiles that no column's first key cuts
    // get code of their own, a third of the instructions (gradients of 64 images of 197
    // rows 84 -> 81 us; the forward pass has no registers for it).
    template <bool Ends>
    __device__ __forceinline__ void hide(const AttendArgs &a, f32x16 &x, int32_t j0, int lane,
                                         float hidden) const
    {
        const bool end = j0 + 31 > last_min, begin = j0 < first_max && j0 + 31 >= a.sinks;
        if (!end && !begin)
            return;
        const int32_t base = fresh(j0 + 4 * (lane >> 5));
        const int32_t to = last - base, from = begin ? first - base : -64, sinks = a.sinks - base;
        if (Ends && !begin) {
#pragma unroll
            for (int e = 0; e < 16; ++e)
                x[e] = 8 * (e >> 2) + (e & 3) <= to ? x[e] : hidden;
            return;
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const int32_t j = 8 * (e >> 2) + (e & 3);
            x[e] = j <= to && (j >= from || j < sinks) ? x[e] : hidden;
        }
    }
};

// The tiles of `Keys` keys that any of queries i0 .. i1 sees: those of the first
// keys (sinks), then a run.
template <int Keys>
struct Walk {
    int32_t head, from, count;
    __device__ __forceinline__ Walk(const AttendArgs &a, const Sequence &s, int32_t i0, int32_t i1)
    {
        i1 = i1 < s.q_length ? i1 : s.q_length - 1;
        const int32_t last = i0 <= i1 ? s.last(a, i1) : -1;
        head = from = count = 0;
        if (last < 0)
            return;
        from = s.first(a, i0) / Keys;
        const int32_t sinks = (a.sinks + Keys - 1) / Keys;
        head = sinks < from ? sinks : from;
        count = head + last / Keys - from + 1;
    }
    __device__ __forceinline__ int32_t tile(int32_t n) const
    {
        return n < head ? n : n - head + from;
    }
};

// Eight values from 16 t + 8 (lane / 32) on of the lane's row, zeros past the head.
template <typename T, int N>
__device__ __forceinline__ void row_operands(const T *row, int32_t dim, int lane,
                                             vec<T, 8> (&v)[2 * N])
{
#pragma unroll
    for (int t = 0; t < 2 * N; ++t) {
        const int32_t d = 16 * t + 8 * (lane >> 5);
        v[t] = load<T, 8>(row + (d < dim ? d : 0));
        if (d >= dim)
            v[t] = (vec<T, 8>)(T)0.0f;
    }
}

// Moves one chunk a lane from base + offset to `to` + 16 * lane in LDS, without
// registers between; zeros where it would pass `bytes` (kNoChunk always does).
// Complete after loads_done and a barrier.
constexpr uint32_t kNoChunk = ~15u;
__device__ __forceinline__ void load_to_lds(const void *base, uint32_t bytes, uint32_t offset,
                                            const char *to)
{
    typedef __attribute__((address_space(3))) void Shared;
    const auto buffer = __builtin_amdgcn_make_buffer_rsrc((void *)base, 0, bytes, 0x00027000);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(buffer, (Shared *)to, 16, offset, 0, 0, 0);
}
__device__ __forceinline__ void loads_done() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// Which chunks of a tile in LDS a lane of `Waves` waves moves: chunk n of its own
// comes from value at(n) of row row(n).
template <typename T, int N, int Rows, int Waves>
struct Share {
    typedef LdsRows<T, N> Layout;
    static constexpr int kTotal = Rows * Layout::kChunks;
    static constexpr int kCount = (kTotal + 64 * Waves - 1) / (64 * Waves);
    static_assert(kTotal % 64 == 0, "whole waves");
    static __device__ __forceinline__ int first(int n, int wave) { return (n * Waves + wave) * 64; }
    static __device__ __forceinline__ bool has(int n, int wave)
    {
        return kTotal % (64 * Waves) == 0 || first(n, wave) < kTotal;
    }
    static __device__ __forceinline__ int row(int n, int wave, int lane)
    {
        return (first(n, wave) + lane) / Layout::kChunks;
    }
    static __device__ __forceinline__ int at(int n, int wave, int lane)
    {
        const int chunk = (first(n, wave) + lane) % Layout::kChunks;
        return (chunk ^ Layout::turn(row(n, wave, lane))) * Layout::kEach;
    }
};

// Rows of keys or values, a stride apart, on their way to tiles in LDS. direct
// (see near_rows in smol_attend.hip): aligned to 16 bytes, no row within another,
// a tile within 2^31 bytes; else they go through registers, and the wave waits
// (queries, keys and values that start an element late: 8192 tokens, 32 heads of 128
// over 8, a window of 2048, 515 us for 298, one token over 32768 keys 66 for 29).
// Offsets within a tile are formed once. Where 64 * Waves chunks are rows that all
// turn alike, one offset serves all of a lane's chunks.
template <typename T, int N, int Rows, int Waves>
struct RowMover {
    typedef Share<T, N, Rows, Waves> Mine;
    typedef LdsRows<T, N> Layout;
    static constexpr bool kAlike = 64 * Waves % (16 * Layout::kChunks) == 0;
    static constexpr int kStep = kAlike ? 64 * Waves / Layout::kChunks : 0;
    uint32_t offset[kAlike ? 1 : Mine::kCount];
    __device__ __forceinline__ RowMover(int64_t stride, int32_t dim, int wave, int lane)
    {
#pragma unroll
        for (int n = 0; n < (kAlike ? 1 : Mine::kCount); ++n) {
            const int at = Mine::at(n, wave, lane);
            offset[n] = at < dim ? ((uint32_t)Mine::row(n, wave, lane) * (uint32_t)stride + at) *
                                       (uint32_t)sizeof(T)
                                 : kNoChunk;
        }
    }
    // Rows row0 .. of `rows`, zeros past them and past the head.
    __device__ __forceinline__ void fetch(const T *p, int64_t stride, bool direct, int32_t dim,
                                          char *tile, int wave, int lane, int32_t row0,
                                          int32_t rows) const
    {
        stride = fresh_scalar(stride);
        p += row0 * stride;
        const int32_t left = rows - row0 < Rows ? rows - row0 : Rows;
        if (direct) {
#pragma unroll
            for (int n = 0; n < Mine::kCount; ++n) {
                const int32_t have = left - n * kStep;
                const uint32_t bytes =
                    have > 0 ? ((uint32_t)(have - 1) * (uint32_t)stride + dim) *
                                   (uint32_t)sizeof(T)
                             : 0;
                if (Mine::has(n, wave))
                    load_to_lds(p + n * kStep * stride, bytes, offset[kAlike ? 0 : n],
                                tile + Mine::first(n, wave) * 16);
            }
            return;
        }
        lane = fresh(lane);
#pragma unroll
        for (int n = 0; n < Mine::kCount; ++n) {
            if (!Mine::has(n, wave))
                break;
            const int row = Mine::row(n, wave, lane), at = Mine::at(n, wave, lane);
            typename Layout::Chunk v = (typename Layout::Chunk)(T)0.0f;
            if (row < left && at < dim)
                v = load<T, Layout::kEach>(p + row * stride + at);
            *(typename Layout::Chunk *)(tile + (Mine::first(n, wave) + lane) * 16) = v;
        }
    }
};

// Whether any of a result's N tiles has a value that is not finite: the only ones
// that 0 times does not make 0. (Or, with another factor, one that times this passes
// fp32.)
template <int N>
__device__ __forceinline__ bool any_not_finite(const f32x16 (&x)[N], float times = 0.0f)
{
    float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
        for (int e = 0; e < 16; ++e)
            s[e & 3] = fmaf(x[n][e], times, s[e & 3]);
    const float all = (s[0] + s[1]) + (s[2] + s[3]);
    return !(fabsf(all) < INFINITY);
}

// Whether any of the workgroup's waves says so (each the same in all its lanes), by way
// of four words of LDS that none reads any more.
__device__ __forceinline__ bool any_wave(int *told, bool so, int wave, int lane)
{
    if (lane == 0)
        told[wave] = so;
    __syncthreads();
    int any = 0;
#pragma unroll
    for (int w = 0; w < kAttendWaves; ++w)
        any |= told[w];
    return __builtin_amdgcn_readfirstlane(any);
}

// Which of 32 rows of a tile in LDS (at its first) hold a value that is not finite:
// bit r for row r.
template <typename T, int N>
__device__ __forceinline__ uint32_t rows_not_finite(const char *tile, int lane)
{
    typedef LdsRows<T, N> Rows;
    static_assert(Rows::kChunks % 2 == 0, "half a row a lane");
    const char *p = tile + (lane & 31) * Rows::kStride + (lane >> 5) * (Rows::kStride / 2);
    float s = 0.0f;
#pragma unroll
    for (int c = 0; c < Rows::kChunks / 2; ++c) {
        const typename Rows::Chunk v = *(const typename Rows::Chunk *)(p + 16 * c);
#pragma unroll
        for (int e = 0; e < Rows::kEach; ++e)
            s = fmaf((float)v[e], 0.0f, s);
    }
    const uint64_t which = __ballot(s != s);
    return (uint32_t)(which | which >> 32);
}

// v with zeros where it is not finite; some: whether any lane's v was not, of those
// that were asked.
template <typename T>
__device__ __forceinline__ vec<T, 8> finite_of(vec<T, 8> v, bool &some)
{
    // an exponent of ones carries into the sign's bit
    constexpr bool half = std::is_same<T, f16>::value, single = sizeof(T) == 4;
    constexpr uint32_t ones = single ? 0x7f800000u : half ? 0x7c007c00u : 0x7f807f80u;
    constexpr uint32_t one = single ? 0x00800000u : half ? 0x04000400u : 0x00800080u;
    typedef uint32_t Words __attribute__((ext_vector_type(2 * sizeof(T))));
    const Words w = __builtin_bit_cast(Words, v);
    uint32_t any = 0;
#pragma unroll
    for (int k = 0; k < 2 * (int)sizeof(T); ++k)
        any |= (w[k] & ones) + one;
    if (__any((any & 0x80008000u) != 0)) {
        some = true;
#pragma unroll
        for (int e = 0; e < 8; ++e)
            v[e] = fabsf((float)v[e]) < INFINITY ? v[e] : (T)0.0f;
    }
    return v;
}

// Adds to a result [values x columns] what a tile's 32 rows hold that is not finite, to
// the columns that see the row (sees(r), of the lane's column): as it is, or as NaN.
// live: whether the lane's column counts. Where all that counts is NaN already nothing
// is added, so that many such rows cost little (all values NaN, 2048 tokens, 16 heads of
// 128: 2.9 ms without).
template <bool AsNan, typename T, int N, typename Sees>
__device__ __forceinline__ void add_not_finite(f32x16 (&sum)[N], const char *tile, int32_t dim,
                                               bool live, int lane, Sees sees)
{
    typedef LdsRows<T, N> Rows;
    uint32_t least = ~0u;  // of the magnitudes' bits: a NaN's are past infinity's
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            if (32 * n + 8 * g >= dim)
                break;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                least = min(least, __builtin_bit_cast(uint32_t, fabsf(sum[n][4 * g + e])));
        }
    if (!__any(least <= 0x7f800000u && live))
        return;
    uint32_t rows = rows_not_finite<T, N>(tile, lane);
#pragma unroll 1
    while (rows) {
        const int r = __builtin_ctz(rows);
        rows &= rows - 1;
        const bool some = sees(r);
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int at = (32 * n + 8 * g + 4 * (lane >> 5)) * (int)sizeof(T);
                const vec<T, 4> v =
                    *(const vec<T, 4> *)(tile + Rows::place(r, at >> 4) + (at & 15));
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float x = some ? (float)v[e] : 0.0f;
                    sum[n][4 * g + e] += AsNan ? x - x : fabsf(x) < INFINITY ? 0.0f : x;
                }
                in_order();
            }
    }
}

// Writes a result [values x rows]: the lane's row at p, times f, and what rounding
// takes from it at rest (or null); zeros for a row that has no pair (its sums may
// hold 0 times a NaN). dim is a multiple of 8, so both halves of the wave write.
template <typename T, int N>
__device__ __forceinline__ void write_row(T *p, T *rest, f32x16 (&sum)[N], float f, bool none,
                                          int32_t dim, int lane)
{
    if (__any(none))
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int e = 0; e < 16; ++e)
                sum[n][e] = none ? 0.0f : sum[n][e];
    f = none ? 0.0f : f;
    p += 4 * (lane >> 5);
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int d = 32 * n + 8 * g;
            if (d >= dim)
                return;
            vec<float, 4> y;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                y[e] = sum[n][4 * g + e] * f;
            const vec<T, 4> z = from_f32<T, 4>(y);
            store<T, 4>(p + d, z);
            if (rest)
                store<T, 4>(rest + 4 * (lane >> 5) + d, from_f32<T, 4>(y - to_f32<4, T>(z)));
        }
}

// A row of up to 128 values over the wave: values lane and lane + 64.
struct Spread {
    float x, y;
};

}  // namespace
}  // namespace smol

#endif  // SMOL_ATTEND_DEVICE_H
