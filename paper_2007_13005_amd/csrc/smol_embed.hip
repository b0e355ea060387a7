// smol_embed.hip -- embedding lookup and its gradient by sorted ids
// (smol_embed, smol_embed_backward).
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "smol.h"
#include "smol_internal.h"
#include "smol_tokens.h"
#include "smol_tokens_device.h"

namespace smol {
namespace {

template <typename I>
__device__ __forceinline__ int64_t id_at(const void *ids, int64_t i)
{
    return (int64_t)((const I *)ids)[i];
}

// Columns col .. col + V - 1 of a row, moved back to end with the row where
// they would pass it; its first `lead` columns then belong to another lane.
template <int V>
struct Span {
    int32_t at, lead;
    __device__ __forceinline__ Span(int32_t col, int32_t dim)
    {
        at = col <= dim - V ? col : dim - V;
        lead = col < dim ? col - at : V;
    }
};

// The elements of a span that are its own.
template <typename T, int V>
__device__ __forceinline__ void store_own(T *p, vec<T, V> v, int32_t lead)
{
    if (lead == 0) {
        store<T, V>(p, v);
        return;
    }
#pragma unroll
    for (int e = 0; e < V; ++e)
        if (e >= lead)
            p[e] = v[e];
}

struct EmbedArgs {
    const void *ids, *table;
    void *out;
    int64_t n, vocab, table_stride, out_stride;
    int32_t dim, keep;
    float scale;
};

// One wave takes kSpans * 64 * V columns of a row, four rows a workgroup; it
// moves bytes and multiplies once a value. 33001 ids (a quarter of them of no
// token) of 1024 fp32 columns to bf16: 23 us, 4.4 TB/s; one id of 4096 fp16
// columns 2.2 us. Narrow rows leave lanes and the second span idle: 65536 ids of
// bf16 rows, columns 512: 21.5 us, 4.7 TB/s, 256: 15.9, 3.1, 128: 14.0, 1.8, 64:
// 12.2, 1.0.
constexpr int kSpans = 2;

template <typename T, typename O, typename I, int V>
__global__ void __launch_bounds__(256) embed_kernel(EmbedArgs a)
{
    const int32_t lane = threadIdx.x & 63;
    const int32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int32_t first = blockIdx.y * kSpans * 64 * V + lane * V;
    for (int64_t i = (int64_t)blockIdx.x * 4 + wave; i < a.n; i += (int64_t)gridDim.x * 4) {
        const int64_t id = id_at<I>(a.ids, i);
        const bool some = id >= 0 && id < a.vocab;
        if (!some && a.keep)
            continue;
        O *out = (O *)a.out + i * a.out_stride;
        vec<T, V> x[kSpans];
        if (some) {
            const T *row = (const T *)a.table + id * a.table_stride;
#pragma unroll
            for (int s = 0; s < kSpans; ++s) {
                const Span<V> c(first + s * 64 * V, a.dim);
                x[s] = load<T, V>(row + c.at);
            }
        } else {
#pragma unroll
            for (int s = 0; s < kSpans; ++s)
                x[s] = (vec<T, V>)(T)0.0f;
        }
#pragma unroll
        for (int s = 0; s < kSpans; ++s) {
            const Span<V> c(first + s * 64 * V, a.dim);
            // a span moved back writes its neighbour's columns alike
            if (c.lead < V)
                store<O, V>(out + c.at,
                            from_f32<O, V>(some ? to_f32<V, T>(x[s]) * a.scale
                                                : (vec<float, V>)0.0f));
        }
    }
}

// The gradient. The ids' keys (the id, or `vocab` for rows without a
// gradient: they come last) are sorted stably with the rows' numbers; pieces
// of a fixed number of sorted rows are summed by a wave per 64 * V columns,
// and sums of ids that reach over pieces are joined in a second launch. Every
// sum runs in an order that depends on the ids alone. Zeros for the rows that
// no id names are written by further workgroups of the sort's launches, which
// leave most of the chip idle.
constexpr int kBits = 9, kDigits = 1 << kBits;
constexpr int kSortThreads = 512, kSortRounds = 2;
constexpr int kSortTile = kSortThreads * kSortRounds;
constexpr int kSortGroups = 64;
// Up to this many rows each row's place is counted directly, in one launch:
// the id and the row's number fit one word for vocabularies below 2^19.
constexpr int kRankBits = 13, kRankRows = 1 << kRankBits;

// Zeros in the words lo .. hi - 1 (dense rows) or the rows lo .. hi - 1 of
// `words` each, `stride` apart; words are 16-bit. first: the launch's first
// workgroup that does this.
struct Fill {
    uint16_t *at;
    int64_t lo, hi, words, stride;
    uint32_t first;
};

__device__ __forceinline__ void fill(const Fill &f)
{
    typedef vec<uint16_t, 8> W;
    const int64_t block = blockIdx.x - f.first, blocks = gridDim.x - f.first;
    const int64_t count = f.words ? f.words : f.hi - f.lo;
    const auto zero = [&](uint16_t *p, int64_t at) {  // words at .. at + 7 of p's `count`
        if (count >= 8)
            // past the caches: the sums that follow read through them
            // (65536 rows of 1024 bf16 values: 117 us -> 109)
            store_past<uint16_t, 8>(p + (at <= count - 8 ? at : count - 8), (W)(uint16_t)0);
        else
            for (int64_t k = at; k < count; ++k)
                p[k] = 0;
    };
    if (!f.words) {
        for (int64_t i = (block * blockDim.x + threadIdx.x) * 8; i < count;
             i += blocks * blockDim.x * 8)
            zero(f.at + f.lo, i);
        return;
    }
    const int64_t waves = blockDim.x / 64;
    for (int64_t r = f.lo + block * waves + threadIdx.x / 64; r < f.hi; r += blocks * waves)
        for (int64_t i = (threadIdx.x & 63) * 8; i < count; i += 512)
            zero(f.at + r * f.stride, i);
}

struct SortArgs {
    const void *ids;
    const uint32_t *key_in, *row_in;
    uint32_t *key, *row;
    uint32_t *table;  // [workgroup][digit] counts
    int64_t vocab, padding;
    uint32_t n, per;  // keys, keys a workgroup
    int32_t shift, groups;
    Fill fill;
};

template <typename I>
__device__ __forceinline__ uint32_t key_of(const SortArgs &a, uint32_t i)
{
    const int64_t id = id_at<I>(a.ids, i);
    return id >= 0 && id < a.vocab && id != a.padding ? (uint32_t)id : (uint32_t)a.vocab;
}

// Every row's place is the number of (key, row) words below its own: n^2
// comparisons, in one launch. 16 rows a workgroup, 16 threads a row, each
// counting every 16th word. us a call, counting / with the four launches of a
// sort by two digits: 321 fp32 columns, a vocabulary of 5003, rows 1025: 12.2 /
// 21.8, 4096: 17.5 / 23.8, 8192: 35.5 / 34.4; 1024 bf16 columns, 32000, rows
// 1025: 33.1 / 33.2, 4096: 35.5 / 38.2, 8192: 51.3 / 51.5.
template <typename I>
__global__ void __launch_bounds__(256) embed_rank_kernel(SortArgs a)
{
    if (blockIdx.x >= a.fill.first) {
        fill(a.fill);
        return;
    }
    __shared__ uint32_t word[kRankRows];
    for (uint32_t i = threadIdx.x; i < ((a.n + 15) & ~15u); i += 256)
        word[i] = i < a.n ? key_of<I>(a, i) << kRankBits | i : 0xffffffffu;
    __shared__ uint32_t part[16][17];
    __syncthreads();
    const uint32_t i = blockIdx.x * 16 + (threadIdx.x & 15), q = threadIdx.x >> 4;
    const uint32_t mine = i < a.n ? word[i] : 0;
    uint32_t below = 0;
#pragma unroll 8
    for (uint32_t j = q; j < a.n; j += 16)
        below += word[j] < mine;
    part[q][threadIdx.x & 15] = below;
    __syncthreads();
    if (q != 0 || i >= a.n)
        return;
    for (int k = 1; k < 16; ++k)
        below += part[k][threadIdx.x];
    a.key[below] = mine >> kRankBits;
    a.row[below] = i;
}

// One pass of the sort over digits of kBits, two launches: counts of each
// workgroup's part, then the moves. 65536 ids: 3 and 6 us, or 13 us each with
// 66 MB of zeros beside them (5 TB/s).
template <typename I, bool First>
__global__ void __launch_bounds__(kSortThreads) embed_count_kernel(SortArgs a)
{
    if (blockIdx.x >= a.fill.first) {
        fill(a.fill);
        return;
    }
    __shared__ uint32_t count[kDigits];
    count[threadIdx.x] = 0;
    __syncthreads();
    const uint32_t lo = blockIdx.x * a.per, end = lo + a.per, hi = end < a.n ? end : a.n;
    for (uint32_t i = lo + threadIdx.x; i < hi; i += kSortThreads) {
        const uint32_t key = First ? key_of<I>(a, i) : a.key_in[i];
        atomicAdd(&count[key >> a.shift & (kDigits - 1)], 1u);
    }
    __syncthreads();
    a.table[blockIdx.x * kDigits + threadIdx.x] = count[threadIdx.x];
}

template <typename I, bool First>
__global__ void __launch_bounds__(kSortThreads) embed_move_kernel(SortArgs a)
{
    static_assert(kSortThreads == kDigits, "a digit a thread");
    if (blockIdx.x >= a.fill.first) {
        fill(a.fill);
        return;
    }
    constexpr int kWaves = kSortThreads / 64;
    __shared__ uint32_t base[kDigits];            // next place of each digit
    __shared__ uint32_t count[kWaves][kDigits];   // this tile's, wave by wave
    __shared__ uint32_t sums[kWaves];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    // base[d]: all keys of smaller digits, and of this digit in earlier groups
    uint32_t total = 0, before = 0;
#pragma unroll 16
    for (int g = 0; g < a.groups; ++g) {
        const uint32_t c = a.table[g * kDigits + threadIdx.x];
        total += c;
        before += g < (int)blockIdx.x ? c : 0;
    }
    uint32_t scan = total;
#pragma unroll
    for (int k = 1; k < 64; k <<= 1) {
        const uint32_t up = __shfl_up(scan, k);
        scan += lane >= k ? up : 0;
    }
    if (lane == 63)
        sums[wave] = scan;
    __syncthreads();
    uint32_t start = scan - total + before;
    for (int w = 0; w < wave; ++w)
        start += sums[w];
    base[threadIdx.x] = start;
    const uint32_t lo = blockIdx.x * a.per, end = lo + a.per, hi = end < a.n ? end : a.n;
    for (uint32_t tile = lo; tile < hi; tile += kSortTile) {
        __syncthreads();
        for (int d = threadIdx.x; d < kWaves * kDigits; d += kSortThreads)
            (&count[0][0])[d] = 0;
        __syncthreads();
        // wave w takes 64 * kSortRounds keys in a row; keys of equal digits
        // among 64 keep their order by the lanes below
        uint32_t key[kSortRounds], row[kSortRounds], rank[kSortRounds];
#pragma unroll
        for (int r = 0; r < kSortRounds; ++r) {
            const uint32_t i = tile + (wave * kSortRounds + r) * 64 + lane;
            const bool in = i < hi;
            key[r] = !in ? 0 : First ? key_of<I>(a, i) : a.key_in[i];
            row[r] = !in || First ? i : a.row_in[i];
        }
#pragma unroll
        for (int r = 0; r < kSortRounds; ++r) {
            const bool in = tile + (wave * kSortRounds + r) * 64 + lane < hi;
            const uint32_t d = key[r] >> a.shift & (kDigits - 1);
            uint64_t same = __ballot(in);
#pragma unroll
            for (int b = 0; b < kBits; ++b) {
                const uint64_t ones = __ballot(d >> b & 1);
                same &= d >> b & 1 ? ones : ~ones;
            }
            const uint32_t below = __popcll(same & ((1ull << lane) - 1));
            const uint32_t had = in ? count[wave][d] : 0;
            rank[r] = had + below;
            // the last of the equal lanes leaves the new count
            if (in && (same >> lane) == 1)
                count[wave][d] = had + below + 1;
            __builtin_amdgcn_wave_barrier();
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < kSortRounds; ++r) {
            if (tile + (wave * kSortRounds + r) * 64 + lane >= hi)
                continue;
            const uint32_t d = key[r] >> a.shift & (kDigits - 1);
            uint32_t to = base[d] + rank[r];
            for (int w = 0; w < wave; ++w)
                to += count[w][d];
            a.key[to] = key[r];
            a.row[to] = row[r];
        }
        __syncthreads();
        uint32_t c = 0;
#pragma unroll
        for (int w = 0; w < kWaves; ++w)
            c += count[w][threadIdx.x];
        base[threadIdx.x] += c;
    }
}

struct GradArgs {
    const void *grad_out;
    const uint32_t *key, *row;
    float *part;  // [piece][2][dim]: sums of the ids that reach in from the
                  // left, and that begin in the piece and reach out
    void *table;
    int64_t grad_stride, table_stride;
    uint32_t n, vocab, pieces;
    int32_t piece;  // rows of a piece, at most 64
    int32_t dim, accumulate;
    float scale;
};

template <typename P, int V>
__device__ __forceinline__ void write_row(const GradArgs &a, uint32_t id, Span<V> c,
                                          vec<float, V> sum)
{
    P *p = (P *)a.table + (int64_t)id * a.table_stride + c.at;
    sum *= a.scale;
    if (a.accumulate)
        sum += to_f32<V, P>(load<P, V>(p));
    store_own<P, V>(p, from_f32<P, V>(sum), c.lead);
}

// A wave sums its piece, kAhead rows on their way at a time. What has arrived
// goes through LDS (each lane's own 16 bytes, so nothing waits for other
// waves): the loop over rows stays a loop, and its code in the instruction
// cache, where unrolled over registers it did not fit. 65536 rows of 1024 bf16
// values, a vocabulary of 64000: 47 us for 101 MB read and 62 MB written; the
// zeros written before are on their way to memory meanwhile (with none before
// it 25 us for the same reads).
template <typename G, typename P, int V>
__global__ void __launch_bounds__(256) embed_grad_kernel(GradArgs a)
{
    constexpr int kAhead = 8;
    __shared__ vec<G, V> arrived[4][kAhead][64];
    const int32_t lane = threadIdx.x & 63;
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t piece = blockIdx.x * 4 + wave;
    if (piece >= a.pieces)
        return;
    const Span<V> c((int32_t)(blockIdx.y * 64 + lane) * V, a.dim);
    const uint32_t lo = piece * a.piece;
    const uint32_t count = a.n - lo < (uint32_t)a.piece ? a.n - lo : a.piece;
    // lane p: the piece's p-th key and row; past the rows, a key of no row
    uint32_t key = a.vocab, row = 0;
    if (lane < (int32_t)count) {
        key = a.key[lo + lane];
        row = a.row[lo + lane];
    }
    const uint32_t left = lo > 0 ? a.key[lo - 1] : a.vocab;
    const uint32_t right = lo + a.piece < a.n ? a.key[lo + a.piece] : a.vocab;
    const uint32_t some = __popcll(__ballot(key != a.vocab));  // they come first
    if (some == 0)
        return;
    vec<float, V> sum = (vec<float, V>)0.0f;
    uint32_t id = __builtin_amdgcn_readlane(key, 0);
    bool first = true;
    vec<G, V> x[kAhead];
    const auto fetch = [&](uint32_t p) {
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const uint32_t q = p + u < some ? p + u : some - 1;
            const int64_t r = (uint32_t)__builtin_amdgcn_readlane(row, q);
            x[u] = load<G, V>((const G *)a.grad_out + r * a.grad_stride + c.at);
        }
        asm volatile("" ::: "memory");
    };
    fetch(0);
    for (uint32_t p = 0; p < some; p += kAhead) {
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
            arrived[wave][u][lane] = x[u];
        if (p + kAhead < some)
            fetch(p + kAhead);
        const uint32_t end = some - p < kAhead ? some : p + kAhead;
#pragma unroll 1
        for (uint32_t q = p; q <= end; ++q) {
            // at the piece's end once more, for the last sum
            const uint32_t k = q < some ? __builtin_amdgcn_readlane(key, q) : ~0u;
            if (k != id && (q < end || end == some)) {
                float *part = a.part + (int64_t)piece * 2 * a.dim + c.at;
                if (first && id == left)
                    store_own<float, V>(part, sum, c.lead);
                else if (q == (uint32_t)a.piece && id == right)
                    store_own<float, V>(part + a.dim, sum, c.lead);
                else
                    write_row<P, V>(a, id, c, sum);
                first = false;
                id = k;
                sum = (vec<float, V>)0.0f;
            }
            if (q < end)
                sum += to_f32<V, G>(arrived[wave][q - p][lane]);
        }
    }
}

// The sums of pieces from..to - 1 after `part`, added in order.
template <int V>
__device__ __forceinline__ vec<float, V> add_parts(const GradArgs &a, const float *part,
                                                   uint32_t from, uint32_t to, vec<float, V> sum)
{
    constexpr uint32_t kAhead = 8;
    for (uint32_t k = from; k < to; k += kAhead) {
        vec<float, V> x[kAhead];
#pragma unroll
        for (uint32_t u = 0; u < kAhead; ++u)
            x[u] = load<float, V>(part + (int64_t)(k + u < to ? k + u : to - 1) * 2 * a.dim);
        asm volatile("" ::: "memory");
#pragma unroll
        for (uint32_t u = 0; u < kAhead; ++u)
            if (k + u < to)
                sum += x[u];
    }
    return sum;
}

// An id that reaches over pieces belongs to the piece in which it begins. A
// wave a piece adds the later pieces' sums to its own, in order; where there
// are more than kAlone of them, the eight waves of the workgroup divide them,
// and the waves' sums are added in order. 65536 rows, the most frequent id 4000
// times: 8 us; one id 49152 times: 18 us (187 with one wave).
template <typename P, int V>
__global__ void __launch_bounds__(512) embed_join_kernel(GradArgs a)
{
    constexpr uint32_t kWaves = 8, kAlone = 16;
    __shared__ vec<float, V> sums[kWaves][64];
    __shared__ uint32_t counts[kWaves];
    const uint32_t lane = threadIdx.x & 63;
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Span<V> c((int32_t)(blockIdx.y * 64 + lane) * V, a.dim);
    const auto own = [&](uint32_t piece) {
        return load<float, V>(a.part + ((int64_t)piece * 2 + 1) * a.dim + c.at);
    };
    const uint32_t piece = blockIdx.x * kWaves + wave, lo = piece * a.piece, hi = lo + a.piece;
    uint32_t count = 0, id = a.vocab;
    if (piece + 1 < a.pieces) {
        id = a.key[hi - 1];
        if (id != a.vocab && a.key[hi] == id &&
            !(lo > 0 && a.key[lo] == id && a.key[lo - 1] == id)) {
            // how many later pieces begin with the id: 64 tried at once, then
            // every (n / 64)th of those that are left
            const uint32_t all = a.pieces - piece - 1;
            uint32_t left = all, step = 1;
            for (;;) {
                const uint32_t at = count + (lane + 1) * step - 1;
                const uint64_t same = __ballot(at < left && a.key[hi + at * a.piece] == id);
                const uint32_t run = ~same ? __builtin_ctzll(~same) : 64;
                count += run * step;
                if (run < 64) {
                    if (step == 1)
                        break;
                    left = count + step < left ? count + step : left;
                }
                if (count == left)
                    break;
                step = left - count > 64 ? (left - count + 63) / 64 : 1;
            }
            if (count <= kAlone) {
                const float *part = a.part + ((int64_t)piece + 1) * 2 * a.dim + c.at;
                write_row<P, V>(a, id, c, add_parts<V>(a, part, 0, count, own(piece)));
            }
        }
    }
    if (lane == 0)
        counts[wave] = count;
    __syncthreads();
    for (uint32_t k = 0; k < kWaves; ++k) {
        const uint32_t many = __builtin_amdgcn_readfirstlane(counts[k]);
        if (many <= kAlone)
            continue;
        const uint32_t at = blockIdx.x * kWaves + k, each = (many + kWaves - 1) / kWaves;
        const uint32_t from = wave * each, to = from + each < many ? from + each : many;
        const float *part = a.part + ((int64_t)at + 1) * 2 * a.dim + c.at;
        vec<float, V> sum = (vec<float, V>)0.0f;
        if (wave == 0)
            sum = own(at);
        sum = add_parts<V>(a, part, from, to, sum);
        sums[wave][lane] = sum;
        __syncthreads();
        if (wave == 0) {
#pragma unroll
            for (uint32_t w = 1; w < kWaves; ++w)
                sum += sums[w][lane];
            write_row<P, V>(a, a.key[at * a.piece + a.piece - 1], c, sum);
        }
        __syncthreads();
    }
}

// Few rows: everything in one launch, without a sort. A wave a row
// looks for its id among all rows (in LDS); the first row of an id has their
// list in order, and its wave adds them, or, where there are more than kAlone,
// the eight waves of the workgroup a part each, joined in order. The grid has
// `groups` workgroups of rows for the first 64 * V columns, as many for the
// next, and so on; those from fill.first on write zeros in the rows of the
// table that no id names: `per` rows each, which they mark in LDS (once for all
// columns: with a copy of them for every 64 * V, which left at once, 64 ids of
// 4096 fp32 columns in a vocabulary of 5003 took 23.3 us, now 15.6; 1024 ids in
// one of 64000, 239 and 205).
//
// Every workgroup of rows goes through all ids, so it is taken up to kFewRows
// rows and kFewLooks ids looked at by all workgroups together. us a call added
// to the table (so without zeros), one launch / with the counting sort, *: taken;
// rows x columns:
//   fp32  777 x 321 9.0* / 13.7   256 x 8192 11.9* / 13.9   256 x 16384 19.2* / 16.7
//         512 x 4096 14.6* / 14.1   700 x 4096 20.5 / 16.0   1024 x 2048 21.8 / 14.7
//         256 x 65536 93 / 38
//   bf16  1024 x 1024 8.8* / 13.6   1024 x 2048 12.7* / 14.3   700 x 4096 12.2* / 15.0
//         128 x 65536 14.0* / 20.1   1024 x 4096 17.3 / 16.8
// One id that all rows name, which
// cannot be known here, is the worst: 1024 x 1024 bf16 20.3 / 11.9, 512 x 1024
// 10.5 / 9.7.
constexpr int kFewRows = 1024;
constexpr int64_t kFewLooks = 1 << 19;
constexpr uint32_t kFewFill = 2048;  // rows of the table a workgroup at most

template <typename I, typename G, typename P, int V>
__global__ void __launch_bounds__(512) embed_few_kernel(SortArgs o, GradArgs a, uint32_t per,
                                                        uint32_t groups)
{
    constexpr uint32_t kWaves = 8, kAlone = 16, kAhead = 8;
    __shared__ uint32_t keys[kFewRows];
    __shared__ uint16_t list[kWaves][kFewRows];
    __shared__ vec<float, V> sums[kWaves][64];
    __shared__ uint32_t counts[kWaves], named[kFewFill / 32];
    const uint32_t lane = threadIdx.x & 63;
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    for (uint32_t i = threadIdx.x; i < ((a.n + 63) & ~63u); i += 512)
        keys[i] = i < a.n ? key_of<I>(o, i) : (uint32_t)o.vocab;
    if (blockIdx.x >= o.fill.first) {
        const uint32_t lo = (blockIdx.x - o.fill.first) * per;
        const uint32_t rows = a.vocab - lo < per ? a.vocab - lo : per;
        if (threadIdx.x < kFewFill / 32)
            named[threadIdx.x] = 0;
        __syncthreads();
        for (uint32_t i = threadIdx.x; i < a.n; i += 512)
            if (keys[i] - lo < rows)
                atomicOr(&named[(keys[i] - lo) / 32], 1u << (keys[i] - lo) % 32);
        __syncthreads();
        // chunks of 16 bytes; a row's last is moved back to end with it
        const uint32_t words = a.dim * (sizeof(P) / 2), chunks = (words + 7) / 8;
        uint16_t *table = (uint16_t *)a.table;
        for (uint32_t e = threadIdx.x; e < rows * chunks; e += 512) {
            const uint32_t r = e / chunks, c = (e - r * chunks) * 8;
            if (named[r / 32] >> r % 32 & 1)
                continue;
            uint16_t *p = table + (int64_t)(lo + r) * a.table_stride * (sizeof(P) / 2);
            if (words >= 8)
                store_past<uint16_t, 8>(p + (c <= words - 8 ? c : words - 8),
                                        (vec<uint16_t, 8>)(uint16_t)0);
            else
                for (uint32_t k = 0; k < words; ++k)
                    p[k] = 0;
        }
        return;
    }
    __syncthreads();
    const uint32_t column = blockIdx.x / groups, first = (blockIdx.x - column * groups) * kWaves;
    const Span<V> c((int32_t)(column * 64 + lane) * V, a.dim);
    const uint32_t row = first + wave;
    const uint32_t id = row < a.n ? keys[row] : a.vocab;
    uint32_t count = 0;
    if (id != a.vocab) {
        for (uint32_t i = 0; i < a.n; i += 64) {
            uint64_t same = __ballot(keys[i + lane] == id);
            if (i < row && (same & (row - i < 64 ? (1ull << (row - i)) - 1 : ~0ull))) {
                count = 0;  // not the first of its id
                break;
            }
            if (same >> lane & 1)
                list[wave][count + __popcll(same & ((1ull << lane) - 1))] = (uint16_t)(i + lane);
            count += __popcll(same);
        }
    }
    // rows k .. to - 1 of wave w's list, added in order
    const auto add = [&](uint32_t w, uint32_t k, uint32_t to) {
        vec<float, V> sum = (vec<float, V>)0.0f;
        for (; k < to; k += kAhead) {
            vec<G, V> x[kAhead];
#pragma unroll
            for (uint32_t u = 0; u < kAhead; ++u) {
                const int64_t r = __builtin_amdgcn_readfirstlane(list[w][k + u < to ? k + u : to - 1]);
                x[u] = load<G, V>((const G *)a.grad_out + r * a.grad_stride + c.at);
            }
            asm volatile("" ::: "memory");
#pragma unroll
            for (uint32_t u = 0; u < kAhead; ++u)
                if (k + u < to)
                    sum += to_f32<V, G>(x[u]);
        }
        return sum;
    };
    if (count > 0 && count <= kAlone)
        write_row<P, V>(a, id, c, add(wave, 0, count));
    if (lane == 0)
        counts[wave] = count;
    __syncthreads();
    for (uint32_t w = 0; w < kWaves; ++w) {
        const uint32_t many = __builtin_amdgcn_readfirstlane(counts[w]);
        if (many <= kAlone)
            continue;
        const uint32_t each = (many + kWaves - 1) / kWaves, from = wave * each;
        vec<float, V> sum = add(w, from, from + each < many ? from + each : many);
        sums[wave][lane] = sum;
        __syncthreads();
        if (wave == 0) {
#pragma unroll
            for (uint32_t k = 1; k < kWaves; ++k)
                sum += sums[k][lane];
            write_row<P, V>(a, keys[first + w], c, sum);
        }
        __syncthreads();
    }
}

int check_ids(int64_t n, int64_t vocab, int32_t dim, int32_t ids_type)
{
    if (n < 0 || vocab < 1 || dim < 1)
        return set_error(SMOL_ERR_INVALID_ARG, "n %lld, vocab %lld or dim %d out of range",
                         (long long)n, (long long)vocab, dim);
    if (ids_type != SMOL_IDS_I32 && ids_type != SMOL_IDS_I64)
        return set_error(SMOL_ERR_INVALID_ARG, "ids_type %d unknown", ids_type);
    if (n > SMOL_MAX_ROWS || vocab > SMOL_MAX_ROWS || dim > SMOL_MAX_EMBED_DIM)
        return set_error(SMOL_ERR_UNSUPPORTED,
                         "n %lld or vocab %lld beyond %d or dim %d beyond %d", (long long)n,
                         (long long)vocab, SMOL_MAX_ROWS, dim, SMOL_MAX_EMBED_DIM);
    return SMOL_OK;
}

// least: the smallest row stride, the width for a matrix that is written.
int check_rows(const char *name, const void *p, int64_t stride, int64_t rows, int64_t least,
               int type)
{
    if (!p)
        return set_error(SMOL_ERR_INVALID_ARG, "%s is NULL", name);
    if (type < SMOL_ELEM_F32 || type > SMOL_ELEM_BF16)
        return set_error(SMOL_ERR_INVALID_ARG, "%s: element type %d unknown", name, type);
    if ((uintptr_t)p % elem_size(type))
        return set_error(SMOL_ERR_INVALID_ARG, "%s is not aligned to its elements", name);
    if (rows > 1 && (stride < least || stride > INT64_MAX / 8 / rows))
        return set_error(SMOL_ERR_INVALID_ARG, "%s: row stride %lld out of range", name,
                         (long long)stride);
    return SMOL_OK;
}

template <typename F>
auto with_ids(int ids_type, F f)
{
    return ids_type == SMOL_IDS_I64 ? f(int64_t{}) : f(int32_t{});
}

// Eight elements a lane where a row has as many, else one.
template <typename F>
void with_width(int dim, F f)
{
    if (dim >= 8)
        f(std::integral_constant<int, 8>{});
    else
        f(std::integral_constant<int, 1>{});
}

struct Workspace {
    int64_t keys, table, part, bytes;
};

// Rows of a piece: few where there are few rows, so that they are summed side
// by side; more where the pieces fill the chip, so that fewer sums are written
// and read again and less room is asked for. us a call in pieces of 8 / 32: 321
// fp32 columns, a vocabulary of 5003, rows 2048: 13.7 / 20.9, 4096: 17.5 / 24.7,
// 8192: 31.0 / 35.5; 1024 bf16 columns, 32000, rows 4096: 35.5 / 43.1, 8192:
// 45.8 / 51.3, 16384: 48.7 / 48.2, 65536: 90.2 / 86.4 (between 4096 and 16384
// pieces of 8 would still be the faster, with four times the room).
int piece_rows(int64_t n) { return n <= 4096 ? 8 : 32; }

Workspace layout(int64_t n, int32_t dim)
{
    Workspace w;
    w.keys = (n * 4 + 15) / 16 * 16;
    w.table = 4 * w.keys;
    w.part = w.table + kDigits * kSortGroups * 4;
    const int piece = piece_rows(n);
    w.bytes = w.part + (n + piece - 1) / piece * 2 * dim * 4 + 16;
    return w;
}

}  // namespace
}  // namespace smol

extern "C" int smol_embed(const smol_embed_args *p, void *stream)
{
    using namespace smol;
    clear_error();
    if (!p)
        return set_error(SMOL_ERR_INVALID_ARG, "args is NULL");
    int st = check_ids(p->n, p->vocab, p->dim, p->ids_type);
    if (st != SMOL_OK)
        return st;
    if (p->reserved[0] || p->reserved[1])
        return set_error(SMOL_ERR_INVALID_ARG, "reserved fields are not zero");
    if (!isfinite(p->scale))
        return set_error(SMOL_ERR_INVALID_ARG, "scale is not finite");
    if (p->keep != 0 && p->keep != 1)
        return set_error(SMOL_ERR_INVALID_ARG, "keep %d is neither 0 nor 1", p->keep);
    if (p->n == 0)
        return SMOL_OK;
    if (!p->ids || (uintptr_t)p->ids % (p->ids_type == SMOL_IDS_I64 ? 8 : 4))
        return set_error(SMOL_ERR_INVALID_ARG, "ids is NULL or not aligned to its elements");
    if ((st = check_rows("table", p->table, p->table_stride, p->vocab, 0, p->table_type)) !=
            SMOL_OK ||
        (st = check_rows("out", p->out, p->out_stride, p->n, p->dim, p->out_type)) != SMOL_OK)
        return st;
    EmbedArgs a;
    a.ids = p->ids;
    a.table = p->table;
    a.out = p->out;
    a.n = p->n;
    a.vocab = p->vocab;
    a.table_stride = p->table_stride;
    a.out_stride = p->out_stride;
    a.dim = p->dim;
    a.keep = p->keep;
    a.scale = p->scale;
    const int64_t groups = (p->n + 3) / 4;
    with_width(p->dim, [&](auto v) {
        const int cols = kSpans * 64 * v.value;
        const dim3 grid((unsigned)(groups < 65536 ? groups : 65536),
                        (unsigned)((p->dim + cols - 1) / cols));
        with_ids(p->ids_type, [&](auto i) {
            with_type(p->table_type, [&](auto t) {
                with_type(p->out_type, [&](auto o) {
                    hipLaunchKernelGGL(
                        (embed_kernel<decltype(t), decltype(o), decltype(i), v.value>), grid,
                        dim3(256), 0, (hipStream_t)stream, a);
                });
            });
        });
    });
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess)
        return set_error(SMOL_ERR_HIP, "embedding launch: %s", hipGetErrorString(e));
    return SMOL_OK;
}

extern "C" int64_t smol_embed_workspace_bytes(int64_t n, int64_t vocab, int32_t dim)
{
    using namespace smol;
    if (n < 0 || n > SMOL_MAX_ROWS || vocab < 1 || vocab > SMOL_MAX_ROWS || dim < 1 ||
        dim > SMOL_MAX_EMBED_DIM)
        return 0;
    return layout(n, dim).bytes;
}

extern "C" int smol_embed_backward(const smol_embed_grad_args *p, void *stream)
{
    using namespace smol;
    clear_error();
    if (!p)
        return set_error(SMOL_ERR_INVALID_ARG, "args is NULL");
    int st = check_ids(p->n, p->vocab, p->dim, p->ids_type);
    if (st != SMOL_OK)
        return st;
    if (!isfinite(p->scale))
        return set_error(SMOL_ERR_INVALID_ARG, "scale is not finite");
    if (p->accumulate != 0 && p->accumulate != 1)
        return set_error(SMOL_ERR_INVALID_ARG, "accumulate %d is neither 0 nor 1", p->accumulate);
    if ((st = check_rows("grad_table", p->grad_table, p->table_stride, p->vocab, p->dim,
                         p->grad_type)) != SMOL_OK)
        return st;
    if (p->n > 0) {
        if (!p->ids || (uintptr_t)p->ids % (p->ids_type == SMOL_IDS_I64 ? 8 : 4))
            return set_error(SMOL_ERR_INVALID_ARG, "ids is NULL or not aligned to its elements");
        if ((st = check_rows("grad_out", p->grad_out, p->grad_stride, p->n, 0,
                             p->out_type)) != SMOL_OK)
            return st;
    }
    const Workspace w = layout(p->n, p->dim);
    if (!p->workspace || (uintptr_t)p->workspace % 16 || p->workspace_bytes < w.bytes)
        return set_error(SMOL_ERR_INVALID_ARG,
                         "workspace must be 16-byte aligned and hold %lld bytes",
                         (long long)w.bytes);
    hipStream_t s = (hipStream_t)stream;
    char *ws = (char *)p->workspace;
    uint32_t *key[2] = {(uint32_t *)ws, (uint32_t *)(ws + w.keys)};
    uint32_t *row[2] = {(uint32_t *)(ws + 2 * w.keys), (uint32_t *)(ws + 3 * w.keys)};

    SortArgs o;
    o.ids = p->ids;
    o.key_in = o.row_in = nullptr;
    o.key = key[0];
    o.row = row[0];
    o.table = (uint32_t *)(ws + w.table);
    o.vocab = p->vocab;
    o.padding = p->padding;
    o.n = (uint32_t)p->n;
    o.shift = 0;
    o.groups = o.per = 0;
    GradArgs a;
    a.grad_out = p->grad_out;
    a.part = (float *)(ws + w.part);
    a.table = p->grad_table;
    a.grad_stride = p->grad_stride;
    a.table_stride = p->table_stride;
    a.n = (uint32_t)p->n;
    a.vocab = (uint32_t)p->vocab;
    a.piece = piece_rows(p->n);
    a.pieces = (uint32_t)((p->n + a.piece - 1) / a.piece);
    a.dim = p->dim;
    a.accumulate = p->accumulate;
    a.scale = p->scale;
    const int lane_columns = p->n && elem_size(p->out_type) == 2 ? 8 : 4;  // of embed_few_kernel
    const int64_t looks =
        (p->n + 7) / 8 * ((p->dim + 64 * lane_columns - 1) / (64 * lane_columns)) * p->n;
    if (p->n <= kFewRows && looks <= kFewLooks) {
        const int64_t bytes = (int64_t)p->dim * elem_size(p->grad_type);
        int64_t per = 65536 / bytes;  // 64 KiB of zeros a workgroup
        per = per < 1 ? 1 : per > kFewFill ? kFewFill : per;
        if ((p->vocab + per - 1) / per > 4096)  // of which there are not too many
            per = (p->vocab + 4095) / 4096 < kFewFill ? (p->vocab + 4095) / 4096 : kFewFill;
        const uint32_t groups = (uint32_t)((p->n + 7) / 8);
        const unsigned zeros = p->accumulate ? 0 : (unsigned)((p->vocab + per - 1) / per);
        with_type(p->grad_type, [&](auto t) {
            typedef decltype(t) P;
            with_type(p->n ? p->out_type : SMOL_ELEM_F32, [&](auto g) {
                typedef decltype(g) G;
                const auto launch = [&](auto v) {
                    constexpr int V = v.value;
                    o.fill.first = groups * (uint32_t)((p->dim + 64 * V - 1) / (64 * V));
                    const dim3 grid(o.fill.first + zeros);
                    with_ids(p->ids_type, [&](auto i) {
                        hipLaunchKernelGGL((embed_few_kernel<decltype(i), G, P, V>), grid,
                                           dim3(512), 0, s, o, a, (uint32_t)per, groups);
                    });
                };
                constexpr int V = 16 / sizeof(G);
                if (groups + zeros == 0)
                    return;
                if (p->dim >= V)
                    launch(std::integral_constant<int, V>{});
                else
                    launch(std::integral_constant<int, 1>{});
            });
        });
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess)
            return set_error(SMOL_ERR_HIP, "embedding backward launch: %s", hipGetErrorString(e));
        return SMOL_OK;
    }
    const bool rank = p->n <= kRankRows && p->vocab < 1 << (32 - kRankBits);
    int passes = 1;
    while (p->vocab >> passes * kBits)
        ++passes;
    // the zeros, a share with each launch of the sort
    const int launches = rank ? 1 : 2 * passes;
    const int64_t words = (int64_t)p->dim * elem_size(p->grad_type) / 2;
    const bool dense = p->vocab == 1 || p->table_stride == p->dim;
    Fill f;
    f.at = (uint16_t *)p->grad_table;
    f.words = dense ? 0 : words;
    f.stride = p->table_stride * elem_size(p->grad_type) / 2;
    const int64_t units = dense ? (p->vocab * words + 7) / 8 : p->vocab;  // of 8 words, or rows
    int launch = 0;
    // The workgroups of the next launch: `sorting` that sort, and those that
    // write zeros after them, 64 KiB each or more.
    const auto with_fill = [&](unsigned sorting, int threads) {
        const int64_t lo = units * launch / launches, hi = units * (launch + 1) / launches;
        ++launch;
        f.first = o.fill.first = sorting;
        if (p->accumulate || lo == hi)
            return dim3(sorting);
        f.lo = dense ? lo * 8 : lo;
        f.hi = dense ? (hi == units ? p->vocab * words : hi * 8) : hi;
        o.fill = f;
        const int64_t bytes = dense ? (hi - lo) * 16 : (hi - lo) * words * 2;
        const int64_t want = bytes / 65536 + 1, most = 2048 * 256 / threads;
        return dim3(sorting + (unsigned)(want < most ? want : most));
    };
    int at = 0;  // which buffer holds the sorted keys
    if (rank) {
        with_ids(p->ids_type, [&](auto i) {
            const dim3 grid = with_fill((unsigned)((p->n + 15) / 16), 256);
            hipLaunchKernelGGL((embed_rank_kernel<decltype(i)>), grid, dim3(256), 0, s, o);
        });
    } else {
        int64_t per = (p->n + kSortGroups - 1) / kSortGroups;
        per = (per + kSortTile - 1) / kSortTile * kSortTile;
        o.per = (uint32_t)per;
        o.groups = (int32_t)((p->n + per - 1) / per);
        at = 1;
        const dim3 block(kSortThreads);
        const auto grid = [&] { return with_fill((unsigned)o.groups, kSortThreads); };
        for (int pass = 0; pass < passes; ++pass) {
            at ^= 1;
            o.shift = pass * kBits;
            o.key = key[at];
            o.row = row[at];
            o.key_in = key[at ^ 1];
            o.row_in = row[at ^ 1];
            if (pass == 0) {
                with_ids(p->ids_type, [&](auto i) {
                    dim3 g = grid();
                    hipLaunchKernelGGL((embed_count_kernel<decltype(i), true>), g, block, 0, s, o);
                    g = grid();
                    hipLaunchKernelGGL((embed_move_kernel<decltype(i), true>), g, block, 0, s, o);
                });
            } else {
                dim3 g = grid();
                hipLaunchKernelGGL((embed_count_kernel<int32_t, false>), g, block, 0, s, o);
                g = grid();
                hipLaunchKernelGGL((embed_move_kernel<int32_t, false>), g, block, 0, s, o);
            }
        }
    }
    a.key = key[at];
    a.row = row[at];
    with_type(p->grad_type, [&](auto t) {
        typedef decltype(t) P;
        with_type(p->out_type, [&](auto g) {
            typedef decltype(g) G;
            const auto launch = [&](auto v) {  // V columns a lane: 16 bytes of grad_out
                constexpr int V = v.value;
                const dim3 grid((a.pieces + 3) / 4,
                                (unsigned)((p->dim + 64 * V - 1) / (64 * V)));
                hipLaunchKernelGGL((embed_grad_kernel<G, P, V>), grid, dim3(256), 0, s, a);
            };
            constexpr int V = 16 / sizeof(G);
            if (p->dim >= V)
                launch(std::integral_constant<int, V>{});
            else
                launch(std::integral_constant<int, 1>{});
        });
        {
            const auto launch = [&](auto v) {
                constexpr int V = v.value;
                const dim3 grid((a.pieces + 7) / 8,
                                (unsigned)((p->dim + 64 * V - 1) / (64 * V)));
                hipLaunchKernelGGL((embed_join_kernel<P, V>), grid, dim3(512), 0, s, a);
            };
            if (p->dim >= 4)
                launch(std::integral_constant<int, 4>{});
            else
                launch(std::integral_constant<int, 1>{});
        }
    });
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess)
        return set_error(SMOL_ERR_HIP, "embedding backward launch: %s", hipGetErrorString(e));
    return SMOL_OK;
}
