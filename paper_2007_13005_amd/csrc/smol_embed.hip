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

// One wave takes kSpans * 64 * V columns of a row, four rows a workgroup.
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
// of kPiece sorted rows are summed by a wave per 64 * V columns, and sums of
// ids that reach over pieces are joined in a second launch. Every sum runs in
// an order that depends on the ids alone.
constexpr int kPiece = 32;
constexpr int kBits = 9, kDigits = 1 << kBits;
constexpr int kSortThreads = 256, kSortRounds = 4;
constexpr int kSortTile = kSortThreads * kSortRounds;
constexpr int kSortGroups = 64;
// Up to this many rows each row's place is counted directly, in one launch:
// the id and the row's number fit one word for vocabularies below 2^19.
constexpr int kRankBits = 13, kRankRows = 1 << kRankBits;

struct SortArgs {
    const void *ids;
    const uint32_t *key_in, *row_in;
    uint32_t *key, *row;
    uint32_t *table;  // [digit][workgroup] counts
    int64_t vocab, padding;
    uint32_t n, per;  // keys, keys a workgroup
    int32_t shift, groups;
};

template <typename I>
__device__ __forceinline__ uint32_t key_of(const SortArgs &a, uint32_t i)
{
    const int64_t id = id_at<I>(a.ids, i);
    return id >= 0 && id < a.vocab && id != a.padding ? (uint32_t)id : (uint32_t)a.vocab;
}

// Every row's place is the number of (key, row) words below its own: 16 rows
// a workgroup, 16 threads a row, each counting every 16th word.
template <typename I>
__global__ void __launch_bounds__(256) embed_rank_kernel(SortArgs a)
{
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
// workgroup's part, then the moves.
template <typename I, bool First>
__global__ void __launch_bounds__(kSortThreads) embed_count_kernel(SortArgs a)
{
    __shared__ uint32_t count[kDigits];
    for (int d = threadIdx.x; d < kDigits; d += kSortThreads)
        count[d] = 0;
    __syncthreads();
    const uint32_t lo = blockIdx.x * a.per, end = lo + a.per, hi = end < a.n ? end : a.n;
    for (uint32_t i = lo + threadIdx.x; i < hi; i += kSortThreads) {
        const uint32_t key = First ? key_of<I>(a, i) : a.key_in[i];
        atomicAdd(&count[key >> a.shift & (kDigits - 1)], 1u);
    }
    __syncthreads();
    for (int d = threadIdx.x; d < kDigits; d += kSortThreads)
        a.table[d * kSortGroups + blockIdx.x] = count[d];
}

template <typename I, bool First>
__global__ void __launch_bounds__(kSortThreads) embed_move_kernel(SortArgs a)
{
    constexpr int kWaves = kSortThreads / 64;
    __shared__ uint32_t base[kDigits];            // next place of each digit
    __shared__ uint32_t count[kWaves][kDigits];   // this tile's, wave by wave
    __shared__ uint32_t sums[kWaves];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    // base[d]: all keys of smaller digits, and of this digit in earlier groups
    uint32_t total[kDigits / kSortThreads], before[kDigits / kSortThreads], sum = 0;
#pragma unroll
    for (int k = 0; k < kDigits / kSortThreads; ++k) {
        const int d = threadIdx.x * (kDigits / kSortThreads) + k;
        uint32_t t = 0, b = 0;
        for (int g = 0; g < a.groups; ++g) {
            const uint32_t c = a.table[d * kSortGroups + g];
            t += c;
            b += g < (int)blockIdx.x ? c : 0;
        }
        total[k] = t;
        before[k] = b;
        sum += t;
    }
    uint32_t scan = sum;
#pragma unroll
    for (int k = 1; k < 64; k <<= 1) {
        const uint32_t up = __shfl_up(scan, k);
        scan += lane >= k ? up : 0;
    }
    if (lane == 63)
        sums[wave] = scan;
    __syncthreads();
    uint32_t start = scan - sum;
    for (int w = 0; w < wave; ++w)
        start += sums[w];
#pragma unroll
    for (int k = 0; k < kDigits / kSortThreads; ++k) {
        base[threadIdx.x * (kDigits / kSortThreads) + k] = start + before[k];
        start += total[k];
    }
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
        for (int d = threadIdx.x; d < kDigits; d += kSortThreads) {
            uint32_t c = 0;
#pragma unroll
            for (int w = 0; w < kWaves; ++w)
                c += count[w][d];
            base[d] += c;
        }
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

template <typename G, typename P, int V>
__global__ void __launch_bounds__(256) embed_grad_kernel(GradArgs a)
{
    constexpr int kAhead = 8;
    const int32_t lane = threadIdx.x & 63;
    const uint32_t piece =
        __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
    if (piece >= a.pieces)
        return;
    const Span<V> c((int32_t)(blockIdx.y * 64 + lane) * V, a.dim);
    const uint32_t lo = piece * kPiece;
    const uint32_t count = a.n - lo < kPiece ? a.n - lo : kPiece;
    // lane p: the piece's p-th key and row; past the rows, a key of no row
    uint32_t key = a.vocab, row = 0;
    if (lane < (int32_t)count) {
        key = a.key[lo + lane];
        row = a.row[lo + lane];
    }
    const uint32_t left = lo > 0 ? a.key[lo - 1] : a.vocab;
    const uint32_t right = lo + kPiece < a.n ? a.key[lo + kPiece] : a.vocab;
    const uint32_t some = __popcll(__ballot(key != a.vocab));  // they come first
    if (some == 0)
        return;
    vec<float, V> sum = (vec<float, V>)0.0f;
    uint32_t id = __builtin_amdgcn_readlane(key, 0);
    bool first = true;
    const auto end_of = [&](bool last) {
        if (first && id == left)
            store_own<float, V>(a.part + (int64_t)piece * 2 * a.dim + c.at, sum, c.lead);
        else if (last && id == right)
            store_own<float, V>(a.part + ((int64_t)piece * 2 + 1) * a.dim + c.at, sum, c.lead);
        else
            write_row<P, V>(a, id, c, sum);
    };
    for (uint32_t p = 0; p < some; p += kAhead) {
        vec<G, V> x[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const uint32_t q = p + u < some ? p + u : some - 1;
            const int64_t r = (uint32_t)__builtin_amdgcn_readlane(row, q);
            x[u] = load<G, V>((const G *)a.grad_out + r * a.grad_stride + c.at);
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (p + u < some) {
                const uint32_t k = __builtin_amdgcn_readlane(key, p + u);
                if (k != id) {
                    end_of(false);
                    first = false;
                    id = k;
                    sum = (vec<float, V>)0.0f;
                }
                sum += to_f32<V, G>(x[u]);
            }
        }
    }
    end_of(some == kPiece);
}

// The wave of the piece in which an id that reaches over pieces begins adds
// the later pieces' sums to its own, in order.
template <typename P, int V>
__global__ void __launch_bounds__(256) embed_join_kernel(GradArgs a)
{
    const int32_t lane = threadIdx.x & 63;
    const uint32_t piece =
        __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
    if (piece + 1 >= a.pieces)
        return;
    const uint32_t lo = piece * kPiece, hi = lo + kPiece;  // hi < n
    const uint32_t id = a.key[hi - 1];
    if (id == a.vocab || a.key[hi] != id)
        return;
    if (lo > 0 && a.key[lo] == id && a.key[lo - 1] == id)
        return;  // begins further left
    const Span<V> c((int32_t)(blockIdx.y * 64 + lane) * V, a.dim);
    const float *part = a.part + c.at;
    vec<float, V> sum = load<float, V>(part + ((int64_t)piece * 2 + 1) * a.dim);
    for (uint32_t q = piece + 1; q < a.pieces;) {
        // how many of the next 64 pieces begin with the id
        const uint32_t at = q + lane;
        const uint64_t more = __ballot(at < a.pieces && a.key[at * kPiece] == id);
        const uint32_t run = more == ~0ull ? 64 : __builtin_ctzll(~more);
#pragma unroll 8
        for (uint32_t k = 0; k < run; ++k)
            sum += load<float, V>(part + (int64_t)(q + k) * 2 * a.dim);
        if (run < 64)
            break;
        q += 64;
    }
    write_row<P, V>(a, id, c, sum);
}

// Zeros in every row.
template <typename P, int V>
__global__ void __launch_bounds__(256) embed_zero_kernel(GradArgs a)
{
    const int32_t lane = threadIdx.x & 63;
    const uint32_t wave = blockIdx.x * 4 + (threadIdx.x >> 6);
    const Span<V> c((int32_t)(blockIdx.y * 64 + lane) * V, a.dim);
    if (c.lead == V)
        return;
    for (uint32_t v = wave; v < a.vocab; v += gridDim.x * 4)
        store<P, V>((P *)a.table + (int64_t)v * a.table_stride + c.at, (vec<P, V>)(P)0.0f);
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

Workspace layout(int64_t n, int32_t dim)
{
    Workspace w;
    w.keys = (n * 4 + 15) / 16 * 16;
    w.table = 4 * w.keys;
    w.part = w.table + kDigits * kSortGroups * 4;
    w.bytes = w.part + (n + kPiece - 1) / kPiece * 2 * dim * 4 + 16;
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
    int at = 0;  // which buffer holds the sorted keys
    if (p->n > 0 && p->n <= kRankRows && p->vocab < 1 << (32 - kRankBits)) {
        with_ids(p->ids_type, [&](auto i) {
            hipLaunchKernelGGL((embed_rank_kernel<decltype(i)>),
                               dim3((unsigned)((p->n + 15) / 16)), dim3(256), 0, s, o);
        });
    } else if (p->n > 0) {
        int64_t per = (p->n + kSortGroups - 1) / kSortGroups;
        per = (per + kSortTile - 1) / kSortTile * kSortTile;
        o.per = (uint32_t)per;
        o.groups = (int32_t)((p->n + per - 1) / per);
        at = 1;
        for (int shift = 0; shift == 0 || p->vocab >> shift; shift += kBits) {
            at ^= 1;
            o.shift = shift;
            o.key = key[at];
            o.row = row[at];
            o.key_in = key[at ^ 1];
            o.row_in = row[at ^ 1];
            const dim3 grid((unsigned)o.groups), block(kSortThreads);
            if (shift == 0) {
                with_ids(p->ids_type, [&](auto i) {
                    hipLaunchKernelGGL((embed_count_kernel<decltype(i), true>), grid, block, 0, s,
                                       o);
                    hipLaunchKernelGGL((embed_move_kernel<decltype(i), true>), grid, block, 0, s,
                                       o);
                });
            } else {
                hipLaunchKernelGGL((embed_count_kernel<int32_t, false>), grid, block, 0, s, o);
                hipLaunchKernelGGL((embed_move_kernel<int32_t, false>), grid, block, 0, s, o);
            }
        }
    }
    GradArgs a;
    a.grad_out = p->grad_out;
    a.key = key[at];
    a.row = row[at];
    a.part = (float *)(ws + w.part);
    a.table = p->grad_table;
    a.grad_stride = p->grad_stride;
    a.table_stride = p->table_stride;
    a.n = (uint32_t)p->n;
    a.vocab = (uint32_t)p->vocab;
    a.pieces = (uint32_t)((p->n + kPiece - 1) / kPiece);
    a.dim = p->dim;
    a.accumulate = p->accumulate;
    a.scale = p->scale;
    with_width(p->dim, [&](auto v) {
        constexpr int V = v.value;
        const unsigned cols = (unsigned)((p->dim + 64 * V - 1) / (64 * V));
        with_type(p->grad_type, [&](auto t) {
            typedef decltype(t) P;
            if (!p->accumulate) {
                const int64_t groups = (p->vocab + 3) / 4;
                hipLaunchKernelGGL((embed_zero_kernel<P, V>),
                                   dim3((unsigned)(groups < 4096 ? groups : 4096), cols),
                                   dim3(256), 0, s, a);
            }
            if (a.pieces == 0)
                return;
            const dim3 grid((a.pieces + 3) / 4, cols);
            with_type(p->out_type, [&](auto g) {
                hipLaunchKernelGGL((embed_grad_kernel<decltype(g), P, V>), grid, dim3(256), 0, s,
                                   a);
            });
            if (a.pieces > 1)
                hipLaunchKernelGGL((embed_join_kernel<P, V>), grid, dim3(256), 0, s, a);
        });
    });
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess)
        return set_error(SMOL_ERR_HIP, "embedding backward launch: %s", hipGetErrorString(e));
    return SMOL_OK;
}
