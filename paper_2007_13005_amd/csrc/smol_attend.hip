// smol_attend.hip -- attention: checks, parts of the keys, launches
// (smol_attend, smol_attend_backward).
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>
#include <initializer_list>

#include "smol.h"
#include "smol_attend.h"
#include "smol_attention.h"
#include "smol_internal.h"

namespace smol {
namespace {

constexpr int64_t kMostColumns = 1 << 30;  // queries times a key head's query heads
constexpr int64_t kMostGroups = (1 << 24) - 1;  // workgroups of 256 threads of a launch

constexpr int64_t kChunkGroups = 512;  // workgroups that run at the same time

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

int check_shape(const smol_attend_shape &s)
{
    if (s.batch < 0 || s.queries < 0 || s.keys < 0 || s.heads < 1 || s.kv_heads < 1 || s.dim < 1)
        return set_error(SMOL_ERR_INVALID_ARG,
                         "batch %d, queries %d, keys %d, heads %d, kv_heads %d or dim %d out of "
                         "range",
                         s.batch, s.queries, s.keys, s.heads, s.kv_heads, s.dim);
    if (s.heads % s.kv_heads)
        return set_error(SMOL_ERR_INVALID_ARG, "%d heads are no multiple of %d kv_heads", s.heads,
                         s.kv_heads);
    if (s.type < SMOL_ELEM_F32 || s.type > SMOL_ELEM_BF16)
        return set_error(SMOL_ERR_INVALID_ARG, "type %d unknown", s.type);
    if (s.causal != 0 && s.causal != 1)
        return set_error(SMOL_ERR_INVALID_ARG, "causal %d is neither 0 nor 1", s.causal);
    if (s.window < 0 || s.sinks < 0 || (!s.causal && (s.window || s.sinks)))
        return set_error(SMOL_ERR_INVALID_ARG,
                         "window %d or sinks %d negative, or given without causal", s.window,
                         s.sinks);
    if (!(s.scale > 0.0f) || isinf(s.scale))
        return set_error(SMOL_ERR_INVALID_ARG, "scale is not positive and finite");
    // (it and its inverse are factors of what is far from 1 too)
    if (s.scale < 0x1p-60f || s.scale > 0x1p60f)
        return set_error(SMOL_ERR_UNSUPPORTED, "scale %g is not within 2^-60 .. 2^60", s.scale);
    if (s.reserved)
        return set_error(SMOL_ERR_INVALID_ARG, "reserved field is not zero");
    if ((uintptr_t)s.q_lengths % 4 || (uintptr_t)s.k_lengths % 4)
        return set_error(SMOL_ERR_INVALID_ARG, "lengths are not aligned to their elements");
    if (s.dim % 8 || s.dim > SMOL_MAX_ATTEND_DIM)
        return set_error(SMOL_ERR_UNSUPPORTED, "dim %d beyond %d or no multiple of 8", s.dim,
                         SMOL_MAX_ATTEND_DIM);
    if (s.batch > SMOL_MAX_ATTEND_BATCH || s.queries > SMOL_MAX_ATTEND_ROWS ||
        s.keys > SMOL_MAX_ATTEND_ROWS || s.heads > SMOL_MAX_HEADS)
        return set_error(SMOL_ERR_UNSUPPORTED,
                         "batch %d beyond %d, queries %d or keys %d beyond %d, or heads %d "
                         "beyond %d",
                         s.batch, SMOL_MAX_ATTEND_BATCH, s.queries, s.keys, SMOL_MAX_ATTEND_ROWS,
                         s.heads, SMOL_MAX_HEADS);
    const int64_t columns = (int64_t)s.queries * (s.heads / s.kv_heads);
    const int64_t pairs = (int64_t)s.batch * s.kv_heads;
    if (columns > kMostColumns || ceil_div(columns, 128) * pairs > kMostGroups ||
        ceil_div(s.keys, 128) * pairs > kMostGroups)
        return set_error(SMOL_ERR_UNSUPPORTED, "too many rows and heads for a launch");
    return SMOL_OK;
}

// Parts of the keys make a workgroup a compute unit (two, where that kernel holds
// two: 28.4 -> 29.7 us for one token over 32768 keys of 8 heads of 128 in fp16, 32
// -> 42 for four over 3000 in fp32, the sums of all parts being written and read;
// 64 tokens over 8192 25 -> 30). A part has 128 keys or more (256: a token over
// 1000 keys 11.2 -> 12.3 us), and up to 512 keys stay whole: the join takes 3 to 4
// us (300 keys: 10.1 us whole, 11 to 12 in parts; 600: 12.6 and 11.2).
constexpr int64_t kSplitGroups = 256, kSplitKeys = 128, kWholeKeys = 512;

// How the forward pass is split.
struct Split {
    bool few;
    int32_t tiles, splits;
};

Split split_of(const smol_attend_shape &s)
{
    Split p;
    const int64_t columns = (int64_t)s.queries * (s.heads / s.kv_heads);
    const int64_t pairs = (int64_t)s.batch * s.kv_heads;
    // a tile of columns that one wave holds: the waves then share the keys
    p.few = columns <= kAttendColumns;
    p.tiles = (int32_t)ceil_div(columns, p.few ? kAttendColumns : kAttendColumns * kAttendWaves);
    int64_t keys = s.keys;
    if (s.causal && s.window)
        keys = std::min<int64_t>(keys, (int64_t)s.window + s.sinks + s.queries);
    const int64_t groups = std::max<int64_t>(1, p.tiles * pairs);
    int64_t splits = std::min<int64_t>(kSplitGroups / groups, ceil_div(keys, kSplitKeys));
    splits = std::max<int64_t>(1, std::min<int64_t>(splits, kAttendSplits));
    if (keys <= kWholeKeys)
        splits = 1;
    p.splits = (int32_t)splits;
    return p;
}

int wide_of(int32_t dim) { return (dim + 31) / 32; }

int64_t part_bytes(const smol_attend_shape &s, const Split &p)
{
    if (p.splits == 1)
        return 0;
    const int64_t rows = (int64_t)s.queries * s.heads * s.batch;
    return p.splits * rows * (wide_of(s.dim) * 32 + 2) * 4;
}

// Parts of the columns of the keys' gradients. They make two workgroups a compute
// unit (four: 4 ragged sequences of 4096 rows 397 -> 443 us, as parts' sums are
// written and read; one: 5906 rows of 8 heads of 96 287 -> 551). A part has 128
// columns or more (512: 1 x 399 rows of 14 heads of 128 over 2 42 -> 52 us, 2 x 148
// of 16 of 80 over 4 24 -> 31), one of a tile of sinks 256 (512: 3 x 271 rows of 32
// heads of 128 over 8, a window of 10, 32 -> 38; 18 x 4422 rows of a head, a window of
// 15, where other workgroups run beside them, 90 -> 88).
constexpr int64_t kTileGroups = 512, kSinkGroups = 256;  // workgroups that parts make
constexpr int64_t kKeyParts = 64;                        // of a tile at most
constexpr int64_t kLeastColumns = 128, kLeastSinkColumns = 256;

// The parts in which the gradients of keys are formed: a tile of 128 keys takes
// the columns of all queries that see it, or a part of them.
struct KeyParts {
    int32_t tiles, sink_tiles;       // of keys; those that hold sinks
    int32_t sink_parts, tile_parts;  // of a tile's columns
    int32_t sink_part, tile_part;    // columns of a part
    int64_t groups, slots;           // workgroups; those that write a part
};

KeyParts key_parts_of(const smol_attend_shape &s)
{
    constexpr int32_t kKeys = kAttendColumns * kAttendWaves;
    KeyParts p;
    const int64_t group = s.heads / s.kv_heads, pairs = (int64_t)s.batch * s.kv_heads;
    const int64_t all = s.queries * group;
    const bool window = s.causal && s.window && s.window < s.keys;
    const int64_t seen =
        window ? std::min<int64_t>(s.queries, (int64_t)s.window + kKeys - 1) * group : all;
    p.tiles = (int32_t)ceil_div(s.keys, kKeys);
    p.sink_tiles = window ? (int32_t)std::min<int64_t>(ceil_div(s.sinks, kKeys), p.tiles) : 0;
    const auto parts = [&](int64_t groups, int64_t tiles, int64_t columns, int64_t least) {
        const int64_t n = std::min(groups / std::max<int64_t>(1, tiles * pairs),
                                   ceil_div(columns, least));
        return (int32_t)std::max<int64_t>(1, std::min<int64_t>(n, kKeyParts));
    };
    p.tile_parts = parts(kTileGroups, p.tiles, seen, kLeastColumns);
    p.tile_part = (int32_t)(ceil_div(ceil_div(seen, p.tile_parts), 32) * 32);
    // those of sinks as long as the others' columns
    p.sink_parts =
        parts(kSinkGroups, p.sink_tiles, all, std::max<int64_t>(p.tile_part, kLeastSinkColumns));
    p.sink_part = (int32_t)(ceil_div(ceil_div(all, p.sink_parts), 32) * 32);
    const int64_t first = (int64_t)p.sink_tiles * p.sink_parts;
    const int64_t rest = (int64_t)(p.tiles - p.sink_tiles) * p.tile_parts;
    p.groups = (first + rest) * pairs;
    // a workgroup's sums stand at its own place
    p.slots = p.tile_parts > 1 ? p.groups : p.sink_parts > 1 ? first * pairs : 0;
    return p;
}

int64_t delta_bytes(const smol_attend_shape &s)
{
    return ((int64_t)s.queries * s.heads * s.batch * 8 + 15) / 16 * 16;
}

// Whatever the mask: the parts that there can be.
int64_t grad_bytes(const smol_attend_shape &s)
{
    const int64_t keys = kAttendColumns * kAttendWaves, group = s.heads / s.kv_heads;
    const int64_t parts = std::min(kKeyParts, ceil_div(s.queries * group, kLeastColumns));
    const int64_t slots = parts > 1 ? std::min(kTileGroups + kSinkGroups,
                                               ceil_div(s.keys, keys) * s.batch * s.kv_heads *
                                                   parts)
                                    : 0;
    return delta_bytes(s) + slots * 2 * keys * wide_of(s.dim) * 32 * 4;
}

// Strides of sequences, rows and heads: those that are read may be 0; what is
// written does not overlap.
int check_rows(const char *name, const void *p, int64_t batch, int64_t rows, int64_t heads,
               const int64_t (&strides)[3], int dim, int type, bool written)
{
    if (!p)
        return set_error(SMOL_ERR_INVALID_ARG, "%s is NULL", name);
    if ((uintptr_t)p % elem_size(type))
        return set_error(SMOL_ERR_INVALID_ARG, "%s is not aligned to its elements", name);
    const int64_t sizes[3] = {batch, rows, heads};
    int order[3] = {0, 1, 2};
    for (int k = 0; k < 3; ++k)
        if (sizes[k] > 1 && (strides[k] < 0 || strides[k] > INT64_MAX / 64 / sizes[k]))
            return set_error(SMOL_ERR_INVALID_ARG, "%s: stride %lld out of range", name,
                             (long long)strides[k]);
    if (!written)
        return SMOL_OK;
    std::sort(order, order + 3, [&](int a, int b) { return strides[a] < strides[b]; });
    int64_t extent = dim;
    for (int k : order) {
        if (sizes[k] <= 1)
            continue;
        if (strides[k] < extent)
            return set_error(SMOL_ERR_INVALID_ARG, "%s: heads or rows overlap", name);
        extent += (sizes[k] - 1) * strides[k];
    }
    return SMOL_OK;
}

template <typename R>
int take(HeadRows *to, const char *name, const R &m, int64_t batch, int64_t rows, int64_t heads,
         int dim, int type, bool written)
{
    to->p = m.data;
    to->batch = m.batch_stride;
    to->row = m.row_stride;
    to->head = m.head_stride;
    if (rows == 0 || batch == 0)
        return SMOL_OK;
    return check_rows(name, m.data, batch, rows, heads,
                      {m.batch_stride, m.row_stride, m.head_stride}, dim, type, written);
}

AttendArgs args_of(const smol_attend_shape &s)
{
    AttendArgs a = {};
    const int32_t group = s.heads / s.kv_heads;
    a.q_lengths = s.q_lengths;
    a.k_lengths = s.k_lengths;
    a.queries = s.queries;
    a.keys = s.keys;
    a.heads = s.heads;
    a.dim = s.dim;
    a.columns = s.queries * group;
    // past all keys a window hides none; nor do more sinks than keys show more
    a.window = s.window < s.keys ? s.window : 0;
    a.sinks = a.window ? std::min(s.sinks, s.keys) : 0;
    a.causal = s.causal;
    a.pairs = s.batch * s.kv_heads;
    a.scale = s.scale;
    a.scale_log2 = (float)(s.scale * 1.44269504088896340736);
    a.per_scale_log2 = 1.0f / a.scale_log2;
    a.group = make_divisor(group);
    a.pair_div = make_divisor(a.pairs);
    a.kv_heads = make_divisor(s.kv_heads);
    a.tile_div = make_divisor(1);
    a.tiles = a.splits = 1;
    return a;
}

// Whether every chunk of 16 bytes is aligned to 16, and `rows` rows of a matrix and
// `heads` of its heads lie within 2^31 bytes.
bool near_rows(const HeadRows &m, int64_t rows, int64_t heads, int type)
{
    const int64_t size = elem_size(type), most = ((int64_t)1 << 31) / size - 256;
    const int64_t any = (int64_t)(uintptr_t)m.p | m.batch * size | m.row * size | m.head * size;
    return any % 16 == 0 && m.row < most / rows && m.head < most / heads &&
           rows * m.row + heads * m.head < most;
}

// The same for rows of keys: what passes the last is told by its offset, so no row
// stands within another.
bool near_keys(const HeadRows &m, int64_t rows, int dim, int type)
{
    return near_rows(m, rows, 1, type) && m.row >= dim;
}

int check_workspace(const void *p, int64_t have, int64_t need)
{
    if (need && (!p || (uintptr_t)p % 16 || have < need))
        return set_error(SMOL_ERR_INVALID_ARG,
                         "workspace must be 16-byte aligned and hold %lld bytes",
                         (long long)need);
    return SMOL_OK;
}

// Whether any of the written matrices stands where another of all does.
int check_apart(std::initializer_list<const void *> written,
                std::initializer_list<const void *> read)
{
    for (auto w = written.begin(); w != written.end(); ++w)
        if (*w && (std::find(w + 1, written.end(), *w) != written.end() ||
                   std::find(read.begin(), read.end(), *w) != read.end()))
            return set_error(SMOL_ERR_INVALID_ARG, "an output stands where another matrix does");
    return SMOL_OK;
}

// Chunks of pairs of `units` workgroups each: 64 images of 197 rows of 16 heads of 64,
// fp16, 33.2 us and their gradients with 12 heads 77.9 (all pairs in one chunk: 37.2
// and 84.5; chunks of 1024 workgroups: 35.9 and 82.9). Workgroups of a causal call
// have unlike lengths, and the longest of all pairs come first (in chunks, gradients
// of 3 x 1376 rows of 16 heads took 153 us for 138).
void set_chunks(AttendArgs *a, int64_t units)
{
    const int64_t chunk =
        a->causal ? a->pairs
                  : std::min<int64_t>(a->pairs,
                                      8 * std::max<int64_t>(1, kChunkGroups / 8 / units));
    a->chunk = make_divisor((uint32_t)chunk);
    a->chunk_last = make_divisor((uint32_t)std::max<int64_t>(1, a->pairs % chunk));
    a->chunk_groups = make_divisor((uint32_t)(chunk * units));
}

int launch(const AttendArgs &a, int kernel, int type, int dim, int64_t grid, void *s)
{
    const bool grad = kernel >= kAttendDelta;
    const auto f = type == SMOL_ELEM_F32   ? grad ? launch_attend_grad_f32 : launch_attend_f32
                   : type == SMOL_ELEM_F16 ? grad ? launch_attend_grad_f16 : launch_attend_f16
                   : grad                  ? launch_attend_grad_bf16
                                           : launch_attend_bf16;
    return f(a, kernel, wide_of(dim), (unsigned)grid, s);
}

}  // namespace
}  // namespace smol

extern "C" int64_t smol_attend_workspace_bytes(const smol_attend_shape *s)
{
    using namespace smol;
    if (!s || check_shape(*s) != SMOL_OK)
        return 0;
    return part_bytes(*s, split_of(*s)) + 16;
}

extern "C" int64_t smol_attend_backward_workspace_bytes(const smol_attend_shape *s)
{
    using namespace smol;
    if (!s || check_shape(*s) != SMOL_OK)
        return 0;
    return grad_bytes(*s) + 16;
}

extern "C" int smol_attend(const smol_attend_args *p, void *stream)
{
    using namespace smol;
    clear_error();
    if (!p)
        return set_error(SMOL_ERR_INVALID_ARG, "args is NULL");
    const smol_attend_shape &s = p->shape;
    int st = check_shape(s);
    if (st != SMOL_OK)
        return st;
    if (s.batch == 0 || s.queries == 0)
        return SMOL_OK;
    AttendArgs a = args_of(s);
    if ((st = take(&a.q, "q", p->q, s.batch, s.queries, s.heads, s.dim, s.type, false)) !=
            SMOL_OK ||
        (st = take(&a.k, "k", p->k, s.batch, s.keys, s.kv_heads, s.dim, s.type, false)) !=
            SMOL_OK ||
        (st = take(&a.v, "v", p->v, s.batch, s.keys, s.kv_heads, s.dim, s.type, false)) !=
            SMOL_OK ||
        (st = take(&a.out, "out", p->out, s.batch, s.queries, s.heads, s.dim, s.type, true)) !=
            SMOL_OK)
        return st;
    if ((uintptr_t)p->lse % 4 || (uintptr_t)p->rest % elem_size(s.type))
        return set_error(SMOL_ERR_INVALID_ARG, "lse or rest is not aligned to its elements");
    const Split split = split_of(s);
    if ((st = check_workspace(p->workspace, p->workspace_bytes, part_bytes(s, split))) !=
            SMOL_OK ||
        (st = check_apart({p->out.data, p->lse, p->rest},
                          {p->q.data, s.keys ? p->k.data : nullptr,
                           s.keys ? p->v.data : nullptr})) != SMOL_OK)
        return st;
    a.direct_keys = near_keys(a.k, kAttendKeys, s.dim, s.type) &&
                    near_keys(a.v, kAttendKeys, s.dim, s.type);
    a.lse = p->lse;
    a.rest = p->rest;
    a.part = (float *)p->workspace;
    a.tiles = split.tiles;
    a.tile_div = make_divisor(split.tiles);
    a.splits = split.splits;
    a.split_div = make_divisor(split.splits);
    set_chunks(&a, (int64_t)split.tiles * split.splits);
    int e = launch(a, split.few ? kAttendFew : kAttendMany, s.type, s.dim,
                   (int64_t)split.tiles * a.pairs * split.splits, stream);
    if (e == hipSuccess && split.splits > 1)
        e = launch(a, kAttendJoin, s.type, s.dim,
                   split.splits <= kAttendJoinParts
                       ? ceil_div((int64_t)a.pairs * a.columns, kAttendWaves)
                       : (int64_t)a.pairs * a.columns,
                   stream);
    if (e != hipSuccess)
        return set_error(SMOL_ERR_HIP, "attention launch: %s", hipGetErrorString((hipError_t)e));
    return SMOL_OK;
}

namespace smol {
namespace {

// kept: the strides of lse and rest, or null: dense.
int attend_backward(const smol_attend_grad_args *p, const smol_attend_kept *kept, void *stream)
{
    const smol_attend_shape &s = p->shape;
    int st = check_shape(s);
    if (st != SMOL_OK)
        return st;
    if (s.batch == 0 || (s.queries == 0 && s.keys == 0))
        return SMOL_OK;
    AttendArgs a = args_of(s);
    const auto of_queries = [&](HeadRows *to, const char *name, const auto &m, bool written) {
        return take(to, name, m, s.batch, s.queries, s.heads, s.dim, s.type, written);
    };
    const auto of_keys = [&](HeadRows *to, const char *name, const auto &m, bool written) {
        return take(to, name, m, s.batch, s.keys, s.kv_heads, s.dim, s.type, written);
    };
    if ((st = of_queries(&a.dout, "grad_out", p->grad_out, false)) != SMOL_OK ||
        (st = of_queries(&a.q, "q", p->q, false)) != SMOL_OK ||
        (st = of_keys(&a.k, "k", p->k, false)) != SMOL_OK ||
        (st = of_keys(&a.v, "v", p->v, false)) != SMOL_OK ||
        (st = of_queries(&a.out, "out", p->out, false)) != SMOL_OK ||
        (st = of_queries(&a.dq, "grad_q", p->grad_q, true)) != SMOL_OK ||
        (st = of_keys(&a.dk, "grad_k", p->grad_k, true)) != SMOL_OK ||
        (st = of_keys(&a.dv, "grad_v", p->grad_v, true)) != SMOL_OK)
        return st;
    const smol_attend_kept dense = {(int64_t)s.queries * s.heads, s.heads, 1,
                                    (int64_t)s.queries * s.heads * s.dim,
                                    (int64_t)s.heads * s.dim, s.dim};
    const smol_attend_kept &at = kept ? *kept : dense;
    const smol_attend_rows lse = {p->lse, at.lse_batch_stride, at.lse_row_stride,
                                  at.lse_head_stride};
    const smol_attend_rows rest = {p->rest, at.rest_batch_stride, at.rest_row_stride,
                                   at.rest_head_stride};
    if ((st = take(&a.lse_in, "lse", lse, s.batch, s.queries, s.heads, 1, SMOL_ELEM_F32,
                   false)) != SMOL_OK ||
        (p->rest && (st = of_queries(&a.rest_in, "rest", rest, false)) != SMOL_OK))
        return st;
    const auto of = [](int32_t rows, const void *x) { return rows ? x : nullptr; };
    if ((st = check_workspace(p->workspace, p->workspace_bytes, grad_bytes(s))) != SMOL_OK ||
        (st = check_apart({of(s.queries, p->grad_q.data), of(s.keys, p->grad_k.data),
                           of(s.keys, p->grad_v.data)},
                          {of(s.queries, p->grad_out.data), of(s.queries, p->q.data),
                           of(s.keys, p->k.data), of(s.keys, p->v.data),
                           of(s.queries, p->out.data), p->rest, p->lse})) != SMOL_OK)
        return st;
    const KeyParts parts = key_parts_of(s);
    a.tiles = (int32_t)ceil_div(a.columns, kAttendColumns * kAttendWaves);
    const int64_t key_groups = s.keys > 0 ? parts.groups : 0;
    const int64_t groups = key_groups + (int64_t)a.tiles * a.pairs;
    if (groups > kMostGroups)
        return set_error(SMOL_ERR_UNSUPPORTED, "too many rows and heads for a launch");
    // (keys of a workgroup; queries of 32 columns)
    a.direct_keys = near_keys(a.k, 128, s.dim, s.type) && near_keys(a.v, 128, s.dim, s.type);
    a.direct_rows = near_rows(a.q, 33, a.group.d, s.type) &&
                    near_rows(a.dout, 33, a.group.d, s.type);
    a.lse_delta = (float *)p->workspace;
    a.part = (float *)((char *)p->workspace + delta_bytes(s));
    a.sink_tiles = parts.sink_tiles;
    a.sink_part = parts.sink_part;
    a.tile_part = parts.tile_part;
    a.sink_div = make_divisor(parts.sink_parts);
    a.tile_div = make_divisor(parts.tile_parts);
    a.key_units = (uint32_t)(key_groups / a.pairs);
    set_chunks(&a, groups / a.pairs);
    int e = hipSuccess;
    if (s.queries > 0) {
        const int64_t lanes = attend_delta_lanes(wide_of(s.dim));
        const int64_t delta_groups = ceil_div(
            (int64_t)s.batch * s.queries * s.heads * lanes, 64 * kAttendWaves);
        a.delta_groups = (uint32_t)delta_groups;
        a.batch = s.batch;
        a.heads_div = make_divisor(s.heads);
        a.queries_div = make_divisor(s.queries);
        e = launch(a, kAttendDelta, s.type, s.dim, std::min(delta_groups, kMostGroups), stream);
    }
    if (e == hipSuccess)
        e = launch(a, kAttendGrad, s.type, s.dim, groups, stream);
    const int64_t joined = s.keys == 0            ? 0
                           : parts.tile_parts > 1 ? parts.tiles
                           : parts.sink_parts > 1 ? parts.sink_tiles
                                                  : 0;
    if (e == hipSuccess && joined)
        e = launch(a, kAttendGradJoin, s.type, s.dim,
                   joined * (kAttendColumns * kAttendWaves / kAttendJoinKeys) * a.pairs, stream);
    if (e != hipSuccess)
        return set_error(SMOL_ERR_HIP, "attention backward launch: %s",
                         hipGetErrorString((hipError_t)e));
    return SMOL_OK;
}

}  // namespace
}  // namespace smol

extern "C" int smol_attend_backward(const smol_attend_grad_args *p, void *stream)
{
    using namespace smol;
    clear_error();
    if (!p)
        return set_error(SMOL_ERR_INVALID_ARG, "args is NULL");
    return attend_backward(p, nullptr, stream);
}

extern "C" int smol_attend_backward_kept(const smol_attend_grad_args *p,
                                         const smol_attend_kept *kept, void *stream)
{
    using namespace smol;
    clear_error();
    if (!p || !kept)
        return set_error(SMOL_ERR_INVALID_ARG, "args or kept is NULL");
    return attend_backward(p, kept, stream);
}
