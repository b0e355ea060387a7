// smol_attention_py.cpp -- the Python binding of the attention operators, as an
// extension module (_smolattention): checks tensors, fills the C ABI's argument
// structures and calls it, as smol_tokens_py.cpp does. Each function takes what
// the function of its name in attention.py takes, all positional.
#include "smol_tokens_py.h"

#include <cmath>
#include <cstring>

#include "smol_attention.h"

namespace {

// The loaded library's functions (bind).
struct Library {
    decltype(&smol_rotate) rotate;
    decltype(&smol_rotate_backward) rotate_backward;
    decltype(&smol_head_norm) norm;
    decltype(&smol_head_norm_backward) norm_backward;
    decltype(&smol_head_norm_workspace_bytes) norm_bytes;
    decltype(&smol_attend) attend;
    decltype(&smol_attend_workspace_bytes) attend_bytes;
    decltype(&smol_attend_backward_kept) attend_backward;
    decltype(&smol_attend_backward_workspace_bytes) attend_backward_bytes;
} lib;

// (..., heads, dim) with dense heads; leading dimensions count as rows, a
// constant stride apart.
struct Heads {
    int64_t rows = 0, heads = 0, dim = 0, row_stride = 0, head_stride = 0;
    Heads() = default;
    Heads(const at::Tensor &t, const char *name)
    {
        if (t.dim() < 2 || t.size(-1) < 1)
            wrong("%s must have dimensions (..., heads, dim)", name);
        dim = t.size(-1);
        heads = t.size(-2);
        if (dim > 1 && t.stride(-1) != 1)
            wrong("%s: the last dimension must be dense", name);
        head_stride = t.stride(-2);
        rows = 1;
        row_stride = heads * dim;
        bool any = false;
        for (int64_t k = t.dim() - 3; k >= 0; --k) {
            if (t.size(k) != 1 && t.numel()) {
                if (!any)
                    row_stride = t.stride(k);
                else if (t.stride(k) != row_stride * rows)
                    wrong("%s: rows do not lie a constant stride apart", name);
                any = true;
            }
            rows *= t.size(k);
        }
    }
    void same(const Heads &o, const char *name) const
    {
        if (rows != o.rows || heads != o.heads || dim != o.dim)
            wrong("%s must have %lld rows of %lld heads of %lld values", name, (long long)o.rows,
                  (long long)o.heads, (long long)o.dim);
    }
};

Heads heads_like(const at::Tensor &t, const Heads &o, at::ScalarType type, const char *name)
{
    same_type(t, type, name);
    const Heads h(t, name);
    h.same(o, name);
    return h;
}

// Positions of `rows` rows.
int positions_type(const at::Tensor &t, int64_t rows)
{
    if (!t.is_contiguous() || (t.scalar_type() != at::kInt && t.scalar_type() != at::kLong) ||
        t.numel() != rows)
        wrong("positions must be a contiguous int32 or int64 tensor of %lld elements",
              (long long)rows);
    return t.scalar_type() == at::kLong ? SMOL_IDS_I64 : SMOL_IDS_I32;
}

int64_t rot_of(const at::Tensor &freqs)
{
    if (freqs.scalar_type() != at::kDouble || freqs.dim() != 1 || !freqs.is_contiguous())
        wrong("freqs must be a contiguous float64 tensor of one dimension");
    return 2 * freqs.numel();
}

int truth(PyObject *o)
{
    const int v = PyObject_IsTrue(o);
    if (v < 0)
        throw Raised();
    return v;
}

// x, positions, freqs, gain, interleaved, out, stream
template <bool Backward>
PyObject *rotation(PyObject *const *o)
{
    Tensors all;
    const char *in = Backward ? "grad_out" : "x", *to = Backward ? "grad_x" : "out";
    const at::Tensor &x = *all.take(o[0], in), &positions = *all.take(o[1], "positions");
    const at::Tensor &freqs = *all.take(o[2], "freqs"), &out = *all.take(o[5], to);
    smol_rotate_args a = {};
    a.type = elem(x, in);
    const Heads h(x, in), y = heads_like(out, h, x.scalar_type(), to);
    a.rows = h.rows;
    a.heads = small(h.heads);
    a.dim = small(h.dim);
    a.x_row_stride = h.row_stride;
    a.x_head_stride = h.head_stride;
    a.out_row_stride = y.row_stride;
    a.out_head_stride = y.head_stride;
    a.rot = small(rot_of(freqs));
    a.positions_type = positions_type(positions, h.rows);
    a.gain = (float)number(o[3]);
    a.interleaved = truth(o[4]);
    all.check_device();
    a.out = all.write(&out);  // first: x may be it
    a.x = ptr(&x);
    a.positions = ptr(&positions);
    a.freqs = (const double *)ptr(&freqs);
    if (!Backward)
        warn_no_graph("rotate", {&x});
    return launch(o[6], all, [&](void *s) {
        return Backward ? lib.rotate_backward(&a, s) : lib.rotate(&a, s);
    });
}

PyObject *rotate(PyObject *const *o) { return rotation<false>(o); }
PyObject *rotate_backward(PyObject *const *o) { return rotation<true>(o); }

// What both directions of the head norm share: shape and positions (both None:
// no rotation).
void fill_shape(Tensors &all, smol_head_shape *s, const Heads &q, const Heads *k,
                PyObject *positions, PyObject *freqs, PyObject *gain, PyObject *eps,
                PyObject *interleaved)
{
    if (k && (k->rows != q.rows || k->dim != q.dim))
        wrong("k must have %lld rows of heads of %lld values", (long long)q.rows,
              (long long)q.dim);
    s->rows = q.rows;
    s->dim = small(q.dim);
    s->gain = (float)number(gain);
    s->eps = (float)number(eps);
    s->interleaved = truth(interleaved);
    const at::Tensor *p = all.take(positions, "positions", true);
    const at::Tensor *f = all.take(freqs, "freqs", true);
    if (!p != !f)
        wrong("positions and freqs go together");
    if (!p)
        return;
    s->rot = small(rot_of(*f));
    s->positions_type = positions_type(*p, q.rows);
    s->positions = ptr(p);
    s->freqs = (const double *)ptr(f);
}

smol_head_side side_of(const Heads &x, const Heads &out)
{
    smol_head_side s = {};
    s.heads = small(x.heads);
    s.x_row_stride = x.row_stride;
    s.x_head_stride = x.head_stride;
    s.out_row_stride = out.row_stride;
    s.out_head_stride = out.head_stride;
    return s;
}

// q, k, q_weight, k_weight, positions, freqs, gain, eps, interleaved, q_out,
// k_out, stream
PyObject *head_norm(PyObject *const *o)
{
    Tensors all;
    const at::Tensor &q = *all.take(o[0], "q"), &q_out = *all.take(o[9], "q_out");
    const at::Tensor *k = all.take(o[1], "k", true), *k_out = all.take(o[10], "k_out", !k);
    const at::Tensor *qw = all.take(o[2], "q_weight", true);
    const at::Tensor *kw = all.take(o[3], "k_weight", true);
    if (!k && (k_out || kw))
        wrong("k_out or k_weight without k");
    smol_head_norm_args a = {};
    a.shape.type = elem(q, "q");
    const Heads hq(q, "q"), yq = heads_like(q_out, hq, q.scalar_type(), "q_out");
    Heads hk, yk;
    if (k) {
        same_type(*k, q.scalar_type(), "k");
        hk = Heads(*k, "k");
        yk = heads_like(*k_out, hk, q.scalar_type(), "k_out");
    }
    fill_shape(all, &a.shape, hq, k ? &hk : nullptr, o[4], o[5], o[6], o[7], o[8]);
    const at::ScalarType w = weight_type(qw, kw, nullptr);
    vector(qw, hq.dim, w, "q_weight");
    vector(kw, hq.dim, w, "k_weight");
    a.shape.weight_type = elem_of(w);
    a.q = side_of(hq, yq);
    a.k = side_of(hk, yk);
    all.check_device();
    a.q.out = all.write(&q_out);  // first: the inputs may be these
    a.k.out = all.write(k_out);
    a.q.x = ptr(&q);
    a.k.x = ptr(k);
    a.q.weight = ptr(qw);
    a.k.weight = ptr(kw);
    warn_no_graph("head_norm", {&q, k, qw, kw});
    return launch(o[11], all, [&](void *s) { return lib.norm(&a, s); });
}

smol_head_grad_side grad_side_of(const Heads &dy, const Heads &x, const Heads &dx)
{
    smol_head_grad_side s = {};
    s.heads = small(x.heads);
    s.grad_out_row_stride = dy.row_stride;
    s.grad_out_head_stride = dy.head_stride;
    s.x_row_stride = x.row_stride;
    s.x_head_stride = x.head_stride;
    s.grad_x_row_stride = dx.row_stride;
    s.grad_x_head_stride = dx.head_stride;
    return s;
}

// grad_q_out, grad_k_out, q, k, q_weight, k_weight, positions, freqs, gain,
// eps, interleaved, grad_q, grad_k, grad_q_weight, grad_k_weight, accumulate,
// workspace, stream
PyObject *head_norm_backward(PyObject *const *o)
{
    Tensors all;
    const at::Tensor &q = *all.take(o[2], "q"), *k = all.take(o[3], "k", true);
    const at::Tensor &dyq = *all.take(o[0], "grad_q_out");
    const at::Tensor *dyk = all.take(o[1], "grad_k_out", !k);
    const at::Tensor *qw = all.take(o[4], "q_weight", true);
    const at::Tensor *kw = all.take(o[5], "k_weight", true);
    const at::Tensor &dq = *all.take(o[11], "grad_q"), *dk = all.take(o[12], "grad_k", !k);
    const at::Tensor *dqw = all.take(o[13], "grad_q_weight", true);
    const at::Tensor *dkw = all.take(o[14], "grad_k_weight", true);
    if (!k && (dyk || dk || kw || dkw))
        wrong("gradients or a weight of k without k");
    smol_head_norm_grad_args a = {};
    a.shape.type = elem(q, "q");
    const at::ScalarType type = q.scalar_type();
    const Heads hq(q, "q"), gq = heads_like(dyq, hq, type, "grad_q_out");
    const Heads xq = heads_like(dq, hq, type, "grad_q");
    Heads hk, gk, xk;
    if (k) {
        same_type(*k, type, "k");
        hk = Heads(*k, "k");
        gk = heads_like(*dyk, hk, type, "grad_k_out");
        xk = heads_like(*dk, hk, type, "grad_k");
    }
    fill_shape(all, &a.shape, hq, k ? &hk : nullptr, o[6], o[7], o[8], o[9], o[10]);
    const at::ScalarType w = weight_type(qw ? qw : kw, dqw, dkw);
    vector(qw, hq.dim, w, "q_weight");
    vector(kw, hq.dim, w, "k_weight");
    vector(dqw, hq.dim, w, "grad_q_weight");
    vector(dkw, hq.dim, w, "grad_k_weight");
    a.shape.weight_type = elem_of(w);
    a.q = grad_side_of(gq, hq, xq);
    a.k = grad_side_of(gk, hk, xk);
    a.accumulate = truth(o[15]);
    const at::Tensor &room = *all.take(o[16], "workspace");
    workspace(room, lib.norm_bytes(hq.rows, a.q.heads, a.k.heads, a.shape.dim));
    all.check_device();
    a.q.grad_x = all.write(&dq);  // first: an input may be it
    a.k.grad_x = all.write(dk);
    a.q.grad_weight = all.write(dqw);
    a.k.grad_weight = all.write(dkw);
    a.workspace = all.write(&room);
    a.workspace_bytes = room.numel();
    a.q.grad_out = ptr(&dyq);
    a.k.grad_out = ptr(dyk);
    a.q.x = ptr(&q);
    a.k.x = ptr(k);
    a.q.weight = ptr(qw);
    a.k.weight = ptr(kw);
    return launch(o[17], all, [&](void *s) { return lib.norm_backward(&a, s); });
}

// rows, q_heads, k_heads, dim
PyObject *head_norm_bytes(PyObject *const *o)
{
    return PyLong_FromLongLong(lib.norm_bytes(integer(o[0]), small(integer(o[1])),
                                              small(integer(o[2])), small(integer(o[3]))));
}

const int32_t *lengths(const at::Tensor *t, int64_t batch, const char *name)
{
    if (t && (t->scalar_type() != at::kInt || t->numel() != batch || !t->is_contiguous()))
        wrong("%s must be a contiguous int32 tensor of %lld elements", name, (long long)batch);
    return (const int32_t *)ptr(t);
}

void four(const at::Tensor &t, const char *name)
{
    if (t.dim() != 4 || (t.size(3) > 1 && t.stride(3) != 1))
        wrong("%s must be a (batch, rows, heads, dim) tensor with dense heads", name);
}

smol_attend_shape shape_of(const at::Tensor &q, const at::Tensor &k)
{
    four(q, "q");
    four(k, "k");
    same_type(k, q.scalar_type(), "k");
    smol_attend_shape s = {};
    s.batch = small(q.size(0));
    s.queries = small(q.size(1));
    s.keys = small(k.size(1));
    s.heads = small(q.size(2));
    s.kv_heads = small(k.size(2));
    s.dim = small(q.size(3));
    s.type = elem(q, "q");
    s.scale = 1.0f;
    if (k.size(0) != q.size(0) || k.size(3) != q.size(3))
        wrong("k must have q's batch %lld and dim %lld", (long long)q.size(0),
              (long long)q.size(3));
    return s;
}

// scale (None: 1 / sqrt(dim)), causal, window, sinks, q_lengths, k_lengths
void fill_mask(Tensors &all, smol_attend_shape *s, PyObject *const *o)
{
    s->scale = o[0] == Py_None ? 1.0f / std::sqrt((float)(s->dim > 0 ? s->dim : 1))
                               : (float)number(o[0]);
    s->causal = truth(o[1]);
    s->window = small(integer(o[2]));
    s->sinks = small(integer(o[3]));
    s->q_lengths = lengths(all.take(o[4], "q_lengths", true), s->batch, "q_lengths");
    s->k_lengths = lengths(all.take(o[5], "k_lengths", true), s->batch, "k_lengths");
}

template <typename M>
M rows_like(const at::Tensor &t, const at::Tensor &like, const char *name)
{
    four(t, name);
    same_type(t, like.scalar_type(), name);
    if (t.sizes() != like.sizes())
        wrong("%s must have %lld x %lld x %lld x %lld elements", name, (long long)like.size(0),
              (long long)like.size(1), (long long)like.size(2), (long long)like.size(3));
    M m = {};
    m.batch_stride = t.stride(0);
    m.row_stride = t.stride(1);
    m.head_stride = t.stride(2);
    return m;
}

// What the forward call wrote for each query and head, on its way back: as many
// elements densely, or the sizes of `like`'s first dimensions (and rest's values,
// dense) at any strides.
void strides_of(const at::Tensor &t, const at::Tensor &like, int64_t dims, at::ScalarType type,
                const char *name, int64_t *batch, int64_t *row, int64_t *head)
{
    const int64_t values = dims == 4 ? like.size(3) : 1;
    const int64_t count = like.size(0) * like.size(1) * like.size(2) * values;
    same_type(t, type, name);
    const bool dense = t.is_contiguous() && t.numel() == count;
    if (!dense && (t.dim() != dims || t.sizes() != like.sizes().slice(0, dims) ||
                   (values > 1 && t.stride(3) != 1)))
        wrong("%s must have q's %s, or %lld elements densely", name,
              dims == 4 ? "sizes with dense heads" : "batch, rows and heads", (long long)count);
    *head = dense ? values : t.stride(2);
    *row = dense ? like.size(2) * values : t.stride(1);
    *batch = dense ? like.size(1) * like.size(2) * values : t.stride(0);
}

// q, k, v, scale, causal, window, sinks, q_lengths, k_lengths, out, lse, rest,
// workspace, stream
PyObject *attend(PyObject *const *o)
{
    Tensors all;
    const at::Tensor &q = *all.take(o[0], "q"), &k = *all.take(o[1], "k");
    const at::Tensor &v = *all.take(o[2], "v"), &out = *all.take(o[9], "out");
    const at::Tensor *lse = all.take(o[10], "lse", true), *rest = all.take(o[11], "rest", true);
    smol_attend_args a = {};
    a.shape = shape_of(q, k);
    fill_mask(all, &a.shape, o + 3);
    a.q = rows_like<smol_attend_rows>(q, q, "q");
    a.k = rows_like<smol_attend_rows>(k, k, "k");
    a.v = rows_like<smol_attend_rows>(v, k, "v");
    a.out = rows_like<smol_attend_out>(out, q, "out");
    vector(lse, q.size(0) * q.size(1) * q.size(2), at::kFloat, "lse");
    vector(rest, q.numel(), q.scalar_type(), "rest");
    const at::Tensor &room = *all.take(o[12], "workspace");
    workspace(room, lib.attend_bytes(&a.shape));
    all.check_device();
    a.out.data = all.write(&out);
    a.lse = (float *)all.write(lse);
    a.rest = all.write(rest);
    a.workspace = all.write(&room);
    a.workspace_bytes = room.numel();
    a.q.data = ptr(&q);
    a.k.data = ptr(&k);
    a.v.data = ptr(&v);
    warn_no_graph("attend", {&q, &k, &v});
    return launch(o[13], all, [&](void *s) { return lib.attend(&a, s); });
}

// q, k, causal, window, sinks
PyObject *attend_bytes(PyObject *const *o)
{
    Tensors all;
    smol_attend_shape s = shape_of(*all.take(o[0], "q"), *all.take(o[1], "k"));
    s.causal = truth(o[2]);
    s.window = small(integer(o[3]));
    s.sinks = small(integer(o[4]));
    return PyLong_FromLongLong(lib.attend_bytes(&s));
}

// grad_out, q, k, v, out, lse, rest, scale, causal, window, sinks, q_lengths,
// k_lengths, grad_q, grad_k, grad_v, workspace, stream
PyObject *attend_backward(PyObject *const *o)
{
    Tensors all;
    const at::Tensor &dy = *all.take(o[0], "grad_out"), &q = *all.take(o[1], "q");
    const at::Tensor &k = *all.take(o[2], "k"), &v = *all.take(o[3], "v");
    const at::Tensor &out = *all.take(o[4], "out"), &lse = *all.take(o[5], "lse");
    const at::Tensor *rest = all.take(o[6], "rest", true);
    const at::Tensor &dq = *all.take(o[13], "grad_q"), &dk = *all.take(o[14], "grad_k");
    const at::Tensor &dv = *all.take(o[15], "grad_v");
    smol_attend_grad_args a = {};
    a.shape = shape_of(q, k);
    fill_mask(all, &a.shape, o + 7);
    a.q = rows_like<smol_attend_rows>(q, q, "q");
    a.k = rows_like<smol_attend_rows>(k, k, "k");
    a.v = rows_like<smol_attend_rows>(v, k, "v");
    a.grad_out = rows_like<smol_attend_rows>(dy, q, "grad_out");
    a.out = rows_like<smol_attend_rows>(out, q, "out");
    a.grad_q = rows_like<smol_attend_out>(dq, q, "grad_q");
    a.grad_k = rows_like<smol_attend_out>(dk, k, "grad_k");
    a.grad_v = rows_like<smol_attend_out>(dv, k, "grad_v");
    smol_attend_kept kept = {};
    strides_of(lse, q, 3, at::kFloat, "lse", &kept.lse_batch_stride, &kept.lse_row_stride,
               &kept.lse_head_stride);
    if (rest)
        strides_of(*rest, q, 4, q.scalar_type(), "rest", &kept.rest_batch_stride,
                   &kept.rest_row_stride, &kept.rest_head_stride);
    const at::Tensor &room = *all.take(o[16], "workspace");
    workspace(room, lib.attend_backward_bytes(&a.shape));
    all.check_device();
    a.grad_q.data = all.write(&dq);
    a.grad_k.data = all.write(&dk);
    a.grad_v.data = all.write(&dv);
    a.workspace = all.write(&room);
    a.workspace_bytes = room.numel();
    a.grad_out.data = ptr(&dy);
    a.q.data = ptr(&q);
    a.k.data = ptr(&k);
    a.v.data = ptr(&v);
    a.out.data = ptr(&out);
    a.rest = ptr(rest);
    a.lse = (const float *)ptr(&lse);
    return launch(o[17], all, [&](void *s) { return lib.attend_backward(&a, &kept, s); });
}

// q, k
PyObject *attend_backward_bytes(PyObject *const *o)
{
    Tensors all;
    const smol_attend_shape s = shape_of(*all.take(o[0], "q"), *all.take(o[1], "k"));
    return PyLong_FromLongLong(lib.attend_backward_bytes(&s));
}

// The addresses of the library's functions, in the order of Library.
PyObject *bind(PyObject *const *o)
{
    void *at[9];
    for (int k = 0; k < 9; ++k)
        if (!(at[k] = PyLong_AsVoidPtr(o[k])))
            wrong("null function address");
    static_assert(sizeof(Library) == sizeof at, "nine functions");
    memcpy((void *)&lib, at, sizeof at);
    Py_RETURN_NONE;
}

#define SMOL_METHOD(name, count)                                                                 \
    {#name, (PyCFunction)(void (*)(void))entry<count, name>, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {SMOL_METHOD(bind, 9),
                         SMOL_METHOD(rotate, 7),
                         SMOL_METHOD(rotate_backward, 7),
                         SMOL_METHOD(head_norm, 12),
                         SMOL_METHOD(head_norm_backward, 18),
                         SMOL_METHOD(head_norm_bytes, 4),
                         SMOL_METHOD(attend, 14),
                         SMOL_METHOD(attend_bytes, 5),
                         SMOL_METHOD(attend_backward, 18),
                         SMOL_METHOD(attend_backward_bytes, 2),
                         {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_smolattention", nullptr, -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__smolattention(void) { return PyModule_Create(&module); }
