// smol_tokens_py.cpp -- the Python binding of the token operators, as an
// extension module (_smoltokens): checks tensors, fills the C ABI's argument
// structures and calls it.
//
// A call of one token's row takes the device less time than a dozen attribute
// lookups take Python; here a tensor's fields are read in place. Each function
// takes what the function of its name in tokens.py takes, all positional, and
// returns the C call's status; a stream of None is torch's current one. Wrong
// arguments raise ValueError before anything is called.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <c10/core/GradMode.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdarg>
#include <cstdio>
#include <exception>
#include <initializer_list>

#include "smol.h"
#include "smol_tokens.h"

namespace {

// The loaded library's functions (bind).
struct Library {
    decltype(&smol_patch_embed) patch;
    decltype(&smol_patch_embed_backward) patch_backward;
    decltype(&smol_patch_workspace_bytes) patch_bytes;
    decltype(&smol_embed) embed;
    decltype(&smol_embed_backward) embed_backward;
    decltype(&smol_embed_workspace_bytes) embed_bytes;
    decltype(&smol_layer_norm) norm;
    decltype(&smol_layer_norm_backward) norm_backward;
    decltype(&smol_norm_workspace_bytes) norm_bytes;
} lib;

struct Raised : std::exception {};  // a Python exception is set

[[noreturn]] void wrong(const char *format, ...)
{
    char text[256];
    va_list args;
    va_start(args, format);
    vsnprintf(text, sizeof text, format, args);
    va_end(args);
    PyErr_SetString(PyExc_ValueError, text);
    throw Raised();
}

// The arguments' tensors, all on one device.
struct Tensors {
    int device = -2;
    // None where it may be: null.
    const at::Tensor *take(PyObject *o, const char *name, bool optional = false)
    {
        if (o == Py_None && optional)
            return nullptr;
        if (!THPVariable_Check(o)) {
            PyErr_Format(PyExc_TypeError, "%s must be a tensor, not %.80s", name,
                         Py_TYPE(o)->tp_name);
            throw Raised();
        }
        const at::Tensor &t = THPVariable_Unpack(o);
        // a lazy negation is not in the memory that the kernels read and write
        if (t.is_neg())
            wrong("%s is a lazily negated view: pass its resolve_neg()", name);
        const int at = t.is_cuda() ? t.get_device() : -1;
        if (device == -2)
            device = at;
        else if (device != at)
            device = -1;
        return &t;
    }
    void check_device() const
    {
        if (device < 0 || device != c10::hip::current_device())
            wrong("tensors must be on the current device");
    }
    // The address of a tensor that the call writes (or null). Asked for as
    // such it gives a lazily cloned tensor memory of its own, which its source
    // then does not share.
    void *write(const at::Tensor *t)
    {
        if (!t)
            return nullptr;
        written[writes++] = t;
        return t->mutable_data_ptr();
    }
    // After the call: autograd counts the writes, and refuses a backward pass
    // that needs what was overwritten. (Inference tensors have no count, and
    // autograd saves none.)
    void count_writes() const
    {
        for (int k = 0; k < writes; ++k)
            if (!written[k]->is_inference())
                written[k]->unsafeGetTensorImpl()->bump_version();
    }

private:
    const at::Tensor *written[4];  // no call writes more
    int writes = 0;
};

int elem(const at::Tensor &t, const char *name)
{
    switch (t.scalar_type()) {
    case at::kFloat: return SMOL_ELEM_F32;
    case at::kHalf: return SMOL_ELEM_F16;
    case at::kBFloat16: return SMOL_ELEM_BF16;
    default: wrong("%s: element type is not float32, float16 or bfloat16", name);
    }
}

const void *ptr(const at::Tensor *t) { return t ? t->const_data_ptr() : nullptr; }

// Rows of `dim` dense elements a constant stride apart; rows < 0: any number.
int64_t rows_of(const at::Tensor &t, int64_t dim, const char *name, int64_t rows, int64_t *stride)
{
    if (t.dim() < 1 || dim < 1 || t.size(-1) != dim)
        wrong("%s: the last dimension must be %lld", name, (long long)dim);
    const int64_t count = t.numel() / dim;
    if (rows >= 0 && count != rows)
        wrong("%s: %lld rows, not %lld", name, (long long)count, (long long)rows);
    *stride = dim;
    if (t.is_contiguous())
        return count;
    if (dim > 1 && t.stride(-1) != 1)
        wrong("%s: the last dimension must be dense", name);
    int64_t inner = 1;
    bool any = false;
    for (int64_t k = t.dim() - 2; k >= 0; --k) {
        if (t.size(k) == 1)
            continue;
        if (!any)
            *stride = t.stride(k);
        else if (t.stride(k) != *stride * inner)
            wrong("%s: rows do not lie a constant stride apart", name);
        any = true;
        inner *= t.size(k);
    }
    return count;
}

void same_type(const at::Tensor &t, at::ScalarType type, const char *name)
{
    if (t.scalar_type() != type)
        wrong("%s must be %s, not %s", name, c10::toString(type), c10::toString(t.scalar_type()));
}

void vector(const at::Tensor *t, int64_t count, at::ScalarType type, const char *name)
{
    if (t && (t->scalar_type() != type || t->numel() != count || !t->is_contiguous()))
        wrong("%s must be a contiguous %s tensor of %lld elements", name, c10::toString(type),
              (long long)count);
}

void workspace(const at::Tensor &t, int64_t need)
{
    if (t.scalar_type() != at::kByte || !t.is_contiguous() || t.numel() < need)
        wrong("workspace must be a contiguous uint8 tensor of >= %lld bytes", (long long)need);
}

double number(PyObject *o)
{
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred())
        throw Raised();
    return v;
}

int64_t integer(PyObject *o)
{
    const int64_t v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred())
        throw Raised();
    return v;
}

int32_t small(int64_t v)  // past 32 bits: a size that the library refuses
{
    return v > INT32_MAX ? INT32_MAX : v < INT32_MIN ? INT32_MIN : (int32_t)v;
}

template <typename F>
PyObject *launch(PyObject *stream, const Tensors &t, F f)
{
    void *s = stream == Py_None
                  ? (void *)c10::hip::getCurrentHIPStream((c10::DeviceIndex)t.device).stream()
                  : PyLong_AsVoidPtr(stream);
    if (!s && PyErr_Occurred())
        throw Raised();
    int status;
    Py_BEGIN_ALLOW_THREADS
    status = f(s);
    Py_END_ALLOW_THREADS
    if (status == SMOL_OK || status == SMOL_ERR_HIP)  // else nothing was enqueued
        t.count_writes();
    return PyLong_FromLong(status);
}

// The forward calls record nothing for autograd: a result that a graph was
// asked for comes with a warning, not in silence.
void warn_no_graph(const char *call, std::initializer_list<const at::Tensor *> inputs)
{
    if (!c10::GradMode::is_enabled())
        return;
    for (const at::Tensor *t : inputs)
        if (t && t->requires_grad()) {
            if (PyErr_WarnFormat(PyExc_UserWarning, 2,
                                 "%s: an input requires grad, and the result has no graph; "
                                 "%s_backward gives the gradients (call under torch.no_grad() or "
                                 "in an autograd function's forward)",
                                 call, call) < 0)
                throw Raised();
            return;
        }
}

// An entry: the number of arguments checked, exceptions turned into Python's.
template <int N, PyObject *(*F)(PyObject *const *)>
PyObject *entry(PyObject *, PyObject *const *args, Py_ssize_t count)
{
    if (count != N) {
        PyErr_Format(PyExc_TypeError, "%d arguments, not %zd", N, count);
        return nullptr;
    }
    try {
        return F(args);
    } catch (const Raised &) {
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    } catch (...) {
        PyErr_SetString(PyExc_RuntimeError, "unknown exception");
    }
    return nullptr;
}

// The type of the weights among those given (float32 where none is).
at::ScalarType weight_type(const at::Tensor *a, const at::Tensor *b, const at::Tensor *c,
                           const char *name = "weight")
{
    const at::Tensor *t = a ? a : b ? b : c;
    if (!t)
        return at::kFloat;
    elem(*t, name);
    return t->scalar_type();
}

int elem_of(at::ScalarType type)  // one of the three
{
    return type == at::kFloat ? SMOL_ELEM_F32 : type == at::kHalf ? SMOL_ELEM_F16 : SMOL_ELEM_BF16;
}

smol_patch_shape shape_of(const at::Tensor &images, int64_t patch, int64_t dim, int64_t layout,
                          int type)
{
    if (layout != 0 && layout != 1)
        wrong("layout %lld unknown", (long long)layout);
    if (images.dim() != 4 || !images.is_contiguous())
        wrong("images must be a contiguous tensor of four dimensions");
    const bool nhwc = layout == 1;
    const auto i = images.sizes();
    smol_patch_shape s = {};
    s.n = small(i[0]);
    s.channels = small(nhwc ? i[3] : i[1]);
    s.height = small(nhwc ? i[1] : i[2]);
    s.width = small(nhwc ? i[2] : i[3]);
    s.patch = small(patch);
    s.dim = small(dim);
    s.layout = (int32_t)layout;
    s.image_type = elem(images, "images");
    s.type = type;
    if (s.patch < 1)
        wrong("a patch's side must be 1 or more");
    return s;
}

smol_patch_shape shape_of(const at::Tensor &images, const at::Tensor &weight, int64_t layout,
                          int type)
{
    if (weight.dim() != 4 || !weight.is_contiguous())
        wrong("weight must be a contiguous tensor of four dimensions");
    const bool nhwc = layout == 1;
    const auto w = weight.sizes();
    const int64_t p = nhwc ? w[1] : w[2], q = nhwc ? w[2] : w[3];
    const smol_patch_shape s = shape_of(images, p, w[0], layout, type);
    if (p != q || (nhwc ? w[3] : w[1]) != images.size(nhwc ? 3 : 1))
        wrong("weight does not fit the images");
    return s;
}

int64_t tokens_of(const smol_patch_shape &s)
{
    return (int64_t)(s.height / s.patch) * (s.width / s.patch);
}

void strides_of(const at::Tensor &t, const smol_patch_shape &s, const char *name,
                int64_t *image_stride, int64_t *row_stride)
{
    const int64_t n = s.n, tokens = tokens_of(s), dim = s.dim;
    if (t.dim() != 3 || t.size(0) != n || t.size(1) != tokens || t.size(2) != dim ||
        (dim > 1 && t.stride(2) != 1))
        wrong("%s must be an (%lld, %lld, %lld) tensor with dense rows", name, (long long)n,
              (long long)tokens, (long long)dim);
    *image_stride = t.stride(0);
    *row_stride = t.stride(1);
}

// images, weight, bias, pos, layout, out, stream
PyObject *patch_embed(PyObject *const *o)
{
    Tensors all;
    const at::Tensor &images = *all.take(o[0], "images"), &weight = *all.take(o[1], "weight");
    const at::Tensor *bias = all.take(o[2], "bias", true), *pos = all.take(o[3], "pos", true);
    smol_patch_args a = {};
    a.shape = shape_of(images, weight, integer(o[4]), elem(weight, "weight"));
    const at::Tensor &out = *all.take(o[5], "out");
    same_type(out, weight.scalar_type(), "out");
    strides_of(out, a.shape, "out", &a.image_stride, &a.row_stride);
    vector(bias, a.shape.dim, weight.scalar_type(), "bias");
    vector(pos, tokens_of(a.shape) * a.shape.dim, weight.scalar_type(), "pos");
    all.check_device();
    a.images = ptr(&images);
    a.weight = ptr(&weight);
    a.bias = ptr(bias);
    a.pos = ptr(pos);
    a.out = all.write(&out);
    warn_no_graph("patch_embed", {&images, &weight, bias, pos});
    return launch(o[6], all, [&](void *s) { return lib.patch(&a, s); });
}

// grad_out, images, grad_weight, grad_bias, grad_pos, layout, accumulate,
// workspace, stream, patch
PyObject *patch_embed_backward(PyObject *const *o)
{
    Tensors all;
    const at::Tensor &grad_out = *all.take(o[0], "grad_out"), &images = *all.take(o[1], "images");
    const at::Tensor *weight = all.take(o[2], "grad_weight", true);
    const at::Tensor *bias = all.take(o[3], "grad_bias", true);
    const at::Tensor *pos = all.take(o[4], "grad_pos", true);
    smol_patch_grad_args a = {};
    const int type = elem(grad_out, "grad_out");
    if (!weight && o[9] == Py_None)
        wrong("without grad_weight the patch's side must be given");
    if (!weight)
        a.shape = shape_of(images, integer(o[9]), grad_out.dim() ? grad_out.size(-1) : 0,
                           integer(o[5]), type);
    else
        a.shape = shape_of(images, *weight, integer(o[5]), type);
    if (o[9] != Py_None && integer(o[9]) != a.shape.patch)
        wrong("patch does not fit grad_weight");
    const at::ScalarType g = weight_type(weight, bias, pos, "a gradient");
    a.grad_type = elem_of(g);
    a.accumulate = (int32_t)integer(o[6]);
    strides_of(grad_out, a.shape, "grad_out", &a.image_stride, &a.row_stride);
    vector(bias, a.shape.dim, g, "grad_bias");
    vector(pos, tokens_of(a.shape) * a.shape.dim, g, "grad_pos");
    const at::Tensor &room = *all.take(o[7], "workspace");
    workspace(room, lib.patch_bytes(&a.shape));
    all.check_device();
    a.grad_out = ptr(&grad_out);
    a.images = ptr(&images);
    a.grad_weight = all.write(weight);
    a.grad_bias = all.write(bias);
    a.grad_pos = all.write(pos);
    a.workspace = all.write(&room);
    a.workspace_bytes = room.numel();
    return launch(o[8], all, [&](void *s) { return lib.patch_backward(&a, s); });
}

int ids_type(const at::Tensor &ids)
{
    if (!ids.is_contiguous() ||
        (ids.scalar_type() != at::kInt && ids.scalar_type() != at::kLong))
        wrong("ids must be a contiguous int32 or int64 tensor");
    return ids.scalar_type() == at::kLong ? SMOL_IDS_I64 : SMOL_IDS_I32;
}

// ids, table, scale, out, keep, stream
PyObject *embed(PyObject *const *o)
{
    Tensors all;
    const at::Tensor &ids = *all.take(o[0], "ids"), &table = *all.take(o[1], "table");
    const at::Tensor &out = *all.take(o[3], "out");
    smol_embed_args a = {};
    a.ids_type = ids_type(ids);
    if (table.dim() != 2)
        wrong("table must have two dimensions");
    a.n = ids.numel();
    a.vocab = rows_of(table, table.size(1), "table", -1, &a.table_stride);
    a.dim = small(table.size(1));
    rows_of(out, a.dim, "out", a.n, &a.out_stride);
    a.table_type = elem(table, "table");
    a.out_type = elem(out, "out");
    a.scale = (float)number(o[2]);
    a.keep = (int32_t)integer(o[4]);
    all.check_device();
    a.ids = ptr(&ids);
    a.table = ptr(&table);
    a.out = all.write(&out);
    warn_no_graph("embed", {&table});
    return launch(o[5], all, [&](void *s) { return lib.embed(&a, s); });
}

// grad_out, ids, grad_table, scale, padding, accumulate, workspace, stream
PyObject *embed_backward(PyObject *const *o)
{
    Tensors all;
    const at::Tensor &grad_out = *all.take(o[0], "grad_out"), &ids = *all.take(o[1], "ids");
    const at::Tensor &table = *all.take(o[2], "grad_table");
    smol_embed_grad_args a = {};
    a.ids_type = ids_type(ids);
    if (table.dim() != 2)
        wrong("grad_table must have two dimensions");
    a.n = ids.numel();
    a.vocab = rows_of(table, table.size(1), "grad_table", -1, &a.table_stride);
    a.dim = small(table.size(1));
    rows_of(grad_out, a.dim, "grad_out", a.n, &a.grad_stride);
    a.out_type = elem(grad_out, "grad_out");
    a.grad_type = elem(table, "grad_table");
    a.scale = (float)number(o[3]);
    a.padding = integer(o[4]);
    a.accumulate = (int32_t)integer(o[5]);
    const at::Tensor &room = *all.take(o[6], "workspace");
    workspace(room, lib.embed_bytes(a.n, a.vocab, a.dim));
    all.check_device();
    a.grad_out = ptr(&grad_out);
    a.ids = ptr(&ids);
    a.grad_table = all.write(&table);
    a.workspace = all.write(&room);
    a.workspace_bytes = room.numel();
    return launch(o[7], all, [&](void *s) { return lib.embed_backward(&a, s); });
}

// x, weight, bias, eps, residual, out, sum_out, mean, rstd, stream
PyObject *layer_norm(PyObject *const *o)
{
    Tensors all;
    const at::Tensor &x = *all.take(o[0], "x"), &out = *all.take(o[5], "out");
    const at::Tensor *weight = all.take(o[1], "weight", true);
    const at::Tensor *bias = all.take(o[2], "bias", true);
    const at::Tensor *residual = all.take(o[4], "residual", true);
    const at::Tensor *sum = all.take(o[6], "sum_out", true);
    const at::Tensor *mean = all.take(o[7], "mean", true), *rstd = all.take(o[8], "rstd", true);
    smol_norm_args a = {};
    a.type = elem(x, "x");
    const int64_t dim = x.dim() ? x.size(-1) : 0;
    a.rows = rows_of(x, dim, "x", -1, &a.x_stride);
    a.dim = small(dim);
    same_type(out, x.scalar_type(), "out");
    rows_of(out, dim, "out", a.rows, &a.out_stride);
    if (residual) {
        same_type(*residual, x.scalar_type(), "residual");
        rows_of(*residual, dim, "residual", a.rows, &a.residual_stride);
    }
    if (sum) {
        same_type(*sum, x.scalar_type(), "sum_out");
        rows_of(*sum, dim, "sum_out", a.rows, &a.sum_stride);
    }
    const at::ScalarType w = weight_type(weight, bias, nullptr);
    vector(weight, dim, w, "weight");
    vector(bias, dim, w, "bias");
    vector(mean, a.rows, at::kFloat, "mean");
    vector(rstd, a.rows, at::kFloat, "rstd");
    a.weight_type = elem_of(w);
    a.eps = (float)number(o[3]);
    all.check_device();
    a.out = all.write(&out);  // first: x and residual may be these
    a.sum = all.write(sum);
    a.mean = (float *)all.write(mean);
    a.rstd = (float *)all.write(rstd);
    a.x = ptr(&x);
    a.residual = ptr(residual);
    a.weight = ptr(weight);
    a.bias = ptr(bias);
    warn_no_graph("layer_norm", {&x, residual, weight, bias});
    return launch(o[9], all, [&](void *s) { return lib.norm(&a, s); });
}

// grad_out, h, weight, mean, rstd, grad_x, grad_weight, grad_bias, grad_sum,
// accumulate, workspace, stream
PyObject *layer_norm_backward(PyObject *const *o)
{
    Tensors all;
    const at::Tensor &grad_out = *all.take(o[0], "grad_out"), &h = *all.take(o[1], "h");
    const at::Tensor *weight = all.take(o[2], "weight", true);
    const at::Tensor *mean = all.take(o[3], "mean"), *rstd = all.take(o[4], "rstd");
    const at::Tensor &grad_x = *all.take(o[5], "grad_x");
    const at::Tensor *grad_weight = all.take(o[6], "grad_weight", true);
    const at::Tensor *grad_bias = all.take(o[7], "grad_bias", true);
    const at::Tensor *grad_sum = all.take(o[8], "grad_sum", true);
    smol_norm_grad_args a = {};
    a.type = elem(h, "h");
    const int64_t dim = h.dim() ? h.size(-1) : 0;
    a.rows = rows_of(h, dim, "h", -1, &a.h_stride);
    a.dim = small(dim);
    same_type(grad_out, h.scalar_type(), "grad_out");
    rows_of(grad_out, dim, "grad_out", a.rows, &a.grad_stride);
    same_type(grad_x, h.scalar_type(), "grad_x");
    rows_of(grad_x, dim, "grad_x", a.rows, &a.x_stride);
    if (grad_sum) {
        same_type(*grad_sum, h.scalar_type(), "grad_sum");
        rows_of(*grad_sum, dim, "grad_sum", a.rows, &a.sum_stride);
    }
    const at::ScalarType w = weight_type(weight, grad_weight, grad_bias);
    vector(weight, dim, w, "weight");
    vector(grad_weight, dim, w, "grad_weight");
    vector(grad_bias, dim, w, "grad_bias");
    vector(mean, a.rows, at::kFloat, "mean");
    vector(rstd, a.rows, at::kFloat, "rstd");
    a.weight_type = elem_of(w);
    a.accumulate = (int32_t)integer(o[9]);
    const at::Tensor &room = *all.take(o[10], "workspace");
    workspace(room, lib.norm_bytes(a.rows, a.dim));
    all.check_device();
    a.grad_x = all.write(&grad_x);  // first: an input may be it
    a.grad_weight = all.write(grad_weight);
    a.grad_bias = all.write(grad_bias);
    a.workspace = all.write(&room);
    a.grad_out = ptr(&grad_out);
    a.h = ptr(&h);
    a.grad_sum = ptr(grad_sum);
    a.weight = ptr(weight);
    a.mean = (const float *)ptr(mean);
    a.rstd = (const float *)ptr(rstd);
    a.workspace_bytes = room.numel();
    return launch(o[11], all, [&](void *s) { return lib.norm_backward(&a, s); });
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
                         SMOL_METHOD(patch_embed, 7),
                         SMOL_METHOD(patch_embed_backward, 10),
                         SMOL_METHOD(embed, 6),
                         SMOL_METHOD(embed_backward, 8),
                         SMOL_METHOD(layer_norm, 10),
                         SMOL_METHOD(layer_norm_backward, 12),
                         {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_smoltokens", nullptr, -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__smoltokens(void) { return PyModule_Create(&module); }
