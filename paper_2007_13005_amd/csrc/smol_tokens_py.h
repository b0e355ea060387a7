// smol_tokens_py.h -- what the Python bindings of the token and attention
// operators share: tensors checked and read in place, streams, errors.
#ifndef SMOL_TOKENS_PY_H
#define SMOL_TOKENS_PY_H

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
    const at::Tensor *written[8];  // no call writes more
    int writes = 0;
};

inline int elem(const at::Tensor &t, const char *name)
{
    switch (t.scalar_type()) {
    case at::kFloat: return SMOL_ELEM_F32;
    case at::kHalf: return SMOL_ELEM_F16;
    case at::kBFloat16: return SMOL_ELEM_BF16;
    default: wrong("%s: element type is not float32, float16 or bfloat16", name);
    }
}

inline const void *ptr(const at::Tensor *t) { return t ? t->const_data_ptr() : nullptr; }

// Rows of `dim` dense elements a constant stride apart; rows < 0: any number.
inline int64_t rows_of(const at::Tensor &t, int64_t dim, const char *name, int64_t rows,
                       int64_t *stride)
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

inline void same_type(const at::Tensor &t, at::ScalarType type, const char *name)
{
    if (t.scalar_type() != type)
        wrong("%s must be %s, not %s", name, c10::toString(type), c10::toString(t.scalar_type()));
}

inline void vector(const at::Tensor *t, int64_t count, at::ScalarType type, const char *name)
{
    if (t && (t->scalar_type() != type || t->numel() != count || !t->is_contiguous()))
        wrong("%s must be a contiguous %s tensor of %lld elements", name, c10::toString(type),
              (long long)count);
}

inline void workspace(const at::Tensor &t, int64_t need)
{
    if (t.scalar_type() != at::kByte || !t.is_contiguous() || t.numel() < need)
        wrong("workspace must be a contiguous uint8 tensor of >= %lld bytes", (long long)need);
}

inline double number(PyObject *o)
{
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred())
        throw Raised();
    return v;
}

inline int64_t integer(PyObject *o)
{
    const int64_t v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred())
        throw Raised();
    return v;
}

inline int32_t small(int64_t v)  // past 32 bits: a size that the library refuses
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
inline void warn_no_graph(const char *call, std::initializer_list<const at::Tensor *> inputs)
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
inline at::ScalarType weight_type(const at::Tensor *a, const at::Tensor *b, const at::Tensor *c,
                                  const char *name = "weight")
{
    const at::Tensor *t = a ? a : b ? b : c;
    if (!t)
        return at::kFloat;
    elem(*t, name);
    return t->scalar_type();
}

inline int elem_of(at::ScalarType type)  // one of the three
{
    return type == at::kFloat ? SMOL_ELEM_F32 : type == at::kHalf ? SMOL_ELEM_F16 : SMOL_ELEM_BF16;
}

}  // namespace

#endif  // SMOL_TOKENS_PY_H
