"""Python binding of the token operators (include/smol_tokens.h): patch
embedding, embedding lookup and layer norm, forward and backward.

Argument marshalling only, as in ``smol``: torch supplies device memory and
the stream, the HIP kernels do the work, and errors of the library raise
``smol.SmolError``. Tensors are device tensors of the current device whose
last dimension is dense; leading dimensions count as rows, and the rows must
lie a constant stride apart. Outputs and workspaces are allocated where they
are not given; a loop keeps its own. The backward functions are plain calls,
not autograd nodes.
"""
from __future__ import annotations

import struct

from . import smol
from .smol import LAYOUT_NCHW, LAYOUT_NHWC, SmolError  # noqa: F401

ELEM_F32 = 0
ELEM_F16 = 1
ELEM_BF16 = 2

IDS_I32 = 0
IDS_I64 = 1

MAX_NORM_DIM = 8192
MAX_EMBED_DIM = 65536
MAX_PATCH_DIM = 65536
MAX_PATCH = 256
MAX_PATCH_VALUES = 262144
MAX_ROWS = 1073741824

# The argument structures of the C ABI, field by field.
_PATCH_SHAPE = struct.Struct("12i")
_PATCH = struct.Struct("12i5Q2q")
_PATCH_GRAD = struct.Struct("12iQ2q5Qq2i")
_EMBED = struct.Struct("3Q4q4ifi2i")
_EMBED_GRAD = struct.Struct("4Q6q4ifi")
_NORM = struct.Struct("8Q5q3if2i")
_NORM_GRAD = struct.Struct("10Q6q4i")

_torch = None
_elems: dict = {}
_ids: dict = {}


def _load():
    global _torch
    if _torch is None:
        smol.lib()
        import torch
        _elems.update({torch.float32: ELEM_F32, torch.float16: ELEM_F16,
                       torch.bfloat16: ELEM_BF16})
        _ids.update({torch.int32: IDS_I32, torch.int64: IDS_I64})
        _torch = torch
    return _torch


def _elem(t, name: str) -> int:
    e = _elems.get(t.dtype)
    if e is None:
        raise ValueError(f"{name}: element type {t.dtype} is not float32, float16 or bfloat16")
    return e


def _here(*tensors) -> None:
    """All tensors lie on the current device."""
    at = _torch.cuda.current_device() if _torch.cuda.is_available() else None
    for t in tensors:
        if t is not None and (not t.is_cuda or t.get_device() != at):
            raise ValueError("tensors must be on the current device")


def _rows(t, dim: int, name: str, rows: int | None = None, dtype=None) -> tuple[int, int]:
    """(rows, row stride) of a tensor whose last dimension is dense."""
    if t.dim() < 1 or dim < 1 or t.shape[-1] != dim:
        raise ValueError(f"{name}: the last dimension must be {dim}, not that of "
                         f"{tuple(t.shape)}")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, not {t.dtype}")
    count = t.numel() // dim
    if rows is not None and count != rows:
        raise ValueError(f"{name}: {count} rows, not {rows}")
    if t.is_contiguous():
        return count, dim
    if dim > 1 and t.stride(-1) != 1:
        raise ValueError(f"{name}: the last dimension must be dense")
    stride, inner = None, 1
    for size, step in zip(reversed(t.shape[:-1]), reversed(t.stride()[:-1])):
        if size == 1:
            continue
        if stride is None:
            stride = step
        elif step != stride * inner:
            raise ValueError(f"{name}: rows do not lie a constant stride apart")
        inner *= size
    return count, dim if stride is None else stride


def _vector(t, dim: int, name: str, dtype) -> int:
    """The address of an optional dense vector."""
    if t is None:
        return 0
    if t.dtype != dtype or t.numel() != dim or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of {dim} elements")
    return t.data_ptr()


def _room(workspace, need: int, device):
    if workspace is None:
        return _torch.empty(max(need, 16), dtype=_torch.uint8, device=device)
    if workspace.dtype != _torch.uint8 or not workspace.is_contiguous() or \
            workspace.numel() < need:
        raise ValueError(f"workspace must be a contiguous uint8 tensor of >= {need} bytes")
    return workspace


def _ptr(t) -> int:
    return 0 if t is None else t.data_ptr()


def _patch_shape(images, patch: int, dim: int, layout: int, dtype) -> tuple:
    if images.dim() != 4 or not images.is_contiguous():
        raise ValueError("images must be a contiguous tensor of four dimensions")
    n, a, b, c = images.shape
    ch, h, w = (a, b, c) if layout == LAYOUT_NCHW else (c, a, b)
    return (n, ch, h, w, patch, dim, layout, _elem(images, "images"), _elems[dtype], 0, 0, 0)


def _weight_shape(weight, images, layout: int) -> tuple[int, int]:
    """(patch, dim) of a projection's weight in the images' layout."""
    if layout not in (LAYOUT_NCHW, LAYOUT_NHWC):
        raise ValueError(f"layout {layout} unknown")
    if weight.dim() != 4 or not weight.is_contiguous() or images.dim() != 4:
        raise ValueError("weight and images must be contiguous tensors of four dimensions")
    d = weight.shape
    ch, p, q = (d[1], d[2], d[3]) if layout == LAYOUT_NCHW else (d[3], d[1], d[2])
    if p != q or ch != images.shape[1 if layout == LAYOUT_NCHW else 3]:
        raise ValueError(f"weight {tuple(d)} does not fit images {tuple(images.shape)}")
    return p, d[0]


def _strides3(t, n: int, tokens: int, dim: int, name: str) -> tuple[int, int]:
    """(image stride, row stride) of an (n, tokens, dim) tensor, dense rows."""
    if tuple(t.shape) != (n, tokens, dim) or (dim > 1 and t.stride(2) != 1):
        raise ValueError(f"{name} must be an ({n}, {tokens}, {dim}) tensor with dense rows")
    return t.stride(0), t.stride(1)


def patch_embed(images, weight, bias=None, pos=None, layout: int = LAYOUT_NCHW, out=None,
                stream=None):
    """Images (n, c, h, w), or (n, h, w, c) with ``LAYOUT_NHWC``, to rows (n,
    tokens, dim) of the weight's type: every patch projected by ``weight``
    (dim, c, p, p), or (dim, p, p, c), plus ``bias`` (dim) and the position
    rows ``pos`` (tokens, dim). ``out`` may be a slice of a longer sequence
    (``smol_patch_embed``)."""
    torch = _load()
    p, dim = _weight_shape(weight, images, layout)
    _elem(weight, "weight")
    dtype = weight.dtype
    shape = _patch_shape(images, p, dim, layout, dtype)
    n, h, w = shape[0], shape[2], shape[3]
    tokens = (h // p) * (w // p)
    if out is None:
        out = torch.empty((n, tokens, dim), dtype=dtype, device=images.device)
    elif out.dtype != dtype:
        raise ValueError(f"out must be {dtype}, not {out.dtype}")
    strides = _strides3(out, n, tokens, dim, "out")
    args = _PATCH.pack(*shape, images.data_ptr(), weight.data_ptr(),
                       _vector(bias, dim, "bias", dtype),
                       _vector(pos, tokens * dim, "pos", dtype), out.data_ptr(), *strides)
    _here(images, weight, bias, pos, out)
    smol._call("smol_patch_embed", args,
               smol._launch_stream(stream, images, weight, bias, pos, out))
    return out


def patch_embed_workspace_bytes(images, grad_weight, dtype, layout: int = LAYOUT_NCHW) -> int:
    """Bytes of workspace of ``patch_embed_backward`` for gradients of type
    ``dtype`` coming in."""
    _load()
    p, dim = _weight_shape(grad_weight, images, layout)
    if dtype not in _elems:
        raise ValueError(f"element type {dtype} is not float32, float16 or bfloat16")
    args = _PATCH_SHAPE.pack(*_patch_shape(images, p, dim, layout, dtype))
    return int(smol.lib().smol_patch_workspace_bytes(args))


def patch_embed_backward(grad_out, images, grad_weight, grad_bias=None, grad_pos=None,
                         layout: int = LAYOUT_NCHW, accumulate: bool = False, workspace=None,
                         stream=None):
    """The projection's gradients from ``grad_out`` (n, tokens, dim): written
    to, or with ``accumulate`` added to, ``grad_weight``, ``grad_bias`` and
    ``grad_pos``, all float32 or all of grad_out's type
    (``smol_patch_embed_backward``). Returns the three."""
    _load()
    p, dim = _weight_shape(grad_weight, images, layout)
    _elem(grad_out, "grad_out")
    grad = _elem(grad_weight, "grad_weight")
    shape = _patch_shape(images, p, dim, layout, grad_out.dtype)
    n, h, w = shape[0], shape[2], shape[3]
    tokens = (h // p) * (w // p)
    strides = _strides3(grad_out, n, tokens, dim, "grad_out")
    need = int(smol.lib().smol_patch_workspace_bytes(_PATCH_SHAPE.pack(*shape)))
    ws = _room(workspace, need, images.device)
    dtype = grad_weight.dtype
    args = _PATCH_GRAD.pack(*shape, grad_out.data_ptr(), *strides, images.data_ptr(),
                            grad_weight.data_ptr(), _vector(grad_bias, dim, "grad_bias", dtype),
                            _vector(grad_pos, tokens * dim, "grad_pos", dtype), ws.data_ptr(),
                            ws.numel(), grad, int(bool(accumulate)))
    _here(grad_out, images, grad_weight, grad_bias, grad_pos, ws)
    smol._call("smol_patch_embed_backward", args,
               smol._launch_stream(stream, grad_out, images, grad_weight, grad_bias, grad_pos,
                                   ws))
    return grad_weight, grad_bias, grad_pos


def _id_type(ids) -> int:
    e = _ids.get(ids.dtype)
    if e is None or not ids.is_contiguous():
        raise ValueError("ids must be a contiguous int32 or int64 tensor")
    return e


def embed(ids, table, scale: float = 1.0, out=None, keep: bool = False, stream=None):
    """Rows ``scale * table[ids]`` (ids.shape + (dim,)); ids outside the table
    give rows of zeros, or with ``keep`` leave their row of ``out`` as it is.
    ``out`` may have another type than the table (``smol_embed``)."""
    torch = _load()
    if table.dim() != 2:
        raise ValueError("table must have two dimensions")
    vocab, dim = table.shape
    n, kind = ids.numel(), _id_type(ids)
    _, table_stride = _rows(table, dim, "table")
    if out is None:
        if keep:
            raise ValueError("keep needs out")
        out = torch.empty((*ids.shape, dim), dtype=table.dtype, device=table.device)
    _, out_stride = _rows(out, dim, "out", n)
    args = _EMBED.pack(ids.data_ptr(), table.data_ptr(), out.data_ptr(), n, vocab, table_stride,
                       out_stride, dim, kind, _elem(table, "table"), _elem(out, "out"), scale,
                       int(bool(keep)), 0, 0)
    _here(ids, table, out)
    smol._call("smol_embed", args, smol._launch_stream(stream, ids, table, out))
    return out


def embed_workspace_bytes(n: int, vocab: int, dim: int) -> int:
    return int(smol.lib().smol_embed_workspace_bytes(n, vocab, dim))


def embed_backward(grad_out, ids, grad_table, scale: float = 1.0, padding: int | None = None,
                   accumulate: bool = False, workspace=None, stream=None):
    """The table's gradient: row v of ``grad_table`` (vocab, dim) becomes, or
    with ``accumulate`` grows by, ``scale`` times the sum of grad_out's rows
    whose id is v; rows of the id ``padding`` count for none
    (``smol_embed_backward``). Any two element types."""
    _load()
    if grad_table.dim() != 2:
        raise ValueError("grad_table must have two dimensions")
    vocab, dim = grad_table.shape
    n, kind = ids.numel(), _id_type(ids)
    _, table_stride = _rows(grad_table, dim, "grad_table")
    _, grad_stride = _rows(grad_out, dim, "grad_out", n)
    ws = _room(workspace, embed_workspace_bytes(n, vocab, dim), grad_table.device)
    args = _EMBED_GRAD.pack(grad_out.data_ptr(), ids.data_ptr(), grad_table.data_ptr(),
                            ws.data_ptr(), ws.numel(), n, vocab, grad_stride, table_stride,
                            -1 if padding is None else padding, dim, kind,
                            _elem(grad_out, "grad_out"), _elem(grad_table, "grad_table"), scale,
                            int(bool(accumulate)))
    _here(grad_out, ids, grad_table, ws)
    smol._call("smol_embed_backward", args,
               smol._launch_stream(stream, grad_out, ids, grad_table, ws))
    return grad_table


def layer_norm(x, weight=None, bias=None, eps: float = 1e-5, residual=None, out=None,
               sum_out=None, mean=None, rstd=None, stats: bool = True, stream=None):
    """Layer norm over the last dimension of ``x``, or of ``x + residual``.

    Returns (out, sum, mean, rstd): the sum x + residual in the type of x
    (None without ``residual``; what the backward pass calls h), and each
    row's statistics in float32 (None with ``stats=False``). ``weight`` and
    ``bias`` are float32 or of x's type. ``out`` or ``sum_out`` may be ``x``
    or ``residual`` itself (``smol_layer_norm``)."""
    torch = _load()
    dim = x.shape[-1] if x.dim() else 0
    kind = _elem(x, "x")
    rows, x_stride = _rows(x, dim, "x")
    if out is None:
        out = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    _, out_stride = _rows(out, dim, "out", rows, x.dtype)
    r_stride = s_stride = 0
    if residual is not None:
        _, r_stride = _rows(residual, dim, "residual", rows, x.dtype)
        if sum_out is None:
            sum_out = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    if sum_out is not None:
        _, s_stride = _rows(sum_out, dim, "sum_out", rows, x.dtype)
    if stats:
        f32 = torch.float32
        if mean is None:
            mean = torch.empty(x.shape[:-1], dtype=f32, device=x.device)
        if rstd is None:
            rstd = torch.empty(x.shape[:-1], dtype=f32, device=x.device)
    w = weight if weight is not None else bias
    weight_kind = ELEM_F32 if w is None else _elem(w, "weight")
    w_dtype = None if w is None else w.dtype
    args = _NORM.pack(x.data_ptr(), _ptr(residual), _vector(weight, dim, "weight", w_dtype),
                      _vector(bias, dim, "bias", w_dtype), out.data_ptr(), _ptr(sum_out),
                      _vector(mean, rows, "mean", torch.float32),
                      _vector(rstd, rows, "rstd", torch.float32), rows, x_stride, r_stride,
                      out_stride, s_stride, dim, kind, weight_kind, eps, 0, 0)
    _here(x, residual, weight, bias, out, sum_out, mean, rstd)
    smol._call("smol_layer_norm", args,
               smol._launch_stream(stream, x, residual, weight, bias, out, sum_out, mean, rstd))
    return out, sum_out, mean, rstd


def layer_norm_workspace_bytes(rows: int, dim: int) -> int:
    return int(smol.lib().smol_norm_workspace_bytes(rows, dim))


def layer_norm_backward(grad_out, h, weight, mean, rstd, grad_x=None, grad_weight=None,
                        grad_bias=None, grad_sum=None, accumulate: bool = False, workspace=None,
                        stream=None):
    """Gradients of ``layer_norm`` from ``grad_out`` (of the output) and
    ``grad_sum`` (of the sum, or None): returns (grad_x, grad_weight,
    grad_bias), the first that of x and of the residual alike. ``h`` is the
    forward pass's sum, or x. ``grad_weight`` and ``grad_bias``, of the
    weight's type, are written to, or with ``accumulate`` added to; None ones
    are not computed (``smol_layer_norm_backward``)."""
    torch = _load()
    dim = h.shape[-1] if h.dim() else 0
    kind = _elem(h, "h")
    rows, h_stride = _rows(h, dim, "h")
    _, g_stride = _rows(grad_out, dim, "grad_out", rows, h.dtype)
    s_stride = 0
    if grad_sum is not None:
        _, s_stride = _rows(grad_sum, dim, "grad_sum", rows, h.dtype)
    if grad_x is None:
        grad_x = torch.empty(h.shape, dtype=h.dtype, device=h.device)
    _, x_stride = _rows(grad_x, dim, "grad_x", rows, h.dtype)
    w = next((t for t in (weight, grad_weight, grad_bias) if t is not None), None)
    weight_kind = ELEM_F32 if w is None else _elem(w, "weight")
    w_dtype = None if w is None else w.dtype
    ws = _room(workspace, layer_norm_workspace_bytes(rows, dim), h.device)
    args = _NORM_GRAD.pack(grad_out.data_ptr(), h.data_ptr(), _ptr(grad_sum),
                           _vector(weight, dim, "weight", w_dtype),
                           _vector(mean, rows, "mean", torch.float32),
                           _vector(rstd, rows, "rstd", torch.float32), grad_x.data_ptr(),
                           _vector(grad_weight, dim, "grad_weight", w_dtype),
                           _vector(grad_bias, dim, "grad_bias", w_dtype), ws.data_ptr(),
                           ws.numel(), rows, g_stride, h_stride, s_stride, x_stride, dim, kind,
                           weight_kind, int(bool(accumulate)))
    _here(grad_out, h, grad_sum, weight, mean, rstd, grad_x, grad_weight, grad_bias, ws)
    smol._call("smol_layer_norm_backward", args,
               smol._launch_stream(stream, grad_out, h, grad_sum, weight, mean, rstd, grad_x,
                                   grad_weight, grad_bias, ws))
    return grad_x, grad_weight, grad_bias
