"""Python binding of the token operators (include/smol_tokens.h): patch
embedding, embedding lookup and layer norm, forward and backward.

Argument marshalling only, as in ``smol``: torch supplies device memory and
the stream, the HIP kernels do the work, and errors of the library raise
``smol.SmolError``. Tensors are device tensors of the current device whose
last dimension is dense; leading dimensions count as rows, and the rows must
lie a constant stride apart. Outputs and workspaces are allocated where they
are not given; a loop keeps its own. Wrong shapes, types and devices raise
ValueError before anything is called (the checks are the native module's,
``csrc/smol_tokens_py.cpp``). All are plain calls, not
autograd nodes: a forward call with an input that requires grad warns (unless
grad mode is off, as it is in an autograd function's ``forward``), and the
backward functions give the gradients. Autograd does count the writes to given
buffers, as it does those of torch's own operations.
"""
from __future__ import annotations

import ctypes

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


class PatchShape(ctypes.Structure):
    _fields_ = [(name, ctypes.c_int32) for name in (
        "n", "channels", "height", "width", "patch", "dim", "layout", "image_type", "type")] + [
        ("reserved", ctypes.c_int32 * 3)]


_torch = None
_native = None

# in the order in which the native module takes them
_FUNCTIONS = ("smol_patch_embed", "smol_patch_embed_backward", "smol_patch_workspace_bytes",
              "smol_embed", "smol_embed_backward", "smol_embed_workspace_bytes",
              "smol_layer_norm", "smol_layer_norm_backward", "smol_norm_workspace_bytes")


def _load():
    """The native module, bound to the library's functions."""
    global _torch, _native
    if _native is None:
        handle = smol.lib()
        import torch
        try:
            from . import _smoltokens as native
        except ImportError as e:
            raise RuntimeError("the _smoltokens extension is missing: build it with "
                               "`python -m paper_2007_13005_amd.build`") from e
        native.bind(*[ctypes.cast(getattr(handle, name), ctypes.c_void_p).value
                      for name in _FUNCTIONS])
        _torch, _native = torch, native
    return _native


def _done(status: int) -> None:
    if status != smol.OK:
        smol._check(status)


def _room(need: int, device):
    return _torch.empty(max(need, 16), dtype=_torch.uint8, device=device)


def _stream(stream, *tensors):
    """None for torch's current stream, else the handle of another one."""
    return None if stream is None else smol._launch_stream(stream, *tensors)


def _tokens(images, patch: int, layout: int) -> int:
    h, w = images.shape[2:4] if layout == LAYOUT_NCHW else images.shape[1:3]
    return (h // patch) * (w // patch)


def patch_embed(images, weight, bias=None, pos=None, layout: int = LAYOUT_NCHW, out=None,
                stream=None):
    """Images (n, c, h, w), or (n, h, w, c) with ``LAYOUT_NHWC``, to rows (n,
    tokens, dim) of the weight's type: every patch projected by ``weight``
    (dim, c, p, p), or (dim, p, p, c), plus ``bias`` (dim) and the position
    rows ``pos`` (tokens, dim). ``out`` may be a slice of a longer sequence
    (``smol_patch_embed``)."""
    native = _native or _load()
    if out is None:
        if images.dim() != 4 or weight.dim() != 4 or weight.shape[2] < 1:
            raise ValueError("images and weight must be tensors of four dimensions")
        out = _torch.empty((images.shape[0], _tokens(images, weight.shape[2], layout),
                            weight.shape[0]), dtype=weight.dtype, device=images.device)
    _done(native.patch_embed(images, weight, bias, pos, layout, out,
                             _stream(stream, images, weight, bias, pos, out)))
    return out


def _patch_bytes(images, patch: int, dim: int, dtype, layout: int) -> int:
    types = {_torch.float32: ELEM_F32, _torch.float16: ELEM_F16, _torch.bfloat16: ELEM_BF16}
    if dtype not in types or images.dtype not in types:
        raise ValueError("element types are float32, float16 and bfloat16")
    if images.dim() != 4:
        raise ValueError("images must be a tensor of four dimensions")
    n, a, b, c = images.shape
    ch, h, w = (a, b, c) if layout == LAYOUT_NCHW else (c, a, b)
    shape = PatchShape(n, ch, h, w, patch, dim, layout, types[images.dtype], types[dtype])
    return int(smol.lib().smol_patch_workspace_bytes(ctypes.byref(shape)))


def patch_embed_workspace_bytes(images, grad_weight, dtype, layout: int = LAYOUT_NCHW) -> int:
    """Bytes of workspace of ``patch_embed_backward`` for gradients of type
    ``dtype`` coming in (0 for shapes that do not fit). ``grad_weight`` stands
    for its shape; the weight itself does as well."""
    _load()
    if grad_weight.dim() != 4:
        raise ValueError("grad_weight must be a tensor of four dimensions")
    return _patch_bytes(images, grad_weight.shape[2], grad_weight.shape[0], dtype, layout)


def patch_embed_backward(grad_out, images, grad_weight, grad_bias=None, grad_pos=None,
                         layout: int = LAYOUT_NCHW, accumulate: bool = False, workspace=None,
                         stream=None, patch: int | None = None):
    """The projection's gradients from ``grad_out`` (n, tokens, dim): written
    to, or with ``accumulate`` added to, ``grad_weight``, ``grad_bias`` and
    ``grad_pos``, all float32 or all of grad_out's type; None ones are not
    computed (``smol_patch_embed_backward``). Without ``grad_weight`` (a frozen
    projection) ``patch`` is the patch's side, and of ``images`` only the shape
    and type count. Returns the three."""
    native = _native or _load()
    if workspace is None:
        if grad_weight is not None:
            need = patch_embed_workspace_bytes(images, grad_weight, grad_out.dtype, layout)
        elif patch is None or grad_out.dim() != 3:
            raise ValueError("without grad_weight the patch's side must be given, and grad_out "
                             "must have three dimensions")
        else:
            need = _patch_bytes(images, patch, grad_out.shape[2], grad_out.dtype, layout)
        workspace = _room(need, images.device)
    _done(native.patch_embed_backward(
        grad_out, images, grad_weight, grad_bias, grad_pos, layout, bool(accumulate), workspace,
        _stream(stream, grad_out, images, grad_weight, grad_bias, grad_pos, workspace), patch))
    return grad_weight, grad_bias, grad_pos


def embed(ids, table, scale: float = 1.0, out=None, keep: bool = False, stream=None):
    """Rows ``scale * table[ids]`` (ids.shape + (dim,)); ids outside the table
    give rows of zeros, or with ``keep`` leave their row of ``out`` as it is.
    ``out`` may have another type than the table (``smol_embed``)."""
    native = _native or _load()
    if out is None:
        if keep:
            raise ValueError("keep needs out")
        out = _torch.empty((*ids.shape, *table.shape[1:]), dtype=table.dtype, device=table.device)
    _done(native.embed(ids, table, scale, out, bool(keep), _stream(stream, ids, table, out)))
    return out


def embed_workspace_bytes(n: int, vocab: int, dim: int) -> int:
    return int(smol.lib().smol_embed_workspace_bytes(n, vocab, dim))


def embed_backward(grad_out, ids, grad_table, scale: float = 1.0, padding: int | None = None,
                   accumulate: bool = False, workspace=None, stream=None):
    """The table's gradient: row v of ``grad_table`` (vocab, dim) becomes, or
    with ``accumulate`` grows by, ``scale`` times the sum of grad_out's rows
    whose id is v; rows of the id ``padding`` count for none
    (``smol_embed_backward``). Any two element types."""
    native = _native or _load()
    if workspace is None:
        if grad_table.dim() != 2:
            raise ValueError("grad_table must have two dimensions")
        workspace = _room(embed_workspace_bytes(ids.numel(), *grad_table.shape),
                          grad_table.device)
    _done(native.embed_backward(grad_out, ids, grad_table, scale,
                                -1 if padding is None else padding, bool(accumulate), workspace,
                                _stream(stream, grad_out, ids, grad_table, workspace)))
    return grad_table


def layer_norm(x, weight=None, bias=None, eps: float = 1e-5, residual=None, out=None,
               sum_out=None, mean=None, rstd=None, stats: bool = True, stream=None):
    """Layer norm over the last dimension of ``x``, or of ``x + residual``.

    Returns (out, sum, mean, rstd): the sum x + residual in the type of x
    (None without ``residual`` or ``sum_out``; what the backward pass calls
    h), and each row's statistics in float32 (None with ``stats=False`` where
    they are not given). ``weight`` and ``bias`` are float32 or of x's type.
    ``out`` or ``sum_out`` may be ``x`` or ``residual`` itself
    (``smol_layer_norm``)."""
    native = _native or _load()
    if out is None:
        out = _torch.empty(x.shape, dtype=x.dtype, device=x.device)
    if residual is not None and sum_out is None:
        sum_out = _torch.empty(x.shape, dtype=x.dtype, device=x.device)
    if stats and mean is None:
        mean = _torch.empty(x.shape[:-1], dtype=_torch.float32, device=x.device)
    if stats and rstd is None:
        rstd = _torch.empty(x.shape[:-1], dtype=_torch.float32, device=x.device)
    _done(native.layer_norm(x, weight, bias, eps, residual, out, sum_out, mean, rstd,
                            _stream(stream, x, weight, bias, residual, out, sum_out, mean,
                                    rstd)))
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
    native = _native or _load()
    if grad_x is None:
        grad_x = _torch.empty(h.shape, dtype=h.dtype, device=h.device)
    if workspace is None:
        dim = h.shape[-1] if h.dim() else 0
        workspace = _room(layer_norm_workspace_bytes(h.numel() // dim if dim else 0, dim),
                          h.device)
    _done(native.layer_norm_backward(
        grad_out, h, weight, mean, rstd, grad_x, grad_weight, grad_bias, grad_sum,
        bool(accumulate), workspace,
        _stream(stream, grad_out, h, weight, mean, rstd, grad_x, grad_weight, grad_bias,
                grad_sum, workspace)))
    return grad_x, grad_weight, grad_bias
