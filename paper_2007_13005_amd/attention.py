"""Python binding of the attention operators (include/smol_attention.h): rotary
positions, norms of queries and keys with the rotation in the same pass, and
attention with a window and first tokens that stay visible, forward and
backward, for training, prompts and single tokens.

As ``tokens``: argument marshalling only, plain calls and not autograd nodes
(a forward call with an input that requires grad warns; the backward functions
give the gradients), wrong shapes, types and devices raise ValueError before
anything is called, errors of the library raise ``smol.SmolError``. Tensors are
device tensors of the current device. Heads are the last two dimensions, (...,
heads, dim), with dense values; rows and heads may lie any stride apart, so that
queries, keys and values may be slices of one projection's rows. Outputs and
workspaces are allocated where they are not given; a loop keeps its own.
"""
from __future__ import annotations

import ctypes
import math

from . import smol
from .smol import SmolError  # noqa: F401

ROTARY_NONE = 0
ROTARY_LINEAR = 1
ROTARY_BASE = 2
ROTARY_PARTS = 3
_SCALINGS = {"none": ROTARY_NONE, "linear": ROTARY_LINEAR, "base": ROTARY_BASE,
             "parts": ROTARY_PARTS}

MAX_HEAD_DIM = 256
MAX_ATTEND_DIM = 128
MAX_HEADS = 1024
MAX_ATTEND_BATCH = 65536
MAX_ATTEND_ROWS = 16777216


class RotaryPlan(ctypes.Structure):
    _fields_ = [(name, ctypes.c_double) for name in ("base", "factor", "length", "low", "high")] + [
        ("dim", ctypes.c_int32), ("scaling", ctypes.c_int32)]


_torch = None
_native = None

# in the order in which the native module takes them
_FUNCTIONS = ("smol_rotate", "smol_rotate_backward", "smol_head_norm", "smol_head_norm_backward",
              "smol_head_norm_workspace_bytes", "smol_attend", "smol_attend_workspace_bytes",
              "smol_attend_backward_kept", "smol_attend_backward_workspace_bytes")


def _load():
    """The native module, bound to the library's functions."""
    global _torch, _native
    if _native is None:
        handle = smol.lib()
        import torch
        try:
            from . import _smolattention as native
        except ImportError as e:
            raise RuntimeError("the _smolattention extension is missing: build it with "
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


def rotary_frequencies(dim: int, base: float = 10000.0, scaling: str = "none",
                       factor: float = 1.0, length: float = 0.0, low: float = 1.0,
                       high: float = 32.0, device="cuda"):
    """(freqs, gain): radians a position of each of the dim / 2 rotated pairs, a
    float64 tensor, and the factor of cosines and sines. ``scaling`` for contexts
    longer than those trained on: "none"; "linear" (positions divided by
    ``factor``); "base" (a larger base); "parts" (frequencies of ``high`` turns or
    more within ``length`` positions stay, those of ``low`` or fewer are divided
    by ``factor``) (``smol_rotary_frequencies``)."""
    _load()
    if scaling not in _SCALINGS:
        raise ValueError(f"scaling {scaling!r} is none of {', '.join(_SCALINGS)}")
    if not 0 <= dim <= 1 << 30:
        raise ValueError(f"dim {dim} out of range")
    plan = RotaryPlan(base, factor, length, low, high, dim, _SCALINGS[scaling])
    freqs = (ctypes.c_double * (MAX_HEAD_DIM // 2))()
    gain = ctypes.c_float()
    _done(smol.lib().smol_rotary_frequencies(ctypes.byref(plan), freqs, ctypes.byref(gain)))
    return _torch.tensor(freqs[:dim // 2], dtype=_torch.float64, device=device), gain.value


def rotate(x, positions, freqs, gain: float = 1.0, interleaved: bool = False, out=None,
           stream=None):
    """``x`` (..., heads, dim) with the first 2 * len(freqs) values of each head
    turned, pair i by positions * freqs[i], and scaled by ``gain``; the others
    are copied. Pairs are the two halves of these values, or neighbours with
    ``interleaved``. ``positions`` (integers) has one element a row. ``out`` may be
    ``x`` itself (``smol_rotate``)."""
    native = _native or _load()
    if out is None:
        out = _torch.empty(x.shape, dtype=x.dtype, device=x.device)
    _done(native.rotate(x, positions, freqs, gain, interleaved, out,
                        _stream(stream, x, positions, freqs, out)))
    return out


def rotate_backward(grad_out, positions, freqs, gain: float = 1.0, interleaved: bool = False,
                    grad_x=None, stream=None):
    """The gradient of ``rotate``: ``grad_out`` turned back, ``gain`` included.
    ``grad_x`` may be ``grad_out`` itself (``smol_rotate_backward``)."""
    native = _native or _load()
    if grad_x is None:
        grad_x = _torch.empty(grad_out.shape, dtype=grad_out.dtype, device=grad_out.device)
    _done(native.rotate_backward(grad_out, positions, freqs, gain, interleaved, grad_x,
                                 _stream(stream, grad_out, positions, freqs, grad_x)))
    return grad_x


def head_norm(q, k, q_weight=None, k_weight=None, positions=None, freqs=None, gain: float = 1.0,
              eps: float = 1e-6, interleaved: bool = False, q_out=None, k_out=None, stream=None):
    """(q_out, k_out): each head of ``q`` and ``k`` (..., heads, dim) divided by
    its root mean square, times the weight (dim, float32 or of q's type), then
    rotated as ``rotate`` does (not without ``positions`` and ``freqs``). ``k`` may
    be None; ``q_out`` and ``k_out`` may be ``q`` and ``k`` themselves
    (``smol_head_norm``)."""
    native = _native or _load()
    if q_out is None:
        q_out = _torch.empty(q.shape, dtype=q.dtype, device=q.device)
    if k is not None and k_out is None:
        k_out = _torch.empty(k.shape, dtype=k.dtype, device=k.device)
    _done(native.head_norm(q, k, q_weight, k_weight, positions, freqs, gain, eps, interleaved,
                           q_out, k_out,
                           _stream(stream, q, k, q_weight, k_weight, positions, freqs, q_out,
                                   k_out)))
    return q_out, k_out


def _head_norm_bytes(native, q, k) -> int:
    if q.dim() < 2 or (k is not None and k.dim() < 2):
        raise ValueError("q and k must have dimensions (..., heads, dim)")
    heads, dim = q.shape[-2:]
    return native.head_norm_bytes(math.prod(q.shape[:-2]), heads,
                                  0 if k is None else k.shape[-2], dim)


def head_norm_workspace_bytes(q, k) -> int:
    """Bytes of workspace of ``head_norm_backward`` (0 for shapes out of range)."""
    return _head_norm_bytes(_native or _load(), q, k)


def head_norm_backward(grad_q_out, grad_k_out, q, k, q_weight=None, k_weight=None, positions=None,
                       freqs=None, gain: float = 1.0, eps: float = 1e-6,
                       interleaved: bool = False, grad_q=None, grad_k=None, grad_q_weight=None,
                       grad_k_weight=None, accumulate: bool = False, workspace=None, stream=None):
    """Gradients of ``head_norm``: returns (grad_q, grad_k, grad_q_weight,
    grad_k_weight). The weights', of the weights' type, are written to, or with
    ``accumulate`` added to; None ones are not computed. ``grad_q`` and ``grad_k``
    may be the incoming gradients or ``q`` and ``k`` themselves
    (``smol_head_norm_backward``)."""
    native = _native or _load()
    if grad_q is None:
        grad_q = _torch.empty(q.shape, dtype=q.dtype, device=q.device)
    if k is not None and grad_k is None:
        grad_k = _torch.empty(k.shape, dtype=k.dtype, device=k.device)
    if workspace is None:
        workspace = _room(_head_norm_bytes(native, q, k), q.device)
    _done(native.head_norm_backward(
        grad_q_out, grad_k_out, q, k, q_weight, k_weight, positions, freqs, gain, eps,
        interleaved, grad_q, grad_k, grad_q_weight, grad_k_weight, accumulate, workspace,
        _stream(stream, grad_q_out, grad_k_out, q, k, q_weight, k_weight, positions, freqs,
                grad_q, grad_k, grad_q_weight, grad_k_weight, workspace)))
    return grad_q, grad_k, grad_q_weight, grad_k_weight


def attend_workspace_bytes(q, k, causal: bool = True, window: int = 0, sinks: int = 0) -> int:
    """Bytes of workspace of ``attend`` (0 for shapes that do not fit)."""
    native = _native or _load()
    return native.attend_bytes(q, k, causal, window, sinks)


def attend(q, k, v, scale: float | None = None, causal: bool = True, window: int = 0,
           sinks: int = 0, q_lengths=None, k_lengths=None, out=None, lse=None, rest=None,
           stats: bool = True, workspace=None, stream=None):
    """(out, lse): softmax(scale * q k^T) v of every head, and the logarithm of
    each softmax's sum (float32, (batch, queries, heads); None with
    ``stats=False`` where it is not given).

    ``q`` (batch, queries, heads, dim), ``k`` and ``v`` (batch, keys, kv_heads,
    dim); heads / kv_heads neighbouring query heads share a key head. The queries
    are the last rows of the first ``k_lengths`` keys (all of them if None), of
    ``q_lengths`` queries each (int32 tensors, (batch)), so prompts, pieces of
    prompts and single tokens over a cache are the same call. With ``causal`` a
    query sees no later key, with ``window`` only the last ``window`` keys, its
    own among them, and the first ``sinks``. ``scale`` is 1 / sqrt(dim) unless
    given. Rows that see nothing are zeros.

    ``rest``, if given, gets what rounding took from ``out``: with it
    ``attend_backward`` is exact to its own rounding (``smol_attend``)."""
    native = _native or _load()
    if out is None:
        out = _torch.empty(q.shape, dtype=q.dtype, device=q.device)
    if stats and lse is None:
        lse = _torch.empty(q.shape[:-1], dtype=_torch.float32, device=q.device)
    if workspace is None:
        workspace = _room(native.attend_bytes(q, k, causal, window, sinks), q.device)
    _done(native.attend(q, k, v, scale, causal, window, sinks, q_lengths, k_lengths, out, lse,
                        rest, workspace,
                        _stream(stream, q, k, v, q_lengths, k_lengths, out, lse, rest,
                                workspace)))
    return out, lse


def attend_backward_workspace_bytes(q, k) -> int:
    """Bytes of workspace of ``attend_backward`` (0 for shapes that do not fit)."""
    native = _native or _load()
    return native.attend_backward_bytes(q, k)


def attend_backward(grad_out, q, k, v, out, lse, rest=None, scale: float | None = None,
                    causal: bool = True, window: int = 0, sinks: int = 0, q_lengths=None,
                    k_lengths=None, grad_q=None, grad_k=None, grad_v=None, workspace=None,
                    stream=None):
    """Gradients of ``attend`` from that of ``out``: returns (grad_q, grad_k,
    grad_v), of the matrices' type. ``out``, ``lse`` and ``rest`` are the forward
    call's (``rest`` may be None; they may lie at any strides, heads before rows for
    instance, or dense in another shape), the other arguments the same as there. Rows
    past the lengths get zeros (``smol_attend_backward_kept``)."""
    native = _native or _load()
    if grad_q is None:
        grad_q = _torch.empty(q.shape, dtype=q.dtype, device=q.device)
    if grad_k is None:
        grad_k = _torch.empty(k.shape, dtype=k.dtype, device=k.device)
    if grad_v is None:
        grad_v = _torch.empty(v.shape, dtype=v.dtype, device=v.device)
    if workspace is None:
        workspace = _room(native.attend_backward_bytes(q, k), q.device)
    _done(native.attend_backward(
        grad_out, q, k, v, out, lse, rest, scale, causal, window, sinks, q_lengths, k_lengths,
        grad_q, grad_k, grad_v, workspace,
        _stream(stream, grad_out, q, k, v, out, lse, rest, q_lengths, k_lengths, grad_q, grad_k,
                grad_v, workspace)))
    return grad_q, grad_k, grad_v
