"""The attention operators' definitions in 64 bits, on the CPU, with bounds on
what correct evaluations may differ from them by (conventions as in
tests/tokens_util.py: U32 a rounding in fp32, UNIT one to the type, first order).

Every function returns (value, bound); the rounding of the output itself is
added by tokens_util.close."""
from __future__ import annotations

import math

import torch

from tests.tokens_util import FLUSH, U32, UNIT

U64 = 2.0 ** -53
# the smallest step of fp16, in halves: what a value near zero is off by
STEP = {torch.float32: 0.0, torch.float16: 2.0 ** -25, torch.bfloat16: 0.0}


def frequencies(rot, base=10000.0, scaling="none", factor=1.0, length=0.0, low=1.0, high=32.0):
    f = []
    if scaling == "base" and rot > 2:
        base = base * factor ** (rot / (rot - 2))
    for i in range(rot // 2):
        v = base ** (-2.0 * i / rot)
        if scaling == "linear":
            v /= factor
        if scaling == "parts":
            keep = (v * length / (2 * math.pi) - low) / (high - low)
            keep = min(1.0, max(0.0, keep))
            v = v * keep + v / factor * (1 - keep)
        f.append(v)
    gain = 0.1 * math.log(factor) + 1.0 if scaling == "parts" else 1.0
    return torch.tensor(f, dtype=torch.float64), gain


def pairs_of(dim, rot, interleaved):
    i = torch.arange(rot // 2)
    return (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)


def turn(x, err, positions, freqs, gain, interleaved, back=False):
    """x (..., heads, dim) in 64 bits, off by err at most, turned.

    The angle's turns are exact to 4 U64 of the angle, reduced to at most half a
    turn and rounded to fp32: pi U32 of an angle; cosine and sine of it are off by
    4 U32 at most, gain and its product by 2 U32, the two products and their
    difference by 3: 16 U32 of the pair's magnitudes together."""
    rot = 2 * freqs.numel()
    angle = positions.reshape(-1).double().view(*positions.shape, 1, 1) * freqs
    c, s = angle.cos() * gain, angle.sin() * (-gain if back else gain)
    a, b = pairs_of(x.shape[-1], rot, interleaved)
    y, e = x.clone(), err.clone()
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., b] * c + x[..., a] * s
    size = (x[..., a].abs() + x[..., b].abs()) * abs(gain) * (16 * U32 + 4 * U64 * angle.abs())
    e[..., a] = err[..., a] * c.abs() + err[..., b] * s.abs() + size
    e[..., b] = err[..., b] * c.abs() + err[..., a] * s.abs() + size
    return y, e


def rotate(x, positions, freqs, gain, interleaved, back=False):
    x = x.double()
    return turn(x, torch.zeros_like(x), positions, freqs, gain, interleaved, back)


def rms(x, eps):
    """r = 1 / sqrt(mean x^2 + eps); dim roundings of the sum halve under the root,
    and the mean's factor, eps, root and division add 4."""
    return 1.0 / (x.square().mean(-1, keepdim=True) + eps).sqrt(), (x.shape[-1] / 2 + 4) * U32


def head_norm(x, weight, eps, positions=None, freqs=None, gain=1.0, interleaved=False):
    x = x.double()
    w = torch.ones(x.shape[-1], dtype=torch.float64) if weight is None else weight.double()
    r, er = rms(x, eps)
    y = x * r * w
    err = y.abs() * (er + 2 * U32)
    if freqs is None:
        return y, err
    return turn(y, err, positions, freqs, gain, interleaved)


def head_norm_backward(dy, x, weight, eps, positions=None, freqs=None, gain=1.0,
                       interleaved=False):
    """((dx, bound), (dweight, bound))."""
    dy, x = dy.double(), x.double()
    dim = x.shape[-1]
    w = torch.ones(dim, dtype=torch.float64) if weight is None else weight.double()
    g, eg = dy, torch.zeros_like(dy)
    if freqs is not None:
        g, eg = turn(dy, eg, positions, freqs, gain, interleaved, back=True)
    r, er = rms(x, eps)
    u, xh = g * w, x * r
    eu = eg * w.abs() + u.abs() * U32
    along = (u * xh).mean(-1, keepdim=True)
    size = (u * xh).abs().mean(-1, keepdim=True)
    ealong = (eu * xh.abs()).mean(-1, keepdim=True) + size * (er + (dim + 4) * U32)
    dx = r * (u - xh * along)
    edx = r * (eu + xh.abs() * ealong + (xh * along).abs() * (er + 2 * U32)
               ) + r * (u.abs() + (xh * along).abs()) * (er + 3 * U32)
    dims = tuple(range(x.dim() - 1))
    n = x.numel() // dim
    dw = (g * xh).sum(dims)
    edw = (eg * xh.abs() + (g * xh).abs() * (er + (n + 4) * U32)).sum(dims)
    return (dx, edx), (dw, edw)


def visible(lq, lk, q_length, k_length, causal, window, sinks):
    """(lq, lk) of one sequence."""
    q_length, k_length = min(max(q_length, 0), lq), min(max(k_length, 0), lk)
    i, j = torch.arange(lq)[:, None], torch.arange(lk)[None, :]
    p = k_length - q_length + i
    see = (i < q_length) & (j < k_length)
    if causal:
        see = see & (j <= p)
        if window:
            see = see & ((j > p - window) | (j < sinks))
    return see


def _scores(q, k, scale, see):
    """Scores of one head in 64 bits, and what fp32 evaluations are off by: dim
    products and their sum, then two roundings of the exponent (of terms as large
    as the score and the row's maximum or lse)."""
    s = scale * (q @ k.t())
    err = scale * (q.abs() @ k.abs().t()) * (q.shape[1] + 6) * U32 + 4 * U32 * s.abs()
    return torch.where(see, s, 0.0), torch.where(see, err, 0.0)


def attend(q, k, v, scale=None, causal=True, window=0, sinks=0, q_lengths=None, k_lengths=None):
    """((out, bound), (lse, bound)); the bound of out takes its weights as rounded to
    the type, and is of the sum before out's own rounding."""
    dtype = q.dtype
    unit = 0.0 if dtype == torch.float32 else UNIT[dtype]
    b, lq, h, d = q.shape
    lk, g = k.shape[1:3]
    scale = d ** -0.5 if scale is None else scale
    out, eout = torch.zeros((b, lq, h, d), dtype=torch.float64), torch.zeros(
        (b, lq, h, d), dtype=torch.float64)
    lse = torch.full((b, lq, h), -math.inf, dtype=torch.float64)
    else_ = torch.zeros_like(lse)
    for n in range(b):
        see = visible(lq, lk, lq if q_lengths is None else int(q_lengths[n]),
                      lk if k_lengths is None else int(k_lengths[n]), causal, window, sinks)
        some = see.any(1)
        if not bool(some.any()):
            continue
        for a in range(h):
            kk, vv = (x[n, :, a // (h // g)].double() for x in (k, v))
            # what no row sees takes no part, whatever it holds
            seen = see.any(0)
            kk, vv = (torch.where(seen[:, None], x, 0.0) for x in (kk, vv))
            qq = torch.where(some[:, None], q[n, :, a].double(), 0.0)
            s, es = _scores(qq, kk, scale, see)
            x = s.masked_fill(~see, -math.inf)
            z = torch.where(some, torch.logsumexp(x, 1), 0.0)
            top = torch.where(some, x.amax(1), 0.0)
            p = (x - z[:, None]).exp()
            count = see.sum(1).double()
            # a weight: its score, the exponent's other term, exp2 itself; scaled when
            # the maximum grows, once a tile of 32 at most
            e = (es.amax(1) + (4 * top.abs() + 8 + 3 * (count / 32 + 8)) * U32)
            total = e + count * U32  # of the sum of weights
            rel = (e + total + unit + (count + 4) * U32)[:, None]
            out[n, :, a] = p @ vv
            # (weights are relative to a maximum rounded up to a power of two: their sum is
            # a half at least, so a step of a weight is two of the quotient)
            eout[n, :, a] = (p @ vv.abs()) * rel + (see.double() @ vv.abs()) * 2 * STEP[dtype]
            lse[n, :, a] = torch.where(some, z, -math.inf)
            else_[n, :, a] = total + 4 * U32 * (top.abs() + z.abs() + 1)
    return (out, eout), (lse, else_)


def attend_backward(grad_out, q, k, v, out, lse, rest=None, scale=None, causal=True, window=0,
                    sinks=0, q_lengths=None, k_lengths=None):
    """(grad_q, bound), (grad_k, bound), (grad_v, bound) from the given out, rest and
    lse; p and d rounded to the type (fp16: carried times 2^6)."""
    dtype = q.dtype
    unit = 0.0 if dtype == torch.float32 else UNIT[dtype]
    step = STEP[dtype] / 64
    b, lq, h, d = q.shape
    lk, g = k.shape[1:3]
    scale = d ** -0.5 if scale is None else scale
    dq, dk, dv = (torch.zeros(x.shape, dtype=torch.float64) for x in (q, k, v))
    eq, ek, ev = (torch.zeros(x.shape, dtype=torch.float64) for x in (q, k, v))
    for n in range(b):
        see = visible(lq, lk, lq if q_lengths is None else int(q_lengths[n]),
                      lk if k_lengths is None else int(k_lengths[n]), causal, window, sinks)
        some, seen = see.any(1)[:, None], see.any(0)[:, None]
        if not bool(some.any()):
            continue
        for a in range(h):
            c = a // (h // g)
            kk, vv = (torch.where(seen, x[n, :, c].double(), 0.0) for x in (k, v))
            qq, dy, y = (torch.where(some, x[n, :, a].double(), 0.0) for x in (q, grad_out, out))
            if rest is not None:
                y = y + torch.where(some, rest[n, :, a].double(), 0.0)
            z = torch.where(some[:, 0], lse[n, :, a].double(), 0.0)[:, None]
            s, es = _scores(qq, kk, scale, see)
            p = torch.where(see, (s - z).exp(), 0.0)
            ep = es + 4 * U32 * (s.abs() + z.abs() + 8)  # relative
            dp = dy @ vv.t()
            delta = (dy * y).sum(1, keepdim=True)
            e = (d + 4) * U32 * (dy.abs() @ vv.abs().t()) + (d + 4) * U32 * (
                dy * y).abs().sum(1, keepdim=True) + 2 * U32 * (dp.abs() + delta.abs())
            ds = p * (dp - delta)
            # below FLUSH exp2's result is zero, which leaves p off by FLUSH and d by that
            # times its other factor; so is an operand or a product of the matrix
            # instructions: FLUSH more of d, and of every term of the sums
            eds = p * e + ds.abs() * (ep + 2 * U32 + unit) + step * see + FLUSH * see * (
                (dp - delta).abs() + 1)
            nq, nk = see.sum(1, keepdim=True).double(), see.sum(0)[:, None].double() * (h // g)
            dq[n, :, a] = scale * (ds @ kk)
            eq[n, :, a] = scale * (eds @ kk.abs() + (nq + 4) * U32 * (ds.abs() @ kk.abs())
                                    + nq * FLUSH)
            dk[n, :, c] += scale * (ds.t() @ qq)
            ek[n, :, c] += scale * (eds.t() @ qq.abs() + (nk + 4) * U32 * (ds.abs().t() @ qq.abs())
                                     + nk * FLUSH)
            dv[n, :, c] += p.t() @ dy
            ev[n, :, c] += ((p * (ep + unit)).t() + (step + FLUSH) * see.t()) @ dy.abs() + (
                nk + 4) * U32 * (p.t() @ dy.abs()) + nk * FLUSH
    return (dq, eq), (dk, ek), (dv, ev)
