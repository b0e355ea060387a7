"""The token operators' definitions in 64 bits, on the CPU, with bounds on
what correct evaluations in fp32 may differ from them by.

U32 = 2^-24 is the relative error of one fp32 rounding; a sum of m terms in
any order is within (m - 1) U32 of the sum of magnitudes (first order). Each
bound below counts the roundings of its formula and adds the output's own:
UNIT of the type relative, and half of its smallest subnormal."""
from __future__ import annotations

import torch

U32 = 2.0 ** -24
UNIT = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 2.0 ** -150, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}
# fp32 values below this may count as zero inside a matrix instruction
FLUSH = 2.0 ** -126


def close(got, want, bound, what: str) -> None:
    """|got - want| <= bound + the rounding to got's type, NaN for NaN."""
    got, dtype = got.detach().cpu().double(), got.dtype
    assert got.shape == want.shape, (what, got.shape, want.shape)
    nan = torch.isnan(want)
    assert torch.equal(torch.isnan(got), nan), f"{what}: NaN in other places"
    inf = torch.isinf(want)
    assert torch.equal(got[inf], want[inf]), f"{what}: infinities differ"
    ok = ~(nan | inf)
    # the rounding is of the computed value, at most bound away from the exact one
    room = bound + UNIT[dtype] * (want.abs() + bound) + TINY[dtype]
    off = ((got - want).abs() - room)[ok]
    if off.numel():
        assert bool((off <= 0).all()), f"{what}: past the bound by {float(off.max())}"


def patches(images, p: int, nhwc: bool):
    """(n, tokens, values), the values in the order of a weight row."""
    if nhwc:
        n, h, w, c = images.shape
        th, tw = h // p, w // p
        x = images[:, :th * p, :tw * p].reshape(n, th, p, tw, p, c).permute(0, 1, 3, 2, 4, 5)
    else:
        n, c, h, w = images.shape
        th, tw = h // p, w // p
        x = images[:, :, :th * p, :tw * p].reshape(n, c, th, p, tw, p).permute(0, 2, 4, 1, 3, 5)
    return x.reshape(n, th * tw, c * p * p)


def patch_embed(images, weight, bias, pos, nhwc: bool):
    """(rows, bound): products exact in 64 bits of the rounded pixels; K + 2
    additions, and the products' own rounding where they have one."""
    d = weight.shape[0]
    p = weight.shape[2] if not nhwc else weight.shape[1]
    a = patches(images.to(weight.dtype).double(), p, nhwc)
    w = weight.double().reshape(d, -1).t()
    y, size = a @ w, a.abs() @ w.abs()
    for t in (bias, pos):
        if t is not None:
            y, size = y + t.double(), size + t.double().abs()
    k = a.shape[2]
    return y, 2 * (k + 4) * (U32 * size + FLUSH)


def patch_embed_backward(grad_out, images, p: int, nhwc: bool):
    """((weight, bias, pos), their bounds); weight as (dim, values)."""
    a = patches(images.to(grad_out.dtype).double(), p, nhwc)
    n, t, k = a.shape
    g = grad_out.double()
    d = g.shape[2]
    g2, a2 = g.reshape(n * t, d), a.reshape(n * t, k)
    want = (g2.t() @ a2, g2.sum(0), g.sum(0))
    size = (g2.abs().t() @ a2.abs(), g2.abs().sum(0), g.abs().sum(0))
    m = n * t
    return want, (2 * (m + 4) * (U32 * size[0] + FLUSH), (m + 4) * U32 * size[1],
                  (n + 4) * U32 * size[2])


def embed(ids, table, scale: float, keep=None):
    some = (ids >= 0) & (ids < table.shape[0])
    out = table.double()[torch.where(some, ids, 0).long()] * scale
    other = torch.zeros_like(out) if keep is None else keep.double()
    out = torch.where(some[..., None], out, other)
    return out, 2 * U32 * out.abs() * some[..., None]


def embed_backward(grad_out, ids, vocab: int, scale: float, padding=None, old=None):
    ids = ids.reshape(-1).long()
    g = grad_out.double().reshape(ids.numel(), -1)
    some = (ids >= 0) & (ids < vocab)
    if padding is not None:
        some &= ids != padding
    ids, g = ids[some], g[some]
    want = torch.zeros((vocab, g.shape[1]), dtype=torch.float64).index_add_(0, ids, g) * scale
    size = torch.zeros_like(want).index_add_(0, ids, g.abs()) * abs(scale)
    count = torch.bincount(ids, minlength=vocab).double()[:, None]
    bound = (count + 3) * U32 * size
    if old is not None:
        want, bound = want + old.double(), bound + 2 * U32 * (size + old.double().abs())
    return want, bound


def layer_norm(h, weight, bias, eps: float):
    """((out, mean, rstd), bounds). The mean of d values is off by d + 2
    roundings of their mean magnitude, the sum of squares by as many of itself
    and by the square of the mean's error; the rest are single roundings."""
    h = h.double()
    d = h.shape[-1]
    w = torch.ones(d, dtype=torch.float64) if weight is None else weight.double()
    b = torch.zeros(d, dtype=torch.float64) if bias is None else bias.double()
    mean = h.mean(-1, keepdim=True)
    rstd = 1 / torch.sqrt(((h - mean) ** 2).mean(-1, keepdim=True) + eps)
    xh = (h - mean) * rstd
    roundings = (d + 16) * U32
    off_mean = roundings * h.abs().mean(-1, keepdim=True)
    off_z = (off_mean + 2 * U32 * (h.abs() + mean.abs())) * rstd  # of xh
    off_rstd = rstd * (roundings + (off_z ** 2).mean(-1, keepdim=True) +
                       2 * (off_z * xh.abs()).mean(-1, keepdim=True))
    bound = w.abs() * (off_z + xh.abs() * off_rstd / rstd) + 8 * U32 * ((xh * w).abs() + b.abs())
    return ((xh * w + b, mean[..., 0], rstd[..., 0]),
            (bound, off_mean[..., 0], off_rstd[..., 0]))


def layer_norm_backward(grad_out, h, weight, mean, rstd, grad_sum):
    """((x, weight, bias), bounds), from the statistics as given."""
    h, dy = h.double(), grad_out.double()
    d = h.shape[-1]
    h, dy = h.reshape(-1, d), dy.reshape(-1, d)
    rows = h.shape[0]
    m, r = mean.double().reshape(-1, 1), rstd.double().reshape(-1, 1)
    w = torch.ones(d, dtype=torch.float64) if weight is None else weight.double()
    xh, g = (h - m) * r, dy * w
    size = (h.abs() + m.abs()) * r  # what xh's roundings are relative to
    dx = r * (g - g.mean(-1, keepdim=True) - xh * (g * xh).mean(-1, keepdim=True))
    bound = (d + 24) * U32 * r * (g.abs() + g.abs().mean(-1, keepdim=True) +
                                  size * (g.abs() * size).mean(-1, keepdim=True))
    if grad_sum is not None:
        s = grad_sum.double().reshape(-1, d)
        dx, bound = dx + s, bound + 2 * U32 * s.abs()
    want = (dx, (dy * xh).sum(0), dy.sum(0))
    return want, (bound, (rows + 8) * U32 * (dy.abs() * size).sum(0),
                  (rows + 4) * U32 * dy.abs().sum(0))


def whole(g, *shape, dtype, most: int = 2):
    """Whole numbers -most .. most. Their products, and sums of up to 2^24 /
    most^2 of them in any order, are exact in fp32, so that a sum with a term too
    few or too many cannot pass for rounding."""
    return torch.randint(-most, most + 1, shape, generator=g).to(dtype)


def same(got, want, what: str) -> None:
    """Exactly the 64-bit values, rounded once to got's type."""
    want = want.to(got.dtype)
    assert got.shape == want.shape, (what, got.shape, want.shape)
    assert torch.equal(got, want.to(got.device)), (
        f"{what}: {int((got != want.to(got.device)).sum())} of {want.numel()} values differ")
