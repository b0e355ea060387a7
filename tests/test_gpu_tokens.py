"""The token operators on the GPU against their definitions in 64 bits
(tests/tokens_util.py, with the bounds derived there): types, layouts, sizes
from one value on, odd sizes, strides, misaligned and overlapping-free
outputs, ids that name no token, accumulation, other streams, graphs, offsets
past 32 bits, and gradients against differences."""
from __future__ import annotations

import pytest
import torch

from paper_2007_13005_amd import tokens
from tests import tokens_util as ref
from tests.gpu_util import note

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
SENTINEL = -77.0


def gen(seed: int) -> torch.Generator:
    return torch.Generator().manual_seed(seed)


def randn(g, *shape, dtype=F32, scale=1.0):
    return (torch.randn(shape, generator=g) * scale).to(dtype)


def dev(t, stride: int | None = None, skew: int = 0):
    """t on the device; with `stride`, as rows that far apart in a buffer of
    sentinels, `skew` elements past its start. Returns the tensor alone."""
    if t is None:
        return None
    if stride is None and skew == 0:
        return t.cuda()
    d = t.shape[-1]
    rows = t.numel() // d
    stride = stride or d
    buf = torch.full((skew + rows * stride + 8,), SENTINEL, dtype=t.dtype, device="cuda")
    view = buf[skew:skew + rows * stride].view(rows, stride)[:, :d]
    view.copy_(t.reshape(rows, d))
    return view if t.dim() == 2 else view.unflatten(0, t.shape[:-1])


def untouched(view, before=None):
    """The sentinels around a strided view are still there."""
    d, stride = view.shape[-1], view.stride(-2)
    whole = view.as_strided((view.shape[0], stride), (stride, 1))
    assert bool((whole[:, d:] == SENTINEL).all())


# --- layer norm -----------------------------------------------------------

DIMS = [1, 2, 3, 4, 7, 8, 9, 15, 63, 64, 65, 130, 255, 257, 511, 512, 513, 768, 1000, 1001, 1023,
        1024, 1025, 1536, 2047, 2048, 2050, 3001, 4095, 4096, 4097, 6000, 8191, 8192]


@pytest.mark.parametrize("dim", DIMS)
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_norm_widths(dim, dtype):
    rows = 1 + (dim * 7) % 11
    note(f"norm dim={dim} rows={rows} {dtype}")
    g = gen(dim)
    x = (randn(g, rows, dim) + randn(g, rows, 1)).to(dtype)
    res = randn(g, rows, dim, dtype=dtype) if dim % 2 else None
    wt = F32 if dim % 3 else dtype
    w = None if dim % 5 == 4 else (1 + randn(g, dim, scale=0.2)).to(wt)
    b = None if dim % 7 == 5 else randn(g, dim, dtype=wt)
    eps = 1e-5
    y, h, mean, rstd = tokens.layer_norm(dev(x), dev(w), dev(b), eps, residual=dev(res))
    want_h = x if res is None else (x.double() + res.double()).to(dtype)
    if res is None:
        assert h is None
    else:
        # the fp32 sum of two 16-bit values may need a second rounding
        ref.close(h, x.double() + res.double(), 2.0 ** -24 * (x.double().abs() +
                                                              res.double().abs()), "sum")
        want_h = h.cpu()
    want, bound = ref.layer_norm(want_h, w, b, eps)
    for got, a, e, name in zip((y, mean, rstd), want, bound, ("out", "mean", "rstd")):
        ref.close(got, a, e, f"norm {name}")
    # backward
    dy = randn(g, rows, dim, dtype=dtype)
    ds = randn(g, rows, dim, dtype=dtype) if dim % 4 == 1 else None
    dw = torch.empty(dim, dtype=wt, device="cuda") if dim % 6 else None
    db = torch.empty(dim, dtype=wt, device="cuda") if dim % 6 != 1 else None
    if w is None and b is None and dw is None and db is None:
        wt = F32
    dx, gw, gb = tokens.layer_norm_backward(dev(dy), dev(want_h), dev(w), mean, rstd,
                                            grad_weight=dw, grad_bias=db, grad_sum=dev(ds))
    want, bound = ref.layer_norm_backward(dy, want_h, w, mean.cpu(), rstd.cpu(), ds)
    for got, a, e, name in zip((dx, gw, gb), want, bound, ("x", "weight", "bias")):
        if got is not None:
            ref.close(got, a, e, f"norm grad {name}")


@pytest.mark.parametrize("rows, dim", [(1, 4096), (2, 1024), (3, 1024), (5, 1500), (257, 320),
                                       (9000, 24), (20011, 8), (2600, 1100), (4099, 2)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_norm_rows(rows, dim, dtype):
    note(f"norm rows={rows} dim={dim} {dtype}")
    g = gen(rows)
    x, dy = randn(g, rows, dim, dtype=dtype), randn(g, rows, dim, dtype=dtype)
    w, b = 1 + randn(g, dim, scale=0.2), randn(g, dim)
    y, _, mean, rstd = tokens.layer_norm(dev(x), dev(w), dev(b))
    want, bound = ref.layer_norm(x, w, b, 1e-5)
    for got, a, e, name in zip((y, mean, rstd), want, bound, ("out", "mean", "rstd")):
        ref.close(got, a, e, f"norm {name}")
    old = randn(g, 2, dim)
    gw, gb = dev(old[0]), dev(old[1])
    dx, _, _ = tokens.layer_norm_backward(dev(dy), dev(x), dev(w), mean, rstd, grad_weight=gw,
                                          grad_bias=gb, accumulate=True)
    want, bound = ref.layer_norm_backward(dy, x, w, mean.cpu(), rstd.cpu(), None)
    ref.close(dx, want[0], bound[0], "norm grad x")
    for got, a, e, o in zip((gw, gb), want[1:], bound[1:], old):
        ref.close(got, a + o.double(), e + 2 * ref.U32 * (a.abs() + o.double().abs()),
                  "accumulated")


@pytest.mark.parametrize("dim, skew, pad", [(64, 1, 3), (513, 3, 1), (1024, 5, 7), (2047, 1, 0),
                                            (5, 1, 2)])
@pytest.mark.parametrize("dtype", [F32, F16])
def test_norm_strides(dim, skew, pad, dtype):
    """Rows with gaps from a misaligned start; nothing between them is written."""
    note(f"norm strides dim={dim} skew={skew} pad={pad} {dtype}")
    g = gen(dim + skew)
    rows = 13
    x, res, dy, ds = (randn(g, rows, dim, dtype=dtype) for _ in range(4))
    w, b = randn(g, dim), randn(g, dim)
    out = dev(torch.zeros_like(x), dim + pad + 2, skew)
    tot = dev(torch.zeros_like(x), dim + pad + 1, skew + 1)
    y, h, mean, rstd = tokens.layer_norm(dev(x, dim + pad, skew), dev(w), dev(b),
                                         residual=dev(res, dim + 2 * pad, skew), out=out,
                                         sum_out=tot)
    want, bound = ref.layer_norm(h.cpu(), w, b, 1e-5)
    ref.close(y, want[0], bound[0], "out")
    untouched(out)
    untouched(tot)
    gx = dev(torch.zeros_like(x), dim + pad + 3, skew)
    gw, gb = (torch.empty(dim, device="cuda") for _ in range(2))
    tokens.layer_norm_backward(dev(dy, dim + pad, skew), h, dev(w), mean, rstd, gx, gw, gb,
                               grad_sum=dev(ds, dim + 1, 1))
    want, bound = ref.layer_norm_backward(dy, h.cpu(), w, mean.cpu(), rstd.cpu(), ds)
    for got, a, e in zip((gx, gw, gb), want, bound):
        ref.close(got, a, e, "grad")
    untouched(gx)


@pytest.mark.parametrize("dim", [40, 700, 1300, 5001])
def test_norm_in_place_and_broadcast(dim):
    """Outputs that are the inputs; one row standing for all (stride 0)."""
    note(f"norm in place dim={dim}")
    g = gen(dim)
    rows = 31
    x, res = randn(g, rows, dim, dtype=BF16), randn(g, 1, dim, dtype=BF16)
    w, b = randn(g, dim), randn(g, dim)
    a, r = dev(x), dev(res).expand(rows, dim)
    y, h, mean, rstd = tokens.layer_norm(a, dev(w), dev(b), residual=r, sum_out=a)
    plain = tokens.layer_norm(dev(x), dev(w), dev(b), residual=dev(res.repeat(rows, 1)))
    assert h is a and torch.equal(h, plain[1]) and torch.equal(y, plain[0])
    c = dev(x)
    tokens.layer_norm(c, dev(w), dev(b), out=c)
    assert torch.equal(c, tokens.layer_norm(dev(x), dev(w), dev(b))[0])
    one = randn(g, 1, dim, dtype=BF16)
    dy = dev(one).expand(rows, dim)  # the gradient of a mean over rows
    ws = [torch.empty(dim, device="cuda") for _ in range(4)]
    d1 = tokens.layer_norm_backward(dy, h, dev(w), mean, rstd, None, ws[0], ws[1])[0]
    full = dev(one.repeat(rows, 1))
    d2 = tokens.layer_norm_backward(full, h, dev(w), mean, rstd, full, ws[2], ws[3])[0]
    assert d2 is full and torch.equal(d1, d2)
    assert torch.equal(ws[0], ws[2]) and torch.equal(ws[1], ws[3])


@pytest.mark.parametrize("dim", [8, 100, 1024, 1500, 4100])
def test_norm_extremes(dim):
    """NaN and infinities stay in their rows; constant rows, large offsets and
    rows of tiny values come out as the definition says."""
    note(f"norm extremes dim={dim}")
    g = gen(dim)
    x = randn(g, 7, dim)
    x[0, dim // 2] = float("nan")
    x[2, 0] = float("inf")
    x[3] = 3.0                              # variance 0
    x[4] = 1e4 + randn(g, dim)              # far from zero
    x[5] = randn(g, dim, scale=1e-18)       # the variance is eps
    y, _, mean, rstd = tokens.layer_norm(dev(x), None, None)
    y = y.cpu()
    assert bool(torch.isnan(y[0]).all()) and bool(torch.isnan(y[2]).all())
    assert bool((y[3] == 0).all())
    keep = [1, 3, 4, 5, 6]
    want, bound = ref.layer_norm(x[keep], None, None, 1e-5)
    for got, a, e, name in zip((y, mean.cpu(), rstd.cpu()), want, bound, ("out", "mean", "rstd")):
        ref.close(got[keep], a, e, name)
    dy = randn(g, 7, dim)
    dx = tokens.layer_norm_backward(dev(dy), dev(x), None, mean, rstd)[0].cpu()
    want, bound = ref.layer_norm_backward(dy[keep], x[keep], None, mean.cpu()[keep],
                                          rstd.cpu()[keep], None)
    ref.close(dx[keep], want[0], bound[0], "grad x")


def test_norm_no_rows():
    x = torch.empty((0, 100), device="cuda")
    y, h, mean, rstd = tokens.layer_norm(x)
    assert y.shape == (0, 100) and mean.shape == (0,)
    gw, gb = torch.full((100,), 5.0, device="cuda"), torch.full((100,), 6.0, device="cuda")
    tokens.layer_norm_backward(x, x, None, mean, rstd, None, gw, gb, accumulate=True)
    assert bool((gw == 5).all()) and bool((gb == 6).all())
    tokens.layer_norm_backward(x, x, None, mean, rstd, None, gw, gb)
    assert bool((gw == 0).all()) and bool((gb == 0).all())


@pytest.mark.parametrize("dim", [6, 200, 1030])
def test_norm_gradient_by_differences(dim):
    """Along random directions, <gradient, v> against (L(x + e v) - L(x - e v)) / 2e
    of the 64-bit forward pass; e = 1e-5 leaves an error of about 1e-10."""
    note(f"norm differences dim={dim}")
    g = gen(dim)
    rows, eps, e = 3, 1e-5, 1e-5
    x, w, b, top = randn(g, rows, dim), randn(g, dim), randn(g, dim), randn(g, rows, dim)
    _, _, mean, rstd = tokens.layer_norm(dev(x), dev(w), dev(b), eps)
    gw, gb = torch.empty(dim, device="cuda"), torch.empty(dim, device="cuda")
    gx = tokens.layer_norm_backward(dev(top), dev(x), dev(w), mean, rstd, None, gw, gb)[0]

    def loss(x, w, b):
        return float((ref.layer_norm(x, w, b, eps)[0][0] * top.double()).sum())

    args = [x.double(), w.double(), b.double()]
    for k, grad in enumerate((gx, gw, gb)):
        for _ in range(4):
            v = torch.randn(args[k].shape, generator=g, dtype=torch.float64)
            hi, lo = list(args), list(args)
            hi[k], lo[k] = args[k] + e * v, args[k] - e * v
            want = (loss(*hi) - loss(*lo)) / (2 * e)
            got = float((grad.cpu().double() * v).sum())
            size = float((grad.cpu().double() * v).abs().sum()) + float(top.abs().sum())
            assert abs(got - want) <= ((dim + 32) * ref.U32 + 1e-8) * size, (k, got, want)


# --- embedding ------------------------------------------------------------

def some_ids(g, n, vocab, holes=0.2, skewed=True):
    u = torch.rand(n, generator=g, dtype=torch.float64)
    ids = (torch.exp(u * torch.log(torch.tensor(vocab + 1.0))) - 1).long() if skewed else (
        u * vocab).long()
    ids.clamp_(0, vocab - 1)
    out = torch.rand(n, generator=g) < holes
    ids[out] = torch.tensor([-1, vocab, -2 ** 31, 2 ** 31 - 1])[
        torch.randint(0, 4, (int(out.sum()),), generator=g)]
    return ids


@pytest.mark.parametrize("dim", [1, 2, 7, 8, 9, 64, 100, 511, 512, 513, 1024, 1025, 2049, 5000])
@pytest.mark.parametrize("kinds", [(F32, F32), (F16, F16), (BF16, BF16), (F32, BF16),
                                   (BF16, F32), (F16, BF16)])
def test_embed_widths(dim, kinds):
    n, vocab, scale = 1 + (dim * 5) % 23, 37, 1.5
    note(f"embed dim={dim} n={n} {kinds}")
    g = gen(dim)
    table = randn(g, vocab, dim, dtype=kinds[0])
    ids = some_ids(g, n, vocab)
    wide = dim % 2 == 0
    out = torch.empty((n, dim), dtype=kinds[1], device="cuda")
    tokens.embed(dev(ids if wide else ids.int()), dev(table), scale, out=out)
    want, bound = ref.embed(ids, table, scale)
    ref.close(out, want, bound, "embed")
    # left rows, gaps and a misaligned start
    old = randn(g, n, dim, dtype=kinds[1])
    out = dev(old, dim + 3, 1)
    tokens.embed(dev(ids), dev(table, dim + 5, 3), scale, out=out, keep=True)
    want, bound = ref.embed(ids, table, scale, keep=old)
    ref.close(out, want, bound, "embed keep")
    if n > 1:
        untouched(out)


@pytest.mark.parametrize("n, vocab, dim, skewed", [
    (1, 1, 1, True), (1, 50, 64, True), (2, 1, 9, True), (31, 5, 33, True), (32, 3, 8, False),
    (33, 1, 700, True), (64, 2, 12, True), (65, 7, 40, True), (777, 5003, 321, True),
    (1000, 4, 100, False), (4097, 300, 72, True), (8192, 1000, 16, True),
    (8193, 1000, 16, True), (20000, 511, 24, True), (20000, 512, 24, True),
    (1023, 3, 40, True), (1024, 900, 520, True), (1025, 900, 520, True), (700, 5000, 3, True),
    (1000, 1, 300, True), (40, 300000, 33, False), (5, 9000, 4100, False), (1024, 2, 8, False),
    (70001, 262143, 8, True), (70001, 262144, 8, True), (9000, 600000, 8, False),
    (3000, 600000, 8, False), (150000, 40, 4, False)])
@pytest.mark.parametrize("kinds", [(F32, F32), (BF16, F32), (F16, F16)])
def test_embed_gradient(n, vocab, dim, skewed, kinds):
    note(f"embed grad n={n} vocab={vocab} dim={dim} {kinds}")
    g = gen(n + vocab)
    ids = some_ids(g, n, vocab, 0.15, skewed)
    dy = randn(g, n, dim, dtype=kinds[0])
    scale = 0.75
    out = torch.full((vocab, dim), SENTINEL, dtype=kinds[1], device="cuda")
    tokens.embed_backward(dev(dy), dev(ids), out, scale)
    want, bound = ref.embed_backward(dy, ids, vocab, scale)
    ref.close(out, want, bound, "embed grad")
    again = torch.empty_like(out)
    tokens.embed_backward(dev(dy), dev(ids.clamp(-2 ** 31, 2 ** 31 - 1).int()), again, scale)
    assert torch.equal(out, again), "32-bit ids or a second run give other bits"
    # added to what is there, one id without a gradient, strided both ways
    old = randn(g, vocab, dim, dtype=kinds[1])
    pad = int(ids[n // 2])
    out = dev(old, dim + 2, 1)
    tokens.embed_backward(dev(dy, dim + 1, 1), dev(ids), out, scale, padding=pad,
                          accumulate=True)
    want, bound = ref.embed_backward(dy, ids, vocab, scale, pad, old)
    ref.close(out, want, bound, "embed grad added")
    if vocab > 1:
        untouched(out)
    seen = torch.zeros(vocab, dtype=torch.bool)
    seen[ids[(ids >= 0) & (ids < vocab) & (ids != pad)]] = True
    assert torch.equal(out.cpu()[~seen], old[~seen]), "rows that no id names were touched"


def test_embed_gradient_without_ids():
    ids = torch.empty(0, dtype=torch.int64, device="cuda")
    out = torch.full((9, 20), 3.0, device="cuda")
    dy = torch.empty((0, 20), device="cuda")
    tokens.embed_backward(dy, ids, out, accumulate=True)
    assert bool((out == 3).all())
    tokens.embed_backward(dy, ids, out)
    assert bool((out == 0).all())
    holes = torch.full((100,), -1, dtype=torch.int64, device="cuda")
    out.fill_(3.0)
    tokens.embed_backward(torch.ones((100, 20), device="cuda"), holes, out)
    assert bool((out == 0).all())
    assert tokens.embed(ids, out).shape == (0, 20)


def test_embed_gradient_bad_values_stay_in_their_rows():
    """A NaN row reaches its own token only, also across pieces; rows that
    name no token count for nothing, whatever they hold."""
    n, vocab, dim = 500, 12, 16
    g = gen(3)
    ids = torch.randint(0, vocab, (n,), generator=g)
    ids[100:120] = -1
    dy = randn(g, n, dim)
    dy[100:120] = float("nan")
    dy[7, 3] = float("inf")
    out = torch.empty((vocab, dim), device="cuda")
    tokens.embed_backward(dev(dy), dev(ids), out)
    want, bound = ref.embed_backward(torch.where(torch.isinf(dy), torch.zeros(()), dy), ids,
                                     vocab, 1.0)
    got = out.cpu().double()
    assert got[ids[7], 3] == float("inf")
    got[ids[7], 3] = want[ids[7], 3]
    ref.close(got.float(), want, bound, "embed grad")


# --- patch embedding ------------------------------------------------------

PATCHES = [  # n, c, h, w, p, dim, nhwc
    (1, 3, 16, 16, 16, 32, False), (1, 1, 1, 1, 1, 1, False), (2, 3, 5, 7, 2, 5, False),
    (2, 3, 5, 7, 2, 5, True), (1, 3, 224, 224, 16, 96, False), (3, 3, 65, 97, 16, 40, False),
    (3, 3, 65, 97, 16, 40, True), (2, 3, 70, 84, 14, 130, False), (2, 3, 70, 84, 14, 130, True),
    (5, 4, 40, 33, 8, 7, False), (2, 1, 50, 50, 7, 65, False), (2, 2, 50, 50, 9, 33, True),
    (7, 3, 60, 40, 20, 33, True), (1, 5, 33, 61, 11, 129, False), (64, 3, 32, 32, 16, 4, False),
    (4, 3, 64, 100, 4, 24, True), (2, 3, 96, 96, 24, 200, False), (2, 3, 7, 7, 8, 16, False),
    (9, 3, 130, 131, 13, 300, False), (40, 3, 112, 112, 14, 384, False)]
# enough rows for the larger tiles: whole chunks, repeated values, short runs;
# ragged last tiles both ways
LARGE = [(33, 3, 160, 176, 16, 1000, False), (70, 3, 140, 154, 14, 520, False),
         (61, 3, 112, 120, 14, 776, True), (130, 2, 63, 70, 7, 264, False),
         (97, 3, 224, 224, 16, 768, False), (260, 1, 112, 112, 8, 1030, True),
         (11, 3, 224, 224, 16, 770, False), (9, 3, 210, 196, 14, 760, False),
         (201, 3, 224, 224, 16, 780, False), (150, 3, 210, 224, 14, 1000, True)]
KINDS = [(F32, F32), (F16, F32), (F16, F16), (F32, F16), (F16, BF16), (F32, BF16), (BF16, BF16)]


def patch_inputs(case, image, dtype, seed):
    n, c, h, w, p, dim, nhwc = case
    g = gen(seed)
    img = randn(g, *((n, h, w, c) if nhwc else (n, c, h, w)), dtype=image)
    weight = randn(g, *((dim, p, p, c) if nhwc else (dim, c, p, p)), dtype=dtype,
                   scale=(c * p * p) ** -0.5)
    t = (h // p) * (w // p)
    return g, img, weight, t


@pytest.mark.parametrize("case", PATCHES)
@pytest.mark.parametrize("image, dtype", KINDS)
def test_patch_embed(case, image, dtype):
    note(f"patch {case} {image} {dtype}")
    n, c, h, w, p, dim, nhwc = case
    g, img, weight, t = patch_inputs(case, image, dtype, dim)
    layout = tokens.LAYOUT_NHWC if nhwc else tokens.LAYOUT_NCHW
    bias = randn(g, dim, dtype=dtype) if dim % 2 else None
    pos = randn(g, t, dim, dtype=dtype) if p % 2 == 0 else None
    out = tokens.patch_embed(dev(img), dev(weight), dev(bias), dev(pos), layout=layout)
    want, bound = ref.patch_embed(img, weight, bias, pos, nhwc)
    ref.close(out, want, bound, "patch")
    # a slice of a longer sequence, rows with gaps
    seq = torch.full((n, t + 3, dim + 1), SENTINEL, dtype=dtype, device="cuda")
    tokens.patch_embed(dev(img), dev(weight), dev(bias), dev(pos), layout=layout,
                       out=seq[:, 2:2 + t, 1:])
    assert torch.equal(seq[:, 2:2 + t, 1:], out)
    assert bool((seq[:, :2] == SENTINEL).all()) and bool((seq[:, 2 + t:] == SENTINEL).all())
    assert bool((seq[:, :, 0] == SENTINEL).all())
    # sequence first: images are the inner dimension
    seq = torch.full((t, n, dim), SENTINEL, dtype=dtype, device="cuda")
    tokens.patch_embed(dev(img), dev(weight), dev(bias), dev(pos), layout=layout,
                       out=seq.transpose(0, 1))
    assert torch.equal(seq.transpose(0, 1), out)


@pytest.mark.parametrize("case", LARGE)
@pytest.mark.parametrize("image, dtype", KINDS)
def test_patch_embed_large(case, image, dtype):
    """The same bounds, from 64 bits on the device."""
    note(f"patch {case} {image} {dtype}")
    n, c, h, w, p, dim, nhwc = case
    g, img, weight, t = patch_inputs(case, image, dtype, dim)
    layout = tokens.LAYOUT_NHWC if nhwc else tokens.LAYOUT_NCHW
    bias, pos = randn(g, dim, dtype=dtype), randn(g, t, dim, dtype=dtype)
    args = [x.cuda() for x in (img, weight, bias, pos)]
    out = tokens.patch_embed(*args, layout=layout)
    want, bound = ref.patch_embed(*args, nhwc)
    ref.close(out, want.cpu(), bound.cpu(), "patch")


@pytest.mark.parametrize("case", PATCHES)
@pytest.mark.parametrize("image, dtype", KINDS)
def test_patch_gradient(case, image, dtype):
    note(f"patch grad {case} {image} {dtype}")
    n, c, h, w, p, dim, nhwc = case
    g, img, weight, t = patch_inputs(case, image, dtype, dim + 1)
    layout = tokens.LAYOUT_NHWC if nhwc else tokens.LAYOUT_NCHW
    kind = F32 if dim % 2 else dtype
    dy = randn(g, n, t, dim, dtype=dtype)
    old = [randn(g, dim, c * p * p, dtype=kind), randn(g, dim, dtype=kind),
           randn(g, t, dim, dtype=kind)]
    want, bound = ref.patch_embed_backward(dy, img, p, nhwc)
    for add in (False, True):
        got = [dev(o) for o in old]
        tokens.patch_embed_backward(dev(dy), dev(img), got[0].view(weight.shape), got[1],
                                    got[2], layout=layout, accumulate=add)
        for a, e, b, o, name in zip(got, want, bound, old, ("weight", "bias", "pos")):
            if add:
                e, b = e + o.double(), b + 2 * ref.U32 * (e.abs() + o.double().abs())
            ref.close(a, e, b, f"patch grad {name} add={add}")
    # a slice of a longer sequence; one gradient row for all (stride 0)
    seq = torch.full((n, t + 2, dim + 1), SENTINEL, dtype=dtype, device="cuda")
    seq[:, 1:1 + t, 1:] = dev(dy)
    first = torch.empty(weight.shape, dtype=kind, device="cuda")
    tokens.patch_embed_backward(seq[:, 1:1 + t, 1:], dev(img), first, layout=layout)
    base = torch.empty_like(first)
    tokens.patch_embed_backward(dev(dy), dev(img), base, layout=layout)
    assert torch.equal(first, base)
    if t:
        one = dev(dy[:1, :1]).expand(n, t, dim)
        tokens.patch_embed_backward(one, dev(img), first, layout=layout)
        tokens.patch_embed_backward(one.contiguous(), dev(img), base, layout=layout)
        assert torch.equal(first, base)


@pytest.mark.parametrize("case", LARGE)
@pytest.mark.parametrize("image, dtype", KINDS)
def test_patch_gradient_large(case, image, dtype):
    note(f"patch grad {case} {image} {dtype}")
    n, c, h, w, p, dim, nhwc = case
    g, img, weight, t = patch_inputs(case, image, dtype, dim + 1)
    layout = tokens.LAYOUT_NHWC if nhwc else tokens.LAYOUT_NCHW
    dy, img = randn(g, n, t, dim, dtype=dtype).cuda(), img.cuda()
    got = [torch.empty(s, device="cuda") for s in (weight.shape, (dim,), (t, dim))]
    tokens.patch_embed_backward(dy, img, *got, layout=layout)
    want, bound = ref.patch_embed_backward(dy, img, p, nhwc)
    got[0] = got[0].view(dim, -1)
    for a, e, b, name in zip(got, want, bound, ("weight", "bias", "pos")):
        ref.close(a, e.cpu(), b.cpu(), f"patch grad {name}")


@pytest.mark.parametrize("case", [
    (2, 3, 70, 84, 14, 130, False), (5, 4, 40, 33, 8, 7, False), (64, 3, 32, 32, 16, 4, False),
    (2, 3, 50, 50, 7, 65, True), (3, 3, 65, 97, 16, 40, True), (17, 3, 112, 112, 14, 384, False),
    (201, 3, 224, 224, 16, 780, False), (2, 3, 7, 7, 8, 16, False)])
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_patch_gradient_without_the_weight(case, dtype):
    """A frozen projection: bias and positions, or one of them, alone; from
    gaps, overwritten and added to. Both ways of the sums (beside products of
    128-wide tiles and after those of 256) give these bits too."""
    note(f"patch grad sums {case} {dtype}")
    n, c, h, w, p, dim, nhwc = case
    g, img, weight, t = patch_inputs(case, F16 if dtype != F32 else F32, dtype, dim + 2)
    layout = tokens.LAYOUT_NHWC if nhwc else tokens.LAYOUT_NCHW
    kind = F32 if dim % 4 else dtype
    dy = randn(g, n, t, dim, dtype=dtype)
    seq = torch.full((n, t + 2, dim + 1), SENTINEL, dtype=dtype, device="cuda")
    seq[:, 1:1 + t, 1:] = dev(dy)
    old = randn(g, dim, dtype=kind), randn(g, t, dim, dtype=kind)
    sums = dy.double().sum((0, 1)), dy.double().sum(0)
    sizes = dy.double().abs().sum((0, 1)), dy.double().abs().sum(0)
    bounds = [(m + 4) * ref.U32 * s for m, s in zip((n * t, n), sizes)]
    img = dev(img)
    for add in (False, True):
        for which in ((True, True), (True, False), (False, True)):
            got = [dev(o) if k else None for o, k in zip(old, which)]
            back = tokens.patch_embed_backward(seq[:, 1:1 + t, 1:], img, None, *got,
                                               layout=layout, accumulate=add, patch=p)
            assert back[0] is None and back[1] is got[0] and back[2] is got[1]
            for a, e, b, o, name in zip(got, sums, bounds, old, ("bias", "pos")):
                if a is None:
                    continue
                if add:
                    e, b = e + o.double(), b + 2 * ref.U32 * (e.abs() + o.double().abs())
                ref.close(a, e, b, f"patch grad {name} alone add={add}")
        if add:
            continue
        both = [torch.empty_like(dev(o)) for o in old]
        gw = torch.empty(weight.shape, dtype=kind, device="cuda")
        tokens.patch_embed_backward(dev(dy), img, gw, *both, layout=layout, patch=p)
        alone = [torch.empty_like(o) for o in both]
        tokens.patch_embed_backward(dev(dy), img, None, *alone, layout=layout, patch=p)
        assert all(torch.equal(a, b) for a, b in zip(both, alone))


def test_patch_no_images():
    img = torch.empty((0, 3, 32, 32), dtype=F16, device="cuda")
    weight = torch.randn((24, 3, 16, 16), device="cuda").half()
    assert tokens.patch_embed(img, weight).shape == (0, 4, 24)
    gw, gb, gp = (torch.full(s, 2.0, device="cuda") for s in ((24, 3, 16, 16), (24,), (4, 24)))
    dy = torch.empty((0, 4, 24), dtype=F16, device="cuda")
    tokens.patch_embed_backward(dy, img, gw, gb, gp, accumulate=True)
    assert all(bool((t == 2).all()) for t in (gw, gb, gp))
    tokens.patch_embed_backward(dy, img, gw, gb, gp)
    assert all(bool((t == 0).all()) for t in (gw, gb, gp))


def test_patch_bad_pixels_stay_in_their_patches():
    """Infinities and NaN beside a patch (the next pixels of its rows, pixels
    past the last whole patch) do not reach it."""
    n, c, h, w, p, dim = 2, 3, 45, 47, 14, 48
    g, img, weight, t = patch_inputs((n, c, h, w, p, dim, False), F16, F16, 5)
    img[:, :, 42:, :] = float("nan")
    img[:, :, :, 42:] = float("inf")
    img[0, 1, 20, 20] = float("nan")  # in patch (1, 1) of image 0
    out = tokens.patch_embed(dev(img), dev(weight)).cpu()
    want, bound = ref.patch_embed(img, weight, None, None, False)
    assert bool(torch.isnan(want[0, 4]).all()) and int(torch.isnan(want).sum()) == dim
    ref.close(out, want, bound, "patch")


def test_patch_gradient_by_differences():
    """The loss is linear in the parameters: one difference of any size is exact
    but for rounding (64-bit forward pass)."""
    case = (2, 3, 30, 44, 14, 20, False)
    g, img, weight, t = patch_inputs(case, F32, F32, 9)
    dim, p = 20, 14
    bias, pos, top = randn(g, dim), randn(g, t, dim), randn(g, 2, t, dim)
    grads = [torch.empty(s.shape, device="cuda") for s in (weight, bias, pos)]
    tokens.patch_embed_backward(dev(top), dev(img), *grads)
    args = [weight.double(), bias.double(), pos.double()]
    img64 = img.double()

    def loss(w, b, q):
        y = ref.patches(img64, p, False) @ w.reshape(dim, -1).t() + b + q
        return float((y * top.double()).sum())

    for k, grad in enumerate(grads):
        v = torch.randn(args[k].shape, generator=g, dtype=torch.float64)
        hi, lo = list(args), list(args)
        hi[k], lo[k] = args[k] + v, args[k] - v
        want = (loss(*hi) - loss(*lo)) / 2
        got = float((grad.cpu().double() * v).sum())
        size = float(top.abs().sum()) * (1 + float(img.abs().max())) * float(v.abs().max())
        assert abs(got - want) <= 64 * ref.U32 * size, (k, got, want)


# --- together: sequences, streams, graphs, long offsets --------------------

def sequence_step(s):
    """One step over a mixed sequence: images to rows 1 .. t, ids elsewhere."""
    t = s["t"]
    tokens.embed(s["ids"], s["table"], 2.0, out=s["seq"], keep=True)
    tokens.patch_embed(s["images"], s["weight"], s["bias"], s["pos"], out=s["seq"][:, 1:1 + t])
    y, _, mean, rstd = tokens.layer_norm(s["seq"], s["gamma"], s["beta"], out=s["y"],
                                         mean=s["mean"], rstd=s["rstd"])
    gx, gw, gb = tokens.layer_norm_backward(s["top"], s["seq"], s["gamma"], mean, rstd, s["gx"],
                                            s["g_gamma"], s["g_beta"], workspace=s["ws_norm"])
    tokens.patch_embed_backward(gx[:, 1:1 + t], s["images"], s["g_weight"], s["g_bias"],
                                s["g_pos"], workspace=s["ws_patch"])
    tokens.embed_backward(gx, s["ids"], s["g_table"], 2.0, workspace=s["ws_embed"])


RESULTS = ("y", "gx", "g_gamma", "g_beta", "g_weight", "g_bias", "g_pos", "g_table")


def sequence_state(seed=1, n=6, p=14, size=70, dim=320, vocab=900, text=40):
    g = gen(seed)
    t = (size // p) ** 2
    length = 1 + t + text
    ids = torch.randint(0, vocab, (n, length), generator=g)
    ids[:, 1:1 + t] = -1
    s = {"t": t, "ids": ids.cuda(), "images": randn(g, n, 3, size, size, dtype=F16).cuda(),
         "table": randn(g, vocab, dim, dtype=BF16).cuda(),
         "weight": randn(g, dim, 3, p, p, dtype=BF16, scale=0.05).cuda(),
         "bias": randn(g, dim, dtype=BF16).cuda(), "pos": randn(g, t, dim, dtype=BF16).cuda(),
         "gamma": randn(g, dim).cuda(), "beta": randn(g, dim).cuda(),
         "top": randn(g, n, length, dim, dtype=BF16).cuda()}
    e = lambda *shape, dtype=F32: torch.empty(shape, dtype=dtype, device="cuda")  # noqa: E731
    s.update(seq=e(n, length, dim, dtype=BF16), y=e(n, length, dim, dtype=BF16),
             gx=e(n, length, dim, dtype=BF16), mean=e(n, length), rstd=e(n, length),
             g_gamma=e(dim), g_beta=e(dim), g_weight=e(dim, 3, p, p), g_bias=e(dim),
             g_pos=e(t, dim), g_table=e(vocab, dim))
    s["ws_norm"] = e(tokens.layer_norm_workspace_bytes(n * length, dim), dtype=torch.uint8)
    s["ws_embed"] = e(tokens.embed_workspace_bytes(n * length, vocab, dim), dtype=torch.uint8)
    s["ws_patch"] = e(tokens.patch_embed_workspace_bytes(s["images"], s["g_weight"], BF16),
                      dtype=torch.uint8)
    return s


def test_sequence_against_definitions():
    note("sequence")
    s = sequence_state()
    sequence_step(s)
    c = {k: v.cpu() if torch.is_tensor(v) else v for k, v in s.items()}
    t, dim = s["t"], c["gamma"].numel()
    # each operator on the rows that the kernels before it made
    want, bound = ref.embed(c["ids"], c["table"], 2.0)
    hole = c["ids"] < 0
    ref.close(c["seq"][~hole], want[~hole], bound[~hole], "text rows")
    want, bound = ref.patch_embed(c["images"], c["weight"], c["bias"], c["pos"], False)
    ref.close(c["seq"][:, 1:1 + t], want, bound, "image rows")
    want, bound = ref.layer_norm(c["seq"], c["gamma"], c["beta"], 1e-5)
    ref.close(c["y"], want[0], bound[0], "norm")
    want, bound = ref.layer_norm_backward(c["top"], c["seq"], c["gamma"], c["mean"], c["rstd"],
                                          None)
    ref.close(c["gx"].reshape(-1, dim), want[0], bound[0], "rows' gradient")
    ref.close(c["g_gamma"], want[1], bound[1], "gamma")
    ref.close(c["g_beta"], want[2], bound[2], "beta")
    want, bound = ref.patch_embed_backward(c["gx"][:, 1:1 + t], c["images"], 14, False)
    ref.close(c["g_weight"].reshape(dim, -1), want[0], bound[0], "projection")
    ref.close(c["g_pos"], want[2], bound[2], "positions")
    want, bound = ref.embed_backward(c["gx"], c["ids"], c["table"].shape[0], 2.0)
    ref.close(c["g_table"], want, bound, "table")


def test_sequence_on_another_stream():
    s, plain = sequence_state(2), sequence_state(2)
    sequence_step(plain)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        sequence_step(s)
    torch.cuda.current_stream().wait_stream(st)
    for k in RESULTS:
        assert torch.equal(s[k], plain[k]), k
    # by argument: the call's stream waits for the current one's work
    x = torch.randn((300, 200), device="cuda")
    want = tokens.layer_norm(x + 1.0)[0]
    got = tokens.layer_norm(x + 1.0, stream=st)[0]
    torch.cuda.current_stream().wait_stream(st)
    assert torch.equal(got, want)


@pytest.mark.parametrize("text", [40, 300, 2500])
def test_sequence_in_a_graph(text):
    """Captured once, replayed with new inputs between eager work: every
    replay gives the eager bits (the ids' gradient without a sort, with one by
    counting and with one by digits)."""
    s, eager = sequence_state(3, text=text), sequence_state(3, text=text)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        sequence_step(s)
    torch.cuda.current_stream().wait_stream(st)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sequence_step(s)
    for turn in range(4):
        new = sequence_state(10 + turn, text=text)
        for k in ("ids", "images", "table", "top"):
            s[k].copy_(new[k])
            eager[k].copy_(new[k])
        for k in RESULTS:
            s[k].fill_(SENTINEL)
        sequence_step(eager)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for k in RESULTS:
            assert torch.equal(s[k], eager[k]), (turn, k)


def test_offsets_past_32_bits():
    """Rows 2^28 elements apart, the last past element 2^31; images past it too."""
    note("long offsets")
    stride, rows, dim = 1 << 28, 10, 100
    buf = torch.empty(stride * (rows - 1) + dim, dtype=F16, device="cuda")
    view = buf.as_strided((rows, dim), (stride, 1))
    g = gen(4)
    x = randn(g, rows, dim, dtype=F16)
    view.copy_(x)
    plain = tokens.layer_norm(dev(x))
    far = tokens.layer_norm(view)
    assert torch.equal(far[0], plain[0]) and torch.equal(far[2], plain[2])
    ids = torch.tensor([9, 0, 8, 8, 3], device="cuda")
    assert torch.equal(tokens.embed(ids, view), tokens.embed(ids, dev(x)))
    top = randn(g, 5, dim, dtype=F16)
    tokens.embed_backward(dev(top), ids, view)
    near = torch.empty((rows, dim), dtype=F16, device="cuda")
    tokens.embed_backward(dev(top), ids, near)
    assert torch.equal(view, near)
    out = tokens.layer_norm(dev(x), out=view)[0]
    assert torch.equal(out, plain[0])
    wide = buf.as_strided((rows, 1, dim), (stride, dim, 1))
    img = randn(g, rows, 1, 8, 8, dtype=F16)
    weight = randn(g, dim, 1, 8, 8, dtype=F16)
    a = tokens.patch_embed(dev(img), dev(weight), out=wide)
    b = tokens.patch_embed(dev(img), dev(weight))
    assert torch.equal(a, b)
    grads = [torch.empty((dim, 1, 8, 8), device="cuda") for _ in range(2)]
    tokens.patch_embed_backward(a, dev(img), grads[0])
    tokens.patch_embed_backward(b, dev(img), grads[1])
    assert torch.equal(*grads)
    del buf, view, wide, a, out, far
    n, size = 700, 1024
    images = torch.zeros((n, 3, size, size), dtype=F16, device="cuda")
    last = randn(g, 2, 3, size, size, dtype=F16)
    images[-2:] = dev(last)
    weight = randn(g, 16, 3, 256, 256, dtype=F16, scale=0.01)
    got = tokens.patch_embed(images, dev(weight))
    want, bound = ref.patch_embed(last, weight, None, None, False)
    ref.close(got[-2:], want, bound, "last images")
    assert bool((got[:-2] == 0).all())


@pytest.mark.parametrize("dim", [40, 1001, 1026, 1537, 2049, 2305, 4098, 4609, 8191])
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_norm_every_place_in_place(dim, dtype):
    """Every output that may be an input, with strides: the bits of the call
    with outputs of their own. From 1025 columns on several waves hold a row, and
    a last chunk that is moved back to end with it can be written by two."""
    note(f"norm in place dim={dim} {dtype}")
    g = gen(dim)
    rows = 23
    x, res, dy, ds = (randn(g, rows, dim, dtype=dtype) for _ in range(4))
    w, b = randn(g, dim), randn(g, dim)

    def new(t):
        return dev(t, dim + 3, 1)

    y, h, mean, rstd = tokens.layer_norm(dev(x), dev(w), dev(b), residual=dev(res))
    for outputs in (("x", None), ("residual", None), (None, "x"), (None, "residual"),
                    ("x", "residual"), ("residual", "x")):
        at = {"x": new(x), "residual": new(res)}
        out, tot = (at.get(k) if k else new(torch.zeros_like(x)) for k in outputs)
        got = tokens.layer_norm(at["x"], dev(w), dev(b), residual=at["residual"], out=out,
                                sum_out=tot)
        assert got[0] is out and got[1] is tot, outputs
        for a, e in zip(got, (y, h, mean, rstd)):
            assert torch.equal(a, e), outputs
        untouched(out)
        untouched(tot)
    # the sum of no residual is x itself
    at = new(x)
    plain = tokens.layer_norm(dev(x), dev(w), dev(b))
    got = tokens.layer_norm(at, dev(w), dev(b), sum_out=at)
    assert torch.equal(got[0], plain[0]) and torch.equal(at, dev(x))
    want = [torch.empty(dim, device="cuda") for _ in range(2)]
    dx = tokens.layer_norm_backward(dev(dy), h, dev(w), mean, rstd, None, *want,
                                    grad_sum=dev(ds))[0]
    for k in ("grad_out", "h", "grad_sum"):
        at = {"grad_out": new(dy), "h": new(h), "grad_sum": new(ds)}
        sums = [torch.empty(dim, device="cuda") for _ in range(2)]
        got = tokens.layer_norm_backward(at["grad_out"], at["h"], dev(w), mean, rstd, at[k],
                                         *sums, grad_sum=at["grad_sum"])[0]
        assert got is at[k] and torch.equal(got, dx), k
        assert torch.equal(sums[0], want[0]) and torch.equal(sums[1], want[1]), k
        untouched(got)
