"""The attention operators on the GPU against their definitions in 64 bits
(tests/attention_util.py, with the bounds derived there): types, layouts, head
widths, grouped heads, windows and sinks, lengths from none on, strides and
misaligned starts, masked NaN and infinities, far positions, offsets past 32
bits, other streams, graphs, gradients against differences, and a run of them
together."""
from __future__ import annotations

import math

import pytest
import torch

from paper_2007_13005_amd import attention
from tests import attention_util as ref
from tests.gpu_util import note
from tests.tokens_util import TINY, UNIT, close

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
NAN, INF = float("nan"), float("inf")
SENTINEL = -77.0


def gen(seed: int) -> torch.Generator:
    return torch.Generator().manual_seed(seed)


def randn(g, *shape, dtype=F32, scale=1.0):
    return (torch.randn(shape, generator=g) * scale).to(dtype)


def dev(t):
    return None if t is None else t.cuda()


def spread(t, pad: int = 3, skew: int = 1):
    """t (..., heads, dim) on the device in a buffer of sentinels: `pad` elements
    between heads, `pad` + 2 more between rows, `skew` before the first. Returns
    (view, buffer)."""
    *lead, h, d = t.shape
    rows = math.prod(lead)
    head, row = d + pad, h * (d + pad) + pad + 2
    buf = torch.full((skew + rows * row + 8,), SENTINEL, dtype=t.dtype, device="cuda")
    strides, step = [], row
    for n in reversed(lead):
        strides.insert(0, step)
        step *= n
    view = buf.as_strided((*lead, h, d), (*strides, head, 1), skew)
    view.copy_(t)
    return view, buf


def untouched(view, buf):
    """The sentinels around a spread view are still there."""
    left = buf.clone()
    left.as_strided(view.shape, view.stride(), view.storage_offset()).fill_(SENTINEL)
    assert bool((left == SENTINEL).all())


# --- rotation and head norm -------------------------------------------------

WIDTHS = [(2, 2), (3, 2), (7, 4), (8, 8), (16, 16), (16, 4), (18, 18), (24, 12), (33, 32), (48, 48),
          (64, 64), (64, 32), (66, 2), (72, 36), (80, 80), (96, 24), (100, 100), (127, 126),
          (128, 128), (128, 64), (130, 130), (160, 160), (194, 98), (255, 254), (256, 256),
          (256, 64)]


@pytest.mark.parametrize("dim, rot", WIDTHS)
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_rotate_widths(dim, rot, dtype):
    g = gen(dim + rot)
    freqs, gain = ref.frequencies(rot, 10000.0, "parts", 4.0, 64.0)
    for rows, heads in ((1, 1), (5, 3), (2, 17), (37, 2)):
        for interleaved in (False, True):
            note(f"rotate dim={dim} rot={rot} {dtype} rows={rows} heads={heads} {interleaved}")
            x = randn(g, rows, heads, dim, dtype=dtype)
            pos = torch.randint(-50, 5000, (rows,), generator=g)
            pos = pos if heads % 2 else pos.int()
            y = attention.rotate(dev(x), dev(pos), dev(freqs), gain, interleaved)
            close(y, *ref.rotate(x, pos, freqs, gain, interleaved), "rotate")
            dx = attention.rotate_backward(dev(x), dev(pos), dev(freqs), gain, interleaved)
            close(dx, *ref.rotate(x, pos, freqs, gain, interleaved, back=True), "backward")
            # the values that do not turn are copied
            assert torch.equal(y[..., rot:].cpu(), x[..., rot:])


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rotate_strides_in_place_and_streams(dtype):
    g = gen(3)
    freqs, _ = ref.frequencies(24)
    for dim, heads, rows in ((40, 5, (3, 4)), (24, 1, (9,)), (33, 4, (2, 3))):
        note(f"rotate strides dim={dim} heads={heads} {dtype}")
        x = randn(g, *rows, heads, dim, dtype=dtype)
        pos = torch.randint(0, 100, rows, generator=g)
        want = ref.rotate(x, pos, freqs, 1.0, False)
        view, _ = spread(x)
        out, buf = spread(torch.zeros_like(x), 5, 2)
        attention.rotate(view, dev(pos), dev(freqs), out=out)
        close(out, *want, "strided")
        untouched(out, buf)
        view, buf = spread(x)
        assert attention.rotate(view, dev(pos), dev(freqs), out=view) is view
        assert torch.equal(view, out)
        untouched(view, buf)
        side = torch.cuda.Stream()
        other = attention.rotate(dev(x), dev(pos), dev(freqs), stream=side)
        side.synchronize()
        assert torch.equal(other, out)
        # one row's and one head's values standing for all
        one = dev(x[..., :1, :]).expand(*rows, heads, dim)
        close(attention.rotate(one, dev(pos), dev(freqs)),
              *ref.rotate(one.cpu(), pos, freqs, 1.0, False), "broadcast")


@pytest.mark.parametrize("pos", [0, 1, -1, 4095, 1 << 20, (1 << 24) + 1, (1 << 31) - 1, 1 << 40])
def test_rotate_far_positions(pos):
    """Angles are formed and reduced in 64 bits."""
    note(f"rotate far {pos}")
    freqs, _ = ref.frequencies(64, 500000.0)
    x = randn(gen(1), 3, 2, 64)
    at = torch.tensor([pos, pos - 1, pos // 2])
    y = attention.rotate(dev(x), dev(at), dev(freqs))
    close(y, *ref.rotate(x, at, freqs, 1.0, False), "far")


def test_rotate_keeps_what_does_not_turn():
    """NaN and infinities stay in their pair."""
    note("rotate NaN")
    for interleaved in (False, True):
        for dim, rot in ((48, 16), (20, 12), (16, 16), (129, 64)):
            x = randn(gen(dim), 4, 3, dim, dtype=BF16)
            x[0, 0, rot - 1] = NAN
            x[1, 1, dim - 1] = INF
            pos = torch.arange(4)
            freqs, _ = ref.frequencies(rot)
            y = attention.rotate(dev(x), dev(pos), dev(freqs), 1.0, interleaved).cpu()
            want = ref.rotate(x, pos, freqs, 1.0, interleaved)[0]
            assert torch.equal(torch.isfinite(y), torch.isfinite(want))
            assert torch.equal(y[..., rot:].isnan(), x[..., rot:].isnan())


@pytest.mark.parametrize("dim, rot", WIDTHS + [(1, 0), (5, 0), (64, 0), (128, 0), (250, 0)])
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_head_norm_widths(dim, rot, dtype):
    g = gen(dim * 3 + rot)
    for rows, hq, hk in ((1, 1, 1), (3, 5, 2), (40, 2, 1), (2, 19, 0)):
        interleaved = (rows + dim) % 2 == 0
        note(f"head norm dim={dim} rot={rot} {dtype} rows={rows} heads={hq},{hk} {interleaved}")
        wt = F32 if dim % 3 else dtype
        q, dyq = (randn(g, rows, hq, dim, dtype=dtype, scale=s) for s in (1.5, 0.5))
        qw = None if rows == 3 and dim % 5 == 0 else (1 + randn(g, dim, scale=0.3)).to(wt)
        k = dyk = kw = None
        if hk:
            k, dyk = (randn(g, rows, hk, dim, dtype=dtype, scale=s) for s in (0.7, 0.5))
            kw = (1 + randn(g, dim, scale=0.3)).to(wt)
        pos = freqs = None
        gain, eps = 1.0, 1e-6
        if rot:
            freqs, gain = ref.frequencies(rot, 10000.0, "parts", 2.0, 100.0)
            pos = torch.randint(0, 3000, (rows,), generator=g)
        args = (dev(qw), dev(kw), dev(pos), dev(freqs), gain, eps, interleaved)
        yq, yk = attention.head_norm(dev(q), dev(k), *args)
        turn = (pos, freqs, gain, interleaved)
        close(yq, *ref.head_norm(q, qw, eps, *turn), "q")
        if hk:
            close(yk, *ref.head_norm(k, kw, eps, *turn), "k")
        dqw = torch.empty(dim, dtype=wt, device="cuda")
        dkw = torch.empty(dim, dtype=wt, device="cuda") if hk and dim % 4 else None
        dq, dk, _, _ = attention.head_norm_backward(
            dev(dyq), dev(dyk), dev(q), dev(k), *args, grad_q_weight=dqw, grad_k_weight=dkw)
        want = ref.head_norm_backward(dyq, q, qw, eps, *turn)
        close(dq, *want[0], "grad q")
        close(dqw, *want[1], "grad q weight")
        if hk:
            want = ref.head_norm_backward(dyk, k, kw, eps, *turn)
            close(dk, *want[0], "grad k")
            if dkw is not None:
                close(dkw, *want[1], "grad k weight")
        # added to what is there, and not computed at all
        old = randn(g, dim, dtype=wt)
        acc = dev(old)
        again = attention.head_norm_backward(dev(dyq), dev(dyk), dev(q), dev(k), *args,
                                             grad_q_weight=acc, accumulate=True)
        assert torch.equal(again[0], dq)
        want = ref.head_norm_backward(dyq, q, qw, eps, *turn)[1]
        total = want[0] + old.double()
        close(acc, total, want[1] + 2 * 2.0 ** -24 * (want[0].abs() + old.double().abs()), "added")


@pytest.mark.parametrize("rows, hq, hk, dim", [(9001, 2, 1, 64), (700, 32, 8, 128), (5000, 1, 1, 8),
                                               (333, 40, 3, 96), (2600, 4, 0, 256)])
def test_head_norm_many_rows(rows, hq, hk, dim):
    """More work than one wave each: rows share waves, waves go round."""
    note(f"head norm rows={rows} heads={hq},{hk} dim={dim}")
    g = gen(rows)
    q, dyq = (randn(g, rows, hq, dim, dtype=BF16) for _ in range(2))
    k, dyk = (randn(g, rows, hk, dim, dtype=BF16) if hk else None for _ in range(2))
    qw, kw = 1 + randn(g, dim, scale=0.2), 1 + randn(g, dim, scale=0.2) if hk else None
    freqs, gain = ref.frequencies(dim)
    pos = torch.randint(0, 9000, (rows,), generator=g)
    turn = (pos, freqs, gain, False)
    args = (dev(qw), dev(kw), dev(pos), dev(freqs), gain, 1e-6, False)
    yq, yk = attention.head_norm(dev(q), dev(k), *args)
    close(yq, *ref.head_norm(q, qw, 1e-6, *turn), "q")
    dqw = torch.empty(dim, device="cuda")
    dkw = torch.empty(dim, device="cuda") if hk else None
    dq, dk, _, _ = attention.head_norm_backward(dev(dyq), dev(dyk), dev(q), dev(k), *args,
                                                grad_q_weight=dqw, grad_k_weight=dkw)
    want = ref.head_norm_backward(dyq, q, qw, 1e-6, *turn)
    close(dq, *want[0], "grad q")
    close(dqw, *want[1], "grad q weight")
    if hk:
        close(yk, *ref.head_norm(k, kw, 1e-6, *turn), "k")
        want = ref.head_norm_backward(dyk, k, kw, 1e-6, *turn)
        close(dk, *want[0], "grad k")
        close(dkw, *want[1], "grad k weight")


def test_head_norm_in_place_strided():
    """Queries and keys as slices of a projection's rows, replaced where they stand."""
    note("head norm in place")
    g = gen(11)
    b, n, hq, hk, dim = 2, 7, 6, 2, 72
    rows = randn(g, b, n, hq + 2 * hk, dim, dtype=F16)
    freqs, _ = ref.frequencies(dim)
    pos = torch.arange(n).expand(b, n).contiguous()
    w = 1 + randn(g, dim, scale=0.1)
    buf = dev(rows)
    q, k = buf[:, :, :hq], buf[:, :, hq:hq + hk]
    yq, yk = attention.head_norm(q, k, dev(w), dev(w), dev(pos), dev(freqs))
    attention.head_norm(q, k, dev(w), dev(w), dev(pos), dev(freqs), q_out=q, k_out=k)
    assert torch.equal(q, yq) and torch.equal(k, yk)
    assert torch.equal(buf[:, :, hq + hk:].cpu(), rows[:, :, hq + hk:])
    # the gradient into the incoming gradient's place
    dy = dev(randn(g, b, n, hq + hk, dim, dtype=F16))
    x = dev(rows)
    args = (x[:, :, :hq], x[:, :, hq:hq + hk], dev(w), dev(w), dev(pos), dev(freqs))
    dyq, dyk = dy[:, :, :hq], dy[:, :, hq:]
    dq, dk, _, _ = attention.head_norm_backward(dyq, dyk, *args)
    attention.head_norm_backward(dyq, dyk, *args, grad_q=dyq, grad_k=dyk)
    assert torch.equal(dyq, dq) and torch.equal(dyk, dk)


def test_head_norm_no_rows():
    note("head norm no rows")
    q = torch.empty((0, 3, 16), device="cuda")
    assert attention.head_norm(q, q)[0].shape == (0, 3, 16)
    freqs, _ = ref.frequencies(16)
    attention.rotate(q, torch.empty(0, dtype=torch.int64, device="cuda"), dev(freqs))
    w = torch.full((16,), 5.0, device="cuda")
    attention.head_norm_backward(q, q, q, q, grad_q_weight=w, accumulate=True)
    assert bool((w == 5).all())
    attention.head_norm_backward(q, q, q, q, grad_q_weight=w)
    assert bool((w == 0).all())


def test_head_norm_extremes():
    """NaN stays in its head; a head of zeros gives zeros, and r = 1 / sqrt(eps)."""
    note("head norm extremes")
    x = randn(gen(5), 3, 4, 40)
    x[0, 1, 7] = NAN
    x[1, 2] = 0.0
    x[2, 0] *= 1e-18
    y, _ = attention.head_norm(dev(x), None)
    want, bound = ref.head_norm(x, None, 1e-6)
    close(y, want, bound, "norm")
    assert int(torch.isnan(y).sum()) == 40


# --- attention ----------------------------------------------------------------

#   b, queries, keys, heads, kv_heads, dim, causal, window, sinks
SHAPES = [
    (1, 1, 1, 1, 1, 8, True, 0, 0),
    (2, 1, 33, 4, 1, 16, True, 0, 0),
    (1, 2, 2, 1, 1, 64, False, 0, 0),
    (2, 5, 5, 3, 3, 40, True, 0, 0),
    (1, 17, 70, 2, 2, 32, False, 0, 0),
    (2, 31, 64, 4, 2, 72, True, 0, 0),
    (1, 64, 64, 2, 1, 128, True, 0, 0),
    (1, 65, 65, 1, 1, 128, True, 1, 0),
    (2, 100, 131, 7, 1, 96, True, 20, 3),
    (1, 129, 200, 4, 4, 80, True, 64, 64),
    (1, 130, 130, 2, 2, 64, False, 0, 0),
    (1, 200, 200, 6, 2, 24, True, 33, 1),
    (1, 257, 300, 2, 1, 128, True, 50, 100),
    (3, 40, 1, 2, 1, 48, True, 0, 0),
    (1, 90, 50, 2, 2, 32, True, 7, 2),      # queries before the first key see nothing
    (1, 3, 700, 8, 2, 128, True, 0, 0),
    (1, 1, 1500, 16, 2, 64, True, 0, 0),
    (2, 1, 900, 64, 1, 32, True, 130, 5),
    (1, 4, 1000, 12, 4, 120, False, 0, 0),
    (1, 30, 2100, 4, 1, 64, True, 0, 0),
    (1, 12, 40, 1, 1, 104, True, 100, 4),   # a window past all keys
    (1, 2, 5000, 4, 1, 72, True, 0, 0),     # the most parts of keys
    (2, 70, 1100, 2, 1, 96, False, 0, 0),
    (60, 140, 90, 15, 5, 16, False, 0, 0),  # pairs in three chunks
    (150, 33, 70, 8, 8, 8, False, 0, 0),
]


def inputs(shape, dtype, seed, sharp=2.0):
    b, lq, lk, h, g_, d = shape[:6]
    g = gen(seed)
    q = randn(g, b, lq, h, d) * (1 + sharp * torch.rand((b, lq, h, 1), generator=g))
    return (q.to(dtype), *(randn(g, b, lk, g_, d, dtype=dtype) for _ in range(2)),
            randn(g, b, lq, h, d, dtype=dtype, scale=0.3))


def mask(shape):
    return {"causal": shape[6], "window": shape[7], "sinks": shape[8]}


def check(q, k, v, dy, what, lengths=None, scale=None, **kw):
    """Forward and backward of one call against the definitions."""
    ql, kl = lengths or (None, None)
    device = dict(kw, scale=scale, q_lengths=dev(ql), k_lengths=dev(kl))
    host = dict(kw, scale=scale, q_lengths=ql, k_lengths=kl)
    rest = torch.empty_like(q, device="cuda")
    out, lse = attention.attend(dev(q), dev(k), dev(v), rest=rest, **device)
    (want, bound), (wlse, blse) = ref.attend(q, k, v, **host)
    close(out, want, bound, f"{what}: out")
    close(lse, wlse, blse, f"{what}: lse")
    whole = out.cpu().double() + rest.cpu().double()
    room = bound + UNIT[q.dtype] * rest.cpu().double().abs() + TINY[q.dtype]
    off = ((whole - want).abs() - room)[torch.isfinite(want)]
    assert off.numel() == 0 or float(off.max()) <= 2.0 ** -24 * float(want.abs().max()) + 1e-30
    grads = attention.attend_backward(dev(dy), dev(q), dev(k), dev(v), out, lse, rest, **device)
    wants = ref.attend_backward(dy, q, k, v, out.cpu(), lse.cpu(), rest.cpu(), **host)
    for got, (a, e), name in zip(grads, wants, "qkv"):
        close(got, a, e, f"{what}: grad {name}")
    return out, lse, rest, grads


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_attend_shapes(shape, dtype):
    note(f"attend {shape} {dtype}")
    q, k, v, dy = inputs(shape, dtype, sum(shape[:6]))
    check(q, k, v, dy, f"{shape}", **mask(shape))


PARTS = [
    # batch, queries, keys, heads, kv_heads, dim, causal, window, sinks
    (129, 100, 100, 8, 1, 40, True, 20, 4),   # sinks in one part, the rest could have more
    (2, 150, 260, 8, 1, 24, True, 40, 150),   # two tiles of sinks
    (1, 700, 700, 8, 2, 64, False, 0, 0),
    (1, 515, 300, 6, 2, 72, True, 100, 130),  # queries before the first key
    (2, 333, 401, 5, 1, 128, True, 64, 3),    # columns of a query across tiles
    (9, 700, 900, 4, 2, 32, False, 0, 0),     # pairs in chunks of 8, 8 and 2
]


@pytest.mark.parametrize("shape", PARTS)
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_attend_parts(shape, dtype):
    """Gradients of keys whose columns are taken in parts, over whole and ragged
    sequences, from tensors that load as they are and from misaligned ones."""
    note(f"attend parts {shape} {dtype}")
    b, lq, lk = shape[:3]
    q, k, v, dy = inputs(shape, dtype, sum(shape[:6]))
    if b == 1 or b > 2:
        out, lse, rest, grads = check(q, k, v, dy, f"{shape}", **mask(shape))
        lengths = {}
    else:
        ql, kl = (torch.tensor([n, n // 2 + 7], dtype=torch.int32) for n in (lq, lk))
        out, lse, rest, grads = check(q, k, v, dy, f"{shape}", (ql, kl), **mask(shape))
        lengths = {"q_lengths": dev(ql), "k_lengths": dev(kl)}
    (sq, _), (sk, _), (sv, _), (sy, _) = spread(q), spread(k, 1, 3), spread(v, 5), spread(dy, 7, 5)
    same = attention.attend(sq, sk, sv, **lengths, **mask(shape))
    assert torch.equal(same[0], out) and torch.equal(same[1], lse)
    got = attention.attend_backward(sy, sq, sk, sv, out, lse, rest, **lengths, **mask(shape))
    for x, y in zip(got, grads):
        assert torch.equal(x, y)


@pytest.mark.parametrize("dim", list(range(8, 129, 8)))
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_attend_widths(dim, dtype):
    note(f"attend dim={dim} {dtype}")
    shape = (1, 37, 75, 2, 1, dim, True, 0, 0)
    check(*inputs(shape, dtype, dim), f"dim {dim}", scale=0.11, **mask(shape))


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("lq, lk", [(45, 45), (1, 80), (20, 300)])
def test_attend_lengths(lq, lk, dtype):
    """Ragged sequences: none, one, all, beyond what there is; what lies past them
    takes no part, and its outputs are zeros."""
    note(f"attend lengths {lq} {lk} {dtype}")
    kl = torch.tensor([0, 1, lk // 2, lk, lk + 100, -3, lk - 1], dtype=torch.int32)
    ql = torch.tensor([lq, 1, lq // 2, lq, lq, lq + 9, 0], dtype=torch.int32)
    for causal, window, sinks in ((True, 0, 0), (False, 0, 0), (True, 9, 2)):
        shape = (7, lq, lk, 4, 2, 40, causal, window, sinks)
        q, k, v, dy = inputs(shape, dtype, lk)
        for n in range(7):
            q[n, max(int(ql[n]), 0):] = NAN
            dy[n, max(int(ql[n]), 0):] = INF
            k[n, max(int(kl[n]), 0):] = INF
            v[n, max(int(kl[n]), 0):] = NAN
        out, lse, _, grads = check(q, k, v, dy, "lengths", (ql, kl), **mask(shape))
        for n in range(7):
            assert bool((out[n, max(int(ql[n]), 0):] == 0).all())
            assert bool((grads[0][n, max(int(ql[n]), 0):] == 0).all())
            for x in grads[1:]:
                assert bool((x[n, max(int(kl[n]), 0):] == 0).all())
        assert bool((out[0] == 0).all()) and bool((lse[0] == -INF).all())


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_attend_masked_values_take_no_part(dtype):
    """NaN, infinities and the type's extremes among keys, values, queries and
    gradients reach exactly the rows that see them."""
    big = torch.finfo(dtype).max
    for shape in ((1, 100, 100, 2, 1, 40, True, 11, 0), (1, 150, 150, 1, 1, 64, True, 0, 0),
                  (1, 4, 200, 4, 2, 32, True, 20, 3), (1, 1, 100, 2, 2, 128, True, 30, 0)):
        note(f"attend masked {shape} {dtype}")
        b, lq, lk = shape[:3]
        see = ref.visible(lq, lk, lq, lk, *shape[6:])
        q, k, v, dy = inputs(shape, dtype, 7)
        (want, bound), (wl, bl) = ref.attend(q, k, v, **mask(shape))
        clean = [x.cpu() for x in attention.attend(dev(q), dev(k), dev(v), **mask(shape))]
        for j, value in ((lk - 1, NAN), (lk // 2, INF), (lk - 40, -big), (lk - 21, NAN)):
            kk, vv = k.clone(), v.clone()
            kk[:, j], vv[:, j] = value, value
            rows = see[:, j]
            blind = ~rows
            out, lse = attention.attend(dev(q), dev(kk), dev(vv), **mask(shape))
            close(out.cpu()[:, blind], want[:, blind], bound[:, blind], "out of others")
            close(lse.cpu()[:, blind], wl[:, blind], bl[:, blind], "lse of others")
            if value != -big:
                assert bool(torch.isnan(out.cpu()[:, rows]).any(-1).all())
            grads = attention.attend_backward(dev(dy), dev(q), dev(kk), dev(vv), out, lse,
                                              **mask(shape))
            mixed = [torch.where(blind.view(1, -1, *[1] * (x.dim() - 2)), y.cpu(), x)
                     for x, y in zip(clean, (out, lse))]
            wants = ref.attend_backward(dy, q, k, v, *mixed, **mask(shape))
            apart = (see.t().float() @ rows.float()) == 0  # keys that none of the rows sees
            for got, (a, e), some in zip(grads, wants, (blind, apart, apart)):
                close(got.cpu()[:, some], a[:, some], e[:, some], "gradients of others")
        # a query and a gradient that are not finite reach the keys that they see
        i = lq // 2
        qq, dd = q.clone(), dy.clone()
        qq[:, i] = dd[:, i] = NAN
        out, lse = attention.attend(dev(qq), dev(k), dev(v), **mask(shape))
        dq, dk, dv = attention.attend_backward(dev(dd), dev(qq), dev(k), dev(v), out, lse,
                                               **mask(shape))
        others = torch.arange(lq) != i
        assert bool(torch.isfinite(dq.cpu()[:, others]).all())
        assert bool(torch.isnan(out.cpu()[:, i]).all())
        for x in (dk, dv):
            assert bool(torch.isfinite(x.cpu()[:, ~see[i]]).all())
            assert bool(torch.isnan(x.cpu()[:, see[i]]).all())


def test_attend_scores_of_minus_infinity():
    """A row all of whose scores are minus infinity has no softmax: NaN; one of
    some has that of the others."""
    note("attend -inf")
    q, k, v, _ = inputs((1, 3, 40, 1, 1, 16, False, 0, 0), F32, 2)
    q[:] = 0.0
    q[..., 0] = 1.0
    k[:, 5:9, :, 0] = -INF
    out, lse = attention.attend(dev(q), dev(k), dev(v), causal=False)
    keep = [j for j in range(40) if not 5 <= j < 9]
    (want, bound), (wl, bl) = ref.attend(q, k[:, keep], v[:, keep], causal=False)
    close(out, want, bound, "out")
    close(lse, wl, bl, "lse")
    k[..., 0] = -INF
    out, lse = attention.attend(dev(q), dev(k), dev(v), causal=False)
    assert bool(torch.isnan(out).all()) and bool((lse == -INF).all())


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_attend_large_scores(dtype):
    """Scores of some hundreds that grow along the keys: the maximum moves in every
    tile, and only the last keys have weight."""
    note(f"attend large scores {dtype}")
    g = gen(9)
    b, n, h, d = 1, 200, 2, 64
    q = torch.full((b, n, h, d), 2.0).to(dtype)
    k = (torch.arange(n).view(1, n, 1, 1) * 0.25 + torch.zeros(b, n, h, d)).to(dtype)
    v, dy = randn(g, b, n, h, d, dtype=dtype), randn(g, b, n, h, d, dtype=dtype)
    check(q, k, v, dy, "growing")
    check(q, k.flip(1).contiguous(), v, dy, "falling")


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_attend_strides(dtype):
    """Queries, keys and values as misaligned slices with gaps between heads and
    rows, outputs likewise; nothing between them is written."""
    shape = (2, 21, 50, 4, 2, 40, True, 0, 0)
    note(f"attend strides {dtype}")
    q, k, v, dy = inputs(shape, dtype, 21)
    plain = attention.attend(dev(q), dev(k), dev(v))
    grads = attention.attend_backward(dev(dy), dev(q), dev(k), dev(v), *plain)
    (sq, _), (sk, _), (sv, _), (sy, _) = spread(q), spread(k, 1, 3), spread(v, 5), spread(dy, 7, 5)
    out, buf = spread(torch.zeros_like(q), 3, 7)
    o, lse = attention.attend(sq, sk, sv, out=out)
    assert o is out and torch.equal(out, plain[0]) and torch.equal(lse, plain[1])
    untouched(out, buf)
    places = [spread(torch.zeros_like(t), 3, 1) for t in (q, k, v)]
    got = attention.attend_backward(sy, sq, sk, sv, out, lse, grad_q=places[0][0],
                                    grad_k=places[1][0], grad_v=places[2][0])
    for a, c, place in zip(got, grads, places):
        assert torch.equal(a, c)
        untouched(*place)
    # heads before rows, one key head standing for all sequences
    t = [x.transpose(1, 2).contiguous().transpose(1, 2) for x in (dev(q), dev(k), dev(v))]
    assert torch.equal(attention.attend(*t)[0], plain[0])
    one = dev(k[:1]).expand(2, -1, -1, -1)
    same = attention.attend(dev(q), one, one)[0]
    both = dev(k[:1].repeat(2, 1, 1, 1))
    assert torch.equal(same, attention.attend(dev(q), both, both)[0])


@pytest.mark.parametrize("dim", [8, 24, 40, 72, 104])
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_attend_gaps_hold_anything(dim, dtype):
    """Heads with NaN between them, aligned (tiles then load as they are) and not,
    give what dense ones give."""
    note(f"attend gaps {dim} {dtype}")
    for shape in ((2, 140, 150, 6, 2, dim, True, 60, 3), (3, 1, 333, 4, 2, dim, True, 0, 0)):
        q, k, v, dy = inputs(shape, dtype, dim)
        plain = attention.attend(dev(q), dev(k), dev(v), **mask(shape))
        grads = attention.attend_backward(dev(dy), dev(q), dev(k), dev(v), *plain, **mask(shape))
        for pad in (24, 3):
            at = []
            for t in (q, k, v, dy):
                b, n, h, d = t.shape
                buf = torch.full((b, n, h, d + pad), NAN, dtype=dtype, device="cuda")
                at.append(buf[..., :d])
                at[-1].copy_(t)
            out, lse = attention.attend(*at[:3], **mask(shape))
            assert torch.equal(out, plain[0]) and torch.equal(lse, plain[1])
            got = attention.attend_backward(at[3], *at[:3], out, lse, **mask(shape))
            for x, y in zip(got, grads):
                assert torch.equal(x, y)


def test_attend_parts_of_no_weight():
    """A long cache taken in parts, of which some have no finite score."""
    note("attend parts of no weight")
    q, k, v, _ = inputs((1, 1, 3000, 1, 1, 16, True, 0, 0), BF16, 6)
    q[..., 0] = 1.0
    k[..., 0] = 0.0
    k[:, 200:2100, :, 0] = -INF
    keep = [j for j in range(3000) if not 200 <= j < 2100]
    out, lse = attention.attend(dev(q), dev(k), dev(v))
    (want, bound), (wl, bl) = ref.attend(q, k[:, keep], v[:, keep])
    close(out, want, bound, "out")
    close(lse, wl, bl, "lse")


@pytest.mark.parametrize("scale", [2.0 ** -60, 1e-9, 2.0 ** 60])
def test_attend_extreme_scales(scale):
    note(f"attend scale {scale}")
    shape = (1, 40, 50, 2, 1, 16, True, 0, 0)
    q, k, v, dy = inputs(shape, F32, 3)
    q, k = (q, k) if scale < 1 else (q * 2.0 ** -30, k * 2.0 ** -30)
    check(q, k, v, dy, f"scale {scale}", scale=scale)


def test_attend_offsets_past_32_bits():
    """Rows of keys and values that far apart that offsets pass 2^31 elements."""
    note("attend far rows")
    n, d, step = 70, 32, (1 << 25) + 8
    q, k, v, dy = inputs((1, 70, n, 1, 1, d), BF16, 4)
    buf = torch.empty(n * step, dtype=BF16, device="cuda")
    fk = buf.as_strided((1, n, 1, d), (0, step, d, 1), 0)
    fv = buf.as_strided((1, n, 1, d), (0, step, d, 1), d)
    gk = buf.as_strided((1, n, 1, d), (0, step, d, 1), 2 * d)
    gv = buf.as_strided((1, n, 1, d), (0, step, d, 1), 3 * d)
    fk.copy_(k)
    fv.copy_(v)
    plain = attention.attend(dev(q), dev(k), dev(v))
    out, lse = attention.attend(dev(q), fk, fv)
    assert torch.equal(out, plain[0]) and torch.equal(lse, plain[1])
    one = attention.attend(dev(q)[:, -1:], fk, fv)[0]
    assert torch.equal(one, attention.attend(dev(q)[:, -1:].contiguous(), dev(k), dev(v))[0])
    want = attention.attend_backward(dev(dy), dev(q), dev(k), dev(v), out, lse)
    got = attention.attend_backward(dev(dy), dev(q), fk, fv, out, lse, grad_k=gk, grad_v=gv)
    for a, c in zip(got, want):
        assert torch.equal(a, c)
    # far heads of queries, in the rotation and the norm
    x = buf.as_strided((3, 66, 16), (32, step, 1), 0)
    src = randn(gen(8), 3, 66, 16, dtype=BF16)
    x.copy_(src)
    freqs, _ = ref.frequencies(16)
    pos = torch.arange(3)
    y = attention.rotate(x, dev(pos), dev(freqs))
    assert torch.equal(y, attention.rotate(dev(src), dev(pos), dev(freqs)))
    attention.head_norm(x, None, None, None, dev(pos), dev(freqs), q_out=x)
    assert torch.equal(x, attention.head_norm(dev(src), None, None, None, dev(pos),
                                              dev(freqs))[0])


def test_attend_nothing():
    note("attend nothing")
    for b, lq, lk in ((0, 4, 4), (2, 0, 4), (2, 4, 0)):
        q = torch.ones((b, lq, 2, 16), device="cuda")
        k = torch.ones((b, lk, 1, 16), device="cuda")
        out, lse = attention.attend(q, k, k)
        assert bool((out == 0).all()) and bool((lse == -INF).all())
        dq, dk, dv = attention.attend_backward(q, q, k, k, out, lse)
        for x in (dq, dk, dv):
            assert bool((x == 0).all())


@pytest.mark.parametrize("lq", [1, 3, 33])
def test_cache_steps_equal_the_prompt(lq):
    """Single tokens and pieces over a longer cache give the prompt's rows."""
    note(f"attend steps {lq}")
    b, n, h, g_, d = 2, 99, 8, 2, 64
    for window, sinks in ((0, 0), (17, 3)):
        q, k, v, _ = inputs((b, n, n, h, g_, d), BF16, 5)
        (want, bound), (wl, bl) = ref.attend(q, k, v, window=window, sinks=sinks)
        ck, cv = (torch.full((b, 160, g_, d), NAN, dtype=BF16, device="cuda") for _ in range(2))
        filled = torch.zeros(b, dtype=torch.int32, device="cuda")
        for at in range(0, n, lq):
            m = min(lq, n - at)
            ck[:, at:at + m], cv[:, at:at + m] = dev(k[:, at:at + m]), dev(v[:, at:at + m])
            filled += m
            out, lse = attention.attend(dev(q[:, at:at + m]), ck, cv, window=window, sinks=sinks,
                                        k_lengths=filled)
            close(out, want[:, at:at + m], bound[:, at:at + m], f"step {at}")
            close(lse, wl[:, at:at + m], bl[:, at:at + m], f"step {at} lse")


@pytest.mark.parametrize("shape", [(1, 9, 9, 2, 1, 16, True, 0, 0), (1, 40, 70, 2, 2, 24, True, 9, 2),
                                   (1, 12, 12, 3, 1, 8, False, 0, 0)])
def test_attend_gradient_by_differences(shape):
    """Along random directions, <gradient, v> against (L(x + e v) - L(x - e v)) / 2e
    of the 64-bit forward pass; e = 1e-5 leaves an error of about 1e-10."""
    note(f"attend differences {shape}")
    q, k, v, top = inputs(shape, F32, 6, sharp=0.5)
    out, lse = attention.attend(dev(q), dev(k), dev(v), **mask(shape))
    grads = attention.attend_backward(dev(top), dev(q), dev(k), dev(v), out, lse, **mask(shape))
    see = ref.visible(shape[1], shape[2], shape[1], shape[2], *shape[6:])
    some = see.any(1)

    def loss(q, k, v):
        r = shape[3] // shape[4]
        kk, vv = k.repeat_interleave(r, 2), v.repeat_interleave(r, 2)
        s = torch.einsum("blhd,bthd->bhlt", q, kk) * shape[5] ** -0.5
        p = torch.softmax(s.masked_fill(~see, -1e300), -1) * some[:, None]
        return float((torch.einsum("bhlt,bthd->blhd", p, vv) * top.double()).sum())

    args, g, e = [x.double() for x in (q, k, v)], gen(1), 1e-5
    for n, grad in enumerate(grads):
        for _ in range(3):
            d = torch.randn(args[n].shape, generator=g, dtype=torch.float64)
            hi, lo = list(args), list(args)
            hi[n], lo[n] = args[n] + e * d, args[n] - e * d
            want = (loss(*hi) - loss(*lo)) / (2 * e)
            got = float((grad.cpu().double() * d).sum())
            size = float((grad.cpu().double() * d).abs().sum()) + float(top.abs().sum())
            assert abs(got - want) <= ((shape[5] + shape[2] + 64) * 2.0 ** -24 + 1e-8) * size


def test_head_norm_gradient_by_differences():
    note("head norm differences")
    g = gen(4)
    rows, heads, dim, e = 3, 2, 20, 1e-5
    x, top, w = randn(g, rows, heads, dim), randn(g, rows, heads, dim), 1 + randn(g, dim, scale=0.2)
    freqs, gain = ref.frequencies(12, 100.0, "parts", 2.0, 50.0)
    pos = torch.tensor([3, 11, 700])
    gw = torch.empty(dim, device="cuda")
    gx = attention.head_norm_backward(dev(top), None, dev(x), None, dev(w), None, dev(pos),
                                      dev(freqs), gain, 1e-6, True, grad_q_weight=gw)[0]

    def loss(x, w):
        return float((ref.head_norm(x, w, 1e-6, pos, freqs, gain, True)[0] * top.double()).sum())

    args = [x.double(), w.double()]
    for n, grad in enumerate((gx, gw)):
        for _ in range(3):
            d = torch.randn(args[n].shape, generator=g, dtype=torch.float64)
            hi, lo = list(args), list(args)
            hi[n], lo[n] = args[n] + e * d, args[n] - e * d
            want = (loss(*hi) - loss(*lo)) / (2 * e)
            got = float((grad.cpu().double() * d).sum())
            size = float((grad.cpu().double() * d).abs().sum()) + float(top.abs().sum())
            assert abs(got - want) <= ((dim + 64) * 2.0 ** -24 + 1e-8) * size


def test_run_together():
    """A block's attention as a training step runs it: norms and rotation of a
    projection's slices, attention, and back into slices of the rows' gradient;
    every stage against its definition on what the stage before gave."""
    note("run together")
    g = gen(31)
    b, n, h, kv, d = 2, 75, 6, 2, 72
    window, sinks = 20, 2
    rows = randn(g, b, n, h + 2 * kv, d, dtype=BF16)
    qw, kw = 1 + randn(g, d, scale=0.2), 1 + randn(g, d, scale=0.2)
    freqs, gain = ref.frequencies(36, 10000.0, "linear", 2.0)
    pos = (torch.arange(n) + torch.tensor([[5], [4000]])).contiguous()
    lengths = torch.tensor([n, 51], dtype=torch.int32)
    dy = randn(g, b, n, h, d, dtype=BF16, scale=0.1)
    x, grad = dev(rows), torch.zeros_like(rows, device="cuda")
    cut = [(slice(None), slice(None), slice(*s)) for s in ((0, h), (h, h + kv), (h + kv, None))]
    turn = dict(positions=dev(pos), freqs=dev(freqs), gain=gain)
    hide = dict(window=window, sinks=sinks, q_lengths=dev(lengths), k_lengths=dev(lengths))
    q, k = attention.head_norm(x[cut[0]], x[cut[1]], dev(qw), dev(kw), **turn)
    rest = torch.empty_like(q)
    out, lse = attention.attend(q, k, x[cut[2]], rest=rest, **hide)
    dq, dk, _ = attention.attend_backward(dev(dy), q, k, x[cut[2]], out, lse, rest,
                                          grad_v=grad[cut[2]], **hide)
    gqw, gkw = torch.empty(d, device="cuda"), torch.empty(d, device="cuda")
    attention.head_norm_backward(dq, dk, x[cut[0]], x[cut[1]], dev(qw), dev(kw), **turn,
                                 grad_q=grad[cut[0]], grad_k=grad[cut[1]], grad_q_weight=gqw,
                                 grad_k_weight=gkw)
    t = (pos, freqs, gain, False)
    close(q, *ref.head_norm(rows[cut[0]], qw, 1e-6, *t), "q")
    close(k, *ref.head_norm(rows[cut[1]], kw, 1e-6, *t), "k")
    host = dict(window=window, sinks=sinks, q_lengths=lengths, k_lengths=lengths)
    (want, bound), (wl, bl) = ref.attend(q.cpu(), k.cpu(), rows[cut[2]], **host)
    close(out, want, bound, "out")
    close(lse, wl, bl, "lse")
    wants = ref.attend_backward(dy, q.cpu(), k.cpu(), rows[cut[2]], out.cpu(), lse.cpu(),
                                rest.cpu(), **host)
    for got, (a, e), name in zip((dq, dk, grad[cut[2]]), wants, "qkv"):
        close(got, a, e, f"grad {name}")
    for c, w, dd, gw, name in ((cut[0], qw, dq, gqw, "q"), (cut[1], kw, dk, gkw, "k")):
        (a, e), (aw, ew) = ref.head_norm_backward(dd.cpu(), rows[c], w, 1e-6, *t)
        close(grad[c], a, e, f"rows' grad {name}")
        close(gw, aw, ew, f"weight grad {name}")


def test_graphs_share_a_workspace():
    """Two captured calls with one workspace, replayed in turn with eager work
    between; every replay equals the eager result."""
    note("attend graphs")
    shapes = ((1, 1, 3000, 8, 2, 64, True, 0, 0), (2, 130, 130, 4, 2, 40, True, 16, 2))
    data = [[dev(x) for x in inputs(s, BF16, 3)] for s in shapes]
    room = torch.empty(max(max(attention.attend_workspace_bytes(d[0], d[1]),
                               attention.attend_backward_workspace_bytes(d[0], d[1]))
                           for d in data), dtype=torch.uint8, device="cuda")

    def call(d, s):
        q, k, v, dy = d
        out, lse = attention.attend(q, k, v, workspace=room, **mask(s))
        return (out, lse, *attention.attend_backward(dy, q, k, v, out, lse, workspace=room,
                                                     **mask(s)))

    eager = [call(d, s) for d, s in zip(data, shapes)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for d, s in zip(data, shapes):
            call(d, s)
    torch.cuda.current_stream().wait_stream(side)
    graphs, outs = [], []
    for d, s in zip(data, shapes):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(call(d, s))
        graphs.append(graph)
    for turn in range(4):
        for graph, got, want in zip(graphs, outs, eager):
            for x in got:
                x.fill_(SENTINEL)
            graph.replay()
            torch.cuda.synchronize()
            for a, c in zip(got, want):
                assert torch.equal(a, c)
            room.fill_(turn)  # the program's own work on the same memory


def test_heads_in_a_graph():
    """Norm, rotation and their gradients captured in one graph: every replay
    takes the positions that stand there then."""
    note("heads graph")
    rows, h, d = 300, 5, 64
    g = gen(12)
    x, dy = (dev(randn(g, rows, h, d, dtype=BF16)) for _ in range(2))
    w, freqs = dev(1 + randn(g, d, scale=0.1)), dev(ref.frequencies(d)[0])
    pos = torch.zeros(rows, dtype=torch.int64, device="cuda")
    gw = torch.empty(d, device="cuda")

    def call():
        y = attention.head_norm(x, None, w, None, pos, freqs)[0]
        z = attention.rotate(x, pos, freqs)
        dz = attention.rotate_backward(dy, pos, freqs)
        dx = attention.head_norm_backward(dy, None, x, None, w, None, pos, freqs,
                                          grad_q_weight=gw)[0]
        return y, z, dz, dx, gw

    call()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = call()
    for start in (0, 17, 100000):
        pos.copy_(torch.arange(rows) + start)
        want = [t.clone() for t in call()]
        for t in got:
            t.fill_(SENTINEL)
        graph.replay()
        torch.cuda.synchronize()
        for a, c in zip(got, want):
            assert torch.equal(a, c)


def test_two_streams_and_repeats():
    """The same bits on every run, and on streams beside each other."""
    note("attend streams")
    shape = (2, 140, 140, 4, 2, 64, True, 33, 1)
    q, k, v, dy = (dev(x) for x in inputs(shape, F16, 8))
    first = attention.attend(q, k, v, **mask(shape))
    grads = attention.attend_backward(dy, q, k, v, *first, **mask(shape))
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for st in streams:
        out, lse = attention.attend(q, k, v, stream=st, **mask(shape))
        with torch.cuda.stream(st):
            got.append((out, lse, attention.attend_backward(dy, q, k, v, out, lse,
                                                            **mask(shape))))
    torch.cuda.synchronize()
    for out, lse, g in got:
        assert torch.equal(out, first[0]) and torch.equal(lse, first[1])
        for a, c in zip(g, grads):
            assert torch.equal(a, c)


def test_forward_calls_warn_without_a_graph():
    note("attend warnings")
    q = torch.zeros((1, 2, 1, 8), device="cuda", requires_grad=True)
    for f in (lambda: attention.attend(q, q, q), lambda: attention.head_norm(q, None),
              lambda: attention.rotate(q, torch.zeros((1, 2), dtype=torch.int64, device="cuda"),
                                       dev(ref.frequencies(8)[0]))):
        with pytest.warns(UserWarning, match="requires grad"):
            f()
    before = torch.empty_like(q, requires_grad=False)
    version = before._version
    with torch.no_grad():
        attention.attend(q, q, q, out=before)
    assert before._version > version
