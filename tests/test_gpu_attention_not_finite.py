"""Attention and its gradients where inputs are not finite: NaN and infinities reach
exactly what sees them. Against the 64-bit definitions of tests/attention_util.py."""
from __future__ import annotations

import math

import pytest
import torch

from paper_2007_13005_amd import attention
from tests import attention_util as ref
from tests.gpu_util import note
from tests.test_gpu_attention import BF16, F16, F32, INF, NAN, dev, inputs, mask
from tests.tokens_util import close

pytestmark = pytest.mark.gpu

TYPES = [F32, F16, BF16]
# batch, queries, keys, heads, kv_heads, dim, causal, window, sinks
SHAPES = [
    (1, 150, 150, 2, 1, 64, True, 0, 0),
    (2, 140, 150, 6, 2, 40, True, 30, 2),   # columns of a query across tiles
    (1, 90, 130, 3, 3, 128, False, 0, 0),
    (1, 700, 700, 8, 2, 24, True, 0, 0),    # gradients of keys in parts
    (1, 3, 700, 4, 2, 72, True, 100, 5),    # few columns, keys in parts
    (2, 1, 90, 8, 2, 32, True, 0, 0),
]


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("what", ["query", "gradient", "key"])
def test_nan_reaches_all_that_sees_it(shape, dtype, what):
    """A NaN in a query, in its output's gradient, or in a key, alone: the weights p =
    exp(s - lse), or d, of every pair of a spoiled row are NaN, so the gradients of all
    keys that the row sees are; nothing else is."""
    note(f"attend nan {shape} {dtype} {what}")
    lq, lk = shape[1:3]
    see = ref.visible(lq, lk, lq, lk, *shape[6:])
    q, k, v, dy = inputs(shape, dtype, 29)
    i, j = lq // 2, int(see[lq // 2].nonzero()[0])
    spoiled = torch.arange(lq) == i
    if what == "query":
        q[:, i, :, 3] = NAN
    elif what == "gradient":
        dy[:, i] = NAN
    else:
        k[:, j, :, 5] = NAN
        spoiled = see[:, j]
    out, lse = attention.attend(dev(q), dev(k), dev(v), **mask(shape))
    if what != "gradient":
        assert torch.equal(torch.isnan(lse.cpu()), spoiled[None, :, None].expand(lse.shape))
        assert bool(torch.isnan(out.cpu()[:, spoiled]).all())
        assert bool(torch.isfinite(out.cpu()[:, ~spoiled]).all())
    dq, dk, dv = (x.cpu() for x in attention.attend_backward(
        dev(dy), dev(q), dev(k), dev(v), out, lse, **mask(shape)))
    touched = see[spoiled].any(0)
    assert bool(torch.isnan(dq[:, spoiled]).all())
    assert bool(torch.isfinite(dq[:, ~spoiled]).all())
    for name, x in (("k", dk), ("v", dv)):
        assert bool(torch.isnan(x[:, touched]).all()), f"grad {name} lost a NaN"
        assert bool(torch.isfinite(x[:, ~touched]).all()), f"grad {name} got a NaN"


def spoil(x, at):
    """x with the values of `at`, {(row, dim): value}, in all heads."""
    bad = x.clone()
    for (row, d), value in at.items():
        bad[:, row, :, d] = value
    return bad


def reach(see, at, rows, dim):
    """(rows, dim): the sum over what is seen of the values of `at`, zeros elsewhere."""
    total = torch.zeros((rows, dim), dtype=torch.float64)
    for (j, d), value in at.items():
        total[:, d] += torch.where(see[:, j], value, 0.0)
    return total


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("dtype", TYPES)
def test_values_that_are_not_finite(shape, dtype):
    """Single NaN and infinities among the values: the rows that see them have them, in
    their column alone, infinities of both signs a NaN, however small the weight."""
    note(f"attend values {shape} {dtype}")
    lq, lk, dim = shape[1], shape[2], shape[5]
    see = ref.visible(lq, lk, lq, lk, *shape[6:])
    q, k, v, _ = inputs(shape, dtype, 31)
    # one key that no query likes: a weight below 2^-200
    k[:, lk // 3] = 0.0
    k[:, lk // 3, :, 0] = -200.0
    q[..., 0] = 0.6 * dim ** 0.5 + 6.0
    at = {(lk // 3, 1): INF, (lk - 1, 0): NAN, (lk - 2, dim - 1): -INF, (lk // 2, 4): INF,
          (lk // 2 + 1, 4): -INF, (lk // 2, 7): -INF, (lk - lq, 6): INF}
    (want, bound), (wl, bl) = ref.attend(q, k, v, **mask(shape))
    want = want + reach(see, at, lq, dim)[None, :, None, :]
    out, lse = attention.attend(dev(q), dev(k), dev(spoil(v, at)), **mask(shape))
    close(out, want, bound, "out")
    close(lse, wl, bl, "lse")


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("dtype", TYPES)
def test_gradients_that_are_not_finite(shape, dtype):
    """Single NaN and infinities in the rows' gradients: grad_v has them in their column
    alone, the keys that such a row sees have no finite grad_k, the row no finite
    grad_q, and the others what they have without."""
    note(f"attend gradients {shape} {dtype}")
    lq, lk, dim = shape[1], shape[2], shape[5]
    see = ref.visible(lq, lk, lq, lk, *shape[6:])
    q, k, v, dy = inputs(shape, dtype, 37)
    rest = torch.empty_like(q, device="cuda")
    out, lse = attention.attend(dev(q), dev(k), dev(v), rest=rest, **mask(shape))
    at = {(lq // 2, 1): INF, (lq - 1, 0): NAN, (lq // 2, 4): -INF, (lq // 3, 4): INF}
    spoiled = torch.zeros(lq, dtype=torch.bool)
    spoiled[[i for i, _ in at]] = True
    (wq, bq), (wk, bk), (wv, bv) = ref.attend_backward(
        dy, q, k, v, out.cpu(), lse.cpu(), rest.cpu(), **mask(shape))
    wv = wv + reach(see.t(), at, lk, dim)[None, :, None, :]
    dq, dk, dv = (x.cpu() for x in attention.attend_backward(
        dev(spoil(dy, at)), dev(q), dev(k), dev(v), out, lse, rest, **mask(shape)))
    touched = see[spoiled].any(0)
    close(dv, wv, bv, "grad v")
    close(dq[:, ~spoiled], wq[:, ~spoiled], bq[:, ~spoiled], "grad q")
    close(dk[:, ~touched], wk[:, ~touched], bk[:, ~touched], "grad k")
    assert not bool(torch.isfinite(dq[:, spoiled]).any())
    assert not bool(torch.isfinite(dk[:, touched]).any())


def test_keys_of_minus_infinity_have_no_weight():
    """A visible key whose score is minus infinity: rows and gradients as without it."""
    note("attend gradients, -inf")
    for dtype in TYPES:
        q, k, v, dy = inputs((1, 70, 70, 1, 1, 16, True, 0, 0), dtype, 2)
        q[..., 0] = 1.0
        k[..., 0] = 0.0
        k[:, 20:23, :, 0] = -INF
        keep = [j for j in range(70) if not 20 <= j < 23]
        out, lse = attention.attend(dev(q), dev(k), dev(v))
        see = ref.visible(70, 70, 70, 70, True, 0, 0)
        assert bool(torch.isfinite(out).all())
        dq, dk, dv = (x.cpu() for x in attention.attend_backward(dev(dy), dev(q), dev(k), dev(v),
                                                                 out, lse))
        # the key's infinite value times a d of zero
        some = see[:, 20:23].any(1)
        assert bool(torch.isfinite(dq[..., 1:]).all())
        assert bool(torch.isfinite(dq[:, ~some]).all())
        assert bool(torch.isfinite(dk[:, keep]).all()) and bool(torch.isfinite(dv[:, keep]).all())
        assert bool((dk[:, 20:23] == 0).all()) and bool((dv[:, 20:23] == 0).all())


@pytest.mark.parametrize("shape", SHAPES + [(1, 515, 300, 6, 2, 72, True, 100, 130),
                                            (1, 300, 300, 1, 1, 96, False, 0, 0)])
@pytest.mark.parametrize("top, wide", [(6000.0, 1.0), (24000.0, 1.0), (60000.0, 1.0),
                                       (60000.0, 4.0)])
@pytest.mark.parametrize("every", [1, 40])
def test_large_gradients_in_fp16(shape, top, wide, every):
    """|d| between 2^10, where d carried times 2^6 passes fp16, and 2^17.5: within the
    bound of smaller ones. A d that would pass is carried so that the largest of its
    row (key) is at least 2^14: half a step of fp16's smallest is then largest *
    2^-39."""
    note(f"attend large gradients {shape} {top} {wide} {every}")
    q, k, v, dy = inputs(shape, F16, 41)
    q, k, v, dy = q * 0.25, k * 0.25, v * wide, dy * 0.01
    dy[:, ::every] = (dy[:, ::every].float() * (top / 0.03)).clamp(-60000, 60000).half()
    k[:, ::7] *= 8.0
    q[:, ::3] *= 8.0
    rest = torch.empty_like(q, device="cuda")
    kw = dict(mask(shape), scale=0.02)  # gradients of queries and keys stay within fp16
    out, lse = attention.attend(dev(q), dev(k), dev(v), rest=rest, **kw)
    wants = ref.attend_backward(dy, q, k, v, out.cpu(), lse.cpu(), rest.cpu(), **kw)
    grads = attention.attend_backward(dev(dy), dev(q), dev(k), dev(v), out, lse, rest, **kw)
    # |d| <= |dy| |v| + |dy| |out + rest| <= 2 |dy| max |v|, of each pair
    lq, lk = shape[1:3]
    most = 2.0 * float(dy.double().norm(dim=-1).max()) * float(v.double().norm(dim=-1).max())
    step = most * 2.0 ** -39 * 0.02
    room = (lk * float(k.double().abs().max()), lq * shape[3] // shape[4] *
            float(q.double().abs().max()), 0.0)
    for got, (a, e), name, n in zip(grads, wants, "qkv", room):
        assert float(a.abs().max()) < 65000.0
        close(got, a, e + step * n, f"grad {name}")


@pytest.mark.parametrize("queries", [1, 70])
def test_many_small_weights_in_fp16(queries):
    """Keys of which each has 2^-26 of a query's weight, 2^13 of them together 2^-13,
    beside one key whose value is zero: a weight's rounding is half a step of 2^-24
    below 2^-14, and weights are carried times 2^7 relative to a whole maximum that is
    8 behind at most: each is off by 2^-25 * 2^-7 * 2 of the largest."""
    note(f"attend small weights {queries}")
    n, d, b = 1 << 13, 32, 300  # (as many sequences as make a cache whole, not in parts)
    q = torch.zeros((1, queries, 1, d), dtype=F16)
    k = torch.zeros((1, n + 1, 1, d), dtype=F16)
    v = torch.full((1, n + 1, 1, d), 500.0, dtype=F16)
    q[..., 0] = 1.0
    k[:, 0, :, 0] = 18.0  # e^18 = 2^25.97
    v[:, 0] = 0.0
    (want, bound), _ = ref.attend(q.float(), k.float(), v.float(), scale=1.0, causal=False)
    assert 0.05 < float(want.min()) < 0.1
    each = 2.0 ** -31 * n * 500.0
    for order in (slice(None), torch.arange(n, -1, -1)):
        args = (dev(t).expand(b, -1, -1, -1) for t in (q, k[:, order], v[:, order]))
        out, _ = attention.attend(*args, scale=1.0, causal=False)
        assert bool((out == out[:1]).all())
        close(out[:1], want, bound + 2.0 ** -11 * want.abs() + each, "out")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shape", [(1, 70, 300, 2, 1, 32, True, 0, 0),
                                   (1, 1, 900, 4, 1, 64, True, 0, 0),
                                   (1, 200, 200, 1, 1, 128, False, 0, 0)])
def test_values_near_the_types_largest(shape, dtype):
    """Rows are means of the values, so finite values have finite rows: values of 2^126
    and scores that grow along the keys."""
    note(f"attend largest values {shape} {dtype}")
    q, k, v, _ = inputs(shape, dtype, 43)
    lk = shape[2]
    q[..., 0] = 1.0
    k[..., 0] = (torch.arange(lk) * 0.125).view(1, lk, 1).to(dtype)
    v = torch.sign(v) * 2.0 ** 126
    (want, bound), (wl, bl) = ref.attend(q, k, v, scale=1.0, **mask(shape))
    out, lse = attention.attend(dev(q), dev(k), dev(v.to(dtype)), scale=1.0, **mask(shape))
    close(out, want, bound, "out")
    close(lse, wl, bl, "lse")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("power", [126, 122, 120, 118, 116, 112, 108])
def test_equal_weights_of_large_values(power, dtype):
    """The same with equal weights, whose sums pass fp32 within a tile, where waves' or
    parts' sums join, or not at all."""
    note(f"attend equal weights {power} {dtype}")
    for queries, keys, heads in ((1, 128, 4), (1, 3000, 2), (1, 20000, 8), (150, 700, 2)):
        q = torch.zeros((1, queries, heads, 16), dtype=dtype)
        k = torch.zeros((1, keys, 1, 16), dtype=dtype)
        v = torch.full((1, keys, 1, 16), 2.0 ** power, dtype=dtype)
        v[..., 1::2] *= -1.0
        out, lse = attention.attend(dev(q), dev(k), dev(v), causal=False)
        want = v[:, :1].double().expand(1, queries, heads, 16)
        # count + 16 roundings of the sums and the quotient
        close(out, want, (keys + 16) * 2.0 ** -24 * want.abs(), f"{keys}")
        total = torch.full(lse.shape, math.log(keys), dtype=torch.float64)
        close(lse, total, 64 * 2.0 ** -24 * (1 + total), f"lse {keys}")


def least_time(call) -> float:
    """Of five calls, in milliseconds."""
    begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    times = []
    for _ in range(6):
        begin.record()
        call()
        end.record()
        end.synchronize()
        times.append(begin.elapsed_time(end))
    return min(times[1:])


def costs(dtype, spoiled):
    """Times of a causal prompt's forward and backward pass, of clean inputs and of ones
    that `spoiled` changes in place."""
    shape = (1, 1024, 1024, 8, 2, 64, True, 0, 0)
    times = []
    for change in (None, spoiled):
        q, k, v, dy = (dev(x) for x in inputs(shape, dtype, 47))
        if change:
            change(q, k, v, dy)
        out, lse = attention.attend(q, k, v)
        grads = [torch.empty_like(x) for x in (q, k, v)]
        room = torch.empty(attention.attend_backward_workspace_bytes(q, k), dtype=torch.uint8,
                           device="cuda")
        times.append((least_time(lambda: attention.attend(q, k, v, out=out, lse=lse)),
                      least_time(lambda: attention.attend_backward(
                          dy, q, k, v, out, lse, grad_q=grads[0], grad_k=grads[1],
                          grad_v=grads[2], workspace=room))))
    return times


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("value, row", [(NAN, 60), (INF, 1000), (-INF, 500)])
def test_a_value_that_is_not_finite_costs_little(value, row, dtype):
    """Rows that are summed again are summed by tiles: a call takes a few times a clean
    one's time (pair by pair it took hundreds of times that)."""
    note(f"attend time, {value} among the values {dtype}")

    def change(q, k, v, dy):
        v[0, row, 0, 5] = value

    clean, spoiled = costs(dtype, change)
    assert spoiled[0] < 20 * clean[0], (clean, spoiled)


SPOIL = {
    "value": lambda q, k, v, dy: v[0, 60, 0].fill_(NAN),
    "query": lambda q, k, v, dy: q[0, 500, 0, 3:4].fill_(NAN),
    "all values": lambda q, k, v, dy: v.fill_(NAN),
    "all queries": lambda q, k, v, dy: q.fill_(NAN),
    "key": lambda q, k, v, dy: k[0, 60, 0, 3:4].fill_(INF),
    "gradient": lambda q, k, v, dy: dy[0, 1000, 0, 3:4].fill_(-INF),
    "large gradients": lambda q, k, v, dy: (dy.mul_(10000.0), q.mul_(4.0)),
}


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("what", sorted(SPOIL))
def test_a_gradient_that_is_not_finite_costs_little(what, dtype):
    """The same for the backward pass, for matrices full of NaN, and for finite gradients
    that fp16 does not hold as they are carried."""
    note(f"attend time, gradients, {what} {dtype}")
    clean, spoiled = costs(dtype, SPOIL[what])
    assert max(s / c for s, c in zip(spoiled, clean)) < 20, (clean, spoiled)
