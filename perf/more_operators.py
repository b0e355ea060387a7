"""The attention operators' workloads, as plain cases: rotary positions, norms of
queries and keys with the rotation in the same pass, and attention with a window
and first tokens that stay visible, for training and for single tokens.

A case is one call as a training or serving loop makes it: weights, frequencies,
output buffers and workspaces are kept by the program, activations change. Its
fields: op; dtype (of activations); b sequences.

  rotate          l rows of h heads of d values each; the first rot of a head's
                  values turn, interleaved or in halves; scaling of the
                  frequencies; far: sequences start at positions below it
  norm, norm_grad the same for h heads of queries and g of keys beside each
                  other in a row that also holds g heads of values; param: type
                  of the weights and their gradients
  attend, attend_grad, attend_token
                  l queries (h heads) of each sequence, the last ones of its t
                  keys (g heads); causal, window (0: none), sinks; ragged: the
                  sequences are shorter, by the rule in _lengths
"""
import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}
EPS = 1e-6
BASE_ANGLE = 500000.0
# frequencies by parts: turns within `LENGTH` positions from which a frequency is
# kept, and up to which it is divided by FACTOR
FACTOR, LENGTH, LOW, HIGH = 8.0, 8192, 1.0, 32.0

ROTATE = {"dtype": "bf16", "b": 1, "l": 1, "h": 16, "d": 128, "rot": 128, "interleaved": False,
          "scaling": "none", "far": 4096}
NORM = {**ROTATE, "h": 32, "g": 8, "param": "f32"}
ATTEND = {"dtype": "bf16", "b": 1, "l": 1, "t": 1, "h": 32, "g": 8, "d": 128, "causal": True,
          "window": 0, "sinks": 0, "ragged": False}
BASE = {"rotate": ROTATE, "norm": NORM, "norm_grad": NORM, "attend": ATTEND,
        "attend_grad": ATTEND, "attend_token": ATTEND}


def _case(name, op, **kw):
    return {"name": name, "op": op, **BASE[op], **kw}


def listed():
    return [
        # one new token of a long context, scaled frequencies: latency of a call
        _case("rotate_one_token", "rotate", dtype="f16", scaling="parts", far=100000),
        # a training batch's queries, a quarter of each head turned in pairs
        _case("rotate_batch", "rotate", b=8, l=4096, rot=32, interleaved=True),
        # the new tokens of 32 requests
        _case("norm_tokens", "norm", b=32, far=30000, scaling="parts"),
        # a training batch of text
        _case("norm_batch", "norm", b=8, l=4096),
        # a few rows of odd heads in single precision
        _case("norm_grad_small", "norm_grad", dtype="f32", b=3, l=331, h=5, g=5, d=72, rot=36),
        # the training batch backwards
        _case("norm_grad_batch", "norm_grad", b=8, l=4096),
        # 64 images of 14 x 14 patches and one more row, every row sees every other
        _case("attend_images", "attend", dtype="f16", b=64, l=197, t=197, h=16, g=16, d=64,
              causal=False),
        # a long prompt through a window with sinks
        _case("attend_prompt", "attend", l=8192, t=8192, window=2048, sinks=4),
        # images backwards, 12 heads
        _case("attend_grad_images", "attend_grad", dtype="f16", b=64, l=197, t=197, h=12, g=12,
              d=64, causal=False),
        # a ragged training batch of text backwards
        _case("attend_grad_text", "attend_grad", b=4, l=4096, t=4096, h=16, g=4, window=1024,
              sinks=4, ragged=True),
        # one request's new token over all of its cache
        _case("attend_token_one", "attend_token", dtype="f16", t=32768),
        # the new tokens of 64 requests of mixed lengths, a window with sinks
        _case("attend_token_batch", "attend_token", b=64, t=6000, window=2048, sinks=16,
              ragged=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng: random.Random):
    op = rng.choice(["rotate", "norm", "norm_grad", "attend", "attend_grad", "attend_token"])
    c = dict(BASE[op], op=op)
    c["dtype"] = rng.choice(["f32", "f16", "f16", "f16", "bf16", "bf16", "bf16", "bf16"])
    if op in ("rotate", "norm", "norm_grad"):
        c["d"] = rng.choice([64, 128, 128, 256, 80, 96, 2 * rng.randrange(8, 120)])
        c["rot"] = rng.choice([c["d"], c["d"], 2 * max(1, c["d"] // 4), 2 * max(1, c["d"] // 8)])
        c["interleaved"] = rng.random() < 0.4
        c["scaling"] = rng.choice(["none", "none", "linear", "base", "parts"])
        c["far"] = _log(rng, 1, 1 << 20)
        c["b"] = _log(rng, 1, 16)
        c["l"] = _log(rng, 1, 4096)
        if op == "rotate":
            c["h"] = _log(rng, 1, 40)
        else:
            c["g"] = rng.choice([1, 2, 4, 8, rng.randrange(1, 17)])
            c["h"] = c["g"] * rng.choice([1, 2, 4, 8])
            c["param"] = rng.choice(["f32", "f32", c["dtype"]])
    else:
        c["d"] = rng.choice([64, 128, 128, 128, 32, 80, 96, 8 * rng.randrange(2, 17)])
        c["g"] = rng.choice([1, 2, 4, 8, rng.randrange(1, 13)])
        c["h"] = c["g"] * rng.choice([1, 1, 2, 4, 4, 7, 8])
        c["ragged"] = rng.random() < 0.5
        if op == "attend_token":
            c["b"] = _log(rng, 1, 64)
            c["t"] = _log(rng, 1, 32768)
            c["l"] = 1
        else:
            c["b"] = _log(rng, 1, 64)
            # (a query that sees one key alone has no gradient of its own)
            c["t"] = _log(rng, 16 if op == "attend_grad" else 2, 8192)
            c["l"] = c["t"] if op == "attend_grad" or rng.random() < 0.7 else _log(rng, 1, c["t"])
            c["causal"] = rng.random() < 0.75
        if c["causal"] and rng.random() < 0.6:
            c["window"] = _log(rng, 8 if op == "attend_grad" else 1, c["t"])
            c["sinks"] = rng.choice([0, 1, 4, 16, rng.randrange(0, 100)])
    most = [work(k) for k in listed() if k["op"] == op]
    while any(work(c)[f] > max(m[f] for m in most) for f in ("bytes", "flops")) or (
            op in ("attend", "attend_grad") and c["b"] * c["h"] * c["l"] * c["t"] > 1 << 31):
        # the plain form holds all scores of a call
        if c["b"] > 1:
            c["b"] = c["b"] * 3 // 4
        elif op in ("rotate", "norm", "norm_grad") or (c["l"] > 1 and c["l"] < c["t"]):
            c["l"] = max(1, c["l"] * 3 // 4)
        else:
            c["l"] = c["t"] = max(1, c["t"] * 3 // 4)
            if op == "attend_token":
                c["l"] = 1
    return c


# What a pass cannot do without

def _lengths(case):
    """Queries and keys of each sequence (lists), all of them unless ragged: then
    from a quarter to the whole, spread evenly by the golden ratio."""
    b, l, t = case["b"], case["l"], case["t"]
    if not case["ragged"]:
        return [l] * b, [t] * b
    keys = [max(1, int(t * (0.25 + 0.75 * math.fmod((k + 1) * 0.6180339887498949, 1.0))))
            for k in range(b)]
    return [n if l == t else min(l, n) for n in keys], keys


def _pairs(case):
    """Pairs of a query and a key it sees, and keys that any query sees, over all sequences."""
    pairs = seen = 0
    for q, k in zip(*_lengths(case)):
        if not case["causal"]:
            pairs += q * k
            seen += k
            continue
        p = torch.arange(k - q, k, dtype=torch.int64)
        w = case["window"] or k
        first = (p - w + 1).clamp(min=0)
        pairs += int((p + 1 - first + torch.minimum(first, torch.tensor(case["sinks"]))).sum())
        lo = max(0, k - q - w + 1)
        seen += k - lo + min(lo, case["sinks"])
    return pairs, seen


def work(case):
    op, d, s = case["op"], case["d"], SIZE[case["dtype"]]
    if op in ("rotate", "norm", "norm_grad"):
        n = case["b"] * case["l"]
        heads = case["h"] if op == "rotate" else case["h"] + case["g"]
        small = 8 * n + 4 * case["rot"]
        if op == "rotate":
            return {"bytes": 2 * n * heads * d * s + small, "flops": 3 * n * heads * case["rot"]}
        q = 2 * d * SIZE[case["param"]]
        if op == "norm":
            return {"bytes": 2 * n * heads * d * s + small + q,
                    "flops": n * heads * (4 * d + 3 * case["rot"])}
        return {"bytes": 3 * n * heads * d * s + small + 2 * q,
                "flops": n * heads * (10 * d + 3 * case["rot"])}
    pairs, seen = _pairs(case)
    rows = sum(_lengths(case)[0])
    q, k = rows * case["h"] * d * s, seen * case["g"] * d * s
    if op == "attend_grad":
        return {"bytes": 4 * q + 4 * k + 4 * rows * case["h"],
                "flops": 10 * pairs * case["h"] * d}
    return {"bytes": 2 * q + 2 * k + 4 * rows * case["h"], "flops": 4 * pairs * case["h"] * d}


# Inputs

def _normal(gen, shape, scale, dtype):
    return (torch.randn(shape, generator=gen, device="cuda") * scale).to(DTYPES[dtype])


def _frequencies(case):
    """Radians a position (64 bits) and the factor of the cosines and sines."""
    rot = case["rot"]
    i = torch.arange(rot // 2, dtype=torch.float64, device="cuda")
    base = BASE_ANGLE
    if case["scaling"] == "base" and rot > 2:
        base = base * FACTOR ** (rot / (rot - 2))
    f = base ** (-2 * i / rot)
    if case["scaling"] == "linear":
        f = f / FACTOR
    if case["scaling"] == "parts":
        keep = ((f * LENGTH / (2 * math.pi) - LOW) / (HIGH - LOW)).clamp(0, 1)
        f = f * keep + f / FACTOR * (1 - keep)
        return f, 0.1 * math.log(FACTOR) + 1.0
    return f, 1.0


def _inputs(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    op, b, d, dt = case["op"], case["b"], case["d"], case["dtype"]
    s = {"case": case}
    if op in ("rotate", "norm", "norm_grad"):
        n, h = case["l"], case["h"]
        start = torch.randint(0, case["far"], (b, 1), generator=gen, device="cuda")
        s["positions"] = start + torch.arange(n, device="cuda")
        s["freqs"], s["gain"] = _frequencies(case)
        if op == "rotate":
            s["x"] = _normal(gen, (b, n, h, d), 1.0, dt)
            return s
        g = case["g"]
        # a projection's rows: queries, keys and values beside each other
        rows = _normal(gen, (b, n, (h + 2 * g), d), 1.5, dt)
        s["q"], s["k"] = rows[:, :, :h], rows[:, :, h:h + g]
        for name in ("q_weight", "k_weight"):
            s[name] = (1 + 0.2 * torch.randn(d, generator=gen, device="cuda")).to(
                DTYPES[case["param"]])
        if op == "norm_grad":
            s["grad_q_out"] = _normal(gen, (b, n, h, d), 0.02, dt)
            s["grad_k_out"] = _normal(gen, (b, n, g, d), 0.02, dt)
        return s
    l, t, h, g = case["l"], case["t"], case["h"], case["g"]
    # normed queries and keys, so that logits are of order one; some rows' are sharper
    sharp = 1 + torch.rand((b, l, 1, 1), generator=gen, device="cuda") ** 4 * 2
    s["q"] = (torch.randn((b, l, h, d), generator=gen, device="cuda") * sharp).to(DTYPES[dt])
    s["k"] = _normal(gen, (b, t, g, d), 1.0, dt)
    if op == "attend_token":
        s["v"] = _normal(gen, (b, t, g, d), 1.0, dt)
    else:  # values as they stand in the projection's rows
        s["v"] = _normal(gen, (b, t, 2 * g, d), 1.0, dt)[:, :, g:]
    s["scale"] = d ** -0.5
    s["q_lengths"] = s["k_lengths"] = None
    if case["ragged"]:
        s["q_lengths"], s["k_lengths"] = (torch.tensor(v, dtype=torch.int32, device="cuda")
                                          for v in _lengths(case))
    if op == "attend_grad":
        s["grad_out"] = _normal(gen, (b, l, h, d), 0.02, dt)
        # what a program kept of the forward pass: the rows, what their rounding
        # took off, and the logarithms of the sums
        y, s["lse"] = _attend(s)
        s["out"] = y.to(DTYPES[dt])
        s["rest"] = (y - s["out"].float()).to(DTYPES[dt])
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if not own:
        return s
    from paper_2007_13005_amd import attention
    op = case["op"]

    def like(x, dtype=None):
        return torch.empty(x.shape, dtype=dtype or x.dtype, device="cuda")

    def room(n):
        return torch.empty((n,), dtype=torch.uint8, device="cuda")

    if op in ("rotate", "norm", "norm_grad"):
        s["freqs"], s["gain"] = attention.rotary_frequencies(
            case["rot"], BASE_ANGLE, case["scaling"], FACTOR, LENGTH, LOW, HIGH)
        if op == "rotate":
            s["x_out"] = like(s["x"])
        else:
            s["q_to"], s["k_to"] = like(s["q"]), like(s["k"])
        if op == "norm_grad":
            s["grad_q_weight"], s["grad_k_weight"] = like(s["q_weight"]), like(s["k_weight"])
            s["workspace"] = room(attention.head_norm_workspace_bytes(s["q"], s["k"]))
        return s
    s["mask"] = {"scale": s["scale"], "causal": case["causal"], "window": case["window"],
                 "sinks": case["sinks"], "q_lengths": s["q_lengths"], "k_lengths": s["k_lengths"]}
    if op == "attend_grad":
        s["grads"] = like(s["q"]), like(s["k"]), like(s["v"])
        s["workspace"] = room(attention.attend_backward_workspace_bytes(s["q"], s["k"]))
    else:
        s["out"] = like(s["q"])
        s["lse"] = torch.empty(s["q"].shape[:3], dtype=torch.float32, device="cuda")
        s["workspace"] = room(attention.attend_workspace_bytes(
            s["q"], s["k"], case["causal"], case["window"], case["sinks"]))
    return s


def _run_own(s):
    from paper_2007_13005_amd import attention
    case = s["case"]
    op = case["op"]
    if op == "rotate":
        return attention.rotate(s["x"], s["positions"], s["freqs"], s["gain"],
                                case["interleaved"], out=s["x_out"])
    if op == "norm":
        return attention.head_norm(s["q"], s["k"], s["q_weight"], s["k_weight"], s["positions"],
                                   s["freqs"], s["gain"], EPS, case["interleaved"],
                                   q_out=s["q_to"], k_out=s["k_to"])
    if op == "norm_grad":
        return attention.head_norm_backward(
            s["grad_q_out"], s["grad_k_out"], s["q"], s["k"], s["q_weight"], s["k_weight"],
            s["positions"], s["freqs"], s["gain"], EPS, case["interleaved"], grad_q=s["q_to"],
            grad_k=s["k_to"], grad_q_weight=s["grad_q_weight"], grad_k_weight=s["grad_k_weight"],
            workspace=s["workspace"])
    if op == "attend_grad":
        q, k, v = s["grads"]
        return attention.attend_backward(s["grad_out"], s["q"], s["k"], s["v"], s["out"],
                                         s["lse"], rest=s["rest"], **s["mask"], grad_q=q,
                                         grad_k=k, grad_v=v, workspace=s["workspace"])
    return attention.attend(s["q"], s["k"], s["v"], **s["mask"], out=s["out"], lse=s["lse"],
                            workspace=s["workspace"])


# The plain forms

def _turn(x, s, sign):
    """x in 32 bits, its first rot values turned by sign times the angles."""
    case = s["case"]
    rot = case["rot"]
    angle = s["positions"].double()[..., None, None] * s["freqs"]
    c, n = (angle.cos() * s["gain"]).float(), (angle.sin() * (s["gain"] * sign)).float()
    if case["interleaved"]:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        turned = torch.stack((a * c - b * n, b * c + a * n), -1).flatten(-2)
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        turned = torch.cat((a * c - b * n, b * c + a * n), -1)
    return torch.cat((turned, x[..., rot:]), -1)


def _norm(x, weight, s):
    z = x.float()
    z = z * (1.0 / torch.sqrt((z * z).mean(-1, keepdim=True) + EPS)) * weight.float()
    return _turn(z, s, 1.0).to(x.dtype)


def _norm_grad(dy, x, weight, s):
    g, z = _turn(dy.float(), s, -1.0), x.float()
    r = 1.0 / torch.sqrt((z * z).mean(-1, keepdim=True) + EPS)
    z = z * r
    u = g * weight.float()
    dx = (u - z * (u * z).mean(-1, keepdim=True)) * r
    return dx.to(x.dtype), (g * z).sum((0, 1, 2)).to(weight.dtype)


def _visible(s):
    """(b, l, t): whether a query sees a key."""
    case = s["case"]
    b, l, t = case["b"], case["l"], case["t"]
    i, j = torch.arange(l, device="cuda"), torch.arange(t, device="cuda")
    ql = s["q_lengths"] if s["q_lengths"] is not None else torch.full((b,), l, device="cuda")
    kl = s["k_lengths"] if s["k_lengths"] is not None else torch.full((b,), t, device="cuda")
    p = (i[None, :] + (kl - ql)[:, None])[:, :, None]
    see = (i[None, :, None] < ql[:, None, None]) & (j < kl[:, None, None])
    if case["causal"]:
        see = see & (j <= p)
        if case["window"]:
            see = see & ((j > p - case["window"]) | (j < case["sinks"]))
    return see


def _by_key_head(x, g):
    """(b, l, h, d) to (b, g, h / g * l, d) in 32 bits."""
    b, l, h, d = x.shape
    return x.float().view(b, l, g, h // g, d).permute(0, 2, 3, 1, 4).reshape(b, g, -1, d)


def _back(x, shape):
    b, l, h, d = shape
    return x.view(b, x.shape[1], -1, l, d).permute(0, 3, 1, 2, 4).reshape(b, l, h, d)


def _scores(s):
    """(b, g, h / g, l, t) in 32 bits, minus infinity where a key is not seen."""
    q, k = s["q"], s["k"]
    b, l, h, d = q.shape
    g = k.shape[2]
    x = torch.matmul(_by_key_head(q, g) * s["scale"], k.float().permute(0, 2, 3, 1).contiguous())
    return x.view(b, g, h // g, l, -1).masked_fill_(~_visible(s)[:, None, None], -math.inf)


def _attend(s):
    """Rows and logarithms of the sums, both in 32 bits."""
    x = _scores(s)
    m = x.amax(-1, keepdim=True).clamp_(min=-3e38)
    x = (x - m).exp_()
    total = x.sum(-1, keepdim=True)
    b, g, r, l, t = x.shape
    y = torch.matmul(x.view(b, g, r * l, t), s["v"].float().permute(0, 2, 1, 3).contiguous())
    y = torch.where(total > 0, y.view(b, g, r, l, -1) / total, 0.0)
    lse = torch.where(total > 0, m + total.log(), -math.inf)
    return (_back(y.reshape(b, g, r * l, -1), s["q"].shape),
            _back(lse.reshape(b, g, r * l, 1), (b, l, g * r, 1))[..., 0])


def _attend_grad(s):
    g = s["k"].shape[2]
    lse = _by_key_head(s["lse"][..., None], g)
    p = _scores(s)
    b, _, r, l, t = p.shape
    p = p.view(b, g, r * l, t)
    p = (p - lse.clamp(min=-3e38)).exp_()
    dy = _by_key_head(s["grad_out"], g)
    y = _by_key_head(s["out"], g) + _by_key_head(s["rest"], g)
    delta = (dy * y).sum(-1, keepdim=True)
    dv = torch.matmul(p.transpose(2, 3).contiguous(), dy)
    ds = torch.matmul(dy, s["v"].float().permute(0, 2, 3, 1).contiguous())
    ds = ds.sub_(delta).mul_(p).mul_(s["scale"])
    dq = torch.matmul(ds, s["k"].float().permute(0, 2, 1, 3).contiguous())
    dk = torch.matmul(ds.transpose(2, 3).contiguous(), _by_key_head(s["q"], g))
    dt = s["q"].dtype
    return (_back(dq, s["q"].shape).to(dt), dk.permute(0, 2, 1, 3).to(dt),
            dv.permute(0, 2, 1, 3).to(dt))


def run(s):
    if own:
        return _run_own(s)
    op = s["case"]["op"]
    if op == "rotate":
        return _turn(s["x"].float(), s, 1.0).to(s["x"].dtype)
    if op == "norm":
        return _norm(s["q"], s["q_weight"], s), _norm(s["k"], s["k_weight"], s)
    if op == "norm_grad":
        dq, dwq = _norm_grad(s["grad_q_out"], s["q"], s["q_weight"], s)
        dk, dwk = _norm_grad(s["grad_k_out"], s["k"], s["k_weight"], s)
        return dq, dk, dwq, dwk
    if op == "attend_grad":
        return _attend_grad(s)
    y, lse = _attend(s)
    return y.to(s["q"].dtype), lse


# The definition in 64 bits

def _turn64(x, s, conj):
    """The pairs as complex numbers times gain e^(i p f), or its conjugate."""
    rot = s["case"]["rot"]
    phase = s["positions"].double()[..., None, None] * s["freqs"]
    z = torch.polar(torch.full_like(phase, s["gain"]), -phase if conj else phase)
    y = x.clone()
    head = x[..., :rot]
    if s["case"]["interleaved"]:
        pair = torch.view_as_complex(head.reshape(*head.shape[:-1], rot // 2, 2).contiguous())
        y[..., :rot] = torch.view_as_real(pair * z).flatten(-2)
    else:
        w = torch.complex(head[..., :rot // 2].contiguous(), head[..., rot // 2:].contiguous()) * z
        y[..., :rot // 2], y[..., rot // 2:rot] = w.real, w.imag
    return y


def _sees(s, n):
    """(l, t) of sequence n."""
    case = s["case"]
    ql, kl = (v[n] for v in _lengths(case))
    p = torch.arange(case["l"], device="cuda")[:, None] + (kl - ql)
    j = torch.arange(case["t"], device="cuda")[None, :]
    hidden = (p >= kl) | (j >= kl)
    if case["causal"]:
        hidden |= j > p
        if case["window"]:
            hidden |= (p - j >= case["window"]) & (j >= case["sinks"])
    return ~hidden


def exact(case, seed):
    s = _inputs(case, seed)
    op = case["op"]
    if op == "rotate":
        return _turn64(s["x"].double(), s, False)
    if op in ("norm", "norm_grad"):
        outs, weights = [], []
        for one in ("q", "k"):
            x, w = s[one].double(), s[one + "_weight"].double()
            length = (x.square().mean(-1, keepdim=True) + EPS).sqrt()
            if op == "norm":
                outs.append(_turn64(x / length * w, s, False))
                continue
            g = _turn64(s["grad_%s_out" % one].double(), s, True)
            u = g * w
            # the Jacobian of x / length: (I - x x^T / (d length^2)) / length
            along = (u * x).sum(-1, keepdim=True) / (x.shape[-1] * length.square())
            outs.append((u - x * along) / length)
            weights.append((g * x / length).sum((0, 1, 2)))
        return (*outs, *weights)
    b, l, t, h, g, d = (case[f] for f in ("b", "l", "t", "h", "g", "d"))
    r = h // g
    grad = op == "attend_grad"
    out = torch.zeros((b, l, h, d), dtype=torch.float64, device="cuda")
    lse = torch.full((b, l, h), -math.inf, dtype=torch.float64, device="cuda")
    if grad:
        dk = torch.zeros((b, t, g, d), dtype=torch.float64, device="cuda")
        dv = torch.zeros_like(dk)
    for n in range(b):
        see = _sees(s, n)
        some = see.any(1)
        for a in range(g):
            q = s["q"][n, :, a * r:(a + 1) * r].double().transpose(0, 1).contiguous()
            k, v = s["k"][n, :, a].double(), s["v"][n, :, a].double()
            x = torch.matmul(q.view(r * l, d), k.t().contiguous()).view(r, l, t) * s["scale"]
            x = x.masked_fill(~see, -math.inf)
            z = torch.where(some, torch.logsumexp(x, -1), 0.0)
            x = (x - z[..., None]).exp_()
            if not grad:
                out[n, :, a * r:(a + 1) * r] = torch.matmul(
                    x.view(r * l, t), v).view(r, l, d).transpose(0, 1)
                lse[n, :, a * r:(a + 1) * r] = torch.where(some, z, -math.inf).t()
                continue
            dy = s["grad_out"][n, :, a * r:(a + 1) * r].double().transpose(0, 1).reshape(r * l, d)
            x = x.view(r * l, t)
            dv[n, :, a] = torch.matmul(x.t().contiguous(), dy)
            dp = torch.matmul(dy, v.t().contiguous())
            ds = x * (dp - (x * dp).sum(1, keepdim=True)) * s["scale"]
            dk[n, :, a] = torch.matmul(ds.t().contiguous(), q.view(r * l, d))
            out[n, :, a * r:(a + 1) * r] = torch.matmul(ds, k).view(r, l, d).transpose(0, 1)
    return (out, dk, dv) if grad else (out, lse)
