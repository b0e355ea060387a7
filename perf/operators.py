"""The token operators' workloads, as plain cases: patch embedding, embedding
lookup and layer norm, each forward and backward, with their plain forms.

A case is one call as a training or serving loop makes it: the weights, output
buffers and workspaces are kept by the program, activations and ids change.
Its fields: op; dtype (of weights and activations, of the table for a lookup).

  patch, patch_grad   n images of h x w pixels in c channels, patch side p,
                      width d, nhwc, image (the pixels' type), pos (position
                      rows), grad (type of the parameters' gradients)
  embed, embed_grad   n ids of a vocabulary of v, width d, act (the rows'
                      type), grad, wide (64-bit ids), holes (share of ids that
                      name no token: places that image rows take)
  norm, norm_grad     n rows of width d, param (type of the weights and their
                      gradients), residual (a second input is added first, or
                      a gradient comes past the norm)
"""
import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}
MEAN = tuple(v * 255.0 for v in (0.485, 0.456, 0.406))
STD = tuple(v * 255.0 for v in (0.229, 0.224, 0.225))
EPS = 1e-5

PATCH = {"n": 1, "c": 3, "h": 224, "w": 224, "p": 16, "d": 768, "nhwc": False, "image": "f16",
         "dtype": "f16", "pos": True, "grad": "f32"}
EMBED = {"n": 1, "v": 32000, "d": 1024, "dtype": "bf16", "act": "bf16", "grad": "f32",
         "wide": True, "holes": 0.0}
NORM = {"n": 1, "d": 1024, "dtype": "bf16", "param": "f32", "residual": True}
BASE = {"patch": PATCH, "patch_grad": PATCH, "embed": EMBED, "embed_grad": EMBED, "norm": NORM,
        "norm_grad": NORM}


def _case(name, op, **kw):
    return {"name": name, "op": op, **BASE[op], **kw}


def listed():
    return [
        # one photo of a request, preprocessed to fp16: latency of a call
        _case("patch_one_photo", "patch"),
        # a training batch of fp16 images into a bf16 model, 14-pixel patches
        _case("patch_batch_p14", "patch", n=256, p=14, d=1024, dtype="bf16"),
        # channels-last fp32 frames of an odd size, everything in single precision
        _case("patch_grad_f32_nhwc", "patch_grad", n=16, h=203, w=331, p=20, d=380, nhwc=True,
              image="f32", dtype="f32"),
        # the training batch's weight gradient, 16-pixel patches
        _case("patch_grad_batch", "patch_grad", n=256, dtype="bf16"),
        # one generated token's row
        _case("embed_one_token", "embed", d=4096, dtype="f16", act="f16"),
        # a batch's text and image places, single-precision table, bf16 rows
        _case("embed_batch", "embed", n=33001, v=65536, dtype="f32", holes=0.25),
        # a small vocabulary and an odd width, fp32
        _case("embed_grad_small", "embed_grad", n=777, v=5003, d=321, dtype="f32", act="f32",
              wide=False, holes=0.1),
        # a training batch's dense gradient
        _case("embed_grad_batch", "embed_grad", n=65536, v=64000, holes=0.25),
        # one generated token after its residual sum
        _case("norm_one_token", "norm", d=4096, dtype="f16", param="f16"),
        # 256 images of 197 rows
        _case("norm_batch", "norm", n=50432),
        # a few rows of an odd width, fp32
        _case("norm_grad_small", "norm_grad", n=331, d=1001, dtype="f32", residual=False),
        # 256 images of 197 rows, backwards
        _case("norm_grad_batch", "norm_grad", n=50432),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng):
    """Half of them whole hundreds of bytes, as models have; half any number."""
    if rng.random() < 0.5:
        return rng.choice([128, 192, 256, 384, 512, 640, 768, 1024, 1280, 1536, 2048, 2560, 4096])
    return _log(rng, 48, 3000)


def draw(rng: random.Random):
    op = rng.choice(["patch", "patch_grad", "embed", "embed_grad", "norm", "norm_grad"])
    c = dict(BASE[op], op=op)
    c["dtype"] = rng.choice(["f32", "f16", "f16", "bf16", "bf16"])
    if op in ("patch", "patch_grad"):
        c["image"] = "f32" if c["dtype"] == "f32" else rng.choice(["f16", "f16", "f32"])
        c["p"] = rng.choice([14, 16, 16, 16, rng.randrange(4, 25)])
        c["h"] = rng.choice([224, 224, 160, 384, rng.randrange(96, 400)])
        c["w"] = rng.choice([c["h"], c["h"], rng.randrange(96, 400)])
        c["d"] = min(_width(rng), 1536)
        c["nhwc"] = rng.random() < 0.25
        c["pos"] = rng.random() < 0.75
        c["grad"] = rng.choice(["f32", "f32", c["dtype"]])
        c["n"] = _log(rng, 1, 256)
    elif op in ("embed", "embed_grad"):
        c["d"] = _width(rng)
        c["v"] = _log(rng, 256, 131072)
        c["n"] = _log(rng, 1, 65536)
        c["act"] = rng.choice([c["dtype"], c["dtype"], "bf16"])
        c["grad"] = rng.choice(["f32", "f32", c["dtype"]])
        c["wide"] = rng.random() < 0.7
        c["holes"] = rng.choice([0.0, 0.25, rng.random()])
    else:
        c["d"] = _width(rng)
        c["n"] = _log(rng, 1, 65536)
        c["param"] = rng.choice(["f32", "f32", c["dtype"]])
        c["residual"] = rng.random() < 0.6
    most = max((work(k) for k in listed() if k["op"] == op), key=lambda k: k["bytes"])
    while work(c)["bytes"] > most["bytes"] or work(c)["flops"] > most["flops"]:
        if op == "embed_grad" and c["v"] > c["n"]:  # its output alone can be too large
            c["v"] = c["v"] * 7 // 8
        else:
            c["n"] = max(1, c["n"] * 3 // 4)
    return c


# What a pass cannot do without

def _grid(case):
    return case["h"] // case["p"], case["w"] // case["p"]


def _distinct(n, v):
    """Expected number of distinct tokens among n drawn with p(i) ~ ln((i+2)/(i+1))."""
    i = torch.arange(v, dtype=torch.float64)
    p = torch.log((i + 2) / (i + 1)) / math.log(v + 1)
    return float(-torch.expm1(n * torch.log1p(-p)).sum())


def work(case):
    op, d, n = case["op"], case["d"], case["n"]
    s = SIZE[case["dtype"]]
    if op in ("patch", "patch_grad"):
        th, tw = _grid(case)
        k, t = case["c"] * case["p"] ** 2, th * tw
        m = n * t
        nbytes = m * k * SIZE[case["image"]] + m * d * s
        params = d * k + d + (t * d if case["pos"] else 0)
        if op == "patch":
            return {"bytes": nbytes + params * s, "flops": 2 * m * k * d}
        return {"bytes": nbytes + params * SIZE[case["grad"]],
                "flops": 2 * m * k * d + 2 * m * d}
    if op in ("embed", "embed_grad"):
        a = SIZE[case["act"]]
        ids = n * (8 if case["wide"] else 4)
        some = n * (1 - case["holes"])
        if op == "embed":
            return {"bytes": int(ids + _distinct(some, case["v"]) * d * s + n * d * a),
                    "flops": int(some * d)}
        return {"bytes": int(ids + some * d * a + case["v"] * d * SIZE[case["grad"]]),
                "flops": int(some * d + case["v"] * d)}
    q = SIZE[case["param"]]
    if op == "norm":
        streams = 4 if case["residual"] else 2
        return {"bytes": streams * n * d * s + 2 * d * q + 8 * n, "flops": 8 * n * d}
    streams = 4 if case["residual"] else 3
    return {"bytes": streams * n * d * s + 3 * d * q + 8 * n, "flops": 14 * n * d}


# Inputs

def _images(gen, case):
    """Normalised pictures: smooth fields and grain, as the preprocessing writes them."""
    n, c, h, w = case["n"], case["c"], case["h"], case["w"]
    y = torch.arange(h, device="cuda", dtype=torch.float32)[None, None, :, None]
    x = torch.arange(w, device="cuda", dtype=torch.float32)[None, None, None, :]
    k = torch.rand((4, n, c, 1, 1), generator=gen, device="cuda") * 0.06
    img = torch.sin(k[0] * x + k[1] * y) * torch.cos(k[2] * x - k[3] * y) * 90.0 + 127.0
    img += torch.randn(img.shape, generator=gen, device="cuda") * 16.0
    img.clamp_(0, 255)
    mean = torch.tensor([MEAN[i % 3] for i in range(c)], device="cuda")[None, :, None, None]
    std = torch.tensor([STD[i % 3] for i in range(c)], device="cuda")[None, :, None, None]
    img = ((img - mean) / std).to(DTYPES[case["image"]])
    return img.permute(0, 2, 3, 1).contiguous() if case["nhwc"] else img


def _normal(gen, shape, scale, dtype):
    return (torch.randn(shape, generator=gen, device="cuda") * scale).to(DTYPES[dtype])


def _ids(gen, case):
    """Token ids by Zipf's law, low ids the frequent ones; -1 where an image row goes."""
    n, v = case["n"], case["v"]
    u = torch.rand(n, generator=gen, device="cuda", dtype=torch.float64)
    ids = (torch.exp(u * math.log(v + 1)) - 1).long().clamp_(0, v - 1)
    hole = torch.rand(n, generator=gen, device="cuda") < case["holes"]
    ids[hole] = -1
    return ids if case["wide"] else ids.int()


def _stream(gen, n, d, dtype):
    """Rows as a residual stream has them: an offset a row, a few large columns."""
    x = torch.randn((n, d), generator=gen, device="cuda")
    x[:, ::173] *= 8.0
    x += torch.randn((n, 1), generator=gen, device="cuda") * 0.3
    return x.to(DTYPES[dtype])


def _inputs(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    op, n, d, dt = case["op"], case["n"], case["d"], case["dtype"]
    s = {"case": case}
    if op in ("patch", "patch_grad"):
        th, tw = _grid(case)
        c, p = case["c"], case["p"]
        s["images"] = _images(gen, case)
        if op == "patch":
            shape = (d, p, p, c) if case["nhwc"] else (d, c, p, p)
            s["weight"] = _normal(gen, shape, (c * p * p) ** -0.5, dt)
            s["bias"] = _normal(gen, (d,), 0.1, dt)
            s["pos"] = _normal(gen, (th * tw, d), 0.2, dt) if case["pos"] else None
        else:
            s["grad_out"] = _normal(gen, (n, th * tw, d), 0.02, dt)
    elif op in ("embed", "embed_grad"):
        s["ids"] = _ids(gen, case)
        s["scale"] = math.sqrt(d)
        if op == "embed":
            s["table"] = _normal(gen, (case["v"], d), 0.02, dt)
        else:
            s["grad_out"] = _normal(gen, (n, d), 0.02, case["act"])
    else:
        s["weight"] = (1 + 0.1 * torch.randn(d, generator=gen, device="cuda")).to(
            DTYPES[case["param"]])
        if op == "norm":
            s["bias"] = _normal(gen, (d,), 0.1, case["param"])
            s["x"] = _stream(gen, n, d, dt)
            s["residual"] = _normal(gen, (n, d), 0.5, dt) if case["residual"] else None
        else:
            s["h"] = _stream(gen, n, d, dt)
            s["grad_out"] = _normal(gen, (n, d), 0.02, dt)
            s["grad_sum"] = _normal(gen, (n, d), 0.02, dt) if case["residual"] else None
            h = s["h"].float()
            s["mean"] = h.mean(1)
            s["rstd"] = torch.rsqrt(((h - s["mean"][:, None]) ** 2).mean(1) + EPS)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if not own:
        return s
    from paper_2007_13005_amd import tokens
    op, n, d = case["op"], case["n"], case["d"]
    dt = DTYPES[case["dtype"]]

    def empty(shape, dtype):
        return torch.empty(shape, dtype=dtype, device="cuda")

    if op in ("patch", "patch_grad"):
        th, tw = _grid(case)
        c, p = case["c"], case["p"]
        s["layout"] = tokens.LAYOUT_NHWC if case["nhwc"] else tokens.LAYOUT_NCHW
        if op == "patch":
            s["out"] = empty((n, th * tw, d), dt)
        else:
            g = DTYPES[case["grad"]]
            s["grad_weight"] = empty((d, p, p, c) if case["nhwc"] else (d, c, p, p), g)
            s["grad_bias"] = empty((d,), g)
            s["grad_pos"] = empty((th * tw, d), g) if case["pos"] else None
            s["workspace"] = empty((tokens.patch_embed_workspace_bytes(
                s["images"], s["grad_weight"], dt, s["layout"]),), torch.uint8)
    elif op == "embed":
        s["out"] = empty((n, d), DTYPES[case["act"]])
    elif op == "embed_grad":
        s["grad_table"] = empty((case["v"], d), DTYPES[case["grad"]])
        s["workspace"] = empty((tokens.embed_workspace_bytes(n, case["v"], d),), torch.uint8)
    elif op == "norm":
        s["out"] = empty((n, d), dt)
        s["sum"] = empty((n, d), dt) if case["residual"] else None
        s["mean"], s["rstd"] = empty((n,), torch.float32), empty((n,), torch.float32)
    else:
        q = DTYPES[case["param"]]
        s["grad_x"] = empty((n, d), dt)
        s["grad_weight"], s["grad_bias"] = empty((d,), q), empty((d,), q)
        s["workspace"] = empty((tokens.layer_norm_workspace_bytes(n, d),), torch.uint8)
    return s


def _run_own(s):
    from paper_2007_13005_amd import tokens
    op = s["case"]["op"]
    if op == "patch":
        return tokens.patch_embed(s["images"], s["weight"], s["bias"], s["pos"],
                                  layout=s["layout"], out=s["out"])
    if op == "patch_grad":
        return tokens.patch_embed_backward(
            s["grad_out"], s["images"], s["grad_weight"], s["grad_bias"], s["grad_pos"],
            layout=s["layout"], workspace=s["workspace"])
    if op == "embed":
        return tokens.embed(s["ids"], s["table"], s["scale"], out=s["out"])
    if op == "embed_grad":
        return tokens.embed_backward(s["grad_out"], s["ids"], s["grad_table"], s["scale"],
                                     workspace=s["workspace"])
    if op == "norm":
        return tokens.layer_norm(s["x"], s["weight"], s["bias"], EPS, residual=s["residual"],
                                 out=s["out"], sum_out=s["sum"], mean=s["mean"], rstd=s["rstd"])
    return tokens.layer_norm_backward(s["grad_out"], s["h"], s["weight"], s["mean"], s["rstd"],
                                      s["grad_x"], s["grad_weight"], s["grad_bias"],
                                      grad_sum=s["grad_sum"], workspace=s["workspace"])


def _patches(img, case):
    """(n, tokens, k) in the weight's order."""
    n, c, p = case["n"], case["c"], case["p"]
    th, tw = _grid(case)
    if case["nhwc"]:
        img = img[:, :th * p, :tw * p].reshape(n, th, p, tw, p, c).permute(0, 1, 3, 2, 4, 5)
    else:
        img = img[:, :, :th * p, :tw * p].reshape(n, c, th, p, tw, p).permute(0, 2, 4, 1, 3, 5)
    return img.reshape(n, th * tw, c * p * p)


def run(s):
    if own:
        return _run_own(s)
    case = s["case"]
    op, n, d, dt = case["op"], case["n"], case["d"], DTYPES[case["dtype"]]
    if op in ("patch", "patch_grad"):
        # the pixels take the weights' type, as every matrix product's operands do
        a = _patches(s["images"].to(dt).float(), case)
        k = a.shape[2]
        if op == "patch":
            y = (a.reshape(-1, k) @ s["weight"].float().reshape(d, k).t()).reshape(n, -1, d)
            y += s["bias"].float()
            if s["pos"] is not None:
                y += s["pos"].float()
            return y.to(dt)
        g = DTYPES[case["grad"]]
        dy = s["grad_out"].float()
        dw = dy.reshape(-1, d).t() @ a.reshape(-1, k)
        c, p = case["c"], case["p"]
        dw = dw.reshape((d, p, p, c) if case["nhwc"] else (d, c, p, p)).to(g)
        dpos = dy.sum(0).to(g) if case["pos"] else None
        return dw, dy.sum((0, 1)).to(g), dpos
    if op in ("embed", "embed_grad"):
        ids = s["ids"].long()
        some = (ids >= 0) & (ids < case["v"])
        at = torch.where(some, ids, 0)
        if op == "embed":
            rows = s["table"][at].float() * s["scale"]
            return (rows * some[:, None]).to(DTYPES[case["act"]])
        rows = s["grad_out"].float() * (some[:, None] * s["scale"])
        dt32 = torch.zeros((case["v"], d), dtype=torch.float32, device=rows.device)
        return dt32.index_add_(0, at, rows).to(DTYPES[case["grad"]])
    if op == "norm":
        h = s["x"]
        if s["residual"] is not None:
            h = (h.float() + s["residual"].float()).to(dt)
        z = h.float()
        mean = z.mean(1)
        z = z - mean[:, None]
        rstd = 1.0 / torch.sqrt((z * z).mean(1) + EPS)
        y = (z * rstd[:, None] * s["weight"].float() + s["bias"].float()).to(dt)
        return (y, h if s["residual"] is not None else None, mean, rstd)
    xh = (s["h"].float() - s["mean"][:, None]) * s["rstd"][:, None]
    dy = s["grad_out"].float()
    g = dy * s["weight"].float()
    dx = (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True)) * s["rstd"][:, None]
    if s["grad_sum"] is not None:
        dx = dx + s["grad_sum"].float()
    q = DTYPES[case["param"]]
    return dx.to(dt), (dy * xh).sum(0).to(q), dy.sum(0).to(q)


# The definition in 64 bits

def exact(case, seed):
    s = _inputs(case, seed)
    op, n, d = case["op"], case["n"], case["d"]
    if op in ("patch", "patch_grad"):
        th, tw = _grid(case)
        p, c = case["p"], case["c"]
        img = s["images"].to(DTYPES[case["dtype"]])
        if case["nhwc"]:
            img = img.permute(0, 3, 1, 2)
        # one (channel, row, column) of every patch at a time would be slow:
        # one channel and row of them, p columns
        strips = []
        for ch in range(c):
            for py in range(p):
                rows = img[:, ch, py:th * p:p, :tw * p].double()
                strips.append(rows.reshape(n * th * tw, p))
        a = torch.cat(strips, 1)  # columns (channel, row, column)
        if op == "patch":
            w = s["weight"].double()
            if case["nhwc"]:
                w = w.permute(0, 3, 1, 2)
            y = torch.mm(a, w.reshape(d, -1).t().contiguous()).view(n, th * tw, d)
            y = y + s["bias"].double()
            return y if s["pos"] is None else y + s["pos"].double()
        dy = s["grad_out"].double()
        dw = torch.mm(dy.view(-1, d).t().contiguous(), a).view(d, c, p, p)
        if case["nhwc"]:
            dw = dw.permute(0, 2, 3, 1).contiguous()
        total = dy.sum(0)
        return dw, total.sum(0), total if case["pos"] else None
    if op in ("embed", "embed_grad"):
        ids = s["ids"].long()
        keep = torch.nonzero((ids >= 0) & (ids < case["v"])).view(-1)
        if op == "embed":
            out = torch.zeros((n, d), dtype=torch.float64, device="cuda")
            out[keep] = s["table"].index_select(0, ids[keep]).double() * s["scale"]
            return out
        out = torch.zeros((case["v"], d), dtype=torch.float64, device="cuda")
        out.index_put_((ids[keep],), s["grad_out"][keep].double() * s["scale"], accumulate=True)
        return out
    if op == "norm":
        h = s["x"]
        if s["residual"] is not None:
            h = (h.double() + s["residual"].double()).to(DTYPES[case["dtype"]])
        v, m = torch.var_mean(h.double(), 1, correction=0)
        r = (v + EPS).rsqrt()
        y = (h.double() - m[:, None]) * r[:, None]
        y = y * s["weight"].double() + s["bias"].double()
        return (y, h.double() if s["residual"] is not None else None, m, r)
    h, dy, w = s["h"].double(), s["grad_out"].double(), s["weight"].double()
    v, m = torch.var_mean(h, 1, correction=0)
    sd = (v + EPS).sqrt()
    xh = (h - m[:, None]) / sd[:, None]
    g = dy * w
    # the Jacobian of a row: (I - 1/d - xh xh^T / d) / sd
    dx = (g - (g.sum(1) / d)[:, None] - xh * ((g * xh).sum(1) / d)[:, None]) / sd[:, None]
    if s["grad_sum"] is not None:
        dx = dx + s["grad_sum"].double()
    return dx, (dy * xh).sum(0), dy.sum(0)
