"""The token operators' checks without a GPU: the structures' layout, every
refusal of the C entry points (all made before any HIP call; the addresses
here are never read), and the binding's own checks."""
from __future__ import annotations

import os
import re
import shutil
import struct
import subprocess

import pytest
import torch

from paper_2007_13005_amd import smol, tokens

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
AT = 0x10000

# the C structures, field by field
SHAPE_PACK = struct.Struct("12i")
PACKS = {"smol_patch_embed": struct.Struct("12i5Q2q"),
         "smol_patch_embed_backward": struct.Struct("12iQ2q5Qq2i"),
         "smol_embed": struct.Struct("3Q4q4ifi2i"),
         "smol_embed_backward": struct.Struct("4Q6q4ifi"),
         "smol_layer_norm": struct.Struct("8Q5q3if2i"),
         "smol_layer_norm_backward": struct.Struct("10Q6q4i")}
SHAPE = ["n", "channels", "height", "width", "patch", "dim", "layout", "image_type", "type",
         "r0", "r1", "r2"]
FIELDS = {
    "smol_patch_embed": (PACKS["smol_patch_embed"], SHAPE + ["images", "weight", "bias", "pos", "out",
                                                 "image_stride", "row_stride"]),
    "smol_patch_embed_backward": (PACKS["smol_patch_embed_backward"], SHAPE + [
        "grad_out", "image_stride", "row_stride", "images", "grad_weight", "grad_bias",
        "grad_pos", "workspace", "workspace_bytes", "grad_type", "accumulate"]),
    "smol_embed": (PACKS["smol_embed"], ["ids", "table", "out", "n", "vocab", "table_stride",
                                   "out_stride", "dim", "ids_type", "table_type", "out_type",
                                   "scale", "keep", "r0", "r1"]),
    "smol_embed_backward": (PACKS["smol_embed_backward"], [
        "grad_out", "ids", "grad_table", "workspace", "workspace_bytes", "n", "vocab",
        "grad_stride", "table_stride", "padding", "dim", "ids_type", "out_type", "grad_type",
        "scale", "accumulate"]),
    "smol_layer_norm": (PACKS["smol_layer_norm"], ["x", "residual", "weight", "bias", "out", "sum", "mean",
                                       "rstd", "rows", "x_stride", "residual_stride",
                                       "out_stride", "sum_stride", "dim", "type", "weight_type",
                                       "eps", "r0", "r1"]),
    "smol_layer_norm_backward": (PACKS["smol_layer_norm_backward"], [
        "grad_out", "h", "grad_sum", "weight", "mean", "rstd", "grad_x", "grad_weight",
        "grad_bias", "workspace", "workspace_bytes", "rows", "grad_stride", "h_stride",
        "sum_stride", "x_stride", "dim", "type", "weight_type", "accumulate"]),
}
SHAPE_GOOD = dict(n=2, channels=3, height=64, width=64, patch=16, dim=128, layout=0,
                  image_type=1, type=1, r0=0, r1=0, r2=0)
GOOD = {
    "smol_patch_embed": dict(SHAPE_GOOD, images=AT, weight=AT, bias=0, pos=0, out=AT,
                             image_stride=16 * 128, row_stride=128),
    "smol_patch_embed_backward": dict(SHAPE_GOOD, grad_out=AT, image_stride=16 * 128,
                                      row_stride=128, images=AT, grad_weight=AT, grad_bias=AT,
                                      grad_pos=AT, workspace=AT, workspace_bytes=1 << 40,
                                      grad_type=0, accumulate=0),
    "smol_embed": dict(ids=AT, table=AT, out=AT, n=10, vocab=100, table_stride=64, out_stride=64,
                       dim=64, ids_type=1, table_type=0, out_type=1, scale=1.0, keep=0, r0=0,
                       r1=0),
    "smol_embed_backward": dict(grad_out=AT, ids=AT, grad_table=AT, workspace=AT,
                                workspace_bytes=1 << 40, n=10, vocab=100, grad_stride=64,
                                table_stride=64, padding=-1, dim=64, ids_type=1, out_type=1,
                                grad_type=0, scale=1.0, accumulate=0),
    "smol_layer_norm": dict(x=AT, residual=0, weight=AT, bias=AT, out=AT, sum=0, mean=AT,
                            rstd=AT, rows=10, x_stride=64, residual_stride=0, out_stride=64,
                            sum_stride=0, dim=64, type=1, weight_type=0, eps=1e-5, r0=0, r1=0),
    "smol_layer_norm_backward": dict(grad_out=AT, h=AT, grad_sum=0, weight=AT, mean=AT, rstd=AT,
                                     grad_x=AT, grad_weight=AT, grad_bias=AT, workspace=AT,
                                     workspace_bytes=1 << 40, rows=10, grad_stride=64,
                                     h_stride=64, sum_stride=0, x_stride=64, dim=64, type=1,
                                     weight_type=0, accumulate=0),
}
BIG = 1 << 62
NAN, INF = float("nan"), float("inf")
INVALID, UNSUPPORTED = smol.ERR_INVALID_ARG, smol.ERR_UNSUPPORTED
BAD_SHAPES = [(dict(n=-1), INVALID), (dict(channels=0), INVALID), (dict(height=0), INVALID),
              (dict(width=-5), INVALID), (dict(patch=0), INVALID), (dict(dim=0), INVALID),
              (dict(layout=2), INVALID), (dict(image_type=2), INVALID),
              (dict(image_type=-1), INVALID), (dict(image_type=3, type=2), INVALID),
              (dict(type=3), INVALID), (dict(type=-1), INVALID), (dict(r1=1), INVALID),
              (dict(height=65536), UNSUPPORTED), (dict(width=2 ** 31 - 1), UNSUPPORTED),
              (dict(patch=257, height=300, width=300), UNSUPPORTED),
              (dict(channels=2 ** 31 - 1), UNSUPPORTED), (dict(channels=2000), UNSUPPORTED),
              (dict(dim=65537), UNSUPPORTED), (dict(n=2 ** 31 - 1), UNSUPPORTED),
              (dict(height=65535, width=65535), UNSUPPORTED),
              (dict(dim=65536, patch=256, height=256, width=256), UNSUPPORTED)]
BAD = {
    "smol_patch_embed": BAD_SHAPES + [
        (dict(images=0), INVALID), (dict(images=AT + 1), INVALID), (dict(weight=0), INVALID),
        (dict(bias=AT + 1), INVALID), (dict(pos=AT + 1), INVALID), (dict(out=0), INVALID),
        (dict(out=AT + 1), INVALID), (dict(row_stride=127), INVALID),
        (dict(row_stride=0), INVALID), (dict(image_stride=0), INVALID),
        (dict(image_stride=15 * 128 + 127), INVALID), (dict(image_stride=-1), INVALID),
        (dict(row_stride=BIG), INVALID), (dict(image_stride=BIG), INVALID)],
    "smol_patch_embed_backward": BAD_SHAPES + [
        (dict(grad_out=0), INVALID), (dict(images=0), INVALID), (dict(images=AT + 1), INVALID),
        (dict(grad_weight=AT + 2), INVALID), (dict(grad_bias=AT + 2), INVALID),
        (dict(grad_pos=AT + 1), INVALID), (dict(workspace=0), INVALID),
        (dict(workspace=AT + 8), INVALID), (dict(workspace_bytes=0), INVALID),
        (dict(workspace_bytes=-1), INVALID), (dict(grad_type=2), INVALID),
        (dict(accumulate=2), INVALID), (dict(row_stride=-1), INVALID),
        (dict(image_stride=-1), INVALID), (dict(image_stride=BIG), INVALID)],
    "smol_embed": [
        (dict(n=-1), INVALID), (dict(vocab=0), INVALID), (dict(dim=0), INVALID),
        (dict(ids_type=2), INVALID), (dict(n=2 ** 30 + 1), UNSUPPORTED),
        (dict(vocab=2 ** 30 + 1), UNSUPPORTED), (dict(dim=65537), UNSUPPORTED),
        (dict(scale=NAN), INVALID), (dict(scale=INF), INVALID), (dict(keep=2), INVALID),
        (dict(ids=0), INVALID), (dict(ids=AT + 4), INVALID), (dict(table=0), INVALID),
        (dict(table=AT + 2), INVALID), (dict(out=0), INVALID), (dict(out=AT + 1), INVALID),
        (dict(table_type=3), INVALID), (dict(out_type=-1), INVALID),
        (dict(table_stride=-1), INVALID), (dict(out_stride=63), INVALID),
        (dict(out_stride=BIG), INVALID), (dict(r0=1), INVALID)],
    "smol_embed_backward": [
        (dict(n=-1), INVALID), (dict(vocab=0), INVALID), (dict(dim=-1), INVALID),
        (dict(ids_type=-1), INVALID), (dict(n=2 ** 31), UNSUPPORTED),
        (dict(vocab=2 ** 31), UNSUPPORTED), (dict(dim=65537), UNSUPPORTED),
        (dict(scale=NAN), INVALID), (dict(accumulate=-1), INVALID), (dict(ids=0), INVALID),
        (dict(ids=AT + 4), INVALID), (dict(grad_out=0), INVALID), (dict(grad_table=0), INVALID),
        (dict(grad_table=AT + 2), INVALID), (dict(out_type=3), INVALID),
        (dict(grad_type=3), INVALID), (dict(grad_stride=-2), INVALID),
        (dict(table_stride=63), INVALID), (dict(workspace=0), INVALID),
        (dict(workspace=AT + 4), INVALID), (dict(workspace_bytes=100), INVALID)],
    "smol_layer_norm": [
        (dict(rows=-1), INVALID), (dict(dim=0), INVALID), (dict(type=3), INVALID),
        (dict(weight_type=2), INVALID), (dict(rows=2 ** 30 + 1), UNSUPPORTED),
        (dict(dim=8193), UNSUPPORTED), (dict(eps=-1e-5), INVALID), (dict(eps=NAN), INVALID),
        (dict(eps=INF), INVALID), (dict(x=0), INVALID), (dict(x=AT + 1), INVALID),
        (dict(out=0), INVALID), (dict(out=AT + 1), INVALID), (dict(residual=AT + 1), INVALID),
        (dict(sum=AT + 1, sum_stride=64), INVALID), (dict(sum=AT, sum_stride=64), INVALID),
        (dict(sum=2 * AT, sum_stride=0), INVALID), (dict(weight=AT + 2), INVALID),
        (dict(bias=AT + 2), INVALID), (dict(mean=AT + 2), INVALID), (dict(rstd=AT + 2), INVALID),
        (dict(x_stride=-1), INVALID), (dict(out_stride=63), INVALID),
        (dict(x_stride=BIG), INVALID), (dict(r1=7), INVALID)],
    "smol_layer_norm_backward": [
        (dict(rows=-1), INVALID), (dict(dim=0), INVALID), (dict(type=-1), INVALID),
        (dict(weight_type=2), INVALID), (dict(rows=2 ** 31), UNSUPPORTED),
        (dict(dim=8193), UNSUPPORTED), (dict(accumulate=2), INVALID),
        (dict(grad_out=0), INVALID), (dict(h=0), INVALID), (dict(grad_x=0), INVALID),
        (dict(mean=0), INVALID), (dict(rstd=0), INVALID), (dict(mean=AT + 2), INVALID),
        (dict(grad_sum=AT + 1), INVALID), (dict(weight=AT + 1), INVALID),
        (dict(grad_weight=AT + 2), INVALID), (dict(grad_bias=AT + 1), INVALID),
        (dict(x_stride=63), INVALID), (dict(h_stride=-1), INVALID), (dict(workspace=0), INVALID),
        (dict(workspace=AT + 1), INVALID), (dict(workspace_bytes=16), INVALID)],
}


def call(name: str, **fields) -> int:
    packer, names = FIELDS[name]
    values = dict(GOOD[name], **fields)
    assert set(values) == set(names)
    return getattr(smol.lib(), name)(packer.pack(*[values[k] for k in names]), None)


@pytest.mark.parametrize("name", sorted(BAD))
def test_refusals(name):
    for fields, status in BAD[name]:
        assert call(name, **fields) == status, (name, fields)
        assert smol.lib().smol_last_error(), (name, fields)
    assert getattr(smol.lib(), name)(None, None) == INVALID


def test_empty_calls_enqueue_nothing():
    # no row: no HIP call is made, whatever the pointers
    assert call("smol_layer_norm", rows=0, x=0, out=0) == smol.OK
    assert call("smol_embed", n=0, ids=0, out=0) == smol.OK
    assert call("smol_patch_embed", n=0, images=0, out=0) == smol.OK
    assert call("smol_patch_embed", patch=65, images=0, out=0) == smol.OK  # no whole patch
    assert call("smol_patch_embed_backward", n=0, grad_weight=0, grad_bias=0, grad_pos=0,
                grad_out=0, images=0) == smol.OK


def test_workspace_sizes():
    lib = smol.lib()
    assert lib.smol_norm_workspace_bytes(0, 64) > 0
    assert lib.smol_norm_workspace_bytes(10 ** 6, 8192) < 1 << 27
    assert lib.smol_norm_workspace_bytes(-1, 64) == 0
    assert lib.smol_norm_workspace_bytes(10, 8193) == 0
    assert lib.smol_embed_workspace_bytes(0, 100, 64) > 0
    assert lib.smol_embed_workspace_bytes(2 ** 30, 2 ** 30, 65536) > 2 ** 40
    assert lib.smol_embed_workspace_bytes(10, 0, 64) == 0
    assert lib.smol_embed_workspace_bytes(10, 100, 65537) == 0
    shape = SHAPE_PACK.pack(*[SHAPE_GOOD[k] for k in SHAPE])
    assert lib.smol_patch_workspace_bytes(shape) > 0
    bad = SHAPE_PACK.pack(*[dict(SHAPE_GOOD, layout=5)[k] for k in SHAPE])
    assert lib.smol_patch_workspace_bytes(bad) == 0
    assert lib.smol_patch_workspace_bytes(None) == 0


C_NAMES = {"smol_patch_embed": "smol_patch_args", "smol_embed": "smol_embed_args",
           "smol_patch_embed_backward": "smol_patch_grad_args",
           "smol_embed_backward": "smol_embed_grad_args", "smol_layer_norm": "smol_norm_args",
           "smol_layer_norm_backward": "smol_norm_grad_args"}


@pytest.mark.skipif(shutil.which("gcc") is None, reason="needs gcc")
def test_structures_match_the_header(tmp_path):
    lines, want = [], []
    for name, (packer, names) in FIELDS.items():
        ctype = C_NAMES[name]
        lines.append(f'printf("%zu\\n", sizeof({ctype}));')
        want.append(packer.size)
        at = 0
        letters = "".join(c * int(k or 1) for k, c in
                          re.findall(r"(\d*)([a-zA-Z])", packer.format))
        assert len(letters) == len(names)
        for field, letter in zip(names, letters):
            size = struct.calcsize(letter)
            at = (at + size - 1) // size * size
            path = f"shape.{field}" if names[0] == "n" and names.index(field) < 12 else field
            if field.startswith("r") and field[1:].isdigit():
                path = ("shape." if path.startswith("shape.") else "") + f"reserved[{field[1:]}]"
            lines.append(f'printf("%zu\\n", offsetof({ctype}, {path}));')
            want.append(at)
            at += size
    src = tmp_path / "layout.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "smol_tokens.h"\n'
                   "int main(void) {" + "\n".join(lines) + "return 0; }\n")
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-std=gnu11", "-I", os.path.join(ROOT, "include"), str(src), "-o",
                    str(exe)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout
    assert [int(v) for v in out.split()] == want


def test_limits_match_the_header():
    text = open(os.path.join(ROOT, "include", "smol_tokens.h")).read()
    for name in ("ELEM_F32", "ELEM_F16", "ELEM_BF16", "IDS_I32", "IDS_I64", "MAX_NORM_DIM",
                 "MAX_EMBED_DIM", "MAX_PATCH_DIM", "MAX_PATCH", "MAX_PATCH_VALUES", "MAX_ROWS"):
        line = next(t for t in text.splitlines() if t.startswith(f"#define SMOL_{name} "))
        assert int(line.split()[2]) == getattr(tokens, name), name


def test_binding_refusals():
    """Wrong shapes, types, devices and row layouts raise ValueError before any call."""
    x = torch.zeros((4, 8))
    with pytest.raises(ValueError, match="current device"):
        tokens.layer_norm(x)
    with pytest.raises(ValueError, match="current device"):
        tokens.embed(torch.zeros(3, dtype=torch.int64), x)
    img, weight = torch.zeros((2, 3, 32, 32)), torch.zeros((8, 3, 16, 16))
    with pytest.raises(ValueError, match="current device"):
        tokens.patch_embed(img, weight)
    for bad in (dict(x=x.double()), dict(x=torch.zeros(())), dict(x=x, weight=torch.zeros(7)),
                dict(x=x, weight=torch.zeros(16)[::2]), dict(x=x, residual=x[:3]),
                dict(x=x, residual=x.half()), dict(x=x.t()), dict(x=x, out=x.half()),
                dict(x=x, weight=torch.zeros(8), bias=torch.zeros(8).half()),
                dict(x=x, mean=torch.zeros(3)), dict(x=torch.zeros((4, 0))),
                dict(x=torch.zeros((4, 6, 8))[:, :5])):
        with pytest.raises(ValueError):
            tokens.layer_norm(**bad)
    stats = torch.zeros(4)
    for bad in (dict(grad_out=x[:3]), dict(mean=stats[:2]), dict(grad_weight=stats),
                dict(workspace=torch.zeros(3, dtype=torch.uint8)), dict(grad_sum=x.half())):
        with pytest.raises(ValueError):
            tokens.layer_norm_backward(**dict(dict(grad_out=x, h=x, weight=None, mean=stats,
                                                   rstd=stats), **bad))
    ids = torch.zeros(3, dtype=torch.int64)
    for args, kw in (((ids.short(), x), {}), ((torch.zeros((3, 2), dtype=torch.int64)[:, 0], x),
                                              {}), ((ids, x[0]), {}), ((ids, x), {"keep": True}),
                     ((ids, x), {"out": torch.zeros((2, 8))}),
                     ((ids, x), {"out": torch.zeros((3, 7))}), ((ids, x.double()), {})):
        with pytest.raises(ValueError):
            tokens.embed(*args, **kw)
    with pytest.raises(ValueError):
        tokens.embed_backward(x, ids, torch.zeros((5, 8)))
    with pytest.raises(ValueError):
        tokens.embed_backward(x[:3], ids, torch.zeros((5, 8)),
                              workspace=torch.zeros(8, dtype=torch.uint8))
    for args, kw in (((img, weight[:, :2]), {}), ((img[0], weight), {}), ((img, weight[0]), {}),
                     ((img, weight), {"layout": tokens.LAYOUT_NHWC}),
                     ((img, weight), {"layout": 7}), ((img, weight.double()), {}),
                     ((img, weight), {"bias": torch.zeros(9)}),
                     ((img, weight), {"pos": torch.zeros((3, 8))}),
                     ((img, weight), {"out": torch.zeros((2, 4, 9))}),
                     ((img, weight), {"out": torch.zeros((2, 4, 8)).half()}),
                     ((img, torch.zeros((8, 3, 16, 8))), {}),
                     ((img.permute(0, 1, 3, 2), weight), {})):
        with pytest.raises(ValueError):
            tokens.patch_embed(*args, **kw)
    dy = torch.zeros((2, 4, 8))
    with pytest.raises(ValueError):
        tokens.patch_embed_backward(dy[:, :3], img, weight)
    with pytest.raises(ValueError):
        tokens.patch_embed_backward(dy, img, weight, workspace=torch.zeros(1, dtype=torch.uint8))
    with pytest.raises(TypeError):
        tokens.layer_norm(x, out=3)
    with pytest.raises(TypeError):
        tokens.embed([1, 2], x, out=x)
    with pytest.raises(TypeError):
        tokens.embed(ids, torch.zeros((5, 8)), "a")


def test_binding_refuses_lazily_negated_views():
    """Their memory holds the values' negatives, which the kernels would take."""
    x = torch.zeros((4, 8))
    negated = torch.zeros((4, 8), dtype=torch.complex64).conj().imag[:, :4]
    assert negated.is_neg()
    ids = torch.zeros(4, dtype=torch.int64)
    img, weight = torch.zeros((1, 3, 16, 16)), torch.zeros((8, 3, 16, 16))
    for function, args in ((tokens.layer_norm, (torch._neg_view(x),)),
                           (tokens.layer_norm, (negated,)),
                           (tokens.embed, (ids, torch._neg_view(x))),
                           (tokens.embed_backward, (torch._neg_view(x), ids, x)),
                           (tokens.patch_embed, (torch._neg_view(img), weight)),
                           (tokens.patch_embed, (img, weight, torch._neg_view(x)[0])),
                           (tokens.patch_embed_backward,
                            (torch.zeros((1, 1, 8)), img, torch._neg_view(weight)))):
        with pytest.raises(ValueError, match="resolve_neg"):
            function(*args)
    with pytest.raises(ValueError, match="resolve_neg"):
        tokens.layer_norm(x, out=torch._neg_view(x.clone()))


def test_patch_gradients_past_a_launch():
    """Every size within its limit, and more joins than one launch takes:
    refused before anything is enqueued, not by the last of the launches."""
    large = dict(n=1, channels=32767, height=181, width=181, patch=1, dim=65536, image_stride=0,
                 row_stride=0)
    assert call("smol_patch_embed_backward", **large) == UNSUPPORTED
    assert b"too many for a launch" in smol.lib().smol_last_error()


def test_binding_patch_gradient_without_the_weight():
    """What then has to be given, and what has to fit."""
    dy, img = torch.zeros((2, 4, 8)), torch.zeros((2, 3, 32, 32))
    bias, weight = torch.zeros(8), torch.zeros((8, 3, 16, 16))
    room = torch.zeros(1 << 20, dtype=torch.uint8)
    with pytest.raises(ValueError, match="side must be given"):
        tokens.patch_embed_backward(dy, img, None, bias)
    with pytest.raises(ValueError, match="side must be given"):
        tokens.patch_embed_backward(dy, img, None, bias, workspace=room)
    for bad in (dict(patch=0), dict(patch=8), dict(patch=16, grad_weight=weight[:, :2]),
                dict(patch=8, grad_weight=weight), dict(patch=16, grad_bias=bias[:7]),
                dict(patch=16, grad_bias=bias.double()), dict(patch=16, grad_out=dy[0]),
                dict(patch=16, grad_bias=bias, grad_pos=torch.zeros((4, 8)).half())):
        for workspace in (None, room):
            args = dict(dict(grad_out=dy, images=img, grad_weight=None, grad_bias=bias,
                             workspace=workspace), **bad)
            with pytest.raises(ValueError) as e:
                tokens.patch_embed_backward(**args)
            assert "current device" not in str(e.value), bad
    with pytest.raises(ValueError, match="current device"):
        tokens.patch_embed_backward(dy, img, None, bias, workspace=room, patch=16)
