"""The attention operators' checks without a GPU: the structures' layout, every
refusal of the C entry points (all made before any HIP call; the addresses here
are never read), frequencies (host code), and the binding's own checks."""
from __future__ import annotations

import ctypes
import os
import re
import shutil
import struct
import subprocess

import pytest
import torch

from paper_2007_13005_amd import attention, smol
from tests import attention_util as ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
AT = 0x10000
BIG = 1 << 62
NAN, INF = float("nan"), float("inf")
INVALID, UNSUPPORTED, OK = smol.ERR_INVALID_ARG, smol.ERR_UNSUPPORTED, smol.OK

# the C structures, field by field: (name, letter of struct, value of a good call)
SIDE = [("x", "Q", AT), ("out", "Q", AT), ("weight", "Q", AT), ("x_row_stride", "q", 256),
        ("x_head_stride", "q", 64), ("out_row_stride", "q", 256), ("out_head_stride", "q", 64),
        ("heads", "i", 4), ("reserved", "i", 0)]
GRAD_SIDE = [("grad_out", "Q", AT), ("x", "Q", AT), ("weight", "Q", AT), ("grad_x", "Q", AT),
             ("grad_weight", "Q", AT), ("grad_out_row_stride", "q", 256),
             ("grad_out_head_stride", "q", 64), ("x_row_stride", "q", 256),
             ("x_head_stride", "q", 64), ("grad_x_row_stride", "q", 256),
             ("grad_x_head_stride", "q", 64), ("heads", "i", 4), ("reserved", "i", 0)]
HEADS = [("positions", "Q", AT), ("freqs", "Q", AT), ("rows", "q", 10), ("dim", "i", 64),
         ("rot", "i", 32), ("type", "i", 1), ("weight_type", "i", 0), ("positions_type", "i", 1),
         ("interleaved", "i", 0), ("eps", "f", 1e-6), ("gain", "f", 1.0),
         ("reserved[0]", "i", 0), ("reserved[1]", "i", 0)]
SHAPE = [("q_lengths", "Q", 0), ("k_lengths", "Q", 0), ("batch", "i", 2), ("queries", "i", 8),
         ("keys", "i", 16), ("heads", "i", 4), ("kv_heads", "i", 2), ("dim", "i", 64),
         ("type", "i", 1), ("causal", "i", 1), ("window", "i", 0), ("sinks", "i", 0),
         ("scale", "f", 0.125), ("reserved", "i", 0)]


def rows(heads, count):
    return [("data", "Q", AT), ("batch_stride", "q", count * heads * 64),
            ("row_stride", "q", heads * 64), ("head_stride", "q", 64)]


def within(name, fields):
    return [(f"{name}.{field}", letter, value) for field, letter, value in fields]


CALLS = {
    "smol_rotate": ("smol_rotate_args", [
        ("x", "Q", AT), ("out", "Q", AT), ("positions", "Q", AT), ("freqs", "Q", AT),
        ("rows", "q", 10), ("x_row_stride", "q", 256), ("x_head_stride", "q", 64),
        ("out_row_stride", "q", 256), ("out_head_stride", "q", 64), ("heads", "i", 4),
        ("dim", "i", 64), ("rot", "i", 32), ("type", "i", 1), ("positions_type", "i", 1),
        ("interleaved", "i", 0), ("gain", "f", 1.0), ("reserved", "i", 0)]),
    "smol_head_norm": ("smol_head_norm_args",
                       within("shape", HEADS) + within("q", SIDE) + within("k", SIDE)),
    "smol_head_norm_backward": ("smol_head_norm_grad_args", (
        within("shape", HEADS) + within("q", GRAD_SIDE) + within("k", GRAD_SIDE) + [
            ("workspace", "Q", AT), ("workspace_bytes", "q", 1 << 40), ("accumulate", "i", 0),
            ("reserved", "i", 0)])),
    "smol_attend": ("smol_attend_args", (
        within("shape", SHAPE) + within("q", rows(4, 8)) + within("k", rows(2, 16)) +
        within("v", rows(2, 16)) + within("out", rows(4, 8)) + [
            ("lse", "Q", AT), ("rest", "Q", 0), ("workspace", "Q", AT),
            ("workspace_bytes", "q", 1 << 40)])),
    "smol_attend_backward": ("smol_attend_grad_args", (
        within("shape", SHAPE) + within("grad_out", rows(4, 8)) + within("q", rows(4, 8)) +
        within("k", rows(2, 16)) + within("v", rows(2, 16)) + within("out", rows(4, 8)) + [
            ("rest", "Q", 0), ("lse", "Q", AT)] + within("grad_q", rows(4, 8)) +
        within("grad_k", rows(2, 16)) + within("grad_v", rows(2, 16)) + [
            ("workspace", "Q", AT), ("workspace_bytes", "q", 1 << 40)])),
}
CALLS["smol_rotate_backward"] = CALLS["smol_rotate"]


def call(name: str, **fields) -> int:
    fields = {k.replace("__", "."): v for k, v in fields.items()}
    # every address its own
    values = {k: v + (n << 24) if v == AT else v for n, (k, _, v) in enumerate(CALLS[name][1])}
    assert set(fields) <= set(values), set(fields) - set(values)
    values.update(fields)
    packed = struct.pack("".join(letter for _, letter, _ in CALLS[name][1]), *values.values())
    return getattr(smol.lib(), name)(packed, None)


def strided(name, written, heads):
    """Refusals of one matrix of rows and heads."""
    bad = [({f"{name}_row_stride": -1}, INVALID), ({f"{name}_head_stride": -1}, INVALID),
           ({f"{name}_row_stride": BIG}, INVALID), ({f"{name}_head_stride": BIG}, INVALID)]
    if written:
        bad += [({f"{name}_row_stride": 63}, INVALID), ({f"{name}_head_stride": 63}, INVALID),
                ({f"{name}_row_stride": 64 * heads - 1}, INVALID)]
    return bad


SIZES = [(dict(rows=-1), INVALID), (dict(dim=0), INVALID), (dict(rot=-2), INVALID),
         (dict(rot=33), INVALID), (dict(rot=66), INVALID), (dict(type=3), INVALID),
         (dict(type=-1), INVALID), (dict(positions_type=2), INVALID),
         (dict(interleaved=2), INVALID), (dict(rows=2 ** 30 + 1), UNSUPPORTED),
         (dict(dim=257), UNSUPPORTED), (dict(positions=0), INVALID),
         (dict(positions=AT + 4), INVALID), (dict(freqs=0), INVALID), (dict(freqs=AT + 4), INVALID),
         (dict(gain=NAN), INVALID), (dict(gain=INF), INVALID)]
ROTATE = SIZES + [(dict(rot=0), INVALID), (dict(heads=0), INVALID), (dict(heads=-1), INVALID),
                  (dict(heads=1025), UNSUPPORTED), (dict(reserved=1), INVALID),
                  (dict(x=0), INVALID), (dict(x=AT + 1), INVALID), (dict(out=0), INVALID),
                  (dict(out=AT + 1), INVALID)] + strided("x", False, 4) + strided("out", True, 4)
NORM_SHAPE = [({f"shape__{k}".replace("reserved1", "reserved[1]"): v for k, v in d.items()}, s)
              for d, s in SIZES + [(dict(weight_type=2), INVALID), (dict(eps=-1e-6), INVALID),
                                   (dict(eps=NAN), INVALID), (dict(eps=INF), INVALID),
                                   (dict(reserved1=1), INVALID)]]


def of_sides(bad):
    return [({f"{side}__{k}": v for k, v in d.items()}, s) for side in "qk" for d, s in bad]


def of_matrix(name, written, heads, count):
    bad = [(dict(data=0), INVALID), (dict(data=AT + 1), INVALID), (dict(batch_stride=-1), INVALID),
           (dict(row_stride=-1), INVALID), (dict(head_stride=-1), INVALID),
           (dict(batch_stride=BIG), INVALID), (dict(row_stride=BIG), INVALID)]
    if written:
        bad += [(dict(head_stride=63), INVALID), (dict(row_stride=64 * heads - 1), INVALID),
                (dict(batch_stride=64 * heads * count - 1), INVALID), (dict(row_stride=0), INVALID)]
    return [({f"{name}__{k}": v for k, v in d.items()}, s) for d, s in bad]


ATTEND_SHAPE = [({f"shape__{k}": v for k, v in d.items()}, s) for d, s in [
    (dict(batch=-1), INVALID), (dict(queries=-1), INVALID), (dict(keys=-1), INVALID),
    (dict(heads=0), INVALID), (dict(kv_heads=0), INVALID), (dict(heads=5), INVALID),
    (dict(dim=0), INVALID), (dict(type=3), INVALID), (dict(causal=2), INVALID),
    (dict(window=-1), INVALID), (dict(sinks=-1), INVALID), (dict(causal=0, window=4), INVALID),
    (dict(causal=0, sinks=4), INVALID), (dict(scale=0.0), INVALID), (dict(scale=-1.0), INVALID),
    (dict(scale=NAN), INVALID), (dict(scale=INF), INVALID), (dict(reserved=1), INVALID),
    (dict(scale=8e-19), UNSUPPORTED), (dict(scale=1.2e18), UNSUPPORTED),
    (dict(q_lengths=AT + 2), INVALID), (dict(k_lengths=AT + 1), INVALID),
    (dict(dim=60), UNSUPPORTED), (dict(dim=136), UNSUPPORTED), (dict(batch=65537), UNSUPPORTED),
    (dict(queries=2 ** 24 + 1), UNSUPPORTED), (dict(keys=2 ** 24 + 1), UNSUPPORTED),
    (dict(heads=1026), UNSUPPORTED), (dict(queries=2 ** 24, heads=1024), UNSUPPORTED),
    (dict(queries=2 ** 24, batch=65536), UNSUPPORTED), (dict(keys=2 ** 24, batch=65536),
                                                        UNSUPPORTED)]]
ROOM = [(dict(workspace=0), INVALID), (dict(workspace=AT + 8), INVALID),
        (dict(workspace_bytes=0), INVALID), (dict(workspace_bytes=-1), INVALID)]
FAR = dict(shape__queries=1, shape__keys=100000)  # keys in parts, which need room
BAD = {
    "smol_rotate": ROTATE,
    "smol_rotate_backward": ROTATE,
    "smol_head_norm": NORM_SHAPE + of_sides(
        [(dict(heads=-1), INVALID), (dict(heads=1025), UNSUPPORTED), (dict(reserved=1), INVALID),
         (dict(x=0), INVALID), (dict(x=AT + 1), INVALID), (dict(out=0), INVALID),
         (dict(out=AT + 1), INVALID), (dict(weight=AT + 2), INVALID)]
        + strided("x", False, 4) + strided("out", True, 4)),
    "smol_head_norm_backward": NORM_SHAPE + ROOM + [(dict(accumulate=2), INVALID),
                                                    (dict(reserved=1), INVALID)] + of_sides(
        [(dict(heads=-1), INVALID), (dict(heads=1025), UNSUPPORTED), (dict(reserved=1), INVALID),
         (dict(x=0), INVALID), (dict(grad_out=0), INVALID), (dict(grad_out=AT + 1), INVALID),
         (dict(grad_x=0), INVALID), (dict(grad_weight=AT + 2), INVALID),
         (dict(weight=AT + 1), INVALID)]
        + strided("x", False, 4) + strided("grad_out", False, 4) + strided("grad_x", True, 4)),
    "smol_attend": ATTEND_SHAPE + of_matrix("q", False, 4, 8) + of_matrix("k", False, 2, 16) +
    of_matrix("v", False, 2, 16) + of_matrix("out", True, 4, 8) + [
        (dict(lse=AT + 2), INVALID), (dict(rest=AT + 1), INVALID)] + [
        (dict(d, **FAR), s) for d, s in ROOM],
    "smol_attend_backward": ATTEND_SHAPE + ROOM + of_matrix("q", False, 4, 8) +
    of_matrix("grad_out", False, 4, 8) + of_matrix("k", False, 2, 16) +
    of_matrix("v", False, 2, 16) + of_matrix("out", False, 4, 8) +
    of_matrix("grad_q", True, 4, 8) + of_matrix("grad_k", True, 2, 16) +
    of_matrix("grad_v", True, 2, 16) + [(dict(lse=0), INVALID), (dict(lse=AT + 2), INVALID),
                                        (dict(rest=AT + 1), INVALID)],
}


SAME = {
    "smol_head_norm": [("q.out", "k.out"), ("q.out", "k.x"), ("k.out", "q.x")],
    "smol_head_norm_backward": [("q.grad_x", "k.grad_x"), ("q.grad_x", "k.x"),
                                ("q.grad_x", "k.grad_out"), ("k.grad_x", "q.x"),
                                ("k.grad_x", "q.grad_out"), ("q.grad_weight", "k.grad_weight")],
    "smol_attend": [("out.data", f"{k}.data") for k in "qkv"] + [("lse", "q.data"),
                                                                 ("rest", "out.data")],
    "smol_attend_backward": [(f"grad_{a}.data", b) for a in "qkv" for b in (
        "q.data", "k.data", "v.data", "out.data", "grad_out.data", "lse")] + [
        ("grad_q.data", "grad_k.data"), ("grad_q.data", "grad_v.data"),
        ("grad_k.data", "grad_v.data")],
}


@pytest.mark.parametrize("name", sorted(SAME))
def test_outputs_stand_apart(name):
    for written, other in SAME[name]:
        assert call(name, **{written: AT, other: AT}) == INVALID, (name, written, other)
        assert b"stands where" in smol.lib().smol_last_error(), (name, written, other)


IN_PLACE = {
    "smol_rotate": [("x", "out", "out")], "smol_rotate_backward": [("x", "out", "out")],
    "smol_head_norm": [("q.x", "q.out", "q.out"), ("k.x", "k.out", "k.x")],
    "smol_head_norm_backward": [("q.x", "q.grad_x", "q.x"), ("k.grad_out", "k.grad_x", "k.grad_x")],
}


@pytest.mark.parametrize("name", sorted(IN_PLACE))
def test_in_place_means_the_same_strides(name):
    for read, written, strides in IN_PLACE[name]:
        for stride, value in (("row_stride", 320), ("head_stride", 2560)):
            change = {read: AT, written: AT, f"{strides}_{stride}": value}
            assert call(name, **change) == INVALID, (name, change)
            assert b"in place" in smol.lib().smol_last_error(), (name, change)


@pytest.mark.parametrize("name", sorted(BAD))
def test_refusals(name):
    for fields, status in BAD[name]:
        assert call(name, **fields) == status, (name, fields)
        assert smol.lib().smol_last_error(), (name, fields)
    assert getattr(smol.lib(), name)(None, None) == INVALID


def test_empty_calls_enqueue_nothing():
    assert call("smol_rotate", rows=0, x=0, out=0, positions=0, freqs=0) == OK
    assert call("smol_head_norm", shape__rows=0, q__x=0, k__out=0, shape__positions=0) == OK
    assert call("smol_head_norm", q__heads=0, k__heads=0, q__x=0) == OK
    assert call("smol_head_norm_backward", shape__rows=0, q__grad_weight=0,
                k__grad_weight=0) == OK
    assert call("smol_attend", shape__batch=0, q__data=0) == OK
    assert call("smol_attend", shape__queries=0, q__data=0, out__data=0) == OK
    assert call("smol_attend_backward", shape__batch=0, q__data=0, workspace=0) == OK
    assert call("smol_attend_backward", shape__queries=0, shape__keys=0, workspace=0) == OK


def test_workspace_sizes():
    lib = smol.lib()
    bytes_of = lib.smol_head_norm_workspace_bytes
    assert bytes_of(0, 4, 4, 64) > 0 and 0 < bytes_of(2 ** 30, 1024, 1024, 256) < 1 << 24
    for bad in ((-1, 1, 1, 64), (2 ** 30 + 1, 1, 1, 64), (1, -1, 1, 64), (1, 1, 1025, 64),
                (1, 1, 1, 0), (1, 1, 1, 257)):
        assert bytes_of(*bad) == 0

    def shape(**kw):
        values = {k: v for k, _, v in SHAPE}
        values.update(kw)
        return struct.pack("".join(letter for _, letter, _ in SHAPE), *values.values())

    for f in (lib.smol_attend_workspace_bytes, lib.smol_attend_backward_workspace_bytes):
        assert f(shape()) > 0 and f(shape(dim=60)) == 0 and f(None) == 0
    few, many = (lib.smol_attend_workspace_bytes(shape(queries=1, keys=n)) for n in (64, 100000))
    assert few < many < 1 << 28
    # a window bounds the keys that there can be
    assert lib.smol_attend_workspace_bytes(shape(queries=1, keys=100000, window=100)) == few


@pytest.mark.skipif(shutil.which("gcc") is None, reason="needs gcc")
def test_structures_match_the_header(tmp_path):
    lines, want = [], []
    for ctype, fields in dict(CALLS.values()).items():
        letters = "".join(letter for _, letter, _ in fields)
        lines.append(f'printf("%zu\\n", sizeof({ctype}));')
        want.append(struct.calcsize(letters))
        for n, (field, letter, _) in enumerate(fields):
            lines.append(f'printf("%zu\\n", offsetof({ctype}, {field}));')
            want.append(struct.calcsize(letters[:n + 1]) - struct.calcsize(letter))
    lines.append('printf("%zu\\n", sizeof(smol_rotary_plan));')
    want.append(ctypes.sizeof(attention.RotaryPlan))
    src = tmp_path / "layout.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "smol_attention.h"\n'
                   "int main(void) {" + "\n".join(lines) + "return 0; }\n")
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-std=gnu11", "-I", os.path.join(ROOT, "include"), str(src), "-o",
                    str(exe)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout
    assert [int(v) for v in out.split()] == want


def test_limits_match_the_header():
    text = open(os.path.join(ROOT, "include", "smol_attention.h")).read()
    names = re.findall(r"#define SMOL_((?:MAX|ROTARY)_\w+)\s+(\d+)", text)
    assert len(names) == 9
    for name, value in names:
        assert int(value) == getattr(attention, name), name


@pytest.mark.parametrize("rot", [2, 4, 36, 128, 256])
def test_frequencies(rot):
    for kw in (dict(), dict(base=500000.0), dict(scaling="linear", factor=4.0),
               dict(scaling="base", factor=8.0),
               dict(scaling="parts", factor=8.0, length=8192.0, low=1.0, high=4.0),
               dict(scaling="parts", factor=1.0, length=64.0)):
        got, gain = attention.rotary_frequencies(rot, device="cpu", **kw)
        want, g = ref.frequencies(rot, **kw)
        # pow, and a few operations, in 64 bits
        assert got.dtype == torch.float64 and bool(((got - want).abs() <= 1e-14 * want).all())
        assert abs(gain - g) <= 1e-7 * g
    # the slowest frequency of the larger base is the slowest divided by the factor
    if rot > 2:
        slow = attention.rotary_frequencies(rot, device="cpu")[0][-1]
        base = attention.rotary_frequencies(rot, scaling="base", factor=8.0, device="cpu")[0]
        assert abs(float(base[-1] * 8 / slow) - 1) < 1e-12 and float(base[0]) == 1.0


def test_frequencies_refusals():
    good = dict(dim=64, scaling="parts", factor=2.0, length=100.0, device="cpu")
    attention.rotary_frequencies(**good)
    for bad in (dict(dim=0), dict(dim=3), dict(dim=258), dict(base=0.0), dict(base=-1.0),
                dict(base=NAN), dict(base=INF), dict(factor=0.5), dict(factor=INF),
                dict(factor=NAN), dict(length=0.0), dict(length=INF), dict(low=32.0),
                dict(high=NAN)):
        with pytest.raises(smol.SmolError):
            attention.rotary_frequencies(**dict(good, **bad))
    for bad in (dict(scaling="other"), dict(dim=-2), dict(dim=1 << 31)):
        with pytest.raises(ValueError):
            attention.rotary_frequencies(**dict(good, **bad))


def test_binding_refusals():
    """Wrong shapes, types, devices and layouts raise ValueError before any call."""
    x = torch.zeros((5, 4, 16))
    pos, freqs = torch.zeros(5, dtype=torch.int64), torch.zeros(8, dtype=torch.float64)
    with pytest.raises(ValueError, match="current device"):
        attention.rotate(x, pos, freqs)
    for bad in (dict(x=x.double()), dict(x=x[0, 0]), dict(x=x.transpose(1, 2)),
                dict(positions=pos[:4]), dict(positions=pos.float()), dict(freqs=freqs.float()),
                dict(freqs=freqs.view(2, 4)), dict(out=x.half()), dict(out=x[:4]),
                dict(x=torch.zeros((2, 6, 4, 16))[:, :5], positions=torch.zeros(12).long()),
                dict(x=torch._neg_view(x)), dict(positions=pos.repeat(2)[::2])):
        with pytest.raises(ValueError):
            attention.rotate(**dict(dict(x=x, positions=pos, freqs=freqs), **bad))
    with pytest.raises(TypeError):
        attention.rotate(x, [0] * 5, freqs)
    w = torch.zeros(16)
    with pytest.raises(ValueError, match="current device"):
        attention.head_norm(x, x[:, :2], w, w, pos, freqs)
    for bad in (dict(k=x[:4]), dict(k=x.half()), dict(k=x[..., :8]), dict(q_weight=w[:8]),
                dict(q_weight=w.half()), dict(k_weight=w.half()), dict(positions=None),
                dict(freqs=None), dict(q_out=x[:, :2]), dict(k=None), dict(q=x[0, 0])):
        args = dict(q=x, k=x, q_weight=w, k_weight=w, positions=pos, freqs=freqs)
        with pytest.raises(ValueError):
            attention.head_norm(**dict(args, **bad))
    room = torch.zeros(1 << 20, dtype=torch.uint8)
    for bad in (dict(grad_q_out=x[:4]), dict(grad_k_out=x.half()), dict(workspace=room[:8]),
                dict(grad_q_weight=w.double()), dict(grad_k_weight=w[:3]), dict(k=None),
                dict(grad_q=x[:, :3])):
        args = dict(grad_q_out=x, grad_k_out=x, q=x, k=x, workspace=room)
        with pytest.raises(ValueError) as e:
            attention.head_norm_backward(**dict(args, **bad))
        assert "current device" not in str(e.value), bad
    q, k = torch.zeros((2, 3, 4, 16)), torch.zeros((2, 6, 2, 16))
    with pytest.raises(ValueError, match="current device"):
        attention.attend(q, k, k)
    lengths = torch.zeros(2, dtype=torch.int32)
    for bad in (dict(q=q[0]), dict(q=q.half()), dict(k=k[:1]), dict(k=k[..., :8]), dict(v=k[:, :5]),
                dict(v=k.half()), dict(out=q[:, :2]), dict(lse=torch.zeros((2, 3, 3))),
                dict(lse=torch.zeros((2, 3, 4)).double()), dict(rest=q.half()),
                dict(rest=q.transpose(1, 2)), dict(q_lengths=lengths.long()),
                dict(k_lengths=lengths[:1]), dict(workspace=room.view(torch.int32)),
                dict(q=q.transpose(2, 3)), dict(v=torch._neg_view(k))):
        with pytest.raises(ValueError) as e:
            attention.attend(**dict(dict(q=q, k=k, v=k), **bad))
        assert "current device" not in str(e.value), bad
    lse = torch.zeros((2, 3, 4))
    for bad in (dict(grad_out=q[:, :2]), dict(out=q.half()), dict(lse=lse[:1]), dict(grad_q=k),
                dict(grad_k=q), dict(grad_v=k.half()), dict(rest=k[:, :5]), dict(workspace=room[:8])):
        args = dict(grad_out=q, q=q, k=k, v=k, out=q, lse=lse, workspace=room)
        with pytest.raises(ValueError) as e:
            attention.attend_backward(**dict(args, **bad))
        assert "current device" not in str(e.value), bad
