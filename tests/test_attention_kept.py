"""What the forward attention call leaves for the backward one (lse and rest) at
strides of its own: refusals of the C call and of the binding, without a GPU (the
addresses here are never read)."""
from __future__ import annotations

import os
import shutil
import struct
import subprocess

import pytest
import torch

from paper_2007_13005_amd import attention, smol
from tests.test_attention_abi import AT, BIG, CALLS, INVALID, OK

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FIELDS = ["lse_batch_stride", "lse_row_stride", "lse_head_stride", "rest_batch_stride",
          "rest_row_stride", "rest_head_stride"]
DENSE = dict(zip(FIELDS, (32, 4, 1, 2048, 256, 64)))


def call(kept=None, **fields) -> int:
    """smol_attend_backward_kept: 2 sequences of 8 queries, 4 heads of 64 values."""
    fields = {k.replace("__", "."): v for k, v in fields.items()}
    layout = CALLS["smol_attend_backward"][1]
    values = {k: v + (n << 24) if v == AT else v for n, (k, _, v) in enumerate(layout)}
    assert set(fields) <= set(values)
    values.update(fields)
    packed = struct.pack("".join(letter for _, letter, _ in layout), *values.values())
    strides = struct.pack("6q", *dict(DENSE, **(kept or {})).values())
    return smol.lib().smol_attend_backward_kept(packed, strides, None)


def test_refusals():
    for name in FIELDS:
        for value in (-1, BIG):
            assert call({name: value}, rest=AT) == INVALID, (name, value)
            assert name.split("_")[0].encode() in smol.lib().smol_last_error()
    for bad in (dict(lse=0), dict(lse=AT + 2), dict(rest=AT + 1), dict(q__data=0),
                dict(shape__dim=0), dict(workspace=0), dict(workspace_bytes=0)):
        assert call(**bad) == INVALID, bad
    # strides of a rest that is not there are not looked at
    assert call({"rest_row_stride": -1}, workspace=0) == INVALID
    assert b"workspace" in smol.lib().smol_last_error()
    lib = smol.lib()
    assert lib.smol_attend_backward_kept(None, struct.pack("6q", *DENSE.values()), None) == INVALID
    assert lib.smol_attend_backward_kept(b"\0" * 4096, None, None) == INVALID
    assert call(shape__batch=0, workspace=0, lse=0) == OK


@pytest.mark.skipif(shutil.which("gcc") is None, reason="needs gcc")
def test_structure_matches_the_header(tmp_path):
    src = tmp_path / "layout.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "smol_attention.h"\n'
                   'int main(void) { printf("%zu", sizeof(smol_attend_kept));' +
                   "".join(f'printf(" %zu", offsetof(smol_attend_kept, {f}));' for f in FIELDS) +
                   "return 0; }\n")
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-std=gnu11", "-I", os.path.join(ROOT, "include"), str(src), "-o",
                    str(exe)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout
    assert [int(v) for v in out.split()] == [48, 0, 8, 16, 24, 32, 40]


def test_binding_takes_any_strides():
    """Layouts that lie as asked get to the device check; others raise before it."""
    b, n, h, d = 2, 3, 4, 16
    q, k = torch.zeros((b, n, h, d)), torch.zeros((b, 6, 2, d))
    lse, rest = torch.zeros((b, h, n)).transpose(1, 2), torch.zeros((b, h, n, d)).transpose(1, 2)
    room = torch.zeros(1 << 20, dtype=torch.uint8)
    args = dict(grad_out=q, q=q, k=k, v=k, out=q, lse=lse, rest=rest, workspace=room)
    for good in (dict(), dict(rest=None), dict(lse=lse.contiguous().view(-1)),
                 dict(rest=rest.contiguous().view(n, -1)), dict(lse=lse[:1].expand(b, n, h)),
                 dict(rest=torch.zeros((b, n, h, d + 1))[..., 1:])):
        with pytest.raises(ValueError, match="current device"):
            attention.attend_backward(**dict(args, **good))
    for bad in (dict(lse=lse[:1]), dict(lse=lse.double()), dict(lse=lse.transpose(1, 2)[:, 1:]),
                dict(lse=torch.zeros((b, n, 1, h)).transpose(1, 3)[..., 0].transpose(1, 2)[:, :2]),
                dict(rest=rest[:, :2]), dict(rest=rest.half()),
                dict(rest=rest.transpose(1, 2)[:, 1:]),
                dict(rest=torch.zeros((b, n, d, h)).transpose(2, 3))):
        with pytest.raises(ValueError, match="lse|rest") as e:
            attention.attend_backward(**dict(args, **bad))
        assert "current device" not in str(e.value), bad
