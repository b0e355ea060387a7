"""Buffers given to the preprocessing calls: autograd counts the writes."""
from __future__ import annotations

import pytest
import torch

from paper_2007_13005_amd import smol, synthetic
from tests.gpu_util import note

pytestmark = pytest.mark.gpu

WORKLOADS = {"rgb": lambda: synthetic.c2(n=3), "yuv": lambda: synthetic.c5(n=2),
             "roi": lambda: synthetic.c6(n=3), "lowres": lambda: synthetic.c7(n=3),
             "jpeg": lambda: synthetic.c8(n=2)}


@pytest.mark.parametrize("name", sorted(WORKLOADS))
def test_outputs(name):
    """An output that autograd saved and a later call wrote again is not used
    as if it had not been: backward raises, as after torch's own writes."""
    note(f"written buffers {name}")
    wl = WORKLOADS[name]()
    src = torch.from_numpy(wl.src).to("cuda")
    if src.dtype != torch.uint8:
        src = src.view(torch.uint8)
    out = smol.run_workload(wl, src)
    again = out.clone()
    factor = torch.ones_like(out, requires_grad=True)
    loss = (out * factor).float().sum()  # saves out
    assert smol.run_workload(wl, src, out=out) is out
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()
    assert torch.equal(out, again)


def test_workspaces_and_planes():
    wl = synthetic.c7(n=2)
    src = torch.from_numpy(wl.src).to("cuda")
    p = smol.make_params(wl.resize_short, wl.crop_h, wl.crop_w, wl.mean, wl.std, wl.out_dtype)
    ws = torch.empty(smol.lowres_workspace_bytes(wl.n, wl.low_res), dtype=torch.uint8,
                     device="cuda")
    before = ws._version
    smol.lowres_preprocess_batch(src, wl.offsets, wl.widths, wl.heights, p, wl.low_res,
                                 wl.pitches, None, ws)
    assert ws._version > before
    wl = synthetic.c8(n=1)
    coef = torch.from_numpy(wl.src).to("cuda").view(torch.int16)
    ws = torch.empty(smol.jpeg_workspace_bytes(wl.widths, wl.heights), dtype=torch.uint8,
                     device="cuda")
    before = ws._version
    smol.jpeg_roi_preprocess_batch(coef, wl.coef_offsets, wl.qtables, wl.widths, wl.heights,
                                   smol.make_params(wl.resize_short, wl.crop_h, wl.crop_w,
                                                    wl.mean, wl.std, wl.out_dtype),
                                   smol._workload_options(wl), ws)
    assert ws._version > before
    # the decoder alone: planes of whole frames
    w, h = int(wl.widths[0]) + 15 & ~15, int(wl.heights[0]) + 15 & ~15
    planes = torch.empty(w * h * 3 // 2, dtype=torch.uint8, device="cuda")
    smol.jpeg_decode_i420(coef, wl.coef_offsets, wl.qtables, wl.widths, wl.heights, planes, [0],
                          [w * h], [w * h * 5 // 4])
    assert planes._version > 0


def test_inference_buffers_are_written():
    wl = synthetic.c2(n=2)
    src = torch.from_numpy(wl.src).to("cuda")
    want = smol.run_workload(wl, src)
    with torch.inference_mode():
        out = torch.empty_like(want)
    assert torch.equal(smol.run_workload(wl, src, out=out).clone(), want)
