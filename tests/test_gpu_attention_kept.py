"""Attention's gradients from lse and rest that lie as a program keeps them: heads
before rows, misaligned with gaps, one row standing for all. The same bits as from
dense ones."""
from __future__ import annotations

import struct

import pytest
import torch

from paper_2007_13005_amd import attention, smol
from tests.gpu_util import note
from tests.test_attention_abi import CALLS
from tests.test_gpu_attention import BF16, F16, F32, dev, inputs, mask, spread

pytestmark = pytest.mark.gpu

SHAPES = [(2, 70, 90, 6, 2, 40, True, 30, 2), (3, 33, 33, 4, 4, 72, False, 0, 0),
          (1, 300, 300, 8, 1, 128, True, 0, 0), (2, 1, 50, 4, 2, 64, True, 0, 0)]


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_any_strides(shape, dtype):
    note(f"attend kept {shape} {dtype}")
    q, k, v, dy = (dev(x) for x in inputs(shape, dtype, 17))
    lengths = {}
    if shape[0] == 2:
        lengths = {"q_lengths": torch.tensor([shape[1], shape[1] // 2], dtype=torch.int32).cuda(),
                   "k_lengths": torch.tensor([shape[2], shape[2] // 2], dtype=torch.int32).cuda()}
    rest = torch.empty_like(q)
    out, lse = attention.attend(q, k, v, rest=rest, **lengths, **mask(shape))

    def grads(lse, rest):
        return attention.attend_backward(dy, q, k, v, out, lse, rest, **lengths, **mask(shape))

    want = grads(lse, rest)
    first = [t.transpose(1, 2).contiguous().transpose(1, 2) for t in (lse, rest)]
    apart = spread(lse[..., None].cpu())[0][..., 0], spread(rest.cpu(), 5, 3)[0]
    for kept in (first, apart, (first[0], rest), (lse, apart[1]), (lse.view(-1), rest.view(-1))):
        for a, c in zip(grads(*kept), want):
            assert torch.equal(a, c)
    # zeros of one row standing for all are no rest
    none = torch.zeros(shape[5], dtype=dtype, device="cuda").expand(q.shape)
    for a, c in zip(grads(lse, none), grads(lse, None)):
        assert torch.equal(a, c)


def test_dense_c_call():
    """smol_attend_backward takes lse and rest densely."""
    note("attend kept dense")
    shape = (2, 40, 50, 4, 2, 64, True, 9, 1)
    q, k, v, dy = (dev(x) for x in inputs(shape, F16, 5))
    rest = torch.empty_like(q)
    out, lse = attention.attend(q, k, v, rest=rest, **mask(shape))
    want = attention.attend_backward(dy, q, k, v, out, lse, rest, **mask(shape))
    got = [torch.empty_like(t) for t in (q, k, v)]
    room = torch.empty(attention.attend_backward_workspace_bytes(q, k), dtype=torch.uint8,
                       device="cuda")
    values = {"shape.batch": 2, "shape.queries": 40, "shape.keys": 50, "shape.window": 9,
              "shape.sinks": 1, "rest": rest.data_ptr(), "lse": lse.data_ptr(),
              "workspace": room.data_ptr(), "workspace_bytes": room.numel()}
    for name, t in (("grad_out", dy), ("q", q), ("k", k), ("v", v), ("out", out),
                    ("grad_q", got[0]), ("grad_k", got[1]), ("grad_v", got[2])):
        values.update({f"{name}.data": t.data_ptr(), f"{name}.batch_stride": t.stride(0),
                       f"{name}.row_stride": t.stride(1), f"{name}.head_stride": t.stride(2)})
    layout = CALLS["smol_attend_backward"][1]
    packed = struct.pack("".join(letter for _, letter, _ in layout),
                         *[values.get(name, value) for name, _, value in layout])
    status = smol.lib().smol_attend_backward(packed, torch.cuda.current_stream().cuda_stream)
    assert status == smol.OK
    torch.cuda.synchronize()
    for a, c in zip(got, want):
        assert torch.equal(a, c)
