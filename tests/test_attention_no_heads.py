"""Norms of heads where one side has no heads: allocated workspaces fit the other's."""
from __future__ import annotations

import pytest
import torch

from paper_2007_13005_amd import attention
from tests import attention_util as ref
from tests.gpu_util import note
from tests.tokens_util import close


def sides(q_heads, k_heads, device):
    g = torch.Generator().manual_seed(3)
    return [torch.randn((2, 5, h, 16), generator=g).to(device)
            for h in (q_heads, k_heads, q_heads, k_heads)]


def test_workspace():
    for heads in ((0, 2), (2, 0), (0, 0)):
        dq, dk, q, k = sides(*heads, "cpu")
        need = attention.head_norm_workspace_bytes(q, k)
        assert need == 10 * sum(heads) * 2 * 16 * 4 + 16
        with pytest.raises(ValueError, match="current device"):
            attention.head_norm_backward(dq, dk, q, k)


@pytest.mark.gpu
def test_gradients():
    for heads in ((0, 2), (2, 0)):
        note(f"head norm without heads {heads}")
        dq, dk, q, k = sides(*heads, "cuda")
        gw = [torch.full((16,), 7.0, device="cuda") for _ in range(2)]
        got = attention.head_norm_backward(dq, dk, q, k, grad_q_weight=gw[0],
                                           grad_k_weight=gw[1])
        for n, dy, x in ((0, dq, q), (1, dk, k)):
            if not heads[n]:
                assert got[n].shape == x.shape and bool((gw[n] == 0).all())
                continue
            (a, e), (aw, ew) = ref.head_norm_backward(dy.cpu(), x.cpu(), None, 1e-6)
            close(got[n], a, e, "grad")
            close(gw[n], aw, ew, "weight's grad")
