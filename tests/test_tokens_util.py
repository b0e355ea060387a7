"""The whole-number checks of the token operators notice one missing row, where
bounds of sums of normal values do not (the mistakes are planted in the oracle)."""
from __future__ import annotations

import pytest
import torch

from tests import tokens_util as ref


@pytest.mark.parametrize("rows, dim, values", [(3630, 16, 24), (39396, 12, 20)])
def test_a_missing_row_is_noticed(rows, dim, values):
    g = torch.Generator().manual_seed(rows)
    dy = ref.whole(g, rows, dim, dtype=torch.bfloat16).double()
    a = ref.whole(g, rows, values, dtype=torch.float16).double()
    assert 4 * rows < 2 ** 24
    total = (dy.t() @ a).float()
    ref.same(total, dy.t() @ a, "all rows")
    # the last row of a part, the first, the last of all, any
    for row in (0, 1, 63, 64, rows // 2, rows - 36, rows - 1):
        with pytest.raises(AssertionError):
            ref.same(total, dy.t() @ a - torch.outer(dy[row], a[row]), f"row {row}")
        with pytest.raises(AssertionError):
            ref.same(dy.sum(0).float(), dy.sum(0) - dy[row], f"row {row}")


def test_one_rounding():
    """A sum is rounded once to 16 bits, and not before it is whole."""
    exact = torch.tensor([2 ** 8 + 1.0, 2 ** 11 + 1.0, 300 * 257.0], dtype=torch.float64)
    for dtype in (torch.bfloat16, torch.float16):
        ref.same(exact.float().to(dtype), exact, "once")
    with pytest.raises(AssertionError):
        ref.same(torch.tensor([256.0 + 1.0 + 2.0]).bfloat16(), torch.tensor([256.0 + 2.0],
                                                                           dtype=torch.float64), "")
