"""The example that runs the preprocessing and the token operators together:
its loss falls step by step."""
from __future__ import annotations

import os
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_losses_fall():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import image_text_tokens
    finally:
        sys.path.pop(0)
    losses = image_text_tokens.run(steps=6, photos=4)
    assert len(losses) == 6 and all(x == x and x > 0 for x in losses)
    assert all(b < a for a, b in zip(losses, losses[1:])), losses
    # the same seeds give the same bits
    assert losses == image_text_tokens.run(steps=6, photos=4)
