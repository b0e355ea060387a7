"""The library is built where no torch is, or one for another device: a user of
the C calls needs none, and only the token operators' Python binding is left out."""
from __future__ import annotations

import sys

import pytest
import torch

from paper_2007_13005_amd import build as hip_build


@pytest.mark.parametrize("torch_is", ["absent", "for the CPU"])
def test_build_without_rocm_torch(monkeypatch, tmp_path, capsys, torch_is):
    if torch_is == "absent":
        monkeypatch.setitem(sys.modules, "torch", None)
    else:
        monkeypatch.setattr(torch.version, "hip", None)
    binding = tmp_path / "binding.so"
    made = []
    monkeypatch.setattr(hip_build, "PYTOKENS", str(binding))
    monkeypatch.setattr(hip_build, "build_pycall", lambda verbose=False: made.append("call"))
    monkeypatch.setattr(hip_build, "_build_library", lambda cc, verbose: made.append("library"))
    hip_build.build()
    assert made == ["call", "library"]
    assert not list(tmp_path.iterdir())
    assert "binding is not built" in capsys.readouterr().err
    assert hip_build.pytokens_command() is None
