"""What the build takes for up to date, and that a build that fails leaves nothing behind."""
import os

import pytest
import torch

from paper_2609_09721_b200 import binding, build


def test_another_torch_makes_the_extension_stale(monkeypatch):
    """efq_tensorcall.so is compiled against torch's C++ headers: the files' times alone do not tell whether it still fits."""
    build.build()
    assert not build._stale()
    monkeypatch.setattr(torch, "__version__", "9.9.9")
    assert build._stale()


def test_an_extension_of_another_torch_is_not_called(monkeypatch):
    build.build()
    monkeypatch.setattr(binding, "_tensors", None)
    assert binding._tensorcall().built_for == build.target()
    monkeypatch.setattr(binding, "_tensors", None)
    monkeypatch.setattr(torch, "__version__", "9.9.9")
    with pytest.raises(RuntimeError, match="was built for torch .* this is torch 9.9.9"):
        binding._tensorcall()
