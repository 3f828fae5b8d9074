"""The module of small calls belongs to one torch and one Python: it is compiled over torch's headers."""
import os

import pytest
import torch

from paper_2606_29758_gb300 import _binding, _build


@pytest.fixture()
def built(monkeypatch):
    _build.build()
    module = _binding.calls()
    monkeypatch.setattr(_binding, "_calls", None)       # (restored after the test)
    return module


@pytest.mark.parametrize("where,name", [(torch, "__version__"), (torch.version, "git_version")])
def test_the_module_of_another_torch_is_not_used(built, monkeypatch, where, name):
    """torch was exchanged since the build: the build is out of date, and the old module is not loaded over the new torch."""
    assert not _build._stale()
    monkeypatch.setattr(where, name, "0.0.1+another")
    assert _build._stale()
    try:
        got = _binding.calls()
    except ImportError:
        return
    assert got is not built and getattr(got, "__file__", None) != built.__file__


def test_it_is_found_again(built):
    got = _binding.calls()
    assert os.path.dirname(got.__file__) == _build.PKG and got.qk_fwd is not None
