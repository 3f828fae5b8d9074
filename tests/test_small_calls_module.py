"""The module of small calls belongs to one torch and one Python: it is compiled over torch's headers."""
import os
import sys

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


@pytest.fixture()
def cannot_build(built, monkeypatch):
    """A torch for which the module is not there and cannot be made: no compiler, no headers."""
    def fails():
        raise RuntimeError("no compiler")
    monkeypatch.setattr(torch, "__version__", "0.0.1+another")
    monkeypatch.setattr(_build, "_build_calls", fails)


def test_the_library_is_built_without_it(cannot_build):
    before = os.path.getmtime(_build.LIB)
    with pytest.warns(UserWarning, match="no compiler"):
        assert _build.build() == _build.LIB
    assert os.path.getmtime(_build.LIB) == before       # and is not made again for it


def test_an_older_module_does_not_stay(cannot_build):
    """The sources have moved on and it could not be made again: it may not fit the library any more."""
    with open(_build.calls_path(), "w"):
        pass
    os.utime(_build.calls_path(), (1, 1))
    with pytest.warns(UserWarning):
        _build.build()
    assert not os.path.exists(_build.calls_path())


def test_the_library_is_built_without_torch(built, monkeypatch):
    monkeypatch.setitem(sys.modules, "torch", None)     # (import torch fails)
    assert _build.build() == _build.LIB and not _build._stale()


def test_holders_without_it_go_their_ordinary_way(cannot_build):
    from paper_2606_29758_gb300 import FFNShape, GatedFFN, QKNormRope, QKShape, RowDropout
    holders = [GatedFFN(FFNShape(4, 16, 24), device="cpu"), QKNormRope(QKShape(4, 2, 1, 16, 0), None, device="cpu")]
    for h in holders:
        assert h._fast_fwd(h._plan, *[None] * 7) is None and h._fast_bwd(h._plan, *[None] * 9) is None
    assert RowDropout(0.5)._fast(*[None] * 10) is None


@pytest.mark.gpu
def test_holders_without_it_give_the_same_bits(built, monkeypatch):
    from paper_2606_29758_gb300 import FFNShape, GatedFFN, QKNormRope, QKShape, RowDropout, rope_table
    g = torch.Generator(device="cuda").manual_seed(1)
    r = lambda *s: torch.randn(*s, device="cuda", generator=g).to(torch.bfloat16)  # noqa: E731
    N, d, F, D = 70, 64, 136, 32
    x, w, qk, pos = r(N, d), (r(F, d), r(F, d), r(d, F)), r(N, 3 * D), torch.arange(1, N + 1, device="cuda", dtype=torch.int32)
    traj = pos // 9

    def run():
        ffn, norms = GatedFFN(FFNShape(N, d, F)), QKNormRope(QKShape(N, 2, 1, D, D), rope_table(N, D))
        out = [ffn.forward(x, *w), *ffn.backward(x, x, *w)]
        q, k = qk[:, :2 * D], qk[:, 2 * D:]
        out += [*norms.forward(q, k, None, None, pos), *norms.backward(q, k, q, k, None, None, pos)]
        return out + [RowDropout(0.3).forward(x, traj, pos, 5, 6, res=x)]
    with_it = run()
    monkeypatch.setattr(torch, "__version__", "0.0.1+another")
    monkeypatch.setattr(_binding, "_calls", None)
    for a, b in zip(with_it, run()):
        assert torch.equal(a, b)
