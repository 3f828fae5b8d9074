"""Arguments of the block operators that are refused on the host, before any CUDA call (no GPU here)."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def L():
    from paper_2606_29758_gb300 import _build, _binding
    _build.build()
    return _binding.lib()


OK, INV, UNSUP, WS = 0, 1, 2, 3
P = ctypes.c_void_p(1 << 20)          # never dereferenced
ODD = ctypes.c_void_p((1 << 20) + 8)


def _ffn(L, N=4, d=64, F=64, dt=0, act=0, X=P, ldx=64, Wd=P, ldy=64, store=None, sb=0):
    return L.ps_gated_ffn_fwd(N, d, F, dt, act, X, ldx, P, P, Wd, P, ldy, store, sb, None, 0, None)


def test_ffn(L):
    for bad in (dict(N=-1), dict(d=12), dict(d=0), dict(F=4), dict(F=65), dict(dt=7), dict(act=2), dict(ldx=63),
                dict(ldx=68), dict(ldy=32), dict(X=None), dict(X=ODD), dict(Wd=ODD), dict(store=ODD, sb=1 << 30)):
        assert _ffn(L, **bad) == INV, bad
    assert _ffn(L, dt=1) == UNSUP                         # f32
    need = L.ps_gated_ffn_store_size(4, 64)
    assert need == 3 * 1024 + 256 and L.ps_gated_ffn_store_size(-1, 64) == 0 and L.ps_gated_ffn_store_size(4, 60) == 0
    assert _ffn(L, store=P, sb=need - 1) == WS
    assert L.ps_gated_ffn_fwd_workspace_size(4, 64, 64, 0) == 256 + 1024
    assert L.ps_gated_ffn_fwd_workspace_size(4, 64, 64, 1) == 256
    # a workspace for N rows holds any fewer
    for d, F in ((64, 64), (136, 4104), (1536, 8192), (3584, 16384)):
        for size in (lambda n: L.ps_gated_ffn_fwd_workspace_size(n, d, F, 1), lambda n: L.ps_gated_ffn_bwd_workspace_size(n, d, F),
                     lambda n: L.ps_gated_ffn_fwd_workspace_size(n, d, F, 0), lambda n: 256 + L.ps_gated_ffn_store_size(n, F)):
            sizes = [size(n) for n in (0, 1, 63, 64, 65, 100, 127, 128, 129, 400, 1000, 5000, 100000)]
            assert sizes == sorted(sizes) and sizes[0] >= 256

    def bwd(N=4, dt=0, dX=P, lddx=64, dxt=0, dWg=P, dWu=P, dwt=0, flags=0, sb=1 << 20, dY=P):
        return L.ps_gated_ffn_bwd(N, 64, 64, dt, dY, 64, P, 64, P, P, P, P, sb, dX, lddx, dxt, dWg, dWu, P, dwt, flags,
                                  None, 0, None)
    for bad in (dict(N=-1), dict(dt=3), dict(dxt=2), dict(dwt=-1), dict(flags=4), dict(lddx=60), dict(dWg=None),
                dict(dWu=ODD), dict(dY=None), dict(dX=ODD)):
        assert bwd(**bad) == INV, bad
    assert bwd(dt=1) == UNSUP and bwd(flags=1) == UNSUP and bwd(flags=2) == UNSUP   # sums over calls in bf16
    assert bwd(sb=need - 1) == WS


def test_qk(L):
    def fwd(N=4, Hq=2, Hk=1, D=64, R=64, dt=0, lay=0, q=P, ldq=128, eps=1e-6, pos=P, T=8, table=P):
        return L.ps_qk_norm_rope_fwd(N, Hq, Hk, D, R, dt, lay, q, ldq, P, 64, None, None, eps, pos, 1, T, table, P, 128,
                                     P, 64, None, 0, None)
    for bad in (dict(N=-1), dict(Hq=-1), dict(D=24), dict(D=528), dict(D=0), dict(R=8), dict(R=80), dict(dt=2), dict(lay=2),
                dict(q=None), dict(q=ODD), dict(ldq=120), dict(ldq=132), dict(eps=-1.0), dict(eps=float("nan")),
                dict(pos=None), dict(T=0), dict(table=None), dict(table=ODD)):
        assert fwd(**bad) == INV, bad
    assert fwd() == WS and fwd(R=0, pos=None, table=None, T=0) == WS      # the workspace is looked at last
    assert L.ps_qk_norm_rope_workspace_size(24) == 0 and L.ps_qk_norm_rope_workspace_size(128) > 256
    assert L.ps_rope_table(0, 64, 1e4, P, None) == INV and L.ps_rope_table(8, 24, 1e4, P, None) == INV
    assert L.ps_rope_table(8, 64, 0.0, P, None) == INV and L.ps_rope_table(8, 64, 1e4, None, None) == INV
    assert L.ps_rope_table(8, 64, float("inf"), P, None) == INV
    assert L.ps_qk_norm_rope_bwd(4, 2, 1, 64, 64, 0, 0, P, 128, P, 64, P, 128, P, 64, None, None, 1e-6, P, 1, 8, P, P, 128,
                                 P, 64, P, P, 2, None, 0, None) == INV    # an unknown flag


def test_dropout(L):
    def run(N=4, d=64, dt=0, x=P, ldx=64, ldr=64, res=None, base=0, p=0.1, step=0, site=0, traj=P):
        return L.ps_dropout_rows(N, d, dt, x, ldx, res, ldr, traj, P, base, p, 1, step, site, P, 64, None)
    for bad in (dict(N=-1), dict(d=0), dict(d=(1 << 19) + 1, ldx=1 << 20), dict(dt=3), dict(x=None), dict(ldx=63),
                dict(res=P, ldr=10), dict(base=-1), dict(base=1 << 32), dict(p=1.0), dict(p=-0.5), dict(p=float("nan")),
                dict(step=1 << 32), dict(site=-1), dict(site=1 << 16), dict(traj=None),
                dict(x=ctypes.c_void_p((1 << 20) + 1))):
        assert run(**bad) == INV, bad
    assert run(N=0) == OK
