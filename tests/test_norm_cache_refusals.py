"""Residual norms, the paged cache and attention over it: what is refused on the host, before any CUDA call (no GPU here)."""
import ctypes

import pytest
import torch

from test_block_devices import BF, HERE, I32, OTHER, Call, Rows

OK, INV, UNSUP, WS = 0, 1, 2, 3
P = ctypes.c_void_p(1 << 20)          # never dereferenced
ODD = ctypes.c_void_p((1 << 20) + 8)
BYTE = ctypes.c_void_p((1 << 20) + 1)
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def L():
    from paper_2606_29758_gb300 import _build, _binding
    _build.build()
    return _binding.lib()


def test_norm(L):
    def fwd(N=4, d=64, dt=0, norms=3, x=P, ldx=64, y=P, ldy=64, gy=P, go=P, gate=P, a=1.0, b=1.0, eps=1e-6, h=P, ldh=64, o=P,
            ldo=64):
        return L.ps_residual_norm_fwd(N, d, dt, norms, x, ldx, y, ldy, gy, go, gate, a, b, eps, h, ldh, o, ldo, None)
    for bad in (dict(N=-1), dict(d=0), dict(d=-5), dict(d=16385, ldx=1 << 15), dict(d=8193, dt=1), dict(dt=2), dict(dt=-1), dict(norms=4),
                dict(norms=-1), dict(a=NAN), dict(a=INF), dict(b=-INF), dict(eps=-1e-9), dict(eps=NAN), dict(eps=INF),
                dict(x=None), dict(x=BYTE), dict(ldx=63), dict(y=BYTE), dict(ldy=63), dict(y=None), dict(y=None, norms=2),
                dict(y=None, norms=0, gate=None), dict(gy=BYTE), dict(go=BYTE), dict(gate=BYTE), dict(h=None), dict(ldh=63),
                dict(o=None), dict(ldo=63), dict(dt=1, x=ctypes.c_void_p((1 << 20) + 2))):
        assert fwd(**bad) == INV, bad
    assert fwd(N=0) == OK and fwd(N=0, x=None, y=None, h=None, o=None) == OK and fwd(N=0, d=0) == INV
    # the widest rows: whole 16 bytes, or a chunk's less
    for d, dt in ((16378, 0), (8190, 1)):
        ld = d + 1
        assert fwd(d=d, dt=dt, ldx=ld, ldy=ld, ldh=ld, ldo=ld) == UNSUP
    assert fwd(d=16384, x=ODD, ldx=16384, ldy=16384, ldh=16384, ldo=16384) == UNSUP
    assert L.ps_residual_norm_workspace_size(0) == 0 and L.ps_residual_norm_workspace_size(16385) == 0
    need = L.ps_residual_norm_workspace_size(64)
    assert need > 256

    def bwd(N=4, d=64, dt=0, norms=3, do=P, lddo=64, dh=P, lddh=64, h=P, ldh=64, y=P, ldy=64, gy=P, go=P, gate=P, eps=1e-6, dx=P,
            lddx=64, dy=P, lddy=64, dgy=P, dgo=P, dgate=P, flags=0, ws=P, wsb=1 << 24):
        return L.ps_residual_norm_bwd(N, d, dt, norms, do, lddo, dh, lddh, h, ldh, y, ldy, gy, go, gate, 1.0, 1.0, eps, dx, lddx, dy,
                                      lddy, dgy, dgo, dgate, flags, ws, wsb, None)
    for bad in (dict(N=-1), dict(d=0), dict(dt=5), dict(norms=8), dict(flags=2), dict(flags=4), dict(do=None), dict(lddo=60),
                dict(dh=BYTE), dict(lddh=60), dict(h=None), dict(ldh=60), dict(ldy=60), dict(dx=None), dict(lddx=60), dict(dy=None),
                dict(lddy=60), dict(dgy=BYTE), dict(dgo=BYTE), dict(dgate=BYTE), dict(gate=BYTE), dict(gate=None),
                dict(norms=1), dict(norms=1, dgo=None, dh=None), dict(y=None), dict(y=None, norms=2, gate=None, dgate=None),
                dict(eps=NAN)):
        assert bwd(**bad) == INV, bad
    assert bwd(wsb=need - 1) == WS and bwd(ws=None) == WS and bwd(ws=ODD) == WS
    assert bwd(dgy=None, dgo=None, wsb=255) == WS                         # (without gain gradients the status alone)
    assert bwd(N=0, wsb=0) == WS


def test_append(L):
    def run(N=4, seqs=2, Hk=2, D=64, dt=0, k=P, ldk=128, v=P, ldv=128, seq=P, pos=P, base=1, table=P, ldt=8, pages=16, page=16, kc=P,
            vc=P, ws=P, wsb=256):
        return L.ps_paged_append(N, seqs, Hk, D, dt, k, ldk, v, ldv, seq, pos, base, table, ldt, pages, page, kc, vc, ws, wsb, None)
    for bad in (dict(N=-1), dict(seqs=-1), dict(Hk=0), dict(Hk=65537), dict(D=0), dict(D=24), dict(D=272), dict(dt=2), dict(k=None),
                dict(k=ODD), dict(v=ODD), dict(ldk=127), dict(ldk=132), dict(ldv=120), dict(seq=None), dict(pos=None),
                dict(table=None), dict(ldt=0), dict(ldt=1 << 28), dict(pages=0), dict(page=0), dict(page=24), dict(page=1 << 17),
                dict(kc=None), dict(vc=ODD)):
        assert run(**bad) == INV, bad
    assert run(wsb=255) == WS and run(ws=None) == WS and run(N=0, ws=None) == WS


def test_decode(L):
    need = L.ps_paged_decode_workspace_size(64)
    assert need > 256 and [L.ps_paged_decode_workspace_size(D) for D in (0, -16, 24, 272)] == [0] * 4
    assert need <= L.ps_paged_decode_workspace_size(80) <= L.ps_paged_decode_workspace_size(256)

    def run(seqs=2, Hq=4, Hk=2, D=64, dt=0, q=P, ldq=256, kc=P, vc=P, pages=16, page=16, table=P, ldt=8, lens=P, window=0, scale=0.1,
            o=P, ldo=256, ws=P, wsb=need):
        return L.ps_paged_decode(seqs, Hq, Hk, D, dt, q, ldq, kc, vc, pages, page, table, ldt, lens, window, scale, o, ldo, None, ws,
                                 wsb, None)
    for bad in (dict(seqs=-1), dict(Hq=3), dict(Hq=1), dict(Hq=0), dict(Hq=1 << 17), dict(Hk=0), dict(D=40), dict(D=512), dict(dt=3),
                dict(q=None), dict(q=ODD), dict(ldq=255), dict(ldq=260), dict(kc=None), dict(vc=ODD), dict(pages=-1), dict(page=12),
                dict(table=None), dict(ldt=0), dict(ldt=1 << 40), dict(lens=None), dict(window=-1), dict(scale=NAN), dict(scale=INF),
                dict(o=None), dict(o=ODD), dict(ldo=128)):
        assert run(**bad) == INV, bad
    assert run(wsb=need - 1) == WS and run(ws=ODD) == WS and run(seqs=0, ws=None) == WS


def test_holders_say_what_is_wrong():
    """CPU tensors: looked at, and refused by name."""
    from paper_2606_29758_gb300 import CacheShape, DecodeAttention, DecodeShape, NormShape, PagedCache, PsppoError, ResidualNorm
    with pytest.raises(ValueError, match="page"):
        PagedCache(CacheShape(2, 8, 24, 1, 16, 64), device="cpu")
    c = PagedCache(CacheShape(3, 8, 4, 1, 16, 20, layers=2), device="cpu")
    for bad, error in ((lambda: c.reserve(3, 1), IndexError), (lambda: c.reserve(-1, 1), IndexError),
                       (lambda: c.reserve(0, 21), ValueError), (lambda: c.reserve(0, -5), ValueError),
                       (lambda: c.release(7), IndexError), (lambda: c.share(0, [1], 1), ValueError),
                       (lambda: c.share(0, [0], 0), ValueError), (lambda: c.share(0, [1, 1], 0), ValueError),
                       (lambda: c.share(0, [3], 0), IndexError), (lambda: c.share(0, [1], -1), ValueError)):
        with pytest.raises(error):
            bad()
    assert c.table.eq(-1).all() and len(c._free) == 8
    c.reserve(0, 17)                                                      # 5 pages
    with pytest.raises(PsppoError):
        c.reserve(1, 16)                                                  # 4 of 3
    with pytest.raises(PsppoError):
        c.reserve(2, 17)
    assert len(c._free) == 3 and c.table[1:].eq(-1).all()
    c.share(0, [1, 2], 18)                                                # (4 whole pages, and a begun one each)
    assert torch.equal(c.table[0, :4], c.table[1, :4]) and len({int(c.table[b, 4]) for b in range(3)}) == 3 and len(c._free) == 1
    c.release(0)
    c.release(0)
    assert len(c._free) == 2
    c.release(2)
    c.release(1)
    assert sorted(c._free) == list(range(8)) and c.table.eq(-1).all() and not any(c._users)
    for name in ("k", "v", "table", "lengths"):
        with pytest.raises(AttributeError):
            setattr(c, name, None)
    m = ResidualNorm(NormShape(4, 16), device="cpu")
    x = torch.zeros(4, 16, dtype=BF)
    with pytest.raises(ValueError, match="without a branch"):
        m.forward(x, gate=torch.ones(4))
    with pytest.raises(ValueError):
        m.forward(torch.zeros(5, 16, dtype=BF))
    with pytest.raises(ValueError):
        m.backward(None, x, x)
    with pytest.raises(RuntimeError):
        ResidualNorm(NormShape(4, 16, train=False), device="cpu").backward(x, x, x)
    with pytest.raises(ValueError, match="heads"):
        DecodeAttention(DecodeShape(3, 2, 2, 16), device="cpu").forward(torch.zeros(3, 32, dtype=BF), c)


# ---------------------------------------------------------------------- devices (made up: none of these calls reaches a GPU)
@pytest.fixture()
def parts(monkeypatch):
    from paper_2606_29758_gb300 import _build, block, cache
    _build.build()
    monkeypatch.setattr(block, "_device", lambda: 0)
    monkeypatch.setattr(block, "_stream", lambda: 0)
    return block, cache


def _holders(parts, at):
    """(name, entry, the call with one tensor's device changed, the names of its tensors), all buffers on `at`."""
    block, cache = parts
    N, d, H, D = 3, 16, 2, 16
    norm = block.ResidualNorm(block.NormShape(4, d), device="cpu")
    c = cache.PagedCache(cache.CacheShape(4, 8, 4, H, D, 16), device="cpu")
    att = cache.DecodeAttention(cache.DecodeShape(4, 2 * H, H, D), device="cpu")
    norm._at = c._at = att._at = at
    norm._fwd, norm._bwd, c._append, att._call = (Call() for _ in range(4))
    F32 = torch.float32

    def on(names, which, device):
        return {n: Rows(s, t, device if n == which else at) for n, (s, t) in names.items()}
    gains = dict(y=((N, d), BF), gy=((d,), BF), go=((d,), BF), gate=((N,), F32))
    fwd_in = dict(x=((N, d), BF), **gains, out=((N, d), BF))
    bwd_in = dict(do=((N, d), BF), dh=((N, d), BF), h=((N, d), BF), **gains)
    app_in = dict(k=((N, H * D), BF), v=((N, H * D), BF), row_seq=((N,), I32), row_pos=((N,), I32))
    dec_in = dict(q=((N, 2 * H * D), BF), out=((N, 2 * H * D), BF), lse=((N, 2 * H), F32))
    return [("norm forward", norm._fwd, lambda w=None, v=None: norm.forward(**on(fwd_in, w, v)), fwd_in),
            ("norm backward", norm._bwd, lambda w=None, v=None: norm.backward(**on(bwd_in, w, v)), bwd_in),
            ("append", c._append, lambda w=None, v=None: c.append(0, **on(app_in, w, v)), app_in),
            ("decode", att._call, lambda w=None, v=None: att.forward(cache=c, **on(dec_in, w, v)), dec_in)], c


def test_a_tensor_on_another_device(parts):
    holders, c = _holders(parts, HERE)
    for name, entry, call, tensors in holders:
        call()
        assert entry.made == 1, name
        for t in tensors:
            with pytest.raises(ValueError):
                call(t, OTHER)
            assert entry.made == 1, (name, t)
    c._at = OTHER                                                         # a cache on another device than the attention
    with pytest.raises(ValueError):
        holders[3][2]()
    assert holders[3][1].made == 1


def test_everything_on_a_device_that_is_not_current(parts):
    for name, entry, call, _ in _holders(parts, OTHER)[0]:
        with pytest.raises(ValueError):
            call()
        assert entry.made == 0, name


def test_small_calls_left_to_the_ordinary_way(L):
    """CPU tensors, other objects, wrong counts, plans of another kind: None, and no error left behind."""
    from paper_2606_29758_gb300 import _binding
    c, x, t = _binding.calls(), torch.zeros(3, 16, dtype=BF), torch.zeros(3, dtype=I32)
    norm = c.norm_plan(4, 16, 0, 3, 2, 1.0, 1.0, 1e-6, *[0] * 9)
    cache = c.cache_plan(4, 1, 16, 0, 1, 8, 4, 2, 0, *[0] * 6)
    att = c.decode_plan(4, 1, 1, 16, 0, 0, 0.25, 0, 0, 0)
    for call in (lambda: c.norm_fwd(norm, x, x, None, None, None, None), lambda: c.norm_fwd(cache, x, x, None, None, None, None),
                 lambda: c.norm_fwd(), lambda: c.norm_fwd(*[None] * 7), lambda: c.norm_bwd(norm, x, x, x, x, None, None, None, False),
                 lambda: c.norm_bwd(*[3] * 9), lambda: c.append(cache, 0, x, x, t, t, 1), lambda: c.append(norm, 0, x, x, t, t, 1),
                 lambda: c.append(1), lambda: c.append(*[None] * 7), lambda: c.decode(att, cache, 0, x, None, None),
                 lambda: c.decode(cache, att, 0, x, None, None), lambda: c.decode(*["x"] * 6), lambda: c.decode()):
        assert call() is None
    for plan in (c.norm_plan, c.cache_plan, c.decode_plan, c.bind_more):
        with pytest.raises(TypeError):
            plan(1, 2)
    names = [n for n in dir(c) if n not in ("bind", "bind_more") and not n.startswith("_")]
    assert all(getattr(_binding._Ordinary, n)() is None for n in names)   # (what stands in where the module is not)
