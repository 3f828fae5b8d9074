"""Calls of the residual norms and of attention over the paged cache that users may make and that sizes alone do not show: other
streams, the widest rows, places far into a cache, scores of minus infinity, gradients against differences, and the two ways of a
call."""
import numpy as np
import pytest
import torch

from oracle import block as ob
from test_gpu_paged import _att, _cache, _check, _queries

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def _rows(g, *shape, dt=BF):
    return torch.randn(*shape, device="cuda", generator=g).to(dt)


def _norm(rows, d, dtype=BF, **kw):
    from paper_2606_29758_gb300 import NormShape, ResidualNorm
    return ResidualNorm(NormShape(rows, d, dtype, **kw))


@pytest.mark.parametrize("post", [True, False])
def test_gradients_are_differences(post):
    """The kernel's f32 gradients against central differences of the float64 forward: 1e-8 from the differences; the kernel's sums of
    24 columns (7 rows) with some ten roundings a term, a few terms each, 64 * 24 * 2^-24 of the largest gradient."""
    N, d, a, b, eps, t = 7, 24, 0.6, 1.5, 1e-4, 1e-5
    rng = np.random.default_rng(1)
    p = {k: rng.standard_normal(s).astype(np.float32).astype(np.float64)
         for k, s in dict(x=(N, d), y=(N, d), gy=d, go=d, gate=N).items()}
    do, dh = rng.standard_normal((2, N, d)).astype(np.float32).astype(np.float64)
    m = _norm(N, d, F32, post=post, res_scale=a, branch_scale=b, eps=eps)
    c = {k: torch.from_numpy(v).float().cuda() for k, v in dict(p, do=do, dh=dh).items()}
    x = c.pop("x")
    h, _ = m.forward(x, c["y"], c["gy"], c["go"], c["gate"])
    got = m.backward(c["do"], c["dh"], h, c["y"], c["gy"], c["go"], c["gate"])

    def loss(p):
        h, o = ob.norm_forward(p["x"], p["y"], p["gy"], p["go"], p["gate"], a, b, eps, post)
        return (dh * h).sum() + (do * o).sum()
    for name, have in zip(("x", "y", "gy", "go", "gate"), got):
        want = np.zeros_like(p[name])
        for i in np.ndindex(want.shape):
            for sign in (1, -1):
                q = dict(p, **{name: p[name].copy()})
                q[name][i] += sign * t
                want[i] += sign * loss(q) / (2 * t)
        off = np.abs(have.double().cpu().numpy() - want).max() / np.abs(want).max()
        assert off <= 64 * 24 * 2.0 ** -24, (name, off)


@pytest.mark.parametrize("N,d", [(300, 1000), (5, 771), (64, 3584), (2000, 40)])
def test_the_sum_is_rounded_alike_however_rows_lie(N, d):
    """bf16 after the branch's norm: h is the f32 nearest to the sum, rounded to bf16, whatever the alignment."""
    g = torch.Generator(device="cuda").manual_seed(d)
    x, y, gy, gate = _rows(g, N, d), _rows(g, N, d), _rows(g, d), torch.rand(N, device="cuda", generator=g)
    want, _ = ob.norm_forward(*(t.double().cpu().numpy() for t in (x, y, gy)), np.ones(d), gate.double().cpu().numpy(), 0.7, 1.1,
                              1e-6, True)
    want = torch.from_numpy(want).float().to(BF).cuda()
    m = _norm(N, d, res_scale=0.7, branch_scale=1.1, train=False)
    for off, pitch in ((0, d), (0, -(-d // 8) * 8), (3, d + 5), (1, d + 8)):
        place = [torch.zeros(N * pitch + 16, dtype=BF, device="cuda")[off:off + N * pitch].view(N, pitch)[:, :d] for _ in range(2)]
        place[0].copy_(x)
        place[1].copy_(y)
        h, _ = m.forward(*place, gy, None, gate)
        assert torch.equal(h, want), (off, pitch, (h != want).sum().item())
        m.forward(*place, gy, None, gate, out=place[0])
        assert torch.equal(place[0], want), (off, pitch)


@pytest.mark.parametrize("d", [40, 300, 3584])
def test_sums_near_the_end_of_the_range(d):
    """A row whose squares add up to 1.5e38 to 3e38, one with zeros alone, one with an infinity: the root's f32 error (d 2^-24) and the
    sum's rounding to bf16. Behind the infinity the root is 0."""
    g = torch.Generator(device="cuda").manual_seed(d)
    x, y = _rows(g, 5, d), _rows(g, 5, d)
    y[0, d // 2] = 1.22e19
    y[1, 0], y[1, d - 1] = -1.22e19, 1.22e19
    y[2] = 0
    y[3, 3] = float("inf")
    h, o = _norm(5, d, train=False).forward(x, y)
    rows = [0, 1, 2, 4]
    hw, _ = ob.norm_forward(*(t[rows].double().cpu().numpy() for t in (x, y)), np.ones(d), np.ones(d), np.ones(4), 1.0, 1.0, 1e-6, True)
    got, size = h[rows].double().cpu().numpy(), np.abs(hw) + np.abs(x[rows].double().cpu().numpy())
    assert (np.abs(got - hw) <= (2.0 ** -8 + d * 2.0 ** -24) * size).all()
    rest = torch.arange(d, device="cuda") != 3
    assert h[3, 3].isnan() and torch.equal(h[3][rest], x[3][rest]) and o[3].isnan().all()


@pytest.mark.parametrize("dt,d", [(BF, 16377), (BF, 16384), (F32, 8189), (F32, 8192)])
def test_the_widest_rows_of_all_alignments(dt, d):
    """Sums of d squares and products: d 2^-24 of the sums of their sizes at most, both ways, plus the output's rounding."""
    N, g = 3, torch.Generator(device="cuda").manual_seed(d)
    x, y, do, dh = (_rows(g, N, d, dt=dt) for _ in range(4))
    gy, go = _rows(g, d, dt=dt), _rows(g, d, dt=dt)
    m = _norm(N, d, dt)
    h, o = m.forward(x, y, gy, go)
    n = lambda *ts: [t.double().cpu().numpy() for t in ts]  # noqa: E731
    hw, ow = ob.norm_forward(*n(x, y, gy, go), np.ones(N), 1.0, 1.0, 1e-6, True)
    r = 2.0 ** -8 if dt == BF else 2.0 ** -24
    tol = (r + d * 2.0 ** -24)
    for got, want in ((h, hw), (o, ow)):
        assert (np.abs(n(got)[0] - want) <= 4 * tol * (np.abs(want) + np.abs(n(x)[0]))).all()
    got = m.backward(do, dh, h, y, gy, go)
    want = ob.norm_backward(*n(do, dh, h, y, gy, go), np.ones(N), 1.0, 1.0, 1e-6, True)
    for name, a, b in zip(("dx", "dy", "dgy", "dgo"), got, want):
        off = np.abs(n(a)[0] - b).max() / np.abs(b).max()
        assert off <= 4 * tol, (name, off)


@pytest.mark.parametrize("d", [1, 2, 3, 5, 7, 8, 9])
@pytest.mark.parametrize("dt", [BF, F32])
def test_narrow_rows_stay_in_their_tensors(d, dt):
    """Chunks of 16 bytes hold several rows; what lies right before and behind the tensors is neither used nor written."""
    N, g = 100, torch.Generator(device="cuda").manual_seed(d)
    for off in (8, 9, 13):
        whole = [torch.full((16 + N * d + 16,), float("nan"), dtype=dt, device="cuda") for _ in range(3)]
        x, y, h = (w[off:off + N * d].view(N, d) for w in whole)
        x.copy_(_rows(g, N, d, dt=dt))
        y.copy_(_rows(g, N, d, dt=dt))
        m = _norm(N, d, dt, post=False)
        m.forward(x, y, out=h)
        assert torch.equal(h, (x.float() + y.float()).to(dt))
        got = m.backward(x, y, h, y)
        assert all(torch.isfinite(t).all() for t in got if t is not None)
        for w in whole:
            assert w[:off].isnan().all() and w[off + N * d:].isnan().all()


def test_two_streams():
    """Holders of their own on streams of their own, both under way at once: the bits of one after the other."""
    lens, Hq, Hk, D = [3000, 700, 1, 2500] * 8, 12, 2, 128
    g = torch.Generator(device="cuda").manual_seed(0)
    sides = []
    for s in range(2):
        c, _ = _cache(lens, Hk, D, 64, BF, seed=s)
        x, y, gain = _rows(g, 4000, 1536), _rows(g, 4000, 1536), _rows(g, 1536)
        sides.append((c, _queries(len(lens), Hq, D, BF, s), _att(len(lens), Hq, Hk, D, BF), _norm(4000, 1536), x, y, gain))

    def work(c, q, att, m, x, y, gain):
        out = []
        for _ in range(3):
            o = att.forward(q, c)
            h, n = m.forward(x, y, gain, gain)
            out = [o, h, n, *m.backward(x, y, h, y, gain, gain)[:4]]
        return [t.clone() for t in out]
    want = [work(*s) for s in sides]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in sides], []
    for _ in range(2):
        got = []
        for s, side in zip(streams, sides):
            with torch.cuda.stream(s):
                got.append(work(*side))
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        for s, t in zip(a, b):
            assert torch.equal(s, t)


@pytest.mark.parametrize("page", [64, 8])
def test_places_behind_2_31_elements(page):
    """A cache of 2^31 elements and more: the last pages, by appending and by attention (chunks by the copy engine, and by lanes)."""
    from paper_2606_29758_gb300 import CacheShape, PagedCache
    Hq, Hk, D, L = 8, 8, 128, 200
    pages = (1 << 31) // (Hk * page * D) + 60
    c = PagedCache(CacheShape(2, pages, page, Hk, D, L + page))
    need = -(-L // page)
    c.table[0, :need] = torch.arange(pages - 1, pages - 1 - need, -1, dtype=torch.int32)
    c.table[1, :need] = torch.arange(need, dtype=torch.int32)
    c.lengths.fill_(L)
    g, kv = torch.Generator(device="cuda").manual_seed(page), []
    pos = torch.arange(1, L + 1, dtype=torch.int32, device="cuda")
    for b in range(2):
        k, v = _rows(g, L, Hk * D), _rows(g, L, Hk * D)
        c.append(0, k, v, torch.full_like(pos, b), pos)
        kv.append(tuple(t.view(L, Hk, D).double().cpu().numpy() for t in (k, v)))
    c.check_status()
    q, lse, m = _queries(2, Hq, D, BF), torch.empty(2, Hq, device="cuda"), _att(2, Hq, Hk, D, BF)
    o = m.forward(q, c, lse=lse)
    m.check_status()
    _check(o, lse, q, kv, Hq, Hk, D, BF)


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("lens", [[100, 40], [3000, 40], [5000] * 40])
def test_scores_that_are_all_minus_infinity(lens, dt):
    """0 / 0, as in a softmax of them: NaN and a sum of minus infinity; a part of them counts nothing; others are as ever."""
    Hq, Hk, D = 4, 2, 64
    c, kv = _cache(lens, Hk, D, 16, dt, seed=3)
    q = _queries(len(lens), Hq, D, dt).abs_()
    m, lse = _att(len(lens), Hq, Hk, D, dt), torch.empty(len(lens), Hq, device="cuda")
    need = -(-lens[0] // 16)
    c.k[0, c.table[0, :need].long()] = float("-inf")
    o = m.forward(q, c, lse=lse)
    m.check_status()
    assert o[0].isnan().all() and (lse[0] == float("-inf")).all()
    rows = range(1, min(4, len(lens)))
    _check(o, lse, q, kv, Hq, Hk, D, dt, rows=rows)
    # only the first page's: its keys have no weight
    part, kv2 = _cache(lens, Hk, D, 16, dt, seed=3)
    part.k[0, part.table[0, 0].long()] = float("-inf")
    part_kv = [(kv2[0][0][16:], kv2[0][1][16:])]
    o = m.forward(q, part, lse=lse)
    _check(o, lse, q, part_kv + kv2[1:], Hq, Hk, D, dt, rows=[0, *rows])


# ---------------------------------------------------------------------- the module of small calls
def _both(parts, call):
    """The call's outputs by the module, and by the ordinary way: the same bits."""
    first = [None if o is None else o.clone() for o in call()]
    kept = [(h, n, getattr(h, n)) for h, n in parts]
    try:
        for h, n in parts:
            setattr(h, n, lambda *a: None)
        second = [None if o is None else o.clone() for o in call()]
    finally:
        for h, n, f in kept:
            setattr(h, n, f)
    for a, b in zip(first, second):
        assert (a is None and b is None) or torch.equal(a, b)


@pytest.mark.parametrize("N", [0, 1, 5, 300])
@pytest.mark.parametrize("dt", [BF, F32])
def test_the_same_bits_both_ways(N, dt):
    from paper_2606_29758_gb300 import CacheShape, PagedCache
    g = torch.Generator(device="cuda").manual_seed(N)
    x, y, do, dh = (_rows(g, N, 104, dt=dt)[:, :96] for _ in range(4))
    gy, go, gate = _rows(g, 96, dt=dt), _rows(g, 96, dt=dt), torch.rand(N, device="cuda", generator=g)
    for pre in (True, False):
        m = _norm(300, 96, dt, pre=pre)
        both = [(m, "_fast_fwd"), (m, "_fast_bwd")]
        go_, do_ = (go, do) if pre else (None, None)
        _both(both, lambda: m.forward(x, y, gy, go_, gate))
        _both(both, lambda: m.forward(x, y, out=torch.empty(N, 112, dtype=dt, device="cuda")[:, :96]))
        _both(both, lambda: m.backward(do_, dh, x, y, gy, go_, gate))
        if pre:
            _both(both, lambda: m.forward(x, go=go))
            _both(both, lambda: m.backward(do, None, x))
            _both(both, lambda: m.backward(do, dh, x, y, dw_accumulate=True)[:2])
    c = PagedCache(CacheShape(300, 900, 4, 2, 48, 12, layers=2, dtype=dt))
    c.table.copy_(torch.arange(900, device="cuda", dtype=torch.int32).view(300, 3))
    c.lengths.copy_(torch.arange(300, device="cuda") % 13)
    for t in (c.k, c.v):
        t.copy_(_rows(g, *t.shape, dt=dt))
    qkv = _rows(g, N, 8 * 48, dt=dt)
    seq, pos = torch.arange(N, device="cuda", dtype=torch.int32), c.lengths[:N].clamp(min=1)

    def append():
        c.append(1, qkv[:, 4 * 48:6 * 48], qkv[:, 6 * 48:], seq, pos)
        return [c.k, c.v]
    _both([(c, "_fast")], append)
    c.check_status()
    m, lse = _att(300, 4, 2, 48, dt, window=5), torch.empty(N, 4, device="cuda")
    for layer in range(2):
        _both([(m, "_fast")], lambda: [m.forward(qkv[:, :4 * 48], c, layer, lse=lse), lse])
        _both([(m, "_fast")], lambda: [m.forward(qkv[:, :4 * 48], c, layer, out=torch.empty(N, 200, dtype=dt, device="cuda")[:, :192])])
    m.check_status()


def test_refusals_come_from_the_ordinary_way():
    from paper_2606_29758_gb300 import CacheShape, PagedCache
    from paper_2606_29758_gb300 import _binding as B
    z = lambda *s, dt=BF: torch.zeros(*s, dtype=dt, device="cuda")  # noqa: E731
    one, m, c, att = torch.zeros(4, dtype=torch.int32, device="cuda"), _norm(4, 16), PagedCache(CacheShape(4, 8, 4, 1, 16, 8)), _att(
        4, 2, 1, 16, BF)
    x, k = z(4, 16), z(4, 16)
    for bad, error in ((lambda: m.forward(x.cpu(), x), ValueError), (lambda: m.forward(z(5, 16)), ValueError),
                       (lambda: m.forward(x, z(4, 15)), ValueError), (lambda: m.forward(x, x.float()), TypeError),
                       (lambda: m.forward(x, x, z(15)), ValueError), (lambda: m.forward(x, x, gate=z(4)), TypeError),
                       (lambda: m.forward(x, x, gate=z(3, dt=F32)), ValueError), (lambda: m.forward(x, out=x), ValueError),
                       (lambda: m.forward(x, z(16, 4).t()), ValueError), (lambda: m.backward(None, x, x), ValueError),
                       (lambda: m.backward(x, x, x, gate=z(4, dt=F32)), ValueError), (lambda: m.backward(x, x, z(3, 16)), ValueError),
                       (lambda: c.append(1, k, k, one, one), IndexError), (lambda: c.append(-1, k, k, one, one), IndexError),
                       (lambda: c.append(0, z(4, 17)[:, 1:], k, one, one), B.PsppoError),
                       (lambda: c.append(0, k, z(4, 8), one, one), ValueError), (lambda: c.append(0, k, k, one.long(), one), TypeError),
                       (lambda: c.append(0, k, k, one, one[:3]), ValueError), (lambda: c.append(0, k.float(), k, one, one), TypeError),
                       (lambda: att.forward(z(5, 32), c), ValueError), (lambda: att.forward(z(4, 16), c), ValueError),
                       (lambda: att.forward(z(4, 32), c, 1), IndexError), (lambda: att.forward(z(4, 32, dt=F32), c), TypeError),
                       (lambda: att.forward(z(4, 33)[:, 1:], c), B.PsppoError),
                       (lambda: att.forward(z(4, 32), c, lse=z(4, 2)), TypeError),
                       (lambda: att.forward(z(4, 32), c, lse=z(2, 4, dt=F32)), ValueError),
                       (lambda: att.forward(z(4, 32), c, out=z(4, 31)), ValueError),
                       (lambda: _att(4, 2, 2, 16, BF).forward(z(4, 32), c), ValueError)):
        with pytest.raises(error):
            bad()


def test_plans_of_another_device_are_left_to_the_holder():
    """(their buffers' addresses are 0: nothing could be launched)"""
    from paper_2606_29758_gb300 import _binding as B
    calls, x = B.calls(), torch.zeros(3, 16, dtype=BF, device="cuda")
    one, here = torch.zeros(3, dtype=torch.int32, device="cuda"), torch.cuda.current_device()
    cache = lambda at: calls.cache_plan(4, 1, 16, 0, 1, 8, 4, 2, 0, *[0] * 6, at)  # noqa: E731
    att = lambda at: calls.decode_plan(4, 1, 1, 16, 0, 0, 0.25, 0, 0, 0, at)  # noqa: E731
    for at in (here + 1, -1):
        norm = calls.norm_plan(4, 16, 0, 3, 2, 1.0, 1.0, 1e-6, *[0] * 9, at)
        assert calls.norm_fwd(norm, x, x, None, None, None, None) is None
        assert calls.norm_bwd(norm, x, x, x, x, None, None, None, False) is None
        assert calls.append(cache(at), 0, x, x, one, one, 1) is None
        for a, b in ((at, at), (here, at), (at, here)):
            assert calls.decode(att(a), cache(b), 0, x, None, None) is None
    assert calls.append(cache(here), 0, x, x, one, one, 1) == B.PS_ERR_INVALID_ARG      # (the library's refusal)
    assert calls.decode(att(here), cache(here), 0, x, None, None) == B.PS_ERR_INVALID_ARG
