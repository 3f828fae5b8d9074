"""The norms before and after a branch with its gate and the residual sum against float64 (oracle.block), forward and backward.

Tolerances, with e = 2^-24 the unit roundoff of f32 (outputs in bf16: plus 2^-8 of the value). A row's sum of d <= 16384
values: 32 in a thread, 5 joins in a warp, 16 warps: under 56 e of the sum of magnitudes; its inverse root has half of a sum of squares'
and 3 e: 31 e. h = a x + w n: n = y r gy under 36 e of |w n|, the sum 2 e: under 40 e of S = |a x| + |w n|, held to 2^-18.
o = h r go: the root's 31 e, and h's 40 e through the mean of squares: 40 e K, K = rms(S) / rms(h): held to
2^-17 r |go| (S + K |h|). dH: its mean under 60 e of mean |go do h|, three roots, four roundings: under 256 e of R = |dh| +
r (|go do| + |h| r^2 mean |go do h|). dy and dgate take dH's 256 e, a sum's 60 e and the branch's root three times: under 512 e of
the same with magnitudes and R for dH. Gain gradients: at most `terms` values in turn in a thread, at most 16 joins, then f64: (terms +
64) e of the sum of magnitudes, dgy with dH's error and the root's (terms + 512) e."""
import numpy as np
import pytest
import torch

from oracle import block as ob

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
E = 2.0 ** -24


def _rows(N, d, dtype, g, pitch=None, shift=0):
    """N(0, 1) rows, if a pitch is given as a column range that begins `shift` elements into rows of it."""
    if pitch is None:
        return torch.randn(N, d, generator=g).to(dtype).cuda()
    return torch.randn(N, pitch, generator=g).to(dtype).cuda()[:, shift:shift + d]


def _case(N, d, dtype, gate=True, seed=0, pitch=None, shift=0):
    g = torch.Generator().manual_seed(seed + 31 * N + d)
    c = {k: _rows(N, d, dtype, g, pitch, shift) for k in ("x", "y", "do", "dh")}
    if N > 2:
        c["y"][1] = 0.0
        c["x"][2] = 0.0
        c["y"][2] = 0.0          # h is 0: r = eps^(-1/2)
        c["do"][0] = 0.0
    c["gy"], c["go"] = ((1 + 0.3 * torch.randn(d, generator=g)).to(dtype).cuda() for _ in range(2))
    c["gate"] = None
    if gate:
        c["gate"] = torch.randn(N, generator=g)
        if N > 4:
            c["gate"][3] = 0.0
        c["gate"] = c["gate"].cuda()
    return c


def _op(N, d, dtype, **kw):
    from paper_2606_29758_gb300 import NormShape, ResidualNorm
    return ResidualNorm(NormShape(rows=N, d=d, dtype=dtype, **kw))


def _n(t):
    return None if t is None else t.detach().double().cpu().numpy()


def _rms(x, eps):
    return 1.0 / np.sqrt(np.mean(x * x, axis=-1, keepdims=True) + eps)


def _check(c, got, dtype, post, pre, a, b, eps, terms, branch=True, do=True, dh=True):
    h, o, dx, dy, dgy, dgo, dgate = got
    half = 2.0 ** -8 if dtype == BF else 0.0
    N, d = c["x"].shape
    x, y, gy, go = (_n(c[k]) for k in ("x", "y", "gy", "go"))
    gate = np.ones(N) if c["gate"] is None else _n(c["gate"])
    if not branch:
        y = None
    hw, ow = ob.norm_forward(x, y, gy, go, gate, a, b, eps, post)

    def near(t, want, reach, part, name):
        t = _n(t)
        bad = ~(np.abs(t - want) <= part * reach + (half * np.abs(want) if part <= 2.0 ** -15 and t.ndim == 2 else 0.0))
        assert not bad.any(), (name, np.argwhere(bad)[:4], t[bad][:4], want[bad][:4])

    w = None
    if branch:
        w = np.abs(b * gate)[:, None]
        ry = _rms(y, eps) if post else np.ones((N, 1))
        S = np.abs(a * x) + w * np.abs(y * ry * gy)
        near(h, hw, S, 2.0 ** -18, "h")
    else:
        S = np.abs(x)
    if pre:
        r = _rms(hw, eps)
        K = np.sqrt(np.mean(S * S, axis=1, keepdims=True) * r * r)
        near(o, ow, r * np.abs(go) * (S + K * np.abs(hw)), 2.0 ** -17, "o")
    if dx is None:
        return
    H = _n(h)                     # the backward has the stream as it is held
    DO = _n(c["do"]) if do and pre else np.zeros((N, d))
    DH = _n(c["dh"]) if dh else np.zeros((N, d))
    want = ob.norm_backward(DO, DH, H, y, gy, go, gate, a, b, eps, post)
    r = _rms(H, eps)
    gd = np.abs(go * DO)
    R = np.abs(DH) + r * (gd + np.abs(H) * r * r * np.mean(gd * np.abs(H), axis=1, keepdims=True))
    near(dx, want[0], abs(a) * R if branch else R, 2.0 ** -16, "dx")
    if pre:
        near(dgo, want[3], np.sum(np.abs(DO * H * r), axis=0), (terms + 64) * E, "dgo")
    if not branch:
        assert dy is None and dgy is None and dgate is None
        return
    reach = np.abs(gy) * R
    if post:
        reach = ry * (reach + np.abs(y) * ry * ry * np.mean(reach * np.abs(y), axis=1, keepdims=True))
    near(dy, want[1], w * reach, 2.0 ** -15, "dy")
    near(dgy, want[2], np.sum(w * R * np.abs(y) * ry, axis=0), (terms + 512) * E, "dgy")
    if c["gate"] is not None:
        near(dgate, want[4], abs(b) * np.sum(R * np.abs(y * ry * gy), axis=1), 2.0 ** -15, "dgate")


SIZES = [(1, 3584), (1, 1), (3, 8), (5, 7), (2, 63), (37, 64), (64, 100), (9, 256), (130, 264), (33, 771), (77, 1025), (300, 1536),
         (7, 3584), (5, 4104), (6, 4100), (3, 8192), (1000, 96), (2500, 392), (1200, 16)]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("post", [True, False])
@pytest.mark.parametrize("N,d", SIZES)
def test_forward_and_backward(N, d, post, dtype):
    c = _case(N, d, dtype)
    a, b, eps = 0.75, 0.5, 1e-6
    m = _op(N, d, dtype, post=post, eps=eps, res_scale=a, branch_scale=b)
    h, o = m.forward(c["x"], c["y"], c["gy"], c["go"], gate=c["gate"])
    g = m.backward(c["do"], c["dh"], h, c["y"], c["gy"], c["go"], gate=c["gate"])
    m_status(m)
    _check(c, (h, o, *g), dtype, post, True, a, b, eps, N)


def m_status(m):
    from paper_2606_29758_gb300 import _binding as B
    assert B.ps_workspace_status(m.ws) == (B.PS_OK, 0)


@pytest.mark.parametrize("N,d", [(3, 16384), (2, 12289), (4, 9000)])
def test_the_widest_rows(N, d):
    c = _case(N, d, BF)
    m = _op(N, d, BF)
    h, o = m.forward(c["x"], c["y"], c["gy"], c["go"], gate=c["gate"])
    _check(c, (h, o, *m.backward(c["do"], c["dh"], h, c["y"], c["gy"], c["go"], gate=c["gate"])), BF, True, True, 1.0, 1.0, 1e-6, N)
    with pytest.raises(Exception, match="invalid"):
        f = _op(1, 8200, F32)
        f.forward(*(torch.ones(1, 8200, device="cuda") for _ in range(2)))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("N,d", [(5, 40), (61, 771), (33, 3584)])
def test_parts_that_are_absent(N, d, dtype):
    """No branch; no normed output; no gate, no gains; one gradient alone."""
    c = _case(N, d, dtype, gate=False)
    one = dict(c, gy=torch.ones(d), go=torch.ones(d))
    m = _op(N, d, dtype)
    h, o = m.forward(c["x"], go=c["go"])
    assert h is c["x"]
    _check(c, (h, o, *m.backward(c["do"], c["dh"], h, go=c["go"])), dtype, False, True, 1.0, 1.0, 1e-6, N, branch=False)
    _check(c, (h, o, *m.backward(c["do"], None, h, go=c["go"])), dtype, False, True, 1.0, 1.0, 1e-6, N, branch=False, dh=False)
    h, o = m.forward(c["x"], c["y"])
    _check(one, (h, o, *m.backward(c["do"], None, h, c["y"])), dtype, True, True, 1.0, 1.0, 1e-6, N, dh=False)
    for post in (True, False):
        m = _op(N, d, dtype, pre=False, post=post, branch_scale=0.3)
        h, o = m.forward(c["x"], c["y"], c["gy"])
        assert o is None
        g = m.backward(None, c["dh"], h, c["y"], c["gy"])
        assert g[3] is None and g[4] is None
        _check(c, (h, o, *g), dtype, post, False, 1.0, 0.3, 1e-6, N)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d,pitch,shift", [(96, 200, 8), (96, 200, 3), (771, 1003, 1), (264, 272, 0), (1, 3, 1)])
def test_strides_and_alignments(d, pitch, shift, dtype):
    N = 40
    c = _case(N, d, dtype, pitch=pitch, shift=shift)
    m = _op(N, d, dtype)
    wide = torch.full((N, pitch), 7.0, dtype=dtype, device="cuda")
    h, o = m.forward(c["x"], c["y"], c["gy"], c["go"], gate=c["gate"], out=wide[:, shift:shift + d])
    _check(c, (h, o, *m.backward(c["do"], c["dh"], h, c["y"], c["gy"], c["go"], gate=c["gate"])), dtype, True, True, 1.0, 1.0, 1e-6,
           N)
    kept = torch.ones(pitch, dtype=torch.bool)
    kept[shift:shift + d] = False
    assert (wide[:, kept.cuda()] == 7.0).all()
    over = dict(c, x=torch.empty(N, pitch, dtype=dtype, device="cuda")[:, shift:shift + d].copy_(c["x"]))
    h2, o2 = m.forward(over["x"], c["y"], c["gy"], c["go"], gate=c["gate"], out=over["x"])   # over its input
    assert h2 is over["x"] and torch.equal(h2, h) and torch.equal(o2, o)        # (the same alignment, the same order of sums)
    h2, o2 = m.forward(c["x"].contiguous(), c["y"], c["gy"], c["go"], gate=c["gate"])        # rows that lie otherwise than the rest
    _check(c, (h2, o2, *m.backward(c["do"].contiguous(), c["dh"], h2, c["y"], c["gy"], c["go"], gate=c["gate"])), dtype, True, True,
           1.0, 1.0, 1e-6, N)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d", [64, 777, 3584])
def test_a_shut_gate_and_values_beyond_it(d, dtype):
    """A gate of 0 leaves out NaN and infinities; those of a row stay in it (the gain gradients have every row)."""
    N = 21
    c = _case(N, d, dtype)
    m = _op(N, d, dtype)
    c["gate"][3] = 0.0
    call = lambda: (m.forward(c["x"], c["y"], c["gy"], c["go"], gate=c["gate"]))  # noqa: E731
    h, o = (t.clone() for t in call())
    g = [t.clone() for t in m.backward(c["do"], c["dh"], h, c["y"], c["gy"], c["go"], gate=c["gate"])]
    assert not g[1][3].any()
    c["y"][3, ::2] = float("nan")
    c["y"][3, 1::2] = float("inf")
    h2, o2 = (t.clone() for t in call())
    g2 = m.backward(c["do"], c["dh"], h, c["y"], c["gy"], c["go"], gate=c["gate"])
    assert torch.equal(h, h2) and torch.equal(o, o2)
    for i in range(4):
        assert torch.equal(g[i], g2[i])
    others = torch.arange(N, device="cuda") != 3
    assert torch.isnan(g2[4][3]) and torch.equal(g[4][others], g2[4][others])
    c["y"][7, 0] = float("nan")
    h2, o2 = call()
    assert torch.isnan(o2[7]).all() and torch.equal(o2[torch.arange(N, device="cuda") != 7], o[torch.arange(N, device="cuda") != 7])


def test_many_rows_reruns_and_sums_over_calls():
    N, d = 9001, 1536
    c = _case(N, d, BF)
    m = _op(N, d, BF)
    h, o = m.forward(c["x"], c["y"], c["gy"], c["go"], gate=c["gate"])
    first = [t.clone() for t in m.backward(c["do"], c["dh"], h, c["y"], c["gy"], c["go"], gate=c["gate"])]
    _check(c, (h, o, *first), BF, True, True, 1.0, 1.0, 1e-6, N)
    for a, b in zip(m.backward(c["do"], c["dh"], h, c["y"], c["gy"], c["go"], gate=c["gate"]), first):
        assert torch.equal(a, b)
    m.backward(c["do"], c["dh"], h, c["y"], c["gy"], c["go"], gate=c["gate"], dw_accumulate=True)
    for a, b in ((m.dgy, first[2]), (m.dgo, first[3])):
        assert ((a - 2 * b).abs() <= 2.0 ** -22 * b.abs()).all()     # the same f64 sum onto it, rounded once
    # fewer rows of the same buffers; the rest stay
    m.h.fill_(5.0)
    m.o.fill_(5.0)
    h, o = m.forward(c["x"][:100], c["y"][:100], c["gy"], c["go"], gate=c["gate"][:100])
    assert h.shape[0] == 100 and (m.h[100:] == 5.0).all() and (m.o[100:] == 5.0).all()


def test_no_rows():
    m = _op(4, 64, BF)
    z = torch.zeros(0, 64, dtype=BF, device="cuda")
    h, o = m.forward(z, z)
    assert h.shape == o.shape == (0, 64)
    m.dgy.fill_(3.0)
    m.dgo.fill_(3.0)
    m.backward(z, z, z, z)
    assert not m.dgy.any() and not m.dgo.any()
    m.dgy.fill_(3.0)
    m.backward(z, z, z, z, dw_accumulate=True)
    assert (m.dgy == 3.0).all()


def test_captured_beside_eager_calls():
    """A replay gives the eager bits; captured forward and backward share the holder's buffers."""
    N, d = 300, 392
    c = _case(N, d, BF)
    m = _op(N, d, BF)

    def step():
        h, o = m.forward(c["x"], c["y"], c["gy"], c["go"], gate=c["gate"])
        return [h, o, *m.backward(c["do"], c["dh"], h, c["y"], c["gy"], c["go"], gate=c["gate"])]
    ref = [t.clone() for t in step()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step()
    for _ in range(2):
        for t in outs:
            t.zero_()
        graph.replay()
        for a, b in zip(outs, ref):
            assert torch.equal(a, b)


def test_rows_further_apart_than_two_gi_elements():
    """Row 1 lies 2^31 elements and more behind row 0 (bf16, 4.3 GB)."""
    d, pitch = 64, (1 << 31) + 64
    base = torch.empty(pitch + d, dtype=BF, device="cuda")
    x = base.as_strided((2, d), (pitch, 1))
    g = torch.Generator().manual_seed(1)
    c = _case(2, d, BF, gate=False)
    x.copy_(torch.randn(2, d, generator=g).to(BF).cuda())
    c["x"] = x
    m = _op(2, d, BF)
    h, o = m.forward(x, c["y"], c["gy"], c["go"])
    _check(c, (h, o, None, None, None, None, None), BF, True, True, 1.0, 1.0, 1e-6, 2)
