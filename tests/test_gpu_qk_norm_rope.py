"""Norms of queries and keys with rotary positions against float64 (oracle.block), forward and backward.

Tolerances, with e = 2^-24 the unit roundoff of f32 (bf16 outputs: plus 2^-8 of the value). A turned value is
a n1 + b n2 of normed values n = x r g: the mean of squares of D <= 512 values (16 in a lane, 5 joins: under 24 e, halved by
the root), rsqrt (2 e), two products, the turn (3 e) and the table's rounding (1 e): under 20 e of |n1| + |n2|, held
to 2^-18 = 64 e. A gradient r (g dn - x r^2 m) has the same steps over, its mean another 24 e: under 64 e of
r (|g dn| + |x| r^2 mean|g dn x|), held to 2^-17 = 128 e. A gain's gradient adds at most n terms per lane in turn, then f64:
(n + 64) e of the sum of magnitudes."""
import numpy as np
import pytest
import torch

from oracle import block as ob

pytestmark = pytest.mark.gpu
THETA, T = 1e6, 4096


def _B():
    from paper_2606_29758_gb300 import _binding as B
    return B


def _data(N, Hq, Hk, D, dtype, seed=0, base=1):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    t = [r(N, Hq * D) * torch.exp(r(N, 1)), r(N, Hk * D), 1 + 0.3 * r(D), 1 + 0.3 * r(D), r(N, Hq * D), r(N, Hk * D)]
    pos = torch.randint(base, base + T, (N,), generator=g, dtype=torch.int32)
    if N > 2:
        pos[0], pos[1] = base, base + T - 1
        t[0][2] = 0.0           # a row of zeros: r = eps^(-1/2)
        t[4][1] = 0.0
    return [v.to(dtype).cuda() for v in t] + [pos.cuda()]


def _make(N, Hq, Hk, D, R, dtype, inter, train=True, eps=1e-6):
    from paper_2606_29758_gb300 import QKNormRope, QKShape, rope_table
    table = rope_table(T, R, THETA) if R else None
    return QKNormRope(QKShape(rows=N, Hq=Hq, Hk=Hk, D=D, R=R, dtype=dtype, interleaved=inter, eps=eps, train=train), table)


def _heads(t, D):
    return t.double().cpu().numpy().reshape(t.shape[0], t.shape[1] // D, D)


def _check_part(x, gain, dy, y, dx, dgain, angles, eps, inter, dtype, terms):
    D = gain.shape[0]
    X, G, DY = _heads(x, D), gain.double().cpu().numpy(), _heads(dy, D)
    cos, sin = np.cos(angles), np.sin(angles)
    half = 2.0 ** -8 if dtype == torch.bfloat16 else 0.0
    want = ob.qk_forward(X, G, eps, cos, sin, inter)
    n = np.abs(ob.qk_forward(X, G, eps, np.ones_like(cos), np.zeros_like(sin), inter))
    reach = np.abs(ob.turn(n, np.ones_like(cos), -np.ones_like(sin), inter)) + n    # |n1| + |n2| of each pair at least
    reach = np.maximum(reach, np.abs(ob.turn(n, np.ones_like(cos), np.ones_like(sin), inter)) + n)
    assert (np.abs(_heads(y, D) - want) <= 2.0 ** -18 * reach + half * np.abs(want)).all()
    if dx is None:
        return
    wdx, wdg = ob.qk_backward(DY, X, G, eps, cos, sin, inter)
    r = 1.0 / np.sqrt(np.mean(X * X, axis=-1, keepdims=True) + eps)
    a = np.abs(DY)
    dn = np.maximum(np.abs(ob.turn(a, np.ones_like(cos), -np.ones_like(sin), inter)),
                    np.abs(ob.turn(a, np.ones_like(cos), np.ones_like(sin), inter)))
    gdn = dn * np.abs(G)
    reach = r * (gdn + np.abs(X) * r * r * np.mean(gdn * np.abs(X), axis=-1, keepdims=True))
    assert (np.abs(_heads(dx, D) - wdx) <= 2.0 ** -17 * reach + half * np.abs(wdx)).all()
    size = np.sum(dn * np.abs(X) * r, axis=(0, 1))
    assert (np.abs(dgain.double().cpu().numpy() - wdg) <= (terms + 64) * 2.0 ** -24 * size).all()


CASES = [(1, 28, 4, 128, 128), (1, 1, 0, 16, 16), (2, 3, 1, 32, 16), (5, 5, 1, 80, 32), (37, 6, 2, 96, 48),
         (64, 12, 2, 128, 64), (130, 16, 16, 64, 64), (571, 3, 0, 256, 256), (33, 2, 3, 512, 512), (20, 4, 4, 192, 0),
         (300, 28, 4, 128, 128), (9, 40, 8, 48, 48)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("N,Hq,Hk,D,R", CASES)
def test_forward_and_backward(N, Hq, Hk, D, R, inter, dtype):
    q, k, gq, gk, dq, dk, pos = _data(N, Hq, Hk, D, dtype, seed=N + D)
    m = _make(N, Hq, Hk, D, R, dtype, inter)
    qo, ko = m.forward(q, k, gq, gk, pos)
    m.check_status()
    a, b, dga, dgb = m.backward(dq, dk, q, k, gq, gk, pos)
    m.check_status()
    angles = ob.rope_angles(pos.cpu().numpy() - 1, R, THETA) if R else np.zeros((N, 0))
    terms = N * max(Hq, Hk)
    _check_part(q, gq, dq, qo, a, dga, angles, 1e-6, inter, dtype, terms)
    if Hk:
        _check_part(k, gk, dk, ko, b, dgb, angles, 1e-6, inter, dtype, terms)
    else:
        assert not dgb.any()


# Rows enough for several a warp, whose heads then come through shared memory (bf16); a lane adds up at most 8 rows of them.
LARGE = [(12500, 13, 3, 128, 64), (12300, 11, 2, 80, 80), (12200, 4, 4, 256, 256)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("N,Hq,Hk,D,R", LARGE)
def test_many_rows(N, Hq, Hk, D, R, dtype):
    q, k, gq, gk, dq, dk, pos = _data(N, Hq, Hk, D, dtype, seed=N)
    m = _make(N, Hq, Hk, D, R, dtype, Hk == 2)
    pos[777] = T + 5                               # outside the table
    qo, ko = m.forward(q, k, gq, gk, pos)
    rc, bits = _B().ps_workspace_status(m.ws)
    assert bits == _B().PS_DEV_BAD_LENGTH and torch.isnan(qo.view(N, Hq, D)[777, :, :R]).all()
    pos[777] = T
    qo, ko = (t.clone() for t in m.forward(q, k, gq, gk, pos))
    first = [t.clone() for t in m.backward(dq, dk, q, k, gq, gk, pos)]
    angles = ob.rope_angles(pos.cpu().numpy() - 1, R, THETA)
    terms = 8 * max(Hq, Hk)
    _check_part(q, gq, dq, qo, first[0], first[2], angles, 1e-6, Hk == 2, dtype, terms)
    _check_part(k, gk, dk, ko, first[1], first[3], angles, 1e-6, Hk == 2, dtype, terms)
    for a, b in zip(m.backward(dq, dk, q, k, gq, gk, pos), first):
        assert torch.equal(a, b)                   # reruns
    m.forward(q, k, gq, gk, pos, in_place=True)
    assert torch.equal(q, qo) and torch.equal(k, ko)
    m.check_status()


def test_the_table():
    from paper_2606_29758_gb300 import rope_table
    t = rope_table(3000, 96, 1e4).cpu().numpy()
    a = ob.rope_angles(np.arange(3000), 96, 1e4)
    # f64 of an angle up to 3000 (half an ulp of it: 2^-42), rounded once to f32
    assert np.abs(t[..., 0] - np.cos(a)).max() <= 2.0 ** -24 and np.abs(t[..., 1] - np.sin(a)).max() <= 2.0 ** -24


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_column_ranges_in_place_and_no_gains(dtype):
    N, Hq, Hk, D = 77, 6, 2, 64
    q, k, gq, gk, dq, dk, pos = _data(N, Hq, Hk, D, dtype, seed=1)
    m = _make(N, Hq, Hk, D, D, dtype, False)
    want = [t.clone() for t in m.forward(q, k, gq, gk, pos)]
    back = [t.clone() for t in m.backward(dq, dk, q, k, gq, gk, pos)]
    v = torch.full((N, Hk * D), 9.0, dtype=dtype, device="cuda")
    qkv = torch.cat([q, k, v], dim=1)
    qs, ks = qkv[:, :Hq * D], qkv[:, Hq * D:(Hq + Hk) * D]
    for a, b in zip(m.backward(dq, dk, qs, ks, gq, gk, pos), back):
        assert torch.equal(a, b)
    m.forward(qs, ks, gq, gk, pos, in_place=True)
    assert torch.equal(qs, want[0]) and torch.equal(ks, want[1]) and bool((qkv[:, (Hq + Hk) * D:] == 9.0).all())
    ones = torch.ones(D, dtype=dtype, device="cuda")
    a = [t.clone() for t in m.forward(q, k, ones, ones, pos)]
    assert all(torch.equal(x, y) for x, y in zip(a, m.forward(q, k, None, None, pos)))


def test_accumulated_gains_reruns_and_no_rows():
    N, Hq, Hk, D = 2000, 4, 2, 64
    q, k, gq, gk, dq, dk, pos = _data(N, Hq, Hk, D, torch.float32, seed=2)
    m = _make(N, Hq, Hk, D, D, torch.float32, True)
    _, _, a, b = (t.clone() for t in m.backward(dq, dk, q, k, gq, gk, pos))
    _, _, a2, b2 = m.backward(dq, dk, q, k, gq, gk, pos)
    assert torch.equal(a, a2) and torch.equal(b, b2)
    m.dgq.fill_(1.0)
    m.backward(dq, dk, q, k, gq, gk, pos, dw_accumulate=True)
    assert torch.allclose(m.dgq, a + 1.0, rtol=2.0 ** -22, atol=2.0 ** -22)      # one rounding more
    qo, ko = m.forward(q[:0], k[:0], gq, gk, pos[:0])
    assert qo.shape[0] == 0 and ko.shape[0] == 0
    _, _, a, b = m.backward(dq[:0], dk[:0], q[:0], k[:0], gq, gk, pos[:0])
    assert not a.any() and not b.any()


def test_position_outside_the_table():
    B = _B()
    N, Hq, Hk, D, R = 50, 2, 1, 64, 32
    q, k, gq, gk, dq, dk, pos = _data(N, Hq, Hk, D, torch.bfloat16, seed=3)
    m = _make(N, Hq, Hk, D, R, torch.bfloat16, False)
    good = m.forward(q, k, gq, gk, pos)[0].clone()
    pos[4], pos[30] = 0, T + 1
    qo = m.forward(q, k, gq, gk, pos)[0].view(N, Hq, D)
    rc, bits = B.ps_workspace_status(m.ws)
    assert rc == B.PS_ERR_DEVICE_DATA and bits == B.PS_DEV_BAD_LENGTH
    bad = torch.zeros(N, dtype=torch.bool)
    bad[[4, 30]] = True
    assert torch.isnan(qo[bad][..., :R]).all() and torch.equal(qo[bad][..., R:], good.view(N, Hq, D)[bad][..., R:])
    assert torch.equal(qo[~bad], good.view(N, Hq, D)[~bad])
    a = m.backward(dq, dk, q, k, gq, gk, pos)[0]
    assert torch.isnan(a[bad]).all() and torch.isfinite(a[~bad]).all()
    pos[4], pos[30] = 1, T
    m.forward(q, k, gq, gk, pos)
    m.check_status()                               # a call clears what the last one reported


@pytest.mark.parametrize("N", [1, 2047, 2048, 2049, 6000])
def test_the_last_row_outside_the_table(N):
    """Whoever looks at the positions: one block, or every one at its own rows."""
    B = _B()
    q, k, gq, gk, dq, dk, pos = _data(N, 4, 1, 64, torch.bfloat16, seed=N)
    m = _make(N, 4, 1, 64, 64, torch.bfloat16, False)
    for call in (lambda: m.forward(q, k, gq, gk, pos), lambda: m.backward(dq, dk, q, k, gq, gk, pos)):
        call()
        m.check_status()
        last = int(pos[-1])
        for wrong in (0, T + 1, -2 ** 31, 2 ** 31 - 1):
            pos[-1] = wrong
            out = call()[0]
            assert B.ps_workspace_status(m.ws) == (B.PS_ERR_DEVICE_DATA, B.PS_DEV_BAD_LENGTH)
            assert torch.isnan(out[-1]).all() and torch.isfinite(out[:-1]).all()
        pos[-1] = last
        assert torch.isfinite(call()[0]).all()
        m.check_status()


def test_nan_stays_in_its_head_and_streams():
    N, Hq, Hk, D = 40, 4, 2, 128
    q, k, gq, gk, dq, dk, pos = _data(N, Hq, Hk, D, torch.bfloat16, seed=4)
    m = _make(N, Hq, Hk, D, D, torch.bfloat16, False)
    good = m.forward(q, k, gq, gk, pos)[0].clone().view(N, Hq, D)
    q[11, 2 * D + 5] = float("nan")
    out = m.forward(q, k, gq, gk, pos)[0].view(N, Hq, D)
    ok = torch.ones(N, Hq, dtype=torch.bool)
    ok[11, 2] = False
    assert torch.isnan(out[11, 2]).all() and torch.equal(out[ok], good[ok])
    q[11, 2 * D + 5] = 1.0
    want = [t.clone() for t in m.backward(dq, dk, q, k, gq, gk, pos)]
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        m.backward(dq, dk, q, k, gq, gk, pos)
    torch.cuda.current_stream().wait_stream(side)
    with torch.cuda.graph(graph):
        m.backward(dq, dk, q, k, gq, gk, pos)
    m.dgq.zero_()
    graph.replay()
    torch.cuda.synchronize()
    for a, b in zip((m.dq, m.dk, m.dgq, m.dgk), want):
        assert torch.equal(a, b)


def test_refusals():
    B = _B()
    q, k, gq, gk, dq, dk, pos = _data(8, 2, 1, 64, torch.bfloat16)
    m = _make(8, 2, 1, 64, 64, torch.bfloat16, False)
    with pytest.raises(TypeError):
        m.forward(q.float(), k, gq, gk, pos)
    with pytest.raises(ValueError):
        m.forward(q[:, :64], k, gq, gk, pos)
    with pytest.raises(ValueError):
        m.forward(q, k[:4], gq, gk, pos)
    with pytest.raises(ValueError):
        m.forward(q, k, gq, gk, pos[:4])
    with pytest.raises(TypeError):
        m.forward(q, k, gq, gk, pos.long())
    with pytest.raises(ValueError):
        _make(8, 2, 1, 64, 64, torch.bfloat16, False).__class__(m.s, None)
    with pytest.raises(RuntimeError):
        _make(8, 2, 1, 64, 64, torch.bfloat16, False, train=False).backward(dq, dk, q, k, gq, gk, pos)
    with pytest.raises(B.PsppoError) as e:
        m.forward(torch.zeros(8, 130, dtype=torch.bfloat16, device="cuda")[:, :128], k, gq, gk, pos)
    assert e.value.status == B.PS_ERR_INVALID_ARG
