"""Dims of a head that are not rotated stand for themselves: an infinity in one of them leaves the others as the formula has
them (oracle.block, float64), whichever dims share its pair in the rotated part."""
import numpy as np
import pytest
import torch

from oracle import block as ob

pytestmark = pytest.mark.gpu
N, HQ, HK, D, T, EPS = 5, 2, 1, 96, 64, 1e-6
INF = float("inf")


def _data(dtype, R):
    g = torch.Generator().manual_seed(R)
    r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    t = [r(N, HQ * D), r(N, HK * D), 1 + 0.3 * r(D), 1 + 0.3 * r(D), r(N, HQ * D), r(N, HK * D)]
    pos = torch.randint(1, T + 1, (N,), generator=g, dtype=torch.int32)
    return [v.to(dtype).cuda() for v in t] + [pos.cuda()]


def _make(dtype, R, inter):
    from paper_2606_29758_gb300 import QKNormRope, QKShape, rope_table
    return QKNormRope(QKShape(N, HQ, HK, D, R, dtype, inter, EPS), rope_table(T, R, 1e4) if R else None)


def _formula(q, g, dq, pos, R, inter):
    heads = lambda t: t.double().cpu().numpy().reshape(N, HQ, D)  # noqa: E731
    a = ob.rope_angles(pos.cpu().numpy() - 1, R, 1e4) if R else np.zeros((N, 0))
    x, g = heads(q), g.double().cpu().numpy()
    with np.errstate(invalid="ignore", over="ignore"):
        return (ob.qk_forward(x, g, EPS, np.cos(a), np.sin(a), inter),
                *ob.qk_backward(heads(dq), x, g, EPS, np.cos(a), np.sin(a), inter))


def _kinds(v):
    """0 finite, 1 and -1 the infinities, 2 NaN."""
    v = v.double().cpu().numpy() if torch.is_tensor(v) else v
    return np.where(np.isnan(v), 2, np.where(np.isinf(v), np.sign(v), 0))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("R", [0, 48])
def test_infinite_values_gains_and_gradients(R, inter, dtype):
    m = _make(dtype, R, inter)
    for u in (48, 51, 59, 64, 95):
        q, k, gq, gk, dq, dk, pos = _data(dtype, R)
        good = m.forward(q, k, gq, gk, pos)[0].clone().view(N, HQ, D)
        others = torch.arange(D, device="cuda") != u
        # a gain: that dim of every head
        g = gq.clone()
        g[u] = INF
        y = m.forward(q, k, g, gk, pos)[0].view(N, HQ, D)
        assert torch.isinf(y[..., u]).all() and torch.equal(y[..., others], good[..., others])
        # a value: r = 0, so 0 inf at the value itself, 0 elsewhere in its head, and the other heads as they were
        x = q.clone()
        x.view(N, HQ, D)[2, 1, u] = INF
        y = m.forward(x, k, gq, gk, pos)[0].view(N, HQ, D)
        want = _formula(x, gq, dq, pos, R, inter)[0]
        assert np.array_equal(_kinds(y), _kinds(want)) and not y[2, 1, others].any()
        keep = torch.ones(N, HQ, dtype=torch.bool, device="cuda")
        keep[2, 1] = False
        assert torch.equal(y[keep], good[keep])
        # a gradient: the gains of the other dims get theirs as ever
        dy = dq.clone()
        dy.view(N, HQ, D)[2, 1, u] = INF
        near = [t.clone() for t in m.backward(dq, dk, q, k, gq, gk, pos)]
        dx, _, dg, dgk = m.backward(dy, dk, q, k, gq, gk, pos)
        _, wdx, wdg = _formula(q, gq, dy, pos, R, inter)
        assert np.array_equal(_kinds(dg), _kinds(wdg)) and torch.equal(dg[others], near[2][others])
        assert torch.equal(dgk, near[3])
        off = _kinds(dx.view(N, HQ, D)) != _kinds(wdx)
        off[2, 1, u] = False                        # (inf less inf x r^2 x: either is its formula's, by rounding)
        assert not off.any()
