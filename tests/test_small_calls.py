"""The module of small calls (csrc/small_calls.cpp): what is not exactly in order is left to the holder's ordinary way, which
says what is wrong; what is in order gives the bits that the ordinary way gives."""
import pytest
import torch

BF = torch.bfloat16


@pytest.fixture(scope="module")
def B():
    from paper_2606_29758_gb300 import _binding, _build
    _build.build()
    return _binding


def test_left_to_the_ordinary_way(B):
    """CPU tensors, other objects, wrong counts, plans of another kind: None, and no error left behind."""
    c = B.calls()
    x, t = torch.zeros(3, 8), torch.zeros(3, dtype=torch.int32)
    qk = c.qk_plan(4, 1, 1, 16, 16, 1, 0, 8, 1e-6, 0, 0, 0, 0, 0, 0, 0, 0, 0)
    ffn = c.ffn_plan(4, 8, 8, 0, 0, 0, *[0] * 11)
    for call in (lambda: c.dropout_rows(x, t, t, 1, 1, None, 0, None, 0.1, 2), lambda: c.dropout_rows(1, 2),
                 lambda: c.dropout_rows(*[None] * 10), lambda: c.qk_fwd(qk, x, x, None, None, t, 1, False),
                 lambda: c.qk_fwd(ffn, x, x, None, None, t, 1, False), lambda: c.qk_fwd(), lambda: c.qk_fwd(*[7] * 8),
                 lambda: c.qk_bwd(qk, x, x, x, x, None, None, t, 1, False), lambda: c.qk_bwd(None, *[x] * 9),
                 lambda: c.ffn_fwd(ffn, x, x, x, x, None), lambda: c.ffn_fwd(qk, *[x] * 5),
                 lambda: c.ffn_bwd(ffn, *[x] * 5, False), lambda: c.ffn_bwd()):
        assert call() is None
    with pytest.raises(TypeError):
        c.qk_plan(1, 2)
    with pytest.raises(TypeError):
        c.ffn_plan("x")


def _both(holder, names, call):
    """The call's outputs, by the module and by the ordinary way."""
    first = [None if o is None else o.clone() for o in call()]
    kept = {n: getattr(holder, n) for n in names}
    try:
        for n in names:
            setattr(holder, n, lambda *a: None)
        second = [None if o is None else o.clone() for o in call()]
    finally:
        for n, f in kept.items():
            setattr(holder, n, f)
    for a, b in zip(first, second):
        assert (a is None and b is None) or torch.equal(a, b)


@pytest.mark.gpu
@pytest.mark.parametrize("N", [0, 1, 5, 300])
def test_the_same_bits(B, N):
    from paper_2606_29758_gb300 import FFNShape, GatedFFN, QKNormRope, QKShape, RowDropout, rope_table
    g = torch.Generator(device="cuda").manual_seed(N)
    r = lambda *s, dt=BF: torch.randn(*s, device="cuda", generator=g).to(dt)  # noqa: E731
    traj = torch.arange(N, device="cuda", dtype=torch.int32) // 7
    pos = torch.arange(N, device="cuda", dtype=torch.int32) % 7 + 1
    for dt in (BF, torch.float32):
        drop, x, res = RowDropout(0.3, site=5), r(N, 104, dt=dt)[:, :96], r(N, 96, dt=dt)
        out = torch.empty(N, 128, dtype=dt, device="cuda")[:, :96]
        for kw in (dict(), dict(res=res), dict(res=res, out=out), dict(traj_base=1 << 31)):
            _both(drop, ["_fast"], lambda: [drop.forward(x, traj, pos, -3, 2 ** 32 - 1, **kw)])
        _both(drop, ["_fast"], lambda: [drop.backward(x, traj, pos, 2 ** 70 + 1, 0)])
        for s in (QKShape(400, 3, 1, 48, 32, dt), QKShape(400, 2, 2, 64, 0, dt, interleaved=True), QKShape(400, 4, 0, 16, 16, dt)):
            m = QKNormRope(s, rope_table(16, s.R) if s.R else None)
            qkv = r(N, (s.Hq + s.Hk) * s.D, dt=dt)
            q, k = qkv[:, :s.Hq * s.D], qkv[:, s.Hq * s.D:]
            gain, p = r(s.D, dt=dt), pos if s.R else None
            names = ["_fast_fwd", "_fast_bwd"]
            _both(m, names, lambda: m.forward(q, k, gain, None, p))
            _both(m, names, lambda: m.forward(q.clone(), k.clone(), None, gain, p, 1, True))
            _both(m, names, lambda: m.backward(q, k, q, k, gain, gain, p))
            m.check_status()
    for train in (False, True):
        m = GatedFFN(FFNShape(400, 64, 136, train=train))
        X, Wg, Wu, Wd = r(N, 72)[:, :64], r(136, 64), r(136, 64), r(64, 136)

        def step():
            y = m.forward(X, Wg, Wu, Wd)
            return [y, *(m.backward(X, X, Wg, Wu, Wd) if train else [])]
        _both(m, ["_fast_fwd", "_fast_bwd"], step)
        out = torch.empty(N, 80, dtype=BF, device="cuda")[:, :64]
        _both(m, ["_fast_fwd", "_fast_bwd"], lambda: [m.forward(X, Wg, Wu, Wd, out=out)])
        m.check_status()


@pytest.mark.gpu
def test_refusals_come_from_the_ordinary_way(B):
    from paper_2606_29758_gb300 import FFNShape, GatedFFN, QKNormRope, QKShape, RowDropout, rope_table
    z = lambda *s, dt=BF: torch.zeros(*s, dtype=dt, device="cuda")  # noqa: E731
    pos = torch.ones(4, dtype=torch.int32, device="cuda")
    drop, m, f = RowDropout(0.5), QKNormRope(QKShape(4, 1, 1, 32, 32), rope_table(8, 32)), GatedFFN(FFNShape(4, 16, 24))
    q = z(4, 32)
    for bad, error in ((lambda: drop.forward(z(4, 8).cpu(), pos, pos, 1, 1), ValueError),
                       (lambda: drop.forward(z(4, 8), pos, pos, 1, 1, res=z(4, 9)), ValueError),
                       (lambda: drop.forward(z(4, 8), pos.long(), pos, 1, 1), TypeError),
                       (lambda: drop.forward(z(8, 4).t(), pos, pos, 1, 1), ValueError),
                       (lambda: drop.forward(z(4, 8), pos, pos, 1, 1, out=z(4, 8, dt=torch.float32)), TypeError),
                       (lambda: drop.forward(z(4, 8), pos, pos, 1, 2 ** 32), B.PsppoError),
                       (lambda: m.forward(z(5, 32), z(5, 32), None, None, pos), ValueError),
                       (lambda: m.forward(q, z(4, 16), None, None, pos), ValueError),
                       (lambda: m.forward(q, q, z(31), None, pos), ValueError),
                       (lambda: m.forward(q, q, None, None, pos[:3]), ValueError),
                       (lambda: m.forward(z(4, 33)[:, 1:], q, None, None, pos), B.PsppoError),
                       (lambda: m.backward(q.float(), q, q, q, None, None, pos), TypeError),
                       (lambda: f.forward(z(5, 16), z(24, 16), z(24, 16), z(16, 24)), ValueError),
                       (lambda: f.forward(z(4, 16), z(16, 24).t(), z(24, 16), z(16, 24)), ValueError),
                       (lambda: f.forward(z(4, 16), z(24, 16).float(), z(24, 16), z(16, 24)), TypeError),
                       (lambda: f.backward(z(4, 16), z(4, 16), z(24, 16), z(24, 16), z(16, 24)), RuntimeError)):
        with pytest.raises(error):
            bad()
