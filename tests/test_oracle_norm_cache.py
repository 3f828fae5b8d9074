"""The oracle's residual norms and attention against differences and plain formulas, in float64."""
import numpy as np
import pytest

from oracle import block as ob


@pytest.mark.parametrize("post", [True, False])
@pytest.mark.parametrize("branch", [True, False])
def test_norm_gradients_are_differences_of_the_forward(branch, post):
    """Central differences of step t: the third derivative's t^2 / 6 and the rounding 2^-53 L / t, both below 1e-7 of the largest
    gradient at t = 1e-5."""
    rng = np.random.default_rng(3)
    N, d, a, b, eps, t = 3, 7, 0.7, 1.3, 1e-3, 1e-5
    p = dict(x=rng.standard_normal((N, d)), y=rng.standard_normal((N, d)) if branch else None, gy=rng.standard_normal(d),
             go=rng.standard_normal(d), gate=rng.standard_normal(N))
    do, dh = rng.standard_normal((2, N, d))

    def loss(p):
        h, o = ob.norm_forward(**p, a=a, b=b, eps=eps, post=post)
        return (dh * h).sum() + (do * o).sum()
    h, _ = ob.norm_forward(**p, a=a, b=b, eps=eps, post=post)
    dx, dy, dgy, dgo, dgate = ob.norm_backward(do, dh, h, p["y"], p["gy"], p["go"], p["gate"], a if branch else 1.0, b, eps, post)
    for name, got in dict(x=dx, y=dy, gy=dgy, go=dgo, gate=dgate).items():
        if got is None:
            continue
        want = np.zeros_like(got)
        for i in np.ndindex(got.shape):
            for sign in (1, -1):
                q = {k: None if v is None else v.copy() for k, v in p.items()}
                q[name][i] += sign * t
                want[i] += sign * loss(q) / (2 * t)
        assert np.abs(got - want).max() <= 1e-7 * max(1, np.abs(want).max()), name


def test_a_gate_of_zero():
    """The branch is left out whatever it holds; the gate's own gradient is that of the branch as it is."""
    rng = np.random.default_rng(4)
    x, y, do = rng.standard_normal((3, 2, 5))
    one = np.ones(5)
    gate = np.array([0.0, 2.0])
    h, _ = ob.norm_forward(x, np.array([[np.inf, np.nan, 0, 1, 2], y[1]]), one, one, gate, 0.5, 1.0, 1e-6, True)
    assert np.array_equal(h[0], 0.5 * x[0]) and np.isfinite(h).all()
    dx, dy, dgy, dgo, dgate = ob.norm_backward(do, 0.0, h, y, one, one, gate, 0.5, 1.0, 1e-6, True)
    assert (dy[0] == 0).all() and dgate[0] != 0


def test_attend():
    """Against one head at a time; a row of equal keys is the values' mean; no keys give zeros and -inf."""
    rng = np.random.default_rng(5)
    q, k, v = rng.standard_normal((4, 6)), rng.standard_normal((9, 2, 6)), rng.standard_normal((9, 2, 6))
    o, lse = ob.attend(q, k, v, 0.3)
    for h in range(4):
        s = 0.3 * k[:, h // 2] @ q[h]
        w = np.exp(s)
        assert np.allclose(o[h], w @ v[:, h // 2] / w.sum(), rtol=1e-13, atol=1e-13) and np.isclose(lse[h], np.log(w.sum()), rtol=1e-13)
    o, lse = ob.attend(q, np.zeros_like(k), v, 0.3)
    assert np.allclose(o, v.mean(axis=0)[[0, 0, 1, 1]], rtol=1e-13, atol=1e-15) and np.allclose(lse, np.log(9))
    o, lse = ob.attend(q, k[:0], v[:0], 0.3)
    assert (o == 0).all() and (lse == -np.inf).all()
    o, lse = ob.attend(200 * q, k, v, 1.0)
    assert np.isfinite(o).all() and np.isfinite(lse).all()
