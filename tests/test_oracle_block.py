"""Pins of the block oracle: its gradients against central differences of its forwards, its activations against
their definitions, the rotation against complex multiplication, its generator against published vectors."""
import numpy as np
import pytest
from scipy.stats import norm

from oracle import block as ob


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_activations(act):
    g = np.linspace(-30.0, 30.0, 601)
    s, slope = ob.activation(g, act)
    want = g / (1.0 + np.exp(-g)) if act == "silu" else g * norm.cdf(g)
    assert np.allclose(s, want, rtol=1e-13, atol=0)
    h = 1e-5
    num = (ob.activation(g + h, act)[0] - ob.activation(g - h, act)[0]) / (2 * h)
    assert np.abs(slope - num).max() < 1e-8
    assert ob.activation(np.array([-2000.0]), act)[0][0] == 0.0


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_ffn_gradients_are_differences_of_the_forward(act):
    r = np.random.default_rng(1)
    N, d, F = 5, 4, 6
    arg = [r.standard_normal(s) for s in ((N, d), (F, d), (F, d), (d, F))]
    dY = r.standard_normal((N, d))
    grads = ob.ffn_backward(dY, *arg, act)
    h = 1e-6
    for i, g in enumerate(grads):
        num = np.zeros_like(g)
        for at in np.ndindex(g.shape):
            hi, lo = [a.copy() for a in arg], [a.copy() for a in arg]
            hi[i][at] += h
            lo[i][at] -= h
            num[at] = np.sum(dY * (ob.ffn_forward(*hi, act) - ob.ffn_forward(*lo, act))) / (2 * h)
        assert np.abs(g - num).max() < 1e-7, i


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("R", [4, 8, 0])
def test_qk_gradients_are_differences_of_the_forward(inter, R):
    r = np.random.default_rng(2)
    N, H, D = 3, 2, 8
    x, dy, gain = r.standard_normal((N, H, D)), r.standard_normal((N, H, D)), r.standard_normal(D)
    a = ob.rope_angles([0, 7, 100], R, 1e4) if R else np.zeros((N, 0))
    cos, sin, eps = np.cos(a), np.sin(a), 1e-3
    dx, dgain = ob.qk_backward(dy, x, gain, eps, cos, sin, inter)
    f = lambda v, g: np.sum(dy * ob.qk_forward(v, g, eps, cos, sin, inter))  # noqa: E731
    h = 1e-6
    for at in np.ndindex(x.shape):
        hi, lo = x.copy(), x.copy()
        hi[at] += h
        lo[at] -= h
        assert abs(dx[at] - (f(hi, gain) - f(lo, gain)) / (2 * h)) < 1e-7
    for j in range(D):
        hi, lo = gain.copy(), gain.copy()
        hi[j] += h
        lo[j] -= h
        assert abs(dgain[j] - (f(x, hi) - f(x, lo)) / (2 * h)) < 1e-7


def test_turn_is_a_complex_product():
    r = np.random.default_rng(3)
    x = r.standard_normal((4, 3, 12))
    a = ob.rope_angles([0, 1, 5, 1000], 8, 1e4)
    z = np.exp(1j * a)[:, None]
    half = ob.turn(x, np.cos(a), np.sin(a), False)
    v = (x[..., :4] + 1j * x[..., 4:8]) * z
    assert np.allclose(half[..., :4], v.real) and np.allclose(half[..., 4:8], v.imag)
    even = ob.turn(x, np.cos(a), np.sin(a), True)
    v = (x[..., 0:8:2] + 1j * x[..., 1:8:2]) * z
    assert np.allclose(even[..., 0:8:2], v.real) and np.allclose(even[..., 1:8:2], v.imag)
    assert np.array_equal(half[..., 8:], x[..., 8:]) and np.array_equal(even[..., 8:], x[..., 8:])
    # position 0 turns nothing, and the score of a turned pair depends on the distance alone
    assert np.allclose(half[0], x[0])
    q, k = r.standard_normal((1, 1, 8)), r.standard_normal((1, 1, 8))
    at = lambda v, p: ob.turn(v, np.cos(ob.rope_angles([p], 8, 1e4)), np.sin(ob.rope_angles([p], 8, 1e4)), False)  # noqa: E731
    assert np.isclose(np.sum(at(q, 9) * at(k, 4)), np.sum(at(q, 105) * at(k, 100)))


def test_philox4x32_vectors():
    """The known-answer vectors published with the generator."""
    f = 0xFFFFFFFF
    for c, k, want in [((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
                       ((f, f, f, f), (f, f), (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
                       ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0),
                        (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1))]:
        assert tuple(int(x) for x in ob.philox4x32_10(np.array(c, dtype=np.uint64), k)) == want


def test_keep_mask_rates_and_keys():
    traj, pos = np.repeat(np.arange(40), 50), np.tile(np.arange(1, 51), 40)
    d, p = 100, 0.3
    m = ob.keep_mask(traj, pos, d, p, 77, 5, 2)
    n = m.size
    q = 1.0 - ob.keep_cut(p) / 65536.0
    assert abs(m.mean() - q) < 5 * np.sqrt(q * (1 - q) / n)
    # neighbouring columns, rows and completions are uncorrelated (5 sigma of n products)
    z = (m - q) / np.sqrt(q * (1 - q))
    for a, b in ((z[:, :-1], z[:, 1:]), (z[:-1], z[1:]), (z[:-50], z[50:])):
        assert abs((a * b).mean()) < 5 / np.sqrt(a.size)
    # a shard's rows, and a prefix of the rows, keep their masks; another seed, step or site changes them
    assert np.array_equal(ob.keep_mask(traj[500:] - 10, pos[500:], d, p, 77, 5, 2, traj_base=10), m[500:])
    assert np.array_equal(ob.keep_mask(traj[:7], pos[:7], 96, p, 77, 5, 2), m[:7, :96])
    for other in (dict(seed=78, step=5, site=2), dict(seed=77 + (1 << 40), step=5, site=2),
                  dict(seed=77, step=6, site=2), dict(seed=77, step=5, site=3)):
        assert 0.2 < (ob.keep_mask(traj, pos, d, p, **other) != m).mean() < 0.6
