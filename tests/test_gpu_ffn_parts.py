"""The two precisions between the feed-forward block's products, on both sides of their edges (64 rows, F = 2048).

One bf16 rounding, to 2^-8 at most, is off by 2^-7 / sqrt(12) over the significand in [1, 2): between 1.13e-3 and 2.26e-3 of
a value in root mean square, and so are f32 gradients, each a sum of independently rounded terms (with the store's f16, 2.8e-4
at most, in quadrature: under 2.3e-3). Two parts leave the f16 and f32 alone: 4e-4."""
import numpy as np
import pytest
import torch

from test_gpu_ffn import _data, _f64, _make, _wanted

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("N,d,F", [(64, 96, 304), (65, 96, 304), (40, 200, 2048), (40, 200, 2056), (64, 72, 2048),
                                   (65, 72, 2048)])
def test_levels_of_error(N, d, F):
    X, Wg, Wu, Wd, dY = _data(N, d, F, seed=N + F)
    want = _wanted(X, Wg, Wu, Wd, dY, "silu")
    m = _make(N, d, F, dx=torch.float32, dw=torch.float32)
    off = lambda got, w: np.linalg.norm(_f64(got)[0] - w[0]) / np.linalg.norm(w[0])  # noqa: E731
    y = off(m.forward(X, Wg, Wu, Wd), want[0])
    grads = [off(g, w) for g, w in zip(m.backward(dY, X, Wg, Wu, Wd), want[1:])]
    if N <= 64 and F <= 2048:
        assert y <= 2.3e-3 and max(grads) <= 4e-4, (y, grads)
    else:
        assert y <= 2.3e-3 * 2 ** 0.5 and 1.1e-3 <= min(grads) and max(grads) <= 2.3e-3, (y, grads)


def test_a_row_in_calls_of_64_and_65_rows():
    """The same rows, within the rounding that the larger call has and the smaller one has not."""
    N, d, F = 65, 96, 304
    X, Wg, Wu, Wd, dY = _data(N, d, F, seed=1)
    m = _make(N, d, F, dx=torch.float32, dw=torch.float32)
    out = []
    for n in (64, 65):
        y = m.forward(X[:n], Wg, Wu, Wd)[:64].double()
        out.append((y, m.backward(dY[:n], X[:n], Wg, Wu, Wd)[0][:64].double()))
    for a, b, own in zip(*out, (2.3e-3, 0.0)):      # (y: its own rounding in each call)
        assert 0 < (a - b).norm() <= (2.3e-3 ** 2 + 2 * own ** 2) ** 0.5 * 1.05 * a.norm()
