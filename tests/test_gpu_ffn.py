"""The gated feed-forward block against float64 (oracle.block), forward and backward.

Tolerances. u = 2^-8 is bf16's unit roundoff. Element by element, an output passes at most one rounding of its own (u of
it) and one of an operand of its last product (u of the sum of its terms' magnitudes, `reach`), the store's f16 (2^-11 of
the same) and f32 arithmetic (accumulation over K terms and the activation: under 2^-11 of it). Over a whole output of
many values and long sums the errors average: u / sqrt(3) = 2.3e-3 in 2-norm for each rounding, 3.2e-3 for both, so 4e-3
with the store's 2.8e-4. (A product that misses one 16-deep step of 1536 is off by 0.1.)"""
import numpy as np
import pytest
import torch

from oracle import block as ob

pytestmark = pytest.mark.gpu
WHOLE, U = 4e-3, 2.0 ** -8


def _B():
    from paper_2606_29758_gb300 import _binding as B
    return B


def _data(N, d, F, seed=0, wscale=None):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    w = wscale or 1.5 / d ** 0.5
    X, Wg, Wu, Wd = r(N, d), r(F, d) * w, r(F, d) * w, r(d, F) / F ** 0.5
    dY = r(N, d) * torch.exp(r(N, 1))
    if N > 2:
        dY[N // 2] = 0.0
    return [t.to(torch.bfloat16).cuda() for t in (X, Wg, Wu, Wd, dY)]


def _f64(*ts):
    return [t.float().cpu().numpy().astype(np.float64) for t in ts]


def _wanted(X, Wg, Wu, Wd, dY, act):
    """(value, reach, length of its last sum) of y, dx, dwg, dwu, dwd."""
    x, wg, wu, wd, dy = _f64(X, Wg, Wu, Wd, dY)
    q, slope = ob.activation(x @ wg.T, act)
    u, da, m = x @ wu.T, dy @ wd, np.abs
    a, dg, du = q * u, da * u * slope, da * q
    y, grads = ob.ffn_forward(x, wg, wu, wd, act), ob.ffn_backward(dy, x, wg, wu, wd, act)
    N, F = a.shape
    reach = (m(a) @ m(wd).T, m(dg) @ m(wg) + m(du) @ m(wu), m(dg).T @ m(x), m(du).T @ m(x), m(dy).T @ m(a))
    return list(zip((y, *grads), reach, (F, 2 * F, N, N, N)))


def _close(got, wanted, what):
    want, reach, terms = wanted
    got = got.float().cpu().numpy().astype(np.float64)
    assert got.shape == want.shape and np.isfinite(got).all(), what
    off = np.abs(got - want) / (U * np.abs(want) + (U + 2.0 ** -10) * reach + 1e-37)
    assert off.max() <= 1.0, (what, off.max())
    if want.size >= 4096 and terms >= 64:
        norm = np.linalg.norm(want)
        assert np.linalg.norm(got - want) <= WHOLE * norm, (what, np.linalg.norm(got - want) / norm)


def _make(N, d, F, act=0, train=True, dx=torch.bfloat16, dw=torch.bfloat16):
    from paper_2606_29758_gb300 import FFNShape, GatedFFN
    return GatedFFN(FFNShape(rows=N, d=d, F=F, act=act, train=train, dx_dtype=dx, dw_dtype=dw))


SIZES = [(1, 8, 8), (2, 8, 264), (3, 24, 40), (1, 1536, 520), (17, 72, 128), (64, 512, 1024), (127, 64, 72),
         (128, 128, 128), (129, 392, 1048), (257, 136, 1056), (300, 1032, 248), (571, 392, 1048), (1100, 264, 4104),
         (5, 2048, 4104), (20, 72, 8200), (33, 1032, 4104), (100, 1032, 4104), (128, 8, 2048)]


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("N,d,F", SIZES)
def test_forward_and_backward(N, d, F, act):
    X, Wg, Wu, Wd, dY = _data(N, d, F, seed=N + d + F)
    code = _B().PS_ACT_GELU if act == "gelu" else _B().PS_ACT_SILU
    want, *grads = _wanted(X, Wg, Wu, Wd, dY, act)
    serve = _make(N, d, F, code, train=False)
    y0 = serve.forward(X, Wg, Wu, Wd).clone()
    _close(y0, want, "y, serving")
    serve.check_status()
    for dt in (torch.bfloat16, torch.float32):
        m = _make(N, d, F, code, dx=dt, dw=dt)
        y = m.forward(X, Wg, Wu, Wd)
        _close(y, want, "y")
        for g, w, name in zip(m.backward(dY, X, Wg, Wu, Wd), grads, ("dx", "dwg", "dwu", "dwd")):
            assert g.dtype == dt
            _close(g, w, name)
        if N > 2:
            assert not m.dX[N // 2].any()      # a row without a gradient
        m.check_status()


@pytest.mark.parametrize("N,d,F", [(2, 4104, 72), (63, 1032, 136), (65, 520, 264), (512, 512, 256), (513, 520, 1032),
                                   (1025, 264, 520), (700, 1544, 2056), (16, 8, 16), (64, 8, 264), (10, 600, 2000)])
def test_more_rows_and_columns_around_the_tiles(N, d, F):
    """Tiles of 512 rows on CTA pairs, long and short K loops beside each other, few rows of dA."""
    X, Wg, Wu, Wd, dY = _data(N, d, F, seed=N + d + F)
    want, *grads = _wanted(X, Wg, Wu, Wd, dY, "silu")
    for dt in (torch.bfloat16, torch.float32):
        m = _make(N, d, F, dx=dt, dw=dt)
        _close(m.forward(X, Wg, Wu, Wd), want, "y")
        for g, w, name in zip(m.backward(dY, X, Wg, Wu, Wd), grads, ("dx", "dwg", "dwu", "dwd")):
            _close(g, w, name)
        m.check_status()


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("N,d,F", [(1, 96, 256), (2, 104, 304), (5, 8, 1048), (16, 136, 72), (33, 256, 512), (64, 128, 1048)])
def test_few_rows_lose_nothing_between_the_products(N, d, F, act):
    """Up to 64 rows of a narrow block A, dG and dU are two bf16 parts: 2^-17 of a value. What is left in f32 gradients is the kept P and Q, in
    f16: 2^-12 to 2^-11 of a value at most, 2.8e-4 in 2-norm where all are at their worst, and f32's own 2^-17 of long sums:
    under 4e-4, where one bf16 rounding gives 1.1e-3 to 2.3e-3. y keeps its own rounding alone, 2.3e-3 at most."""
    X, Wg, Wu, Wd, dY = _data(N, d, F, seed=3 * N + d + F)
    want, *grads = _wanted(X, Wg, Wu, Wd, dY, act)
    code = _B().PS_ACT_GELU if act == "gelu" else _B().PS_ACT_SILU
    m = _make(100, d, F, code, dx=torch.float32, dw=torch.float32)     # (buffers for more rows)
    off = lambda got, w: np.linalg.norm(_f64(got)[0] - w[0]) / np.linalg.norm(w[0])  # noqa: E731
    assert off(m.forward(X, Wg, Wu, Wd), want) <= 2.4e-3
    for g, w, name in zip(m.backward(dY, X, Wg, Wu, Wd), grads, ("dx", "dwg", "dwu", "dwd")):
        assert off(g, w) <= 4e-4, (name, off(g, w))
    m.check_status()


def test_backward_is_the_difference_of_the_forward():
    """The loss sum(Y dY) along random directions, in float64, against the library's f32 gradients. The gradient's 2-norm
    error is WHOLE of its norm, so along a unit direction it is at most that."""
    N, d, F = 40, 64, 136
    X, Wg, Wu, Wd, dY = _data(N, d, F, seed=5)
    m = _make(N, d, F, dx=torch.float32, dw=torch.float32)
    m.forward(X, Wg, Wu, Wd)
    grads = [g.double().cpu().numpy() for g in m.backward(dY, X, Wg, Wu, Wd)]
    arg, dy = _f64(X, Wg, Wu, Wd), _f64(dY)[0]
    r = np.random.default_rng(0)
    h = 1e-6
    for i, g in enumerate(grads):
        v = g / np.linalg.norm(g) + 0.3 * r.standard_normal(g.shape) / np.sqrt(g.size)
        hi, lo = list(arg), list(arg)
        hi[i], lo[i] = arg[i] + h * v, arg[i] - h * v
        num = np.sum(dy * (ob.ffn_forward(*hi, "silu") - ob.ffn_forward(*lo, "silu"))) / (2 * h)
        assert abs(num - np.sum(g * v)) <= 1.2 * WHOLE * np.linalg.norm(g)


@pytest.mark.parametrize("scale", [1e-5, 1e-3, 30.0])
def test_sizes_of_values(scale):
    """Gates and ups of 1e-5 (far below f16's normal numbers) or of hundreds: the store is relative to each slice."""
    N, d, F = 70, 128, 200
    X, Wg, Wu, Wd, dY = _data(N, d, F, seed=9, wscale=scale)
    want = _wanted(X, Wg, Wu, Wd, dY, "silu")
    m = _make(N, d, F)
    _close(m.forward(X, Wg, Wu, Wd), want[0], "y")
    for g, w in zip(m.backward(dY, X, Wg, Wu, Wd), want[1:]):
        _close(g, w, "gradient")


def test_values_beyond_f16_in_one_slice():
    """Ups of 1e6 and of 1 in the same slices: beyond f16's range, and 2^-20 below the slice's largest."""
    N, d, F = 64, 64, 96
    X, Wg, Wu, Wd, dY = _data(N, d, F, seed=3)
    Wu[::7] *= 1e6
    want = _wanted(X, Wg, Wu, Wd, dY, "silu")
    m = _make(N, d, F)
    _close(m.forward(X, Wg, Wu, Wd), want[0], "y")
    # (rows of dWg for ups of 1e6 and of 1: each is held to the sum of its own terms)
    for g, w in zip(m.backward(dY, X, Wg, Wu, Wd), want[1:]):
        _close(g, w, "gradient")


def test_nonfinite_rows_stay_in_their_rows():
    N, d, F = 150, 64, 104
    X, Wg, Wu, Wd, dY = _data(N, d, F, seed=4)
    X[7, 3] = float("nan")
    X[130, 5] = float("inf")
    dY[20, 1] = float("nan")
    m = _make(N, d, F)
    y = m.forward(X, Wg, Wu, Wd)
    ok = torch.ones(N, dtype=torch.bool)
    ok[[7, 130]] = False
    assert torch.isfinite(y[ok]).all() and not torch.isfinite(y[7]).any() and not torch.isfinite(y[130]).all()
    zero = torch.zeros_like(dY)
    _close(y[ok], _wanted(X[ok], Wg, Wu, Wd, zero[ok], "silu")[0], "y")
    dX = m.backward(dY, X, Wg, Wu, Wd)[0]
    ok[20] = False
    assert torch.isfinite(dX[ok]).all() and torch.isnan(dX[20]).any() and torch.isnan(dX[7]).any()
    _close(dX[ok], _wanted(X[ok], Wg, Wu, Wd, dY[ok], "silu")[1], "dx")


@pytest.mark.parametrize("N", [60, 150])
def test_an_infinite_up_leaves_its_neighbours(N):
    """One up overflows (row n, column f): the other columns of its slice keep that row's share of their gradients."""
    d, F, n, f, j = 64, 104, 33, 5, 7
    X, Wg, Wu, Wd, dY = _data(N, d, F, seed=11)
    Wg[:, j] = 0.0
    Wu[:, j] = 0.0
    Wu[f, j] = 1e20
    X[:, j] = 0.0
    X[n, j] = 1e30
    m = _make(N, d, F)
    y = m.forward(X, Wg, Wu, Wd)
    dX, dWg, dWu, dWd = m.backward(dY, X, Wg, Wu, Wd)
    rows, cols, dims = (torch.arange(k) != i for k, i in ((N, n), (F, f), (d, j)))
    Xs, Wus = X.clone(), Wu.clone()
    Wus[f, j] = 0.0                                # (finite; differs in column f alone)
    want = _wanted(Xs, Wg, Wus, Wd, dY, "silu")
    part = lambda w, a, b: (w[0][a][:, b], w[1][a][:, b], w[2])  # noqa: E731
    every = lambda k: torch.ones(k, dtype=torch.bool)  # noqa: E731
    assert not torch.isfinite(y[n]).any() and not torch.isfinite(dX[n]).all()
    _close(y[rows], part(want[0], rows.numpy(), every(d).numpy()), "y")
    # (dim j of dX has the weight that the finite copy lacks)
    _close(dX[rows][:, dims], part(want[1], rows.numpy(), dims.numpy()), "dx")
    _close(dWg[cols][:, dims], part(want[2], cols.numpy(), dims.numpy()), "dwg")
    _close(dWu[:, dims], part(want[3], every(F).numpy(), dims.numpy()), "dwu")
    _close(dWd[:, cols], part(want[4], every(d).numpy(), cols.numpy()), "dwd")


def test_pitches_reruns_and_accumulation():
    N, d, F = 200, 136, 264
    X, Wg, Wu, Wd, dY = _data(N, d, F, seed=6)
    m = _make(N, d, F, dx=torch.float32, dw=torch.float32)
    y = m.forward(X, Wg, Wu, Wd).clone()
    first = [g.clone() for g in m.backward(dY, X, Wg, Wu, Wd)]
    # rows inside wider buffers, weights as the halves of one
    wide = torch.full((N, d + 24), 7.0, dtype=torch.bfloat16, device="cuda")
    wide[:, 8:8 + d] = X
    wide_dy = torch.full((N, 2 * d), -3.0, dtype=torch.bfloat16, device="cuda")
    wide_dy[:, d:] = dY
    out = torch.full((N, d + 8), 5.0, dtype=torch.bfloat16, device="cuda")
    both = torch.cat([Wg, Wu])
    y2 = m.forward(wide[:, 8:8 + d], both[:F], both[F:], Wd, out=out[:, :d])
    assert torch.equal(y2, y) and bool((out[:, d:] == 5.0).all())
    again = m.backward(wide_dy[:, d:], wide[:, 8:8 + d], both[:F], both[F:], Wd)
    for a, b in zip(first, again):
        assert torch.equal(a, b)
    # added to what the buffers hold: the overwritten result plus the buffer, one rounding
    before = [torch.randn_like(g) for g in (m.dWg, m.dWu, m.dWd)]
    for g, b in zip((m.dWg, m.dWu, m.dWd), before):
        g.copy_(b)
    m.forward(X, Wg, Wu, Wd)
    for g, b, f in zip(m.backward(dY, X, Wg, Wu, Wd, dw_accumulate=True)[1:], before, first[1:]):
        assert torch.equal(g, b + f)
    # fewer rows than the holder was built for: the same rows
    y3 = m.forward(X[:129], Wg, Wu, Wd)
    assert y3.shape == (129, d)
    _close(y3, _wanted(X[:129], Wg, Wu, Wd, dY[:129], "silu")[0], "y")


def test_no_rows():
    d, F = 64, 72
    X, Wg, Wu, Wd, dY = _data(4, d, F)
    m = _make(4, d, F)
    assert m.forward(X[:0], Wg, Wu, Wd).shape == (0, d)
    m.dWg.fill_(3.0)
    dX, dWg, dWu, dWd = m.backward(dY[:0], X[:0], Wg, Wu, Wd)
    assert dX.shape == (0, d) and not dWg.any() and not dWu.any() and not dWd.any()
    m.check_status()


def test_another_stream_and_a_graph():
    N, d, F = 130, 72, 136
    X, Wg, Wu, Wd, dY = _data(N, d, F, seed=8)
    m = _make(N, d, F)
    y = m.forward(X, Wg, Wu, Wd).clone()
    want = [g.clone() for g in m.backward(dY, X, Wg, Wu, Wd)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        m.forward(X, Wg, Wu, Wd)
        m.backward(dY, X, Wg, Wu, Wd)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        m.forward(X, Wg, Wu, Wd)
        m.backward(dY, X, Wg, Wu, Wd)
    outs = (m.dX, m.dWg, m.dWu, m.dWd)
    for _ in range(2):
        m.Y.zero_()
        for g in outs:
            g.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(m.Y, y)
        for g, w in zip(outs, want):
            assert torch.equal(g, w)


def test_refusals():
    B = _B()
    N, d, F = 8, 64, 72
    X, Wg, Wu, Wd, dY = _data(N, d, F)
    m = _make(N, d, F)
    with pytest.raises(RuntimeError):
        m.backward(dY, X, Wg, Wu, Wd)              # no forward before it
    m.forward(X, Wg, Wu, Wd)
    m.backward(dY, X, Wg, Wu, Wd)
    with pytest.raises(RuntimeError):
        m.backward(dY, X, Wg, Wu, Wd)              # a second one
    with pytest.raises(RuntimeError):
        _make(N, d, F, train=False).backward(dY, X, Wg, Wu, Wd)
    with pytest.raises(ValueError):
        m.forward(torch.cat([X, X]), Wg, Wu, Wd)   # more rows than it was built for
    with pytest.raises(TypeError):
        m.forward(X.float(), Wg, Wu, Wd)
    with pytest.raises(ValueError):
        m.forward(X, Wg.t(), Wu, Wd)
    with pytest.raises(ValueError):
        m.forward(X.t().contiguous().t(), Wg, Wu, Wd)
    with pytest.raises(B.PsppoError) as e:         # a row pitch of 4 bytes more than whole 16-byte units
        m.forward(torch.zeros(N, d + 2, dtype=torch.bfloat16, device="cuda")[:, :d], Wg, Wu, Wd)
    assert e.value.status == B.PS_ERR_INVALID_ARG
    small = torch.zeros(B.ps_gated_ffn_store_size(N, F) - 1, dtype=torch.uint8, device="cuda")
    with pytest.raises(B.PsppoError) as e:
        B.ps_gated_ffn_fwd(N, d, F, B.PS_DTYPE_BF16, 0, X, Wg, Wu, Wd, m.Y, small, m.ws_fwd)
    assert e.value.status == B.PS_ERR_WORKSPACE
    m16 = _make(N, d, F)
    m16.forward(X, Wg, Wu, Wd)
    with pytest.raises(B.PsppoError) as e:         # a sum over calls in bf16
        m16.backward(dY, X, Wg, Wu, Wd, dw_accumulate=True)
    assert e.value.status == B.PS_ERR_UNSUPPORTED
