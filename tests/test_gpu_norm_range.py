"""Residual norms at the ends of their ranges, against float64 (oracle.block): eps of 0 with small rows, rows that are not there, gates of
0 with scales that f32 rounds, infinities in the stream and in a gate.

Tolerances: those of test_gpu_residual_norm.py hold, whose sums and roots are relative to the rows themselves. A square below f32's
smallest normal number is off by 2^-150; at a mean square of 1e-38 that is 2^-23 of it at most."""
import numpy as np
import pytest
import torch

from oracle import block as ob
from test_gpu_residual_norm import _case, _check, _n, _op

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def _rounded(h):
    """The f32 nearest to h, rounded to bf16."""
    return torch.from_numpy(h).float().to(BF).cuda()


@pytest.mark.parametrize("d", [40, 256, 300, 771, 3584, 16384])
def test_small_rows_without_an_epsilon(d):
    """bf16 rows of 1e-12 to 1e-19 of teams below a warp, of one and of several: h is the f32 nearest to the sum, rounded, while the
    squares that count are exact in f32 (down to 1e-18); at 1e-19 it is near the sum."""
    g = torch.Generator().manual_seed(d)
    sizes = torch.tensor([1e-12, 1e-16, 1e-18, 3e-19, 1e-19, 1.0])[:, None]
    N = len(sizes)
    x, gy = torch.randn(N, d, generator=g).to(BF), (1 + 0.3 * torch.randn(d, generator=g)).to(BF)
    y = (sizes.double() * torch.randn(N, d, generator=g).double()).to(BF)
    for a, b in ((1.0, 1.0), (0.7, 1.1)):
        h, o = _op(N, d, BF, eps=0.0, res_scale=a, branch_scale=b, train=False).forward(x.cuda(), y.cuda(), gy.cuda())
        want, norm = ob.norm_forward(_n(x), _n(y), _n(gy), np.ones(d), np.ones(N), a, b, 0.0, True)
        exact = [0, 1, 2, 5]
        assert torch.equal(h[exact], _rounded(want[exact])), (a, b)
        size = np.abs(a * _n(x)) + np.abs(want - a * _n(x))
        assert (np.abs(_n(h) - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -18 * size).all()
        assert (np.abs(_n(o) - norm) <= 2.0 ** -8 * np.abs(norm) + 2.0 ** -16 * (np.abs(norm) + size)).all()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("N,d", [(1, 8), (3, 64), (1, 128), (3, 128), (5, 128), (1, 256), (5, 256), (3, 771), (2, 3584)])
@pytest.mark.parametrize("size", [1.0, 1e-15])
def test_both_ways_without_an_epsilon(size, N, d, dtype):
    """Rows that no row lies beside in their warp, aligned and not: nothing of a row that is not there counts."""
    for pitch, shift in ((None, 0), (d + 3, 1)):
        c = _case(N, d, dtype, seed=5, pitch=pitch, shift=shift)
        g = torch.Generator().manual_seed(d)
        c["x"].copy_(torch.randn(N, d, generator=g).to(dtype))
        c["y"].copy_((size * torch.randn(N, d, generator=g)).to(dtype))
        c["gate"] = 0.5 + torch.rand(N, generator=g).cuda()
        for post in (True, False):
            m = _op(N, d, dtype, post=post, eps=0.0, res_scale=0.75, branch_scale=0.5)
            h, o = m.forward(c["x"], c["y"], c["gy"], c["go"], gate=c["gate"])
            got = m.backward(c["do"], c["dh"], h, c["y"], c["gy"], c["go"], gate=c["gate"])
            _check(c, (h, o, *got), dtype, post, True, 0.75, 0.5, 0.0, N)
        m, one = _op(N, d, dtype, eps=0.0), dict(c, gate=None)
        one["x"].copy_((size * torch.randn(N, d, generator=g)).to(dtype))
        h, o = m.forward(one["x"], go=c["go"])
        _check(one, (h, o, *m.backward(c["do"], c["dh"], h, go=c["go"])), dtype, False, True, 1.0, 1.0, 0.0, N, branch=False)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d", [40, 771, 3584])
@pytest.mark.parametrize("post", [True, False])
@pytest.mark.parametrize("a", [1.0, 0.75, 2.0])
def test_infinities_of_the_stream_and_of_a_gate(a, post, d, dtype):
    """An infinity of x, one that a scale makes, a gate of 0 beside one: h as the sum has it, o 0 beside an infinity and NaN in its
    place. An infinite gate leaves nothing finite."""
    N, g = 5, torch.Generator().manual_seed(d)
    x, y = (torch.randn(N, d, generator=g).to(dtype) for _ in range(2))
    gate = torch.ones(N)
    x[0, 3], x[0, d - 1] = float("inf"), float("-inf")
    x[1, 5] = torch.finfo(dtype).max          # (2: beyond the range)
    gate[2] = float("inf")
    x[3, 0], gate[3] = float("inf"), 0.0
    y = torch.where(y == 0, 1, y)
    h, o = _op(N, d, dtype, post=post, res_scale=a, train=False).forward(x.cuda(), y.cuda(), gate=gate.cuda())
    with np.errstate(invalid="ignore"):
        want, norm = ob.norm_forward(_n(x), _n(y), np.ones(d), np.ones(d), _n(gate), a, 1.0, 1e-6, post)
    want = torch.from_numpy(want).float().to(dtype)
    assert not torch.isfinite(h[2]).any() and o[2].isnan().all()
    want[2] = h[2] = 0.0
    fine = torch.isfinite(want)
    assert torch.equal(h.cpu()[~fine], want[~fine])
    off = (h.cpu()[fine].double() - want[fine].double()).abs()      # (a rounding each, and some e of terms below 16)
    assert (off <= 2.0 ** -7 * want[fine].double().abs() + 2.0 ** -15).all()
    for i in (0, 3):
        place = torch.isinf(want[i])
        assert o.cpu()[i][place].isnan().all() and not o.cpu()[i][~place].any(), i
    assert torch.isfinite(o[4]).all()


@pytest.mark.parametrize("a", [0.53, 0.65, 1.05, 1.3, 0.7, 1.0])
def test_shut_gates_and_scales_that_f32_rounds(a):
    """bf16 after the branch's norm: a x alone is rounded like the sum, from the scale as it was given."""
    for d in (64, 256, 1024):
        powers = 2.0 ** (torch.arange(d // 64) - d // 128)
        x = (torch.arange(128, 256).repeat(d // 64) * powers.repeat_interleave(128)).to(BF).view(2, d).repeat(2, 1)
        g = torch.Generator().manual_seed(d)
        y, gate = torch.randn(4, d, generator=g).to(BF), torch.tensor([0.0, 0.0, 1.0, 0.5])
        h, _ = _op(4, d, BF, res_scale=a, train=False).forward(x.cuda(), y.cuda(), gate=gate.cuda())
        want, _ = ob.norm_forward(_n(x), _n(y), np.ones(d), np.ones(d), _n(gate), a, 1.0, 1e-6, True)
        assert torch.equal(h, _rounded(want)), d


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("post", [True, False])
def test_shut_gates_and_gains_that_are_not_finite(post, dtype):
    """The branch is left out whatever its gain holds."""
    N, d, g = 6, 300, torch.Generator().manual_seed(0)
    x, y = (torch.randn(N, d, generator=g).to(dtype).cuda() for _ in range(2))
    gy, gate = torch.ones(d, dtype=dtype, device="cuda"), (torch.arange(N) % 2).float().cuda()
    gy[5], gy[77], gy[299] = float("inf"), float("nan"), float("-inf")
    h, o = _op(N, d, dtype, post=post, train=False).forward(x, y, gy, gate=gate)
    assert torch.equal(h[::2], x[::2]) and torch.isfinite(o[::2]).all()
    assert not torch.isfinite(h[1::2, [5, 77, 299]]).any()
