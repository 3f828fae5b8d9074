"""Weights of attention over a bf16 cache are f32: two of nearly the same size, whose difference a smaller type would lose."""
import numpy as np
import pytest
import torch

from oracle import block as ob
from test_gpu_paged import BF, _att

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("page", [16, 4])       # (chunks by the copy engine, and by lanes)
@pytest.mark.parametrize("Hq", [8, 16])
def test_a_difference_of_two_weights(page, Hq):
    """Three keys with scores 0, b and b - 2^-13 and values 0, 1 and -1. The scores are exact. A weight's exponent (|x| < 1.8, its
    factor log2 e and the product rounded: 2^-24 and 2^-24 at most) and ex2 (2^-22 of itself) leave 1.4 * 2^-22 of each weight; the
    sums of three products some 2^-23 of the larger: under 2^-20 of the two. And the output's rounding, 2^-8 of the difference
    (2^-14 of the weights, so 2^-22 of them)."""
    from paper_2606_29758_gb300 import CacheShape, PagedCache
    n, D = 60, 16
    c = PagedCache(CacheShape(n, n, page, 1, D, page))
    c.table.copy_(torch.arange(n, dtype=torch.int32).view(n, 1))
    c.lengths.fill_(3)
    c.k.zero_()
    c.v.zero_()
    base = (-0.05 - 0.01 * torch.arange(n)).to(BF).cuda()
    c.k[0, :, 0, 1:3, 0] = base[:, None]
    c.k[0, :, 0, 2, 1] = -1.0
    c.v[0, :, 0, 1], c.v[0, :, 0, 2] = 1.0, -1.0
    q = torch.zeros(n, Hq, D, dtype=BF)
    q[:, :, 0], q[:, :, 1] = 1.0 + torch.arange(Hq) / 16, 2.0 ** -13
    q = q.cuda()
    o = _att(n, Hq, 1, D, BF, scale=1.0).forward(q.view(n, -1), c).view(n, Hq, D).double().cpu().numpy()
    for b in range(n):
        k, v = (t[0, b, 0, :3].double().cpu().numpy()[:, None] for t in (c.k, c.v))
        qb = q[b].double().cpu().numpy()
        want, lse = ob.attend(qb, k, v, 1.0)
        both = np.exp(qb @ k[1:, 0].T - lse[:, None]).sum(axis=1)[:, None]
        assert (np.abs(o[b] - want) <= 2.0 ** -20 * both + 2.0 ** -8 * np.abs(want)).all(), b
