"""Dropout of a branch's rows added to the residual rows: masks equal to the oracle's bit for bit, values to one
rounding (2^-8 of the value in bf16; in f32 2^-22 of |x| scale + |res|, two roundings)."""
import numpy as np
import pytest
import torch

from oracle import block as ob

pytestmark = pytest.mark.gpu
SEED, STEP, SITE = 0x123456789ABCDEF0, 41, 9


def _B():
    from paper_2606_29758_gb300 import _binding as B
    return B


def _rows(N, seed=0):
    g = np.random.default_rng(seed)
    n = g.integers(1, 60, size=N)
    traj = np.repeat(np.arange(N), n)[:N].astype(np.int32)
    pos = np.concatenate([np.arange(1, m + 1) for m in n])[:N].astype(np.int32)
    return torch.from_numpy(traj).cuda(), torch.from_numpy(pos).cuda()


def _data(N, d, dtype, seed=0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(N, d, generator=g)
    x = torch.where(x.abs() < 0.01, torch.ones(()), x)          # nothing kept looks dropped
    return x.to(dtype).cuda(), torch.randn(N, d, generator=g).to(dtype).cuda()


def _check(y, x, res, keep, p, dtype):
    X = x.double().cpu().numpy()
    base = np.zeros_like(X) if res is None else res.double().cpu().numpy()
    scale = 65536.0 / (65536 - ob.keep_cut(p))
    want = base + np.where(keep, X, 0.0) * scale
    got = y.double().cpu().numpy()
    assert np.array_equal(got[~keep], base[~keep])
    tol = 2.0 ** -8 * np.abs(want) if dtype == torch.bfloat16 else 0.0
    assert (np.abs(got - want) <= tol + 2.0 ** -22 * (np.abs(X) * scale + np.abs(base))).all()
    if res is None:
        assert (got[keep] != 0).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("N,d,p", [(1, 1, 0.5), (1, 8, 0.5), (3, 7, 0.25), (2, 3584, 0.1), (50, 48, 0.1), (33, 255, 0.3),
                                   (100, 256, 0.9), (65, 771, 0.1), (7, 4097, 0.01), (300, 136, 0.0), (20, 8192, 0.5)])
def test_masks_and_values(N, d, p, dtype):
    from paper_2606_29758_gb300 import RowDropout
    x, res = _data(N, d, dtype, seed=d)
    traj, pos = _rows(N)
    m = RowDropout(p, site=SITE)
    keep = ob.keep_mask(traj.cpu().numpy(), pos.cpu().numpy(), d, p, SEED, STEP, SITE, traj_base=1000)
    _check(m.forward(x, traj, pos, SEED, STEP, res=res, traj_base=1000), x, res, keep, p, dtype)
    # the backward: the same mask on the gradient
    _check(m.backward(res, traj, pos, SEED, STEP, traj_base=1000), res, None, keep, p, dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_pitches_alignment_and_in_place(dtype):
    from paper_2606_29758_gb300 import RowDropout
    N, d, p = 90, 264, 0.2
    x, res = _data(N, d, dtype)
    traj, pos = _rows(N)
    m = RowDropout(p, site=SITE)
    want = m.forward(x, traj, pos, SEED, STEP, res=res)
    for shift in (0, 1, 3):                         # rows of an odd pitch that start anywhere
        wide = torch.zeros(N, d + 5, dtype=dtype, device="cuda")
        wide[:, shift:shift + d] = x
        out = torch.full((N, d + 5), 3.0, dtype=dtype, device="cuda")
        y = m.forward(wide[:, shift:shift + d], traj, pos, SEED, STEP, res=res, out=out[:, shift:shift + d])
        assert torch.equal(y, want)
        assert bool((out[:, :shift] == 3.0).all()) and bool((out[:, shift + d:] == 3.0).all())
    a, b = x.clone(), res.clone()
    assert torch.equal(m.forward(a, traj, pos, SEED, STEP, res=res, out=a), want)
    assert torch.equal(m.forward(x, traj, pos, SEED, STEP, res=b, out=b), want)


def test_masks_do_not_depend_on_packing_or_shard():
    from paper_2606_29758_gb300 import RowDropout
    N, d, p = 400, 136, 0.3
    x, _ = _data(N, d, torch.bfloat16)
    traj, pos = _rows(N)
    m = RowDropout(p, site=SITE)
    whole = m.forward(x, traj, pos, SEED, STEP, traj_base=5)
    some = torch.arange(0, N, 3, device="cuda")      # the rows that shorter prefixes would keep
    part = m.forward(x[some].contiguous(), traj[some].contiguous(), pos[some].contiguous(), SEED, STEP, traj_base=5)
    assert torch.equal(part, whole[some])
    first = int(traj[200])
    cut = int((traj < first).sum())
    shard = m.forward(x[cut:], (traj[cut:] - first).contiguous(), pos[cut:], SEED, STEP, traj_base=5 + first)
    assert torch.equal(shard, whole[cut:])
    assert not torch.equal(m.forward(x, traj, pos, SEED, STEP + 1, traj_base=5), whole)
    assert not torch.equal(RowDropout(p, site=SITE + 1).forward(x, traj, pos, SEED, STEP, traj_base=5), whole)


def test_dropped_values_count_as_zero_whatever_they_are():
    from paper_2606_29758_gb300 import RowDropout
    N, d, p = 40, 64, 0.5
    traj, pos = _rows(N)
    keep = torch.from_numpy(ob.keep_mask(traj.cpu().numpy(), pos.cpu().numpy(), d, p, SEED, STEP, SITE)).cuda()
    for width in (d, d - 1):
        x = torch.where(keep, 1.0, float("nan"))[:, :width].contiguous()
        y = RowDropout(p, site=SITE).forward(x, traj, pos, SEED, STEP)
        assert torch.equal(y, torch.where(keep[:, :width], 2.0, 0.0))


def test_no_rows_a_graph_and_refusals():
    from paper_2606_29758_gb300 import RowDropout
    B = _B()
    x, res = _data(30, 72, torch.bfloat16)
    traj, pos = _rows(30)
    m = RowDropout(0.1)
    assert m.forward(x[:0], traj[:0], pos[:0], 1, 1).shape == (0, 72)
    out = torch.empty_like(x)
    want = m.forward(x, traj, pos, 1, 1, res=res).clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        m.forward(x, traj, pos, 1, 1, res=res, out=out)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)
    for p in (1.0, -0.1, float("nan"), 0.999999):
        with pytest.raises(B.PsppoError) as e:
            RowDropout(p).forward(x, traj, pos, 1, 1)
        assert e.value.status == B.PS_ERR_INVALID_ARG
    with pytest.raises(B.PsppoError):
        m.forward(x, traj, pos, 1, 1 << 32)
    with pytest.raises(B.PsppoError):
        RowDropout(0.1, site=65536).forward(x, traj, pos, 1, 1)
    with pytest.raises(TypeError):
        m.forward(x.half(), traj, pos, 1, 1)
    with pytest.raises(ValueError):
        m.forward(x, traj[:5], pos, 1, 1)
    with pytest.raises(TypeError):
        m.forward(x, traj.long(), pos, 1, 1)
    with pytest.raises(TypeError):
        m.forward(x, traj, pos, 1, 1, res=res.float())
