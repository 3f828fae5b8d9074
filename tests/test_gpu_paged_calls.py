"""Calls of attention over the paged cache whose values are looked at, not only that two of them agree."""
import pytest
import torch

from test_gpu_paged import BF, F32, _att, _cache, _check, _queries

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF, F32])
def test_the_first_sequences_alone(dtype):
    """A call with fewer queries than sequences: their values, and the buffers' other rows left as they were."""
    lens, Hq, Hk, D = [100, 300, 0, 777, 16], 12, 2, 128
    c, kv = _cache(lens, Hk, D, 16, dtype)
    q, m = _queries(5, Hq, D, dtype), _att(5, Hq, Hk, D, dtype)
    for n in (5, 4, 2, 1):
        m.o.fill_(5.0)
        lse = torch.full((n, Hq), 7.0, device="cuda")
        o = m.forward(q[:n], c, lse=lse)
        m.check_status()
        assert o.shape == (n, Hq * D) and (m.o[n:] == 5.0).all()
        _check(o, lse, q[:n], kv[:n], Hq, Hk, D, dtype)


def test_a_sequence_that_ends_and_one_that_takes_its_pages():
    """Two completions keep their values while a third one's pages go to a new sequence."""
    from paper_2606_29758_gb300 import CacheShape, PagedCache
    Hq, Hk, D, page, i32 = 4, 2, 64, 8, dict(dtype=torch.int32, device="cuda")
    c = PagedCache(CacheShape(4, 14, page, Hk, D, 64))
    c.k.zero_()
    c.v.zero_()
    g = torch.Generator().manual_seed(2)
    prompt = torch.randn(21, 2 * Hk * D, generator=g).to(BF).cuda()
    new = torch.randn(4, 9, 2 * Hk * D, generator=g).to(BF).cuda()
    w = Hk * D

    def put(rows, seq, first):
        n = len(rows)
        c.append(0, rows[:, :w], rows[:, w:], torch.full((n,), seq, **i32), torch.arange(first, first + n, **i32))
        c.check_status()
    c.reserve(0, 21)
    put(prompt, 0, 1)
    c.share(0, [1, 2], 21)
    for b in range(3):
        c.reserve(b, 30)
        put(new[b], b, 22)
    c.lengths.copy_(torch.tensor([30, 30, 30, 0], dtype=torch.int32))
    q, m, lse = _queries(4, Hq, D, BF), _att(4, Hq, Hk, D, BF), torch.empty(4, Hq, device="cuda")
    full = [torch.cat([prompt, new[b]]) for b in range(3)] + [prompt[:0]]

    def check():
        kv = [tuple(t.double().cpu().numpy().reshape(-1, Hk, D) for t in (x[:, :w], x[:, w:])) for x in full]
        _check(m.forward(q, c, lse=lse), lse, q, kv, Hq, Hk, D, BF)
        m.check_status()
    check()
    c.release(0)
    full[0] = prompt[:0]
    check()
    c.reserve(3, 40)
    put(torch.cat([new[3], prompt]), 3, 1)
    c.lengths[3] = 30
    full[3] = torch.cat([new[3], prompt])
    check()
