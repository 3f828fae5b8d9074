"""Pages that the cache hands out: the table and the bookkeeping agree, whatever device is current and whatever fails."""
import pytest
import torch

from paper_2606_29758_gb300 import CacheShape, PagedCache, PsppoError


def _cache():
    c = PagedCache(CacheShape(4, 12, 4, 1, 16, 20, layers=2), device="cpu")
    for t in (c.k, c.v):
        t.copy_(torch.randn(t.shape))
    return c


def _agrees(c):
    """Each sequence's row names its pages and nothing else; pages are free or someone's; users are counted."""
    users = [0] * c.s.pages
    for b, own in enumerate(c._own):
        assert c.table[b].tolist() == own + [-1] * (c.width - len(own)), b
        for p in own:
            users[p] += 1
    assert users == c._users
    assert sorted(c._free) == [p for p in range(c.s.pages) if users[p] == 0]


@pytest.mark.parametrize("name", ["cuda", "cuda:1", "cpu"])
def test_the_table_is_written_where_it_is(name):
    """Not on the device that the name means by now (here one that is not there)."""
    c = _cache()
    c.device = name
    c.reserve(0, 10)
    c.share(0, [1, 3], 10)
    c.reserve(1, 17)
    _agrees(c)
    for x in (c.k, c.v):
        for b in (1, 3):
            assert torch.equal(x[:, c._own[b][2]], x[:, c._own[0][2]])      # the begun page, copied
            assert c._own[b][:2] == c._own[0][:2] and c._own[b][2] != c._own[0][2]
    c.lengths[1] = 17
    c.release(0)
    c.release(1)
    _agrees(c)
    assert c.lengths.tolist() == [0] * 4 and len(c._own[3]) == 3


def test_whole_pages_are_shared_without_a_copy():
    c = _cache()
    c.reserve(2, 8)
    c.share(2, [0, 1], 8)
    _agrees(c)
    assert c._own[0] == c._own[1] == c._own[2] and len(c._free) == 10
    c.share(2, [], 8)
    c.share(2, [3], 0)
    _agrees(c)
    assert c._own[3] == []


def test_a_call_that_fails_leaves_the_cache_as_it_was(monkeypatch):
    c = _cache()
    c.reserve(0, 10)
    c.share(0, [1], 6)
    kept = [list(c._free), list(c._users), [list(o) for o in c._own], c.table.clone()]

    def fails(own):
        raise RuntimeError("no memory")
    for call in (lambda: c.reserve(0, 20), lambda: c.reserve(2, 3), lambda: c.share(0, [2, 3], 10), lambda: c.release(1)):
        monkeypatch.setattr(c, "_publish", fails)
        with pytest.raises(RuntimeError, match="no memory"):
            call()
        monkeypatch.undo()
        assert kept[:3] == [c._free, c._users, c._own] and torch.equal(kept[3], c.table)
        _agrees(c)
    c.reserve(2, 20)
    c.reserve(3, 12)                          # 3 + 1 + 5 + 3 of 12
    with pytest.raises(PsppoError):
        c.reserve(0, 20)
    _agrees(c)
