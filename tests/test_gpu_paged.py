"""The paged cache and attention of one new token over it against float64 (oracle.block).

Appending copies: equal bits. Tolerances of attention, e = 2^-24: a score sums D products (exact of bf16 operands, f32 sums of the
tensor cores counted 2 e each): |ds| <= 2 D e A, A = scale sum |q k|; the exponent's product and difference 2 e |x| with |x| <= 2 A;
ex2 2^-22; so a weight is off by at most 2 (2 D e A + 4 e A) + 2^-22 of itself, its two bf16 parts by 2^-17 (bf16); sums of n keys'
weights and weighted values: n / 64 + 64 additions in turn, 2 e each. All of that of sum_j w_j |v_j|, twice, as the total's error counts like
the weights'. bf16 outputs: plus 2^-8 of the value. lse: |ds| and the total's error."""
import numpy as np
import pytest
import torch

from oracle import block as ob

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
E = 2.0 ** -24


def _B():
    from paper_2606_29758_gb300 import _binding as B
    return B


def _cache(lens, Hk, D, page, dtype, seed=0, spare=5, width=None, layers=1):
    """A cache of such sequences: pages in no order, NaN wherever nothing of a sequence lies."""
    from paper_2606_29758_gb300 import CacheShape, PagedCache
    g = torch.Generator().manual_seed(seed)
    need = [-(-n // page) for n in lens]
    pages = sum(need) + spare
    width = width or max(1, max(need))
    c = PagedCache(CacheShape(len(lens), pages, page, Hk, D, width * page, layers, dtype))
    c.k.fill_(float("nan"))
    c.v.fill_(float("nan"))
    c.table.fill_(-(2 ** 31))
    ids = torch.randperm(pages, generator=g)
    kv, at = [], 0
    for b, n in enumerate(lens):
        own = ids[at:at + need[b]]
        at += need[b]
        c.table[b, :need[b]] = own.to(torch.int32)
        k, v = (torch.randn(n, Hk, D, generator=g).to(dtype) for _ in range(2))
        kv.append((k.double().numpy(), v.double().numpy()))
        for i, p in enumerate(own.tolist()):
            part = slice(i * page, min(n, (i + 1) * page))
            c.k[layers - 1, p, :, :part.stop - part.start] = k[part].transpose(0, 1).cuda()
            c.v[layers - 1, p, :, :part.stop - part.start] = v[part].transpose(0, 1).cuda()
    c.lengths.copy_(torch.tensor(lens, dtype=torch.int32))
    return c, kv


def _queries(n, Hq, D, dtype, seed=1, size=1.0):
    g = torch.Generator().manual_seed(seed)
    return (size * torch.randn(n, Hq * D, generator=g)).to(dtype).cuda()


def _att(seqs, Hq, Hk, D, dtype, **kw):
    from paper_2606_29758_gb300 import DecodeAttention, DecodeShape
    return DecodeAttention(DecodeShape(seqs, Hq, Hk, D, dtype, **kw))


def _check(o, lse, q, kv, Hq, Hk, D, dtype, window=0, scale=None, rows=None):
    scale = D ** -0.5 if scale is None else scale
    o, lse, q = o.double().cpu().numpy(), lse.double().cpu().numpy(), q.double().cpu().numpy()
    of = np.arange(Hq) // (Hq // Hk)
    for b, (k, v) in enumerate(kv):
        if rows is not None and b not in rows:
            continue
        if window:
            k, v = k[-window:], v[-window:]
        qb, n = q[b].reshape(Hq, D), len(k)
        want, wl = ob.attend(qb, k, v, scale)
        got = o[b].reshape(Hq, D)
        if n == 0:
            assert (got == 0).all() and (lse[b] == -np.inf).all()
            continue
        A = abs(scale) * np.einsum("hd,jhd->hj", np.abs(qb), np.abs(k[:, of])).max(axis=1)
        w = np.exp(scale * np.einsum("hd,jhd->hj", qb, k[:, of]) - wl[:, None])
        reach = np.einsum("hj,jhd->hd", w, np.abs(v[:, of]))
        ds = 2 * D * E * A + 4 * E * A
        part = 2 * ds + 2.0 ** -22 + (2.0 ** -17 if dtype == BF else 0.0) + 2 * (n / 64 + 64) * E
        ok = np.abs(got - want) <= 2 * part[:, None] * reach + (2.0 ** -8 if dtype == BF else E) * np.abs(want)
        assert ok.all(), (b, n, np.argwhere(~ok)[:4], got[~ok][:4], want[~ok][:4])
        assert (np.abs(lse[b] - wl) <= ds + part + 4 * E * np.abs(wl)).all(), (b, n)


def _run(lens, Hq, Hk, D, page, dtype, window=0, scale=None, seed=0, size=1.0, **kw):
    c, kv = _cache(lens, Hk, D, page, dtype, seed, **kw)
    q = _queries(len(lens), Hq, D, dtype, seed + 1, size)
    m = _att(len(lens), Hq, Hk, D, dtype, window=window, scale=scale)
    lse = torch.full((len(lens), Hq), 9.0, device="cuda")
    o = m.forward(q, c, c.s.layers - 1, lse=lse)
    m.check_status()
    _check(o, lse, q, kv, Hq, Hk, D, dtype, window, scale)
    return m, c, q, kv, o, lse


EDGES = [0, 1, 2, 15, 16, 17, 31, 33, 63, 64, 65, 127, 128, 129, 300, 0]
HEADS = [(28, 4, 128), (16, 16, 128), (5, 1, 64), (6, 2, 96), (12, 2, 80), (9, 1, 128), (32, 2, 64), (20, 1, 128), (8, 1, 256),
         (12, 1, 192), (3, 3, 16), (2, 1, 48)]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("Hq,Hk,D", HEADS)
def test_lengths_around_the_tiles(Hq, Hk, D, dtype):
    _run(EDGES, Hq, Hk, D, 16, dtype)


@pytest.mark.parametrize("page", [1, 2, 8, 32, 64, 256, 4096])
def test_pages(page):
    _run([1, 30, 64, 65, 200, 7], 12, 2, 128, page, BF, seed=page, width=-(-200 // page) + 2)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("window", [1, 16, 50, 64, 100, 1000])
def test_windows(window, dtype):
    _run([0, 1, 15, 64, 99, 100, 101, 300, 700], 6, 2, 64, 16, dtype, window=window)


@pytest.mark.parametrize("lens", [[16384], [16384, 1], [1, 16384, 0, 0, 5000], [0] * 9, [3] * 700, [5000, 40] * 12])
def test_splits_over_the_ctas(lens):
    """One long sequence over many CTAs, short ones many to a CTA, empty ones at all places."""
    _run(lens, 28, 4, 128, 64, BF, seed=len(lens))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_long_sequences_of_all_widths(dtype):
    for Hq, Hk, D in ((7, 1, 64), (16, 1, 96), (4, 2, 256)):
        _run([3001, 1, 2500], Hq, Hk, D, 32, dtype, seed=D)


def test_a_workspace_after_longer_calls():
    """Nothing of an earlier call's parts is taken for this one's."""
    Hq, Hk, D = 12, 2, 128
    m = _att(40, Hq, Hk, D, BF)
    for lens in ([4000] * 40, [70, 100], [64 * 7, 1, 0, 65], [4000, 3], [130], [2] * 40):
        c, kv = _cache(lens, Hk, D, 16, BF, seed=len(lens), width=250)
        q = _queries(len(lens), Hq, D, BF)
        lse = torch.empty(len(lens), Hq, device="cuda")
        _check(m.forward(q, c, lse=lse), lse, q, kv, Hq, Hk, D, BF)


def test_few_keys_take_all_the_weight():
    """Large scores of both signs, and a negative scale."""
    _run([64, 500, 3000], 8, 2, 128, 16, BF, size=20.0)
    _run([64, 500, 3000], 8, 2, 128, 16, BF, size=20.0, scale=-0.05)
    _run([64, 500], 8, 2, 128, 16, F32, size=20.0, scale=0.0)


def test_strides_places_and_reruns():
    lens, Hq, Hk, D = [100, 3, 0, 777], 12, 2, 128
    m, c, q, kv, o, lse = _run(lens, Hq, Hk, D, 16, BF, layers=3)
    o, first = o.clone(), lse.clone()
    wide = torch.zeros(4, Hq * D + 64, dtype=BF, device="cuda")
    wide[:, 32:-32] = q
    place = torch.full((4, Hq * D + 128), 5.0, dtype=BF, device="cuda")
    got = m.forward(wide[:, 32:-32], c, 2, out=place[:, 64:-64])
    assert torch.equal(got, o) and (place[:, :64] == 5).all() and (place[:, -64:] == 5).all()
    m.forward(wide[:, 32:-32], c, 2, out=wide[:, 32:-32])                  # over the queries
    assert torch.equal(wide[:, 32:-32], o)
    m.forward(q, c, 2, lse=lse)
    assert torch.equal(m.o, o) and torch.equal(lse, first)
    m.o.fill_(5.0)
    assert torch.equal(m.forward(q[:2], c, 2)[0], m.o[0]) and (m.o[2:] == 5.0).all()   # the first two sequences


def test_infinities_and_nan_of_a_sequence_stay_in_it():
    lens, Hq, Hk, D = [100, 70, 300], 4, 2, 64
    c, kv = _cache(lens, Hk, D, 16, BF)
    q = _queries(3, Hq, D, BF)
    m = _att(3, Hq, Hk, D, BF)
    lse = torch.empty(3, Hq, device="cuda")
    c.v[0, c.table[1, 2].item(), 1, 3, 5] = float("inf")      # a value of key head 1: position 35
    c.k[0, c.table[2, 0].item(), 0, 0] = float("nan")
    o = m.forward(q, c, lse=lse).view(3, Hq, D)
    _check(o.view(3, -1), lse, q, kv, Hq, Hk, D, BF, rows=[0])
    # (inf by a weight's second part, which may be 0 or negative: an infinity or NaN, in its own dim)
    finite = torch.isfinite(o[1])
    assert finite[:2].all() and not finite[2:, 5].any() and finite[2:, :5].all() and finite[2:, 6:].all()
    assert torch.isnan(o[2, :2]).all() and torch.isfinite(o[2, 2:]).all()


def test_lengths_and_pages_that_cannot_be():
    B = _B()
    lens, Hq, Hk, D = [100, 70, 300, 40], 4, 2, 64
    c, kv = _cache(lens, Hk, D, 16, BF)
    q, m = _queries(4, Hq, D, BF), _att(4, Hq, Hk, D, BF)
    lse = torch.empty(4, Hq, device="cuda")
    for bad in (-1, c.width * 16 + 1, 2 ** 31 - 1):
        c.lengths[1] = bad
        o = m.forward(q, c, lse=lse)
        assert B.ps_workspace_status(m.ws) == (B.PS_ERR_DEVICE_DATA, B.PS_DEV_BAD_LENGTH)
        assert torch.isnan(o[1]).all() and torch.isnan(lse[1]).all()
        _check(o, lse, q, kv, Hq, Hk, D, BF, rows=[0, 2, 3])
    c.lengths[1] = 70
    for bad in (-1, c.s.pages, 2 ** 31 - 1):
        kept = c.table[2, 18].item()                          # its last page
        c.table[2, 18] = bad
        o = m.forward(q, c, lse=lse)
        assert B.ps_workspace_status(m.ws) == (B.PS_ERR_DEVICE_DATA, B.PS_DEV_BAD_PAGE)
        assert torch.isnan(o[2]).all() and torch.isnan(lse[2]).all()
        _check(o, lse, q, kv, Hq, Hk, D, BF, rows=[0, 1, 3])
        c.table[2, 18] = kept
    o = m.forward(q, c, lse=lse)
    m.check_status()
    _check(o, lse, q, kv, Hq, Hk, D, BF)


def test_captured_steps_with_growing_lengths():
    """A captured step appends, counts and attends; replays give what eager calls give; two graphs take turns with a workspace."""
    from paper_2606_29758_gb300 import CacheShape, PagedCache
    Hq, Hk, D, n = 8, 2, 64, 5
    g = torch.Generator().manual_seed(3)
    kv = torch.randn(40, n, 2 * Hk * D, generator=g).to(BF).cuda()
    qs = torch.randn(40, n, Hq * D, generator=g).to(BF).cuda()

    def fresh():
        c = PagedCache(CacheShape(n, 40, 8, Hk, D, 64))
        for b in range(n):
            c.reserve(b, 48)
        return c
    seq = torch.arange(n, device="cuda", dtype=torch.int32)
    m = _att(n, Hq, Hk, D, BF)

    def step(c, q, row):
        c.lengths.add_(1)
        c.append(0, row[:, :Hk * D], row[:, Hk * D:], seq, c.lengths)
        return m.forward(q, c)
    c, want = fresh(), []
    for t in range(40):
        want.append(step(c, qs[t], kv[t]).clone())
    c.check_status()
    c2, q_in, kv_in = fresh(), torch.empty_like(qs[0]), torch.empty_like(kv[0])
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = step(c2, q_in, kv_in)
        graphs.append(graph)
    c2.lengths.zero_()
    for t in range(40):
        q_in.copy_(qs[t])
        kv_in.copy_(kv[t])
        graphs[t % 2].replay()
        assert torch.equal(out, want[t]), t
    m.check_status()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("Hk,D,page,lens", [(4, 128, 64, [100, 1, 64, 0, 300]), (1, 16, 1, [3, 5]), (2, 80, 16, [700, 33]),
                                            (16, 256, 8, [9, 8, 7]), (2, 64, 16, [900, 900, 900])])
def test_append(Hk, D, page, lens, dtype):
    from paper_2606_29758_gb300 import CacheShape, PagedCache
    g = torch.Generator().manual_seed(D)
    pages = sum(-(-n // page) for n in lens) + 2
    c = PagedCache(CacheShape(len(lens), pages, page, Hk, D, (-(-max(lens) // page) + 1) * page, 2, dtype))
    c.k.fill_(7.0)
    c.v.fill_(7.0)
    for b, n in enumerate(lens):
        c.reserve(b, n)
    seq = torch.cat([torch.full((n,), b, dtype=torch.int32) for b, n in enumerate(lens)])
    pos = torch.cat([torch.arange(1, n + 1, dtype=torch.int32) for n in lens])
    order = torch.randperm(len(seq), generator=g)
    kv = torch.randn(len(seq), 2 * Hk * D, generator=g).to(dtype)
    want = [x.cpu().clone() for x in (c.k, c.v)]
    table = c.table.cpu()
    for i in range(len(seq)):
        p = int(pos[i]) - 1
        for x, part in zip(want, (kv[i, :Hk * D], kv[i, Hk * D:])):
            x[1, table[seq[i], p // page], :, p % page] = part.view(Hk, D)
    seq[order[0]], skipped = -1, order[0]                      # a row that is passed by
    p = int(pos[skipped]) - 1
    b = [b for b in range(len(lens)) if sum(lens[:b]) <= skipped < sum(lens[:b + 1])][0]
    for x in want:
        x[1, table[b, p // page], :, p % page] = 7.0
    kv = kv[order].cuda()
    c.append(1, kv[:, :Hk * D], kv[:, Hk * D:], seq[order].cuda(), pos[order].cuda())
    c.check_status()
    assert torch.equal(c.k.cpu(), want[0]) and torch.equal(c.v.cpu(), want[1])


@pytest.mark.parametrize("N", [6, 3000])
def test_append_refuses_rows_on_the_device(N):
    """Rows to places that are not there are not written, whether the call has few rows or many."""
    from paper_2606_29758_gb300 import CacheShape, PagedCache
    B = _B()
    c = PagedCache(CacheShape(3, 400, 8, 1, 16, 2400))
    c.k.zero_()
    c.v.zero_()
    c.reserve(0, 2392)
    c.reserve(1, 8)
    kv = torch.ones(N, 16, dtype=BF, device="cuda")
    good = torch.zeros(N, dtype=torch.int32)
    at = torch.arange(1, N + 1, dtype=torch.int32).clamp(max=2300)
    good[2300:] = -1
    for what, seq, pos, bit in (("sequence", 3, 1, B.PS_DEV_BAD_LENGTH), ("sequence", -2, 1, B.PS_DEV_BAD_LENGTH),
                                ("position", 0, 0, B.PS_DEV_BAD_LENGTH), ("position", 0, 2401, B.PS_DEV_BAD_LENGTH),
                                ("position", 1, -5, B.PS_DEV_BAD_LENGTH), ("page", 1, 9, B.PS_DEV_BAD_PAGE),
                                ("page", 2, 1, B.PS_DEV_BAD_PAGE)):
        s, p = good.clone(), at.clone()
        s[4], p[4] = seq, pos
        c.k.zero_()
        c.append(0, kv, kv, s.cuda(), p.cuda())
        assert B.ps_workspace_status(c.ws) == (B.PS_ERR_DEVICE_DATA, bit), what
        assert c.k.float().sum().item() == 16 * ((good >= 0).sum().item() - 1), what
    c.append(0, kv, kv, good.cuda(), at.cuda())
    c.check_status()


def test_pages_handed_out_and_shared():
    """Completions share their prompt's whole pages; what each writes after that is its own."""
    from paper_2606_29758_gb300 import CacheShape, PagedCache
    B = _B()
    Hq, Hk, D = 4, 2, 64
    c = PagedCache(CacheShape(4, 14, 8, Hk, D, 64, 2))
    c.k.zero_()
    c.v.zero_()
    g = torch.Generator().manual_seed(0)
    prompt = torch.randn(21, 2 * Hk * D, generator=g).to(BF).cuda()
    c.reserve(0, 21)
    i32 = dict(dtype=torch.int32, device="cuda")
    for layer in range(2):
        c.append(layer, prompt[:, :Hk * D], prompt[:, Hk * D:], torch.zeros(21, **i32), torch.arange(1, 22, **i32))
    c.share(0, [1, 2], 21)
    assert torch.equal(c.table[0, :2], c.table[1, :2]) and len(set(c.table[:3, 2].tolist())) == 3
    for b in range(3):
        c.reserve(b, 30)
    new = torch.randn(3, 9, 2 * Hk * D, generator=g).to(BF).cuda()
    rows = new.reshape(27, -1)
    c.append(1, rows[:, :Hk * D], rows[:, Hk * D:], torch.arange(27, **i32) // 9, torch.arange(27, **i32) % 9 + 22)
    c.lengths.copy_(torch.tensor([30, 30, 30, 0], dtype=torch.int32))
    q, m = _queries(4, Hq, D, BF), _att(4, Hq, Hk, D, BF)
    lse = torch.empty(4, Hq, device="cuda")
    o = m.forward(q, c, 1, lse=lse)
    full = [torch.cat([prompt, new[b]]).double().cpu().numpy() for b in range(3)]
    kv = [(x[:, :Hk * D].reshape(30, Hk, D), x[:, Hk * D:].reshape(30, Hk, D)) for x in full] + [(np.zeros((0, Hk, D)),) * 2]
    _check(o, lse, q, kv, Hq, Hk, D, BF)
    # 2 shared, 3 begun and copied, 3 more: 6 of 14 are free
    with pytest.raises(B.PsppoError):
        c.reserve(3, 56)
    c.release(0)
    assert c.lengths[0] == 0 and (c.table[0] == -1).all()
    c.reserve(3, 64)                                      # its two own pages came back, the shared ones not
    taken = set(c.table[3].tolist())
    assert len(taken) == 8 and not taken & (set(c.table[1].tolist()) | set(c.table[2].tolist()))
    o2 = m.forward(q, c, 1, lse=lse)
    assert torch.equal(o2[1:3], m.o[1:3])
    _check(o2, lse, q, kv, Hq, Hk, D, BF, rows=[1, 2])
