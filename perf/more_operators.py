"""What a policy block takes beside its feed-forward block, its q/k norms and its dropout: cases, plain and 64-bit forms.

  norm    the norm after a branch, its gate, the scaled residual sum and the norm before the next branch, forward and, in
          training, backward: ResidualNorm
  append  keys and values of new tokens written into a paged cache: PagedCache.append
  decode  attention of one new token a sequence over the paged cache: DecodeAttention

Rows of training are those of a packed batch. Sequences of sampling are the completions of a batch, prompts x completions of
each, with lengths of a lognormal law (its quantiles, in an order that the seed decides); their pages lie in the cache in no
order. Gradients are of very different size per row, with some rows 0, as where the clip binds.
"""
import math
from statistics import NormalDist

import torch

own = False
DEVICE = "cuda"
DTYPE = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-6


def listed():
    return [
        # One token of a 7B-shaped policy (d of the benchmark's head) between two of its branches, in sampling: latency.
        dict(name="norm_token_7b", op="norm", N=1, d=3584, dtype="bf16", post=True, gate=False, a=1.0, b=1.0, train=False),
        # A full-precision reference run of an odd width, with a gate per token, forward and backward.
        dict(name="norm_train_f32", op="norm", N=1571, d=771, dtype="f32", post=True, gate=True, a=1.0, b=0.5, train=True),
        # An ordinary micro-batch of the 1.5B-shaped policy, branches added as they are, forward and backward.
        dict(name="norm_train_1.5b", op="norm", N=6030, d=1536, dtype="bf16", post=False, gate=False, a=1.0, b=1.0, train=True),
        # Sixty thousand rows, about a third of the 7B-shaped benchmark batch, gated, forward and backward.
        dict(name="norm_train_7b", op="norm", N=60000, d=3584, dtype="bf16", post=True, gate=True, a=1.0, b=0.7, train=True),
        # The new keys and values of one sampling step of 16 prompts x 8 completions.
        dict(name="append_step_7b", op="append", seqs=128, median=700, sigma=0.5, most=2048, step=True, Hk=4, D=128, page=64,
             dtype="bf16"),
        # A whole batch of prompts and answers laid into the cache at once.
        dict(name="append_batch_7b", op="append", seqs=64, median=1024, sigma=0.5, most=4096, step=False, Hk=4, D=128,
             page=64, dtype="bf16"),
        # The first answer tokens of one completion after a short question.
        dict(name="decode_token_short", op="decode", seqs=1, median=37, sigma=0.0, most=64, Hq=28, Hk=4, D=128, page=16,
             dtype="bf16", window=0, done=False),
        # One long completion alone: as many keys as the long traces have at most.
        dict(name="decode_token_long", op="decode", seqs=1, median=16384, sigma=0.0, most=16384, Hq=28, Hk=4, D=128, page=64,
             dtype="bf16", window=0, done=False),
        # A full-precision reference run: every query head with keys of its own, heads of 96, a sliding window.
        dict(name="decode_f32", op="decode", seqs=24, median=300, sigma=0.5, most=1000, Hq=6, Hk=6, D=96, page=16, dtype="f32",
             window=256, done=False),
        # A step of 32 prompts x 8 completions of the 1.5B-shaped policy, some of which have ended.
        dict(name="decode_step_1.5b", op="decode", seqs=256, median=1024, sigma=0.5, most=4096, Hq=12, Hk=2, D=128, page=16,
             dtype="bf16", window=0, done=True),
        # A step of 16 x 8 completions of the 7B-shaped policy.
        dict(name="decode_step_7b", op="decode", seqs=128, median=2048, sigma=0.5, most=8192, Hq=28, Hk=4, D=128, page=64,
             dtype="bf16", window=0, done=False),
        # A step of 8 x 16 long completions.
        dict(name="decode_step_long", op="decode", seqs=128, median=12288, sigma=0.2, most=16384, Hq=28, Hk=4, D=128, page=64,
             dtype="bf16", window=0, done=False),
    ]


def _log(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def draw(rng):
    """One more case of the ranges that the listed ones stand for."""
    op = rng.choice(["norm", "norm", "append", "decode", "decode"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    e = 4 if dtype == "f32" else 2
    if op == "norm":
        d = int(_log(rng, 64, 8192))
        d = d // 8 * 8 if rng.random() < 0.75 else d
        most = 60000 * 3584 * 2 / (d * e)
        return dict(op=op, N=int(_log(rng, 1, min(most, 200000))), d=d, dtype=dtype, post=rng.random() < 0.6,
                    gate=rng.random() < 0.4, a=1.0, b=rng.choice([1.0, 0.7, 0.25]), train=rng.random() < 0.7)
    page = rng.choice([16, 16, 32, 64, 128])
    D = rng.choice([64, 80, 96, 128, 128, 128, 192, 256])
    Hq, Hk = rng.choice([(28, 4), (12, 2), (16, 16), (6, 2), (5, 1), (40, 8), (32, 1), (64, 8)])
    seqs = int(_log(rng, 1, 300))
    per_key = 2.0 * Hk * D * e                                    # bytes of a key and its value in all heads
    if op == "append":
        median = int(_log(rng, 1, max(2.0, min(2048.0, 6e8 / (seqs * per_key)))))
        return dict(op=op, seqs=seqs, median=median, sigma=0.5, most=4 * median, step=rng.random() < 0.5, Hk=Hk, D=D,
                    page=page, dtype=dtype)
    median = int(_log(rng, 1, max(2.0, min(16384.0, 2.4e9 / (seqs * per_key)))))
    return dict(op=op, seqs=seqs, median=median, sigma=rng.choice([0.0, 0.2, 0.5]), most=2 * median, Hq=Hq, Hk=Hk, D=D,
                page=page, dtype=dtype, window=rng.choice([0, 0, 0, max(1, median // 2)]), done=rng.random() < 0.3)


# ----------------------------------------------------------------------------- inputs
def _generator(seed):
    return torch.Generator(device=DEVICE).manual_seed(seed)


def _activations(N, d, g, dtype):
    x = torch.randn(N, d, device=DEVICE, generator=g)
    x[:, torch.randint(0, d, (max(1, d // 100),), device=DEVICE, generator=g)] *= 8.0
    return x.to(dtype)


def _gradients(N, d, g, dtype):
    size = torch.exp(torch.randn(N, 1, device=DEVICE, generator=g)) * 1e-3
    size *= torch.rand(N, 1, device=DEVICE, generator=g) > 0.1 if N > 1 else 1.0
    return (torch.randn(N, d, device=DEVICE, generator=g) * size).to(dtype)


def _lengths(case):
    """The law's quantiles; with `done` every seventh completion has ended and holds no keys."""
    n = case["seqs"]
    z = [NormalDist().inv_cdf((i + 0.5) / n) for i in range(n)]
    lens = [max(1, min(case["most"], round(case["median"] * math.exp(case["sigma"] * v)))) for v in z]
    return [0 if case.get("done") and i % 7 == 3 else v for i, v in enumerate(lens)]


class State:
    pass


def prepare(case, seed):
    s = State()
    s.case = case
    (_prepare_norm if case["op"] == "norm" else _prepare_cache)(s, case, seed)
    return s


def _prepare_norm(s, case, seed):
    g, t = _generator(seed), DTYPE[case["dtype"]]
    N, d = case["N"], case["d"]
    s.x, s.y = _activations(N, d, g, t), _activations(N, d, g, t)
    s.gy, s.go = ((1.0 + 0.3 * torch.randn(d, device=DEVICE, generator=g)).to(t) for _ in range(2))
    s.gate = None
    if case["gate"]:      # a token's gate, 0 for those that pass the branch by
        s.gate = torch.sigmoid(torch.randn(N, device=DEVICE, generator=g))
        s.gate *= torch.rand(N, device=DEVICE, generator=g) > 0.1
    if case["train"]:
        s.do, s.dh = _gradients(N, d, g, t), _gradients(N, d, g, t)
    if own:
        from paper_2606_29758_gb300 import NormShape, ResidualNorm
        s.op = ResidualNorm(NormShape(rows=N, d=d, dtype=t, post=case["post"], eps=EPS, res_scale=case["a"],
                                      branch_scale=case["b"], train=case["train"]))


def _prepare_cache(s, case, seed):
    g, t = _generator(seed), DTYPE[case["dtype"]]
    Hk, D, page, n = case["Hk"], case["D"], case["page"], case["seqs"]
    order = torch.randperm(n, device=DEVICE, generator=g)
    s.lens = torch.tensor(_lengths(case), dtype=torch.int32, device=DEVICE)[order]
    need = (s.lens.long() + page - 1) // page
    total, most = int(need.sum()), max(1, int(need.max()))
    pages = total + 3
    ids = torch.randperm(pages, device=DEVICE, generator=g)[:total].to(torch.int32)
    s.table = torch.full((n, most), -1, dtype=torch.int32, device=DEVICE)
    s.table[torch.arange(most, device=DEVICE)[None, :] < need[:, None]] = ids
    s.kc, s.vc = (torch.randn(pages, Hk, page, D, device=DEVICE, generator=g, dtype=t) for _ in range(2))
    if case["op"] == "decode":
        q = torch.randn(n, case["Hq"], D, device=DEVICE, generator=g)
        q *= torch.exp(0.7 * torch.randn(1, case["Hq"], 1, device=DEVICE, generator=g))   # some heads look at few keys
        s.q = q.reshape(n, -1).to(t)
    else:
        seq = torch.arange(n, device=DEVICE, dtype=torch.int32)
        if case["step"]:                       # the last token of each
            s.seq, s.pos = seq, s.lens.clone()
        else:
            s.seq = torch.repeat_interleave(seq, s.lens.long())
            start = torch.cumsum(s.lens.long(), 0) - s.lens.long()
            s.pos = (torch.arange(len(s.seq), device=DEVICE) - start[s.seq.long()] + 1).to(torch.int32)
        # keys and values lie in one projection's rows
        kv = torch.randn(len(s.seq), 2 * Hk * D, device=DEVICE, generator=g).to(t)
        s.k, s.v = kv[:, :Hk * D], kv[:, Hk * D:]
    if own:
        from paper_2606_29758_gb300 import CacheShape, DecodeAttention, DecodeShape, PagedCache
        s.cache = PagedCache(CacheShape(seqs=n, pages=pages, page=page, Hk=Hk, D=D, max_len=most * page, dtype=t))
        s.cache.k[0].copy_(s.kc)
        s.cache.v[0].copy_(s.vc)
        s.cache.table.copy_(s.table)
        s.cache.lengths.copy_(s.lens)
        s.kc, s.vc = s.cache.k[0], s.cache.v[0]
        if case["op"] == "decode":
            s.op = DecodeAttention(DecodeShape(seqs=n, Hq=case["Hq"], Hk=Hk, D=D, dtype=t, window=case["window"]))


def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    op = s.case["op"]
    if op == "append":
        s.cache.append(0, s.k, s.v, s.seq, s.pos, pos_base=1)
        return dict(k=s.kc, v=s.vc)
    if op == "decode":
        return dict(o=s.op.forward(s.q, s.cache, 0))
    h, o = s.op.forward(s.x, s.y, s.gy, s.go, gate=s.gate)
    out = dict(h=h, o=o)
    if s.case["train"]:
        out.update(zip(("dx", "dy", "dgy", "dgo", "dgate"),
                       s.op.backward(s.do, s.dh, h, s.y, s.gy, s.go, gate=s.gate)))
        if s.gate is None:
            del out["dgate"]
    return out


# ----------------------------------------------------------------------------- the plain forms, in 32 bits
def _run_plain(s):
    return {"norm": _norm_plain, "append": _append_plain, "decode": _decode_plain}[s.case["op"]](s)


def _norm_plain(s):
    c, t = s.case, s.x.dtype
    y, gy, go = s.y.float(), s.gy.float(), s.go.float()
    ry = torch.rsqrt((y * y).mean(dim=1, keepdim=True) + EPS) if c["post"] else 1.0
    b = c["b"] if s.gate is None else c["b"] * s.gate[:, None]
    n = y * ry * gy
    hf = c["a"] * s.x.float() + b * n
    o = (hf * torch.rsqrt((hf * hf).mean(dim=1, keepdim=True) + EPS) * go).to(t)
    held = hf.to(t)
    out = dict(h=held, o=o)
    if not c["train"]:
        return out
    h, do = held.float(), s.do.float()           # the backward has the stream as it is held
    rh = torch.rsqrt((h * h).mean(dim=1, keepdim=True) + EPS)
    dgo = (do * h * rh).sum(dim=0)
    do = do * go
    dH = s.dh.float() + rh * (do - h * (rh * rh) * (do * h).mean(dim=1, keepdim=True))
    dn = b * dH
    dgy = (dn * y * ry).sum(dim=0)
    dy = dn * gy
    if c["post"]:
        dy = ry * (dy - y * (ry * ry) * (dy * y).mean(dim=1, keepdim=True))
    out.update(dx=(c["a"] * dH).to(t), dy=dy.to(t), dgy=dgy, dgo=dgo)
    if s.gate is not None:
        out["dgate"] = c["b"] * (dH * n).sum(dim=1)
    return out


def _append_plain(s):
    c = s.case
    p = s.pos.long() - 1
    at = s.table[s.seq.long(), p // c["page"]].long()
    for cache, rows in ((s.kc, s.k), (s.vc, s.v)):
        cache[at, :, p % c["page"]] = rows.reshape(-1, c["Hk"], c["D"])
    return dict(k=s.kc, v=s.vc)


def _decode_plain(s):
    c = s.case
    n, Hk, D, page = c["seqs"], c["Hk"], c["D"], c["page"]
    most = int(s.table.shape[1]) * page
    j = torch.arange(most, device=DEVICE)
    lens = s.lens.long()[:, None]
    seen = j[None, :] < lens
    if c["window"]:
        seen &= j[None, :] >= lens - c["window"]
    at = s.table.clamp(min=0).long()[:, j // page]
    out = []
    part = max(1, int(4e9 / (most * Hk * D * 4.0)))               # as many sequences at a time as lie side by side
    for i in range(0, n, part):
        w = seen[i:i + part]
        k, v = (x[at[i:i + part], :, (j % page)[None, :]].float() for x in (s.kc, s.vc))   # [n][key][head][D]
        q = s.q[i:i + part].float().reshape(-1, Hk, c["Hq"] // Hk, D)
        x = torch.einsum("bhgd,bjhd->bhgj", q, k) * D ** -0.5
        x = torch.where(w[:, None, None, :], x, -math.inf)
        top = x.amax(dim=-1, keepdim=True)
        e = torch.where(w[:, None, None, :], torch.exp(x - torch.where(top == -math.inf, 0.0, top)), 0.0)
        total = e.sum(dim=-1, keepdim=True)
        o = torch.einsum("bhgj,bjhd->bhgd", e / torch.where(total == 0.0, 1.0, total), v)
        out.append(o.reshape(o.shape[0], -1))
    return dict(o=torch.cat(out).to(s.q.dtype))


# ----------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    e = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "norm":
        n = float(case["N"]) * case["d"]
        # forward: x, y, h, o; backward: do, dh, dx, dy, and h and y as read by the forward's
        return dict(bytes=n * e * (8 if case["train"] else 4) + (8.0 * case["N"] if case["gate"] else 0.0),
                    flops=n * (34 if case["train"] else 9))
    lens = _lengths(case)
    if case["op"] == "append":
        rows = float(len(lens) if case["step"] else sum(lens))
        return dict(bytes=rows * (4.0 * case["Hk"] * case["D"] * e + 8.0), flops=rows)
    keys = float(sum(min(v, case["window"]) if case["window"] else v for v in lens))
    return dict(bytes=2.0 * e * case["D"] * (keys * case["Hk"] + len(lens) * case["Hq"]),
                flops=4.0 * keys * case["Hq"] * case["D"])


# ----------------------------------------------------------------------------- the definitions, in 64 bits
def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    return {"norm": _norm_exact, "append": _append_exact, "decode": _decode_exact}[case["op"]](s)


def _norm_exact(s):
    c, t = s.case, s.x.dtype
    N, d = s.x.shape
    gy, go = s.gy.double(), s.go.double()
    parts = {}
    dgy, dgo = (torch.zeros(d, dtype=torch.float64, device=DEVICE) for _ in range(2))
    for r0 in range(0, N, 16384):
        rows = slice(r0, min(N, r0 + 16384))
        y = s.y[rows].double()
        size = (y.square().sum(1, keepdim=True) / d + EPS).sqrt() if c["post"] else torch.ones_like(y[:, :1])
        branch = y / size * gy
        weight = torch.full_like(size, c["b"]) if s.gate is None else c["b"] * s.gate[rows].double()[:, None]
        h = c["a"] * s.x[rows].double() + weight * branch
        got = dict(h=h, o=h / (h.square().sum(1, keepdim=True) / d + EPS).sqrt() * go)
        if c["train"]:
            h = h.to(t).double()
            norm = (h.square().sum(1, keepdim=True) / d + EPS).sqrt()
            do = s.do[rows].double()
            dgo += (do * (h / norm)).sum(0)
            do = do * go
            dh = s.dh[rows].double() + do / norm - h * ((do * h).sum(1, keepdim=True) / d / norm ** 3)
            dn = weight * dh
            dgy += (dn * (y / size)).sum(0)
            dy = dn * gy
            if c["post"]:
                dy = dy / size - y * ((dy * y).sum(1, keepdim=True) / d / size ** 3)
            got.update(dx=c["a"] * dh, dy=dy)
            if s.gate is not None:
                got["dgate"] = c["b"] * (dh * branch).sum(1)
        for k, v in got.items():
            parts.setdefault(k, []).append(v)
    out = {k: torch.cat(v) for k, v in parts.items()}
    if c["train"]:
        out.update(dgy=dgy, dgo=dgo)
    return out


def _append_exact(s):
    """A row at a time on the host for few rows, a sequence at a time otherwise."""
    c = s.case
    page, Hk, D = c["page"], c["Hk"], c["D"]
    out = dict(k=s.kc.double(), v=s.vc.double())
    table = s.table.tolist()
    seq, pos = s.seq.tolist(), s.pos.tolist()
    i = 0
    while i < len(seq):                            # a run of rows of one page
        p = pos[i] - 1
        n = 1
        while i + n < len(seq) and seq[i + n] == seq[i] and pos[i + n] == pos[i] + n and (p + n) % page:
            n += 1
        for name, rows in (("k", s.k), ("v", s.v)):
            part = rows[i:i + n].double().reshape(n, Hk, D).transpose(0, 1)
            out[name][table[seq[i]][p // page], :, p % page:p % page + n] = part
        i += n
    return out


def _decode_exact(s):
    c = s.case
    Hq, Hk, D, page = c["Hq"], c["Hk"], c["D"], c["page"]
    out = torch.zeros(c["seqs"], Hq, D, dtype=torch.float64, device=DEVICE)
    for b, n in enumerate(s.lens.tolist()):
        if n == 0:
            continue
        ids = s.table[b, :(n + page - 1) // page].long()
        first = max(0, n - c["window"]) if c["window"] else 0
        k, v = (x[ids].double().transpose(0, 1).reshape(Hk, -1, D)[:, first:n] for x in (s.kc, s.vc))
        q = s.q[b].double().reshape(Hk, Hq // Hk, D)
        weight = torch.softmax(torch.bmm(q, k.transpose(1, 2)) / math.sqrt(D), dim=-1)
        out[b] = torch.bmm(weight, v).reshape(Hq, D)
    return dict(o=out.reshape(c["seqs"], -1))
