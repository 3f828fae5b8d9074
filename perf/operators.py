"""The row-wise operators of a policy block over packed prefix rows: their cases, plain forms and 64-bit forms.

  ffn      the gated feed-forward block: GatedFFN.forward and, in training, GatedFFN.backward
  qk       norms of queries and keys per head with the rotary positions: QKNormRope
  dropout  dropout of a branch's rows added to the residual rows, from a counter-based generator: RowDropout

Rows are those of a packed batch: completion after completion, each with the positions 1..n of its prefix.
Weights are N(0, 0.02), activations N(0, 1) with some loud channels, incoming gradients of very different size
per row (small advantages, large inverse-survival weights) with some rows 0, as where the clip binds.
"""
import math

import numpy as np
import torch

own = False
DEVICE = "cuda"
DTYPE = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS, THETA = 1e-6, 1e6
TABLE_ROWS = 16384


def listed():
    return [
        # One token of one completion through the feed-forward block of a 7B-shaped policy (d of the
        # benchmark's head): serving, bound by reading the weights.
        dict(name="ffn_token_7b", op="ffn", N=1, d=3584, F=16384, act="silu", train=False),
        # One sampling step of 128 completions (16 prompts x 8) of a 1.5B-shaped policy.
        dict(name="ffn_step_1.5b", op="ffn", N=128, d=1536, F=8192, act="silu", train=False),
        # A small policy with sizes that are a multiple of no tile, forward and backward: debugging, where
        # launches count.
        dict(name="ffn_train_mid", op="ffn", N=571, d=392, F=1048, act="gelu", train=True),
        # An ordinary micro-batch of the 1.5B-shaped policy, forward and backward.
        dict(name="ffn_train_1.5b", op="ffn", N=6030, d=1536, F=8192, act="silu", train=True),
        # One group of four ordinary completions of the 7B-shaped policy, forward and backward.
        dict(name="ffn_train_7b", op="ffn", N=7835, d=3584, F=16384, act="silu", train=True),
        # The queries and keys of one token, in serving.
        dict(name="qk_token_7b", op="qk", N=1, Hq=28, Hk=4, D=128, R=128, dtype="bf16", pairs="half", train=False),
        # A full-precision reference run: heads of 96, half of each rotated, neighbouring pairs.
        dict(name="qk_train_f32", op="qk", N=571, Hq=6, Hk=2, D=96, R=48, dtype="f32", pairs="even", train=True),
        # Half of the 7B-shaped benchmark batch, forward and backward.
        dict(name="qk_train_7b", op="qk", N=106000, Hq=28, Hk=4, D=128, R=128, dtype="bf16", pairs="half", train=True),
        # The residual branch of the smallest 7B-shaped micro-batch (two groups of short answers).
        dict(name="dropout_short_7b", op="dropout", N=185, d=3584, dtype="bf16", p=0.05, res=True),
        # f32 rows of an odd width.
        dict(name="dropout_f32", op="dropout", N=6330, d=771, dtype="f32", p=0.1, res=True),
        # Sixty thousand rows, about a third of the 7B-shaped benchmark batch.
        dict(name="dropout_7b", op="dropout", N=60000, d=3584, dtype="bf16", p=0.1, res=True),
    ]


def _log(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def draw(rng):
    """One more case of the ranges that the listed ones stand for."""
    op = rng.choice(["ffn", "ffn", "qk", "dropout"])
    if op == "ffn":
        d = int(_log(rng, 96, 3600)) // 8 * 8
        F = min(16384, int(d * rng.uniform(1.4, 5.4)) // 8 * 8)
        N = int(_log(rng, 1, 8000))
        return dict(op=op, N=N, d=d, F=F, act=rng.choice(["silu", "silu", "gelu"]), train=rng.random() < 0.6)
    if op == "qk":
        D = rng.choice([64, 80, 96, 128, 128, 192, 256])
        R = rng.choice([D, D, D // 32 * 16])
        Hq, Hk = rng.choice([(28, 4), (12, 2), (16, 16), (6, 2), (5, 1), (40, 8), (3, 0)])
        dtype = rng.choice(["bf16", "bf16", "f32"])
        most = 106000 * 32 * 128 * 2 / ((Hq + Hk) * D * (4 if dtype == "f32" else 2))
        return dict(op=op, N=int(_log(rng, 1, min(most, 106000))), Hq=Hq, Hk=Hk, D=D, R=R, dtype=dtype,
                    pairs=rng.choice(["half", "half", "even"]), train=rng.random() < 0.6)
    dtype = rng.choice(["bf16", "bf16", "f32"])
    d = int(_log(rng, 48, 8192))
    most = 60000 * 3584 * 2 / (d * (4 if dtype == "f32" else 2))
    return dict(op=op, N=int(_log(rng, 1, min(most, 200000))), d=d, dtype=dtype,
                p=round(rng.uniform(0.01, 0.5), 3), res=rng.random() < 0.75)


# ----------------------------------------------------------------------------- inputs
def _generator(seed):
    return torch.Generator(device=DEVICE).manual_seed(seed)


def _normal(shape, g, dtype=torch.bfloat16, scale=1.0):
    return (torch.randn(shape, device=DEVICE, generator=g) * scale).to(dtype)


def _activations(N, d, g, dtype=torch.bfloat16):
    x = torch.randn(N, d, device=DEVICE, generator=g)
    x[:, torch.randint(0, d, (max(1, d // 100),), device=DEVICE, generator=g)] *= 8.0
    return x.to(dtype)


def _gradients(N, d, g, dtype=torch.bfloat16):
    size = torch.exp(torch.randn(N, 1, device=DEVICE, generator=g)) * 1e-3
    size *= torch.rand(N, 1, device=DEVICE, generator=g) > 0.1 if N > 1 else 1.0
    return (torch.randn(N, d, device=DEVICE, generator=g) * size).to(dtype)


def _packed(N, seed):
    """Completion and 1-based position of each of N packed rows; a single row is some way into its completion."""
    rng = np.random.default_rng([seed, 9])
    if N == 1:
        return (torch.full((1,), int(rng.integers(0, 64)), dtype=torch.int32, device=DEVICE),
                torch.full((1,), int(rng.integers(1, TABLE_ROWS + 1)), dtype=torch.int32, device=DEVICE))
    n = np.minimum(np.maximum(1, np.rint(np.exp(math.log(max(2.0, min(1024.0, N / 6))) +
                                                0.5 * rng.standard_normal(N)))), TABLE_ROWS).astype(np.int64)
    n = n[:int(np.searchsorted(np.cumsum(n), N)) + 1]
    n[-1] -= n.sum() - N
    start = np.cumsum(n) - n
    traj = np.repeat(np.arange(len(n)), n)
    pos = np.arange(N) - np.repeat(start, n) + 1
    return (torch.from_numpy(traj.astype(np.int32)).to(DEVICE), torch.from_numpy(pos.astype(np.int32)).to(DEVICE))


def _table(T, R):
    """cos and sin of position t (from 0) and pair i, f32 [T][R/2][2]."""
    i = torch.arange(R // 2, device=DEVICE, dtype=torch.float64)
    a = torch.arange(T, device=DEVICE, dtype=torch.float64)[:, None] * THETA ** (-2.0 * i / R)
    return torch.stack([torch.cos(a), torch.sin(a)], dim=2).float()


class State:
    pass


def prepare(case, seed):
    s = State()
    s.case, op = case, case["op"]
    g = _generator(seed)
    if op == "ffn":
        N, d, F = case["N"], case["d"], case["F"]
        s.x = _activations(N, d, g)
        s.wg, s.wu, s.wd = (_normal(shape, g, scale=0.02) for shape in ((F, d), (F, d), (d, F)))
        s.dy = _gradients(N, d, g) if case["train"] else None
        if own:
            from paper_2606_29758_gb300 import PS_ACT_GELU, PS_ACT_SILU, FFNShape, GatedFFN
            s.ffn = GatedFFN(FFNShape(rows=N, d=d, F=F, act=PS_ACT_GELU if case["act"] == "gelu" else PS_ACT_SILU,
                                      train=case["train"], dx_dtype=torch.bfloat16, dw_dtype=torch.bfloat16))
        return s
    s.traj, s.pos = _packed(case["N"], seed)
    if op == "qk":
        N, Hq, Hk, D, R = (case[k] for k in ("N", "Hq", "Hk", "D", "R"))
        t = DTYPE[case["dtype"]]
        # queries and keys lie in one projection's rows, followed by as many values as keys
        qkv = _activations(N, (Hq + 2 * Hk) * D, g, t)
        s.q, s.k = qkv[:, :Hq * D], qkv[:, Hq * D:(Hq + Hk) * D]
        s.gq, s.gk = ((1.0 + 0.3 * torch.randn(D, device=DEVICE, generator=g)).to(t) for _ in range(2))
        s.table = _table(TABLE_ROWS, R)
        if case["train"]:
            s.dq, s.dk = _gradients(N, Hq * D, g, t), _gradients(N, Hk * D, g, t)
        if own:
            from paper_2606_29758_gb300 import QKNormRope, QKShape
            s.op = QKNormRope(QKShape(rows=N, Hq=Hq, Hk=Hk, D=D, R=R, dtype=t, interleaved=case["pairs"] == "even",
                                      eps=EPS, train=case["train"]), s.table)
        return s
    t = DTYPE[case["dtype"]]
    s.x = _activations(case["N"], case["d"], g, t)
    s.res = _activations(case["N"], case["d"], g, t) if case["res"] else None
    s.dy = _gradients(case["N"], case["d"], g, t)
    s.seed, s.step, s.site, s.traj_base = seed * 2654435761 + 12345, 3 + seed % 5, 7, 1000
    if own:
        from paper_2606_29758_gb300 import RowDropout
        s.op = RowDropout(case["p"], site=s.site)
    return s


def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    case = s.case
    if case["op"] == "ffn":
        out = dict(y=s.ffn.forward(s.x, s.wg, s.wu, s.wd))
        if case["train"]:
            out["dx"], out["dwg"], out["dwu"], out["dwd"] = s.ffn.backward(s.dy, s.x, s.wg, s.wu, s.wd)
        return out
    if case["op"] == "qk":
        out = dict(zip(("q", "k"), s.op.forward(s.q, s.k, s.gq, s.gk, s.pos, pos_base=1)))
        if case["train"]:
            out.update(zip(("dq", "dk", "dgq", "dgk"),
                           s.op.backward(s.dq, s.dk, s.q, s.k, s.gq, s.gk, s.pos, pos_base=1)))
        return out
    return dict(y=s.op.forward(s.x, s.traj, s.pos, s.seed, s.step, res=s.res, traj_base=s.traj_base),
                dx=s.op.backward(s.dy, s.traj, s.pos, s.seed, s.step, traj_base=s.traj_base))


# ----------------------------------------------------------------------------- the plain forms, in 32 bits
def _run_plain(s):
    return {"ffn": _ffn_plain, "qk": _qk_plain, "dropout": _dropout_plain}[s.case["op"]](s)


def _act_plain(g, act):
    """s(g) and s'(g)."""
    if act == "silu":
        e = 1.0 / (1.0 + torch.exp(-g))
        return g * e, e * (1.0 + g * (1.0 - e))
    c = 0.5 * (1.0 + torch.erf(g * math.sqrt(0.5)))
    return g * c, c + g * torch.exp(-0.5 * g * g) * (1.0 / math.sqrt(2.0 * math.pi))


def _ffn_plain(s):
    x, wg, wu, wd = (v.float() for v in (s.x, s.wg, s.wu, s.wd))
    t = s.x.dtype
    g, u = x @ wg.T, x @ wu.T
    q, slope = _act_plain(g, s.case["act"])
    a = q * u
    out = dict(y=(a @ wd.T).to(t))
    if s.case["train"]:
        dy = s.dy.float()
        da = dy @ wd
        du, dg = da * q, da * u * slope
        out.update(dx=(dg @ wg + du @ wu).to(t), dwg=(dg.T @ x).to(t), dwu=(du.T @ x).to(t), dwd=(dy.T @ a).to(t))
    return out


def _pairs(x, R, pairs):
    """The two members of each rotated pair, and the dims that are not rotated."""
    rot, rest = x[..., :R], x[..., R:]
    if pairs == "half":
        return rot[..., :R // 2], rot[..., R // 2:], rest
    return rot[..., 0::2], rot[..., 1::2], rest


def _joined(a, b, rest, pairs):
    rot = torch.cat([a, b], dim=-1) if pairs == "half" else torch.stack([a, b], dim=-1).flatten(-2)
    return torch.cat([rot, rest], dim=-1)


def _qk_part(x, gain, dy, cs, sn, D, R, pairs):
    n, t = x.shape[0], x.dtype
    x, gain = x.float().reshape(n, -1, D), gain.float()
    r = torch.rsqrt((x * x).mean(dim=-1, keepdim=True) + EPS)
    a, b, rest = _pairs(x * r * gain, R, pairs)
    y = _joined(a * cs - b * sn, a * sn + b * cs, rest, pairs).reshape(n, -1).to(t)
    if dy is None:
        return y, None, None
    a, b, rest = _pairs(dy.float().reshape(n, -1, D), R, pairs)
    dn = _joined(a * cs + b * sn, b * cs - a * sn, rest, pairs)
    dgain = (dn * (x * r)).sum(dim=(0, 1))
    dn = dn * gain
    dx = r * (dn - x * (r * r) * (dn * x).mean(dim=-1, keepdim=True))
    return y, dx.reshape(n, -1).to(t), dgain


def _qk_plain(s):
    c = s.case
    at = s.table[s.pos.long() - 1]
    cs, sn = at[:, None, :, 0], at[:, None, :, 1]
    dq, dk = (s.dq, s.dk) if c["train"] else (None, None)
    q, dq, dgq = _qk_part(s.q, s.gq, dq, cs, sn, c["D"], c["R"], c["pairs"])
    k, dk, dgk = _qk_part(s.k, s.gk, dk, cs, sn, c["D"], c["R"], c["pairs"])
    return dict(q=q, k=k, dq=dq, dk=dk, dgq=dgq, dgk=dgk) if c["train"] else dict(q=q, k=k)


def _round_of(c, k0, k1):
    """One round of Philox4x32 on words held in 64 bits (a product wraps to its exact 64 low bits)."""
    p0, p1 = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
    lo, hi = 0xFFFFFFFF, 32
    return [((p1 >> hi) & lo) ^ c[1] ^ k0, p1 & lo, ((p0 >> hi) & lo) ^ c[3] ^ k1, p0 & lo]


def _keep_plain(s, d):
    """Which of N x d values are kept: 16 bits of the generator each, eight to a block."""
    n, blocks = s.traj.shape[0], -(-d // 8)
    lo = 0xFFFFFFFF
    c = [(s.site * 65536 + torch.arange(blocks, device=DEVICE, dtype=torch.int64))[None, :].expand(n, blocks),
         (s.pos.long() & lo)[:, None], ((s.traj.long() + s.traj_base) & lo)[:, None],
         torch.full((1, 1), s.step & lo, dtype=torch.int64, device=DEVICE)]
    k0, k1 = s.seed & lo, (s.seed >> 32) & lo
    c = _round_of(c, k0, k1)
    c = _round_of(c, k0 + 0x9E3779B9 & lo, k1 + 0xBB67AE85 & lo)
    c = _round_of(c, k0 + 2 * 0x9E3779B9 & lo, k1 + 2 * 0xBB67AE85 & lo)
    c = _round_of(c, k0 + 3 * 0x9E3779B9 & lo, k1 + 3 * 0xBB67AE85 & lo)
    c = _round_of(c, k0 + 4 * 0x9E3779B9 & lo, k1 + 4 * 0xBB67AE85 & lo)
    c = _round_of(c, k0 + 5 * 0x9E3779B9 & lo, k1 + 5 * 0xBB67AE85 & lo)
    c = _round_of(c, k0 + 6 * 0x9E3779B9 & lo, k1 + 6 * 0xBB67AE85 & lo)
    c = _round_of(c, k0 + 7 * 0x9E3779B9 & lo, k1 + 7 * 0xBB67AE85 & lo)
    c = _round_of(c, k0 + 8 * 0x9E3779B9 & lo, k1 + 8 * 0xBB67AE85 & lo)
    c = _round_of(c, k0 + 9 * 0x9E3779B9 & lo, k1 + 9 * 0xBB67AE85 & lo)
    u = torch.stack([c[0] & 0xFFFF, c[0] >> 16, c[1] & 0xFFFF, c[1] >> 16, c[2] & 0xFFFF, c[2] >> 16,
                     c[3] & 0xFFFF, c[3] >> 16], dim=2)
    return u.reshape(n, blocks * 8)[:, :d] >= _threshold(s.case["p"])


def _threshold(p):
    return int(math.floor(p * 65536.0 + 0.5))


def _dropout_plain(s):
    keep = _keep_plain(s, s.case["d"])
    scale = 65536.0 / (65536 - _threshold(s.case["p"]))
    y = torch.where(keep, s.x.float() * scale, 0.0)
    if s.res is not None:
        y = s.res.float() + y
    return dict(y=y.to(s.x.dtype), dx=torch.where(keep, s.dy.float() * scale, 0.0).to(s.x.dtype))


# ----------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    if case["op"] == "ffn":
        N, d, F = case["N"], case["d"], case["F"]
        # x and y (and dy, dx), the weights (and their gradients), two bytes each
        rows, weights = 2.0 * N * d * 2, 3.0 * d * F * 2
        return dict(bytes=(rows + weights) * (2 if case["train"] else 1),
                    flops=(18.0 if case["train"] else 6.0) * N * d * F)
    e = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "qk":
        n = float(case["N"]) * (case["Hq"] + case["Hk"]) * case["D"]
        # forward: x, y; backward: x is read with the forward's, dy, dx
        return dict(bytes=n * e * (4 if case["train"] else 2) + case["N"] * 4.0, flops=n * (20 if case["train"] else 8))
    n = float(case["N"]) * case["d"]
    return dict(bytes=n * e * (5 if case["res"] else 4) + case["N"] * 8.0, flops=n * 12)


# ----------------------------------------------------------------------------- the definitions, in 64 bits
def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    if case["op"] == "ffn":
        return _ffn_exact(s) if 18.0 * case["N"] * case["d"] * case["F"] <= 1.2e13 else None
    return _qk_exact(s) if case["op"] == "qk" else _dropout_exact(s)


def _ffn_exact(s):
    x, wg, wu, wd = (v.double() for v in (s.x, s.wg, s.wu, s.wd))
    g, u = torch.mm(x, wg.t()), torch.mm(x, wu.t())
    if s.case["act"] == "silu":
        gate = g * torch.sigmoid(g)
        slope = torch.sigmoid(g) + gate * torch.sigmoid(-g)
    else:
        cdf = 0.5 * torch.erfc(-g / math.sqrt(2.0))
        gate, slope = g * cdf, cdf + g * torch.exp(-g.square() / 2) / math.sqrt(2 * math.pi)
    out = dict(y=torch.mm(gate * u, wd.t()))
    if s.case["train"]:
        dy = s.dy.double()
        dwd = torch.mm(dy.t(), gate * u)
        da = torch.mm(dy, wd)
        du = da * gate
        dg = da.mul_(u).mul_(slope)
        out.update(dx=torch.mm(dg, wg) + torch.mm(du, wu), dwg=torch.mm(dg.t(), x), dwu=torch.mm(du.t(), x), dwd=dwd)
    return out


def _qk_exact(s):
    c = s.case
    D, R = c["D"], c["R"]
    i = torch.arange(R // 2, device=DEVICE, dtype=torch.float64)
    turn = torch.polar(torch.ones((), device=DEVICE, dtype=torch.float64),
                       (s.pos.double() - 1)[:, None] * THETA ** (-2.0 * i / R))
    first = torch.arange(R // 2, device=DEVICE) * (1 if c["pairs"] == "half" else 2)
    second = first + (R // 2 if c["pairs"] == "half" else 1)

    def rotated(v, by):
        z = torch.complex(v[..., first], v[..., second]) * by[:, None]
        v = v.clone()
        v[..., first], v[..., second] = z.real, z.imag
        return v

    out = {}
    for name, x, gain in (("q", s.q, s.gq), ("k", s.k, s.gk)):
        # a part of the rows at a time, so that the largest case fits
        ys, dxs, dgain = [], [], torch.zeros(D, dtype=torch.float64, device=DEVICE)
        dy = getattr(s, "d" + name, None)
        for r0 in range(0, c["N"], 16384):
            rows = slice(r0, min(c["N"], r0 + 16384))
            v, w = x[rows].double().unflatten(1, (-1, D)) if x.shape[1] else None, gain.double()
            if v is None:
                break
            norm = torch.sqrt(v.square().mean(-1, keepdim=True) + EPS)
            ys.append(rotated(v / norm * w, turn[rows]).flatten(1))
            if dy is not None:
                back = rotated(dy[rows].double().unflatten(1, (-1, D)), turn[rows].conj())
                dgain += (back * v / norm).sum((0, 1))
                back = back * w
                dxs.append((back / norm - v * (back * v).mean(-1, keepdim=True) / norm ** 3).flatten(1))
        out[name] = torch.cat(ys) if ys else x.double()
        if dy is not None:
            out["d" + name], out["dg" + name] = torch.cat(dxs) if dxs else x.double(), dgain
    return out


def _dropout_exact(s):
    """The generator by 32-bit words of numpy, a part of the rows at a time."""
    N, d = s.x.shape
    blocks = (d + 7) // 8
    cut = _threshold(s.case["p"])
    scale = 65536.0 / (65536.0 - cut)
    traj, pos = s.traj.cpu().numpy().astype(np.uint64), s.pos.cpu().numpy().astype(np.uint64)
    y, dx = (torch.empty(N, d, dtype=torch.float64, device=DEVICE) for _ in range(2))
    part = max(1, 400000 // blocks)
    low = np.uint64(0xFFFFFFFF)
    for r0 in range(0, N, part):
        r1 = min(N, r0 + part)
        shape = (r1 - r0, blocks)
        w = [np.broadcast_to(np.uint64(s.site << 16) + np.arange(blocks, dtype=np.uint64), shape),
             np.broadcast_to(pos[r0:r1, None], shape),
             np.broadcast_to((traj[r0:r1, None] + np.uint64(s.traj_base)) & low, shape),
             np.full(shape, s.step, dtype=np.uint64)]
        key = [s.seed & 0xFFFFFFFF, (s.seed >> 32) & 0xFFFFFFFF]
        for _ in range(10):
            a, b = np.uint64(0xD2511F53) * w[0], np.uint64(0xCD9E8D57) * w[2]
            w = [(b >> np.uint64(32)) ^ w[1] ^ np.uint64(key[0]), b & low,
                 (a >> np.uint64(32)) ^ w[3] ^ np.uint64(key[1]), a & low]
            key = [(key[0] + 0x9E3779B9) & 0xFFFFFFFF, (key[1] + 0xBB67AE85) & 0xFFFFFFFF]
        words = np.stack([v.astype("<u4") for v in w], axis=-1).view("<u2")
        kept = torch.from_numpy(words.reshape(r1 - r0, blocks * 8)[:, :d] >= cut).to(DEVICE)
        y[r0:r1] = s.x[r0:r1].double() * scale * kept
        dx[r0:r1] = s.dy[r0:r1].double() * scale * kept
    if s.res is not None:
        y += s.res.double()
    return dict(y=y, dx=dx)
