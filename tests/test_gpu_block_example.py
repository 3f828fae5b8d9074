"""The example that trains a block through the head: the block operators, the packed rows and the head together.

The first update's gradients against float64 autograd of the whole chain (block, dropout by the oracle's masks, head,
surrogate at ratio 1), on the same bf16 weights and rows. Every tensor that passes between the steps is rounded to bf16
(unit roundoff 2^-8, some ten of them on the way back, averaging over the sums): 2-norm within 2e-2, the tolerance of the head's
own gradients; a missing branch, rotation or mask is off by more than 0.1. Then the loss falls."""
import importlib.util
import os

import pytest
import torch

from oracle import block as ob

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    spec = importlib.util.spec_from_file_location("block_update", os.path.join(ROOT, "examples", "block_update.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def _chain(f, w, x):
    """The surrogate's loss at ratio 1: its gradient is that of -weight * logp."""
    b = f["block"]
    Hq, Hk, D = b.Hq, b.Hk, b.D
    pos, traj = f["pos"].cpu().numpy(), f["traj"].cpu().numpy()
    a = torch.from_numpy(ob.rope_angles(pos - 1, D, 10000.0)).cuda()
    cs, sn = torch.cos(a)[:, None], torch.sin(a)[:, None]
    scale = 65536.0 / (65536 - ob.keep_cut(f["p"]))
    masks = [torch.from_numpy(ob.keep_mask(traj, pos, x.shape[1], f["p"], b.seed, f["step"], i)).cuda() * scale
             for i in range(2)]

    def head(t, H, gain):
        t = t.view(-1, H, D)
        t = t / torch.sqrt(t.square().mean(-1, keepdim=True) + 1e-6) * gain
        u, v = t[..., :D // 2], t[..., D // 2:]
        return torch.cat([u * cs - v * sn, u * sn + v * cs], dim=-1).flatten(1)

    qkv = x @ w["qkv"].T
    q, k, v = qkv.split([Hq * D, Hk * D, Hk * D], dim=1)
    q, k = head(q, Hq, w["gq"]), head(k, Hk, w["gk"])
    out = []
    for i, j in zip(f["cu"][:-1], f["cu"][1:]):
        n = j - i
        qs = q[i:j].view(n, Hq, D).transpose(0, 1)
        ks, vs = (t[i:j].view(n, Hk, D).transpose(0, 1).repeat_interleave(Hq // Hk, dim=0) for t in (k, v))
        s = (qs @ ks.transpose(1, 2)) / D ** 0.5
        s = s.masked_fill(torch.ones(n, n, dtype=torch.bool, device="cuda").triu(1), float("-inf"))
        out.append((torch.softmax(s, -1) @ vs).transpose(0, 1).reshape(n, -1))
    h = x + masks[0] * (torch.cat(out) @ w["o"].T)
    g = h @ w["gate"].T
    h = h + masks[1] * ((g * torch.sigmoid(g) * (h @ w["up"].T)) @ w["down"].T)
    logp = torch.log_softmax(h @ f["W"].double().T, dim=1).gather(1, f["tok"].long()[:, None])[:, 0]
    return -(f["weight"].double() * logp).sum()


def test_gradients_and_loss():
    losses, f = _example().run(updates=4)
    w = {k: t.double().requires_grad_() for k, t in f["w"].items()}
    x = f["x"].double().requires_grad_()
    want = torch.autograd.grad(_chain(f, w, x), [x, *w.values()])
    for name, got, exact in zip(["x", *w], [f["dx"], *(f["grads"][k] for k in w)], want):
        off = (torch.linalg.norm(got.double() - exact) / torch.linalg.norm(exact)).item()
        print(name, off)
        assert off < 2e-2, (name, off)
    assert all(b < a for a, b in zip(losses, losses[1:])), losses
