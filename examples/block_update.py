"""A policy block trained through the head: the packed-prefix update with one transformer block under it.

The rows that the cutoffs keep pass a block -- attention over each completion's prefix, with normed and rotated
queries and keys, and a gated feed-forward block, dropout on both residual branches -- and then the LM head's
clipped surrogate. dH from the head goes back through the block. Only the kept prefixes are computed: the attention
is causal, so a row needs nothing after it.

    python examples/block_update.py [--updates 3]

The library runs the cutoffs, the packing, the norms and rotations, the dropouts, the feed-forward block and the
head; the projections and the attention itself are plain torch. The masks are a function of (seed, step, completion,
position): the updates on one batch keep the step, so they all see the masks under which the old log-probabilities
were taken, and the ratio moves with the weights alone.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2606_29758_gb300 import (FFNShape, GatedFFN, PassShape, QKNormRope, QKShape, RowDropout, UpdatePass,  # noqa: E402
                                    rope_table)
from synthetic import get_config, make_batch  # noqa: E402

BF16 = torch.bfloat16


def attention(q, k, v, cu, Hq, Hk, D):
    """Causal attention within each completion's rows [cu[i], cu[i+1]); heads of queries share keys in groups."""
    out = []
    for a, b in zip(cu[:-1], cu[1:]):
        n = b - a
        qs = q[a:b].view(n, Hq, D).transpose(0, 1).float()
        ks, vs = (t[a:b].view(n, Hk, D).transpose(0, 1).float().repeat_interleave(Hq // Hk, dim=0) for t in (k, v))
        s = qs @ ks.transpose(1, 2) / D ** 0.5
        s = s.masked_fill(torch.ones(n, n, dtype=torch.bool, device=s.device).triu(1), float("-inf"))
        out.append((torch.softmax(s, dim=-1) @ vs).transpose(0, 1).reshape(n, Hq * D))
    return torch.cat(out).to(q.dtype)


class PolicyBlock:
    """x -> x + drop(attention(x) Wo^T) =: h -> h + drop(ffn(h)), and its gradients, over packed rows."""

    def __init__(self, rows, d, F, Hq, Hk, D, T, p=0.1, seed=1, device="cuda"):
        g = torch.Generator(device=device).manual_seed(seed)
        w = lambda *s: (torch.randn(*s, device=device, generator=g) * 0.5 / s[-1] ** 0.5).to(BF16)  # noqa: E731
        self.Hq, self.Hk, self.D, self.seed = Hq, Hk, D, seed
        self.w = dict(qkv=w((Hq + 2 * Hk) * D, d), o=w(d, Hq * D), gate=w(F, d), up=w(F, d), down=w(d, F),
                      gq=torch.ones(D, dtype=BF16, device=device), gk=torch.ones(D, dtype=BF16, device=device))
        self.qk = QKNormRope(QKShape(rows, Hq, Hk, D, D), rope_table(T, D, device=device), device)
        self.ffn = GatedFFN(FFNShape(rows, d, F), device)
        self.drops = [RowDropout(p, site=i) for i in range(2)]      # one site per branch

    def forward(self, x, traj, pos, cu, step):
        w, nq, nk = self.w, self.Hq * self.D, self.Hk * self.D
        qkv = x @ w["qkv"].t()
        q, k, v = qkv[:, :nq], qkv[:, nq:nq + nk], qkv[:, nq + nk:]
        heads = [t.detach().requires_grad_() for t in (*self.qk.forward(q, k, w["gq"], w["gk"], pos), v)]
        with torch.enable_grad():
            att = attention(*heads, cu, self.Hq, self.Hk, self.D)
        h = self.drops[0].forward(att.detach() @ w["o"].t(), traj, pos, self.seed, step, res=x)
        y = self.ffn.forward(h, w["gate"], w["up"], w["down"])
        self.saved = (x, traj, pos, step, q, k, heads, att, h)
        return self.drops[1].forward(y, traj, pos, self.seed, step, res=h)

    def backward(self, dout):
        """dx and the weights' gradients from the gradient of the block's output rows."""
        w = self.w
        x, traj, pos, step, q, k, heads, att, h = self.saved
        dy = self.drops[1].backward(dout, traj, pos, self.seed, step)
        dh, dgate, dup, ddown = self.ffn.backward(dy, h, w["gate"], w["up"], w["down"])
        dh = dh + dout
        do = self.drops[0].backward(dh, traj, pos, self.seed, step)
        dqn, dkn, dv = torch.autograd.grad(att, heads, do @ w["o"])
        dq, dk, dgq, dgk = self.qk.backward(dqn, dkn, q, k, w["gq"], w["gk"], pos)
        dqkv = torch.cat([dq, dk, dv], dim=1)
        grads = dict(qkv=dqkv.t() @ x, o=do.t() @ att.detach(), gate=dgate, up=dup, down=ddown, gq=dgq, gk=dgk)
        return dqkv @ w["qkv"] + dh, grads

    def check_status(self):
        self.qk.check_status()
        self.ffn.check_status()


def run(updates=3, lr=0.01, p=0.1):
    """Updates of the block on one batch; returns the losses, and what the first update saw and computed."""
    cfg = get_config("mid")
    b = make_batch(cfg, device="cuda")
    D = b.dev
    up = UpdatePass(PassShape(cfg.P, cfg.K, b.T_max, cfg.d, cfg.V, b.total_len, BF16), eps=cfg.eps,
                    loss_scale=cfg.loss_scale)
    up.sample(D["q"], D["L"], cfg.seed, cfg.step)
    N = up.pack(D["L"], D["R"], D["tok_full"], D["oldlogp_full"], D["hid_full"])
    x, traj, pos = up.hid[:N].clone(), up.row_traj[:N], up.row_pos[:N]
    cu = [a for i, a in enumerate(up.cu_seqlens.tolist()) if i == 0 or a > up.cu_seqlens[i - 1]]
    block = PolicyBlock(b.total_len, cfg.d, 1048, 4, 2, 96, b.T_max, p)
    losses, first = [], {}
    for i in range(updates):
        up.hid[:N].copy_(block.forward(x, traj, pos, cu, cfg.step))
        if i == 0:                     # the policy that rolled out is the one before the first update
            up.forward(D["W"])
            up.oldlogp[:N].copy_(up.logp[:N])
        up.forward(D["W"])
        up.backward(D["W"])
        dx, grads = block.backward(up.dH[:N].to(BF16))
        losses.append(up.loss.item())
        if i == 0:
            first = dict(x=x, traj=traj.clone(), pos=pos.clone(), cu=cu, W=D["W"], tok=up.tok[:N].clone(),
                         weight=(up.adv[:N] * up.w[:N] * up.loss_scale).clone(), dx=dx, grads={k: g.clone() for k, g in grads.items()},
                         w={k: t.clone() for k, t in block.w.items()}, block=block, step=cfg.step, p=p)
        for k, g in grads.items():
            block.w[k] -= (lr * g).to(BF16)
    up.check_status()
    block.check_status()
    return losses, first


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--updates", type=int, default=3)
    losses, first = run(ap.parse_args().updates)
    print(f"{first['x'].shape[0]} packed rows; loss " + " -> ".join(f"{v:.5f}" for v in losses))


if __name__ == "__main__":
    main()
