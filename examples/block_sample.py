"""Completions sampled from a policy block: a paged cache of keys and values, and one token of every sequence a step.

Each prompt has K completions. A prompt's tokens go through the block into the pages of its first completion, the other
completions share those pages, and then all of them take a token a step: the norm before attention, queries, keys and
values, their norms and rotation, the new keys and values into the cache, attention over it, the residual sum with the
norm after attention and the one before the feed-forward block, the feed-forward block, and its norm and sum.

    python examples/block_sample.py [--steps 24]

The library runs the norms, the rotation, the cache, the attention and the feed-forward block; the projections, the head
and the choice of the tokens are plain torch. The step is captured in a CUDA graph: the lengths that it counts up, the
table of pages and the rows are read where they lie.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2606_29758_gb300 import (CacheShape, DecodeAttention, DecodeShape, FFNShape, GatedFFN, NormShape,  # noqa: E402
                                    PagedCache, QKNormRope, QKShape, ResidualNorm, rope_table)

BF16, I32 = torch.bfloat16, torch.int32


class SampleBlock:
    """x -> x + norm(attention(norm(x)) Wo^T) =: h -> h + norm(ffn(norm(h))), for one new token a sequence."""

    def __init__(self, seqs, d, F, Hq, Hk, D, max_len, page=16, seed=1, device="cuda"):
        g = torch.Generator(device=device).manual_seed(seed)
        w = lambda *s: (torch.randn(*s, device=device, generator=g) / s[-1] ** 0.5).to(BF16)  # noqa: E731
        gain = lambda n: (1 + 0.2 * torch.randn(n, device=device, generator=g)).to(BF16)  # noqa: E731
        self.Hq, self.Hk, self.D = Hq, Hk, D
        self.w = dict(qkv=w((Hq + 2 * Hk) * D, d), o=w(d, Hq * D), gate=w(F, d), up=w(F, d), down=w(d, F), gq=gain(D),
                      gk=gain(D), n0=gain(d), n1=gain(d), n2=gain(d), n3=gain(d))
        self.first = ResidualNorm(NormShape(seqs, d, train=False), device)
        self.middle = ResidualNorm(NormShape(seqs, d, train=False), device)
        self.last = ResidualNorm(NormShape(seqs, d, pre=False, train=False), device)
        self.qk = QKNormRope(QKShape(seqs, Hq, Hk, D, D, train=False), rope_table(max_len, D, device=device), device)
        self.ffn = GatedFFN(FFNShape(seqs, d, F, train=False), device)
        self.cache = PagedCache(CacheShape(seqs, seqs * -(-max_len // page), page, Hk, D, max_len), device)
        self.attention = DecodeAttention(DecodeShape(seqs, Hq, Hk, D), device)

    def step(self, x, row_seq):
        """Rows x [n][d] of the first n sequences' new tokens, which their lengths count already. row_seq: i, or -1 for a
        sequence without a new token (its row comes out all the same, and nobody wants it)."""
        w, n, nq, nk = self.w, x.shape[0], self.Hq * self.D, self.Hk * self.D
        pos = self.cache.lengths[:n]
        _, o = self.first.forward(x, go=w["n0"])
        qkv = o @ w["qkv"].t()
        q, k = self.qk.forward(qkv[:, :nq], qkv[:, nq:nq + nk], w["gq"], w["gk"], pos, in_place=True)
        self.cache.append(0, k, qkv[:, nq + nk:], row_seq, pos)
        att = self.attention.forward(q, self.cache)
        h, o = self.middle.forward(x, att @ w["o"].t(), w["n1"], w["n2"])
        return self.last.forward(h, self.ffn.forward(o, w["gate"], w["up"], w["down"]), w["n3"])[0]

    def check_status(self):
        for holder in (self.qk, self.ffn, self.cache, self.attention):
            holder.check_status()


def run(steps=24, prompts=3, K=4, d=256, F=520, V=1000, longest=40, capture=True, seed=0):
    """Returns the block, the embeddings, the tokens [prompts * K][length] and the rows out of the last step, whose new
    tokens are the last ones. Sequence k * prompts + p is completion k of prompt p."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = prompts * K
    block = SampleBlock(n, d, F, 4, 2, 64, longest + steps)
    cache, table = block.cache, torch.randn(V, d, device="cuda", generator=g).to(BF16)    # embeddings, and the head
    lens = torch.randint(5, longest + 1, (prompts,), device="cuda", generator=g).tolist()
    words = torch.randint(0, V, (prompts, longest), device="cuda", generator=g)
    seqs = torch.arange(n, dtype=I32, device="cuda")

    for p in range(prompts):                             # a prompt's tokens, into its first completion's pages
        cache.reserve(p, lens[p])
    has = torch.tensor(lens, dtype=I32, device="cuda")
    rows = torch.empty(n, d, dtype=BF16, device="cuda")
    for t in range(max(lens)):
        cache.lengths[:prompts] = has.clamp(max=t + 1)
        out = block.step(table[words[:, t]], torch.where(has > t, seqs[:prompts], -1))
        for p in range(prompts):
            if t == lens[p] - 1:
                rows[p::prompts] = out[p]
    for p in range(prompts):
        cache.share(p, range(p + prompts, n, prompts), lens[p])
    for b in range(n):
        cache.reserve(b, lens[b % prompts] + steps)
    cache.lengths.copy_(has.repeat(K))

    x = torch.empty(n, d, dtype=BF16, device="cuda")

    def step():
        cache.lengths.add_(1)
        rows.copy_(block.step(x, seqs))

    graph, new = None, []
    for t in range(steps):
        noise = -torch.log(-torch.log(torch.rand(n, V, device="cuda", generator=g).clamp(1e-6, 1 - 1e-6)))
        tokens = ((rows @ table.t()).float() / d + noise).argmax(dim=1)
        new.append(tokens)
        x.copy_(table[tokens])
        if graph is not None:
            graph.replay()
            continue
        step()
        if capture:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                step()
    block.check_status()
    new = torch.stack(new, dim=1)
    return block, table, [torch.cat([words[b % prompts, :lens[b % prompts]], new[b]]) for b in range(n)], rows


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=24)
    _, _, tokens, _ = run(ap.parse_args().steps)
    print(f"{len(tokens)} completions of {min(map(len, tokens))} to {max(map(len, tokens))} tokens, prompts among them")


if __name__ == "__main__":
    main()
