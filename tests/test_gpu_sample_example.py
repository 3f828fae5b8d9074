"""The example that samples from a block: norms, rotation, cache, attention and feed-forward block together, step after step.

The last step's rows against float64 of the whole block over each completion's tokens at once (causal attention, no cache), on the
same bf16 weights. Between the row and the output lie ten tensors rounded to bf16 (the two normed rows, q k v, the heads, attention,
its projection, h, the product in the feed-forward block, its output, the row): 2^-8 at most and 0.4 of that in the mean of squares
each, 5e-3 in all if they are independent: 2-norm within 2e-2. Another completion's pages, a missing norm or a wrong position is off by
more than 0.1."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    spec = importlib.util.spec_from_file_location("block_sample", os.path.join(ROOT, "examples", "block_sample.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def _last_row(block, x):
    """The block's output for the last of a sequence's rows x [n][d]."""
    w = {k: t.double() for k, t in block.w.items()}
    Hq, Hk, D, n = block.Hq, block.Hk, block.D, len(x)
    norm = lambda t, g: t / torch.sqrt(t.square().mean(-1, keepdim=True) + 1e-6) * g  # noqa: E731
    a = torch.arange(n, device="cuda", dtype=torch.float64)[:, None] * 10000.0 ** (
        -2 * torch.arange(D // 2, device="cuda", dtype=torch.float64) / D)
    cs, sn = torch.cos(a)[:, None], torch.sin(a)[:, None]

    def head(t, gain):
        t = norm(t.view(n, -1, D), gain)
        u, v = t[..., :D // 2], t[..., D // 2:]
        return torch.cat([u * cs - v * sn, u * sn + v * cs], dim=-1).transpose(0, 1)
    q, k, v = (norm(x, w["n0"]) @ w["qkv"].T).split([Hq * D, Hk * D, Hk * D], dim=1)
    q, k, v = head(q, w["gq"]), head(k, w["gk"]), v.view(n, Hk, D).transpose(0, 1)
    s = q[:, -1:] @ k.repeat_interleave(Hq // Hk, dim=0).transpose(1, 2) / D ** 0.5
    att = (torch.softmax(s, -1) @ v.repeat_interleave(Hq // Hk, dim=0)).reshape(1, Hq * D)
    h = x[-1:] + norm(att @ w["o"].T, w["n1"])
    o = norm(h, w["n2"])
    g = o @ w["gate"].T
    return (h + norm((g * torch.sigmoid(g) * (o @ w["up"].T)) @ w["down"].T, w["n3"]))[0]


@pytest.mark.parametrize("capture", [False, True])
@pytest.mark.parametrize("steps,prompts,K", [(24, 3, 4), (1, 1, 1), (70, 2, 3)])
def test_the_last_step(steps, prompts, K, capture):
    block, table, tokens, rows = _example().run(steps, prompts, K, capture=capture)
    assert len(tokens) == prompts * K and block.cache.lengths.tolist() == [len(t) for t in tokens]
    assert len({tuple(t.tolist()) for t in tokens}) == len(tokens)        # (sampled: completions differ)
    for b, t in enumerate(tokens):
        want = _last_row(block, table[t].double())
        off = (torch.linalg.norm(rows[b].double() - want) / torch.linalg.norm(want)).item()
        print(b, len(t), off)
        assert off < 2e-2, (b, len(t), off)
