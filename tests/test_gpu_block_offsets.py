"""Rows further apart than 2^31 elements in all: the same bits as the rows side by side."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def _apart(rows, cols, pitch, dtype):
    """A [rows][cols] view of that pitch, and its values side by side."""
    wide = torch.empty(rows, pitch, dtype=dtype, device="cuda")
    assert wide.numel() > 2 ** 31
    g = torch.Generator(device="cuda").manual_seed(3)
    packed = torch.randn(rows, cols, device="cuda", generator=g).to(dtype)
    view = wide[:, pitch - cols:]
    view.copy_(packed)
    return view, packed


def test_qk():
    from paper_2606_29758_gb300 import QKNormRope, QKShape, rope_table
    N, Hq, Hk, D = 70000, 3, 1, 64
    rows, packed = _apart(N, (Hq + Hk) * D, 32768, torch.bfloat16)
    pos = (torch.arange(N, device="cuda", dtype=torch.int32) % 500) + 1
    g = torch.linspace(0.5, 1.5, D, device="cuda").to(torch.bfloat16)
    m = QKNormRope(QKShape(N, Hq, Hk, D, D), rope_table(500, D))
    part = lambda t: (t[:, :Hq * D], t[:, Hq * D:])  # noqa: E731
    near = [t.clone() for t in (*m.forward(*part(packed), g, g, pos), *m.backward(*part(packed), *part(packed), g, g, pos))]
    for a, b in zip((*m.forward(*part(rows), g, g, pos), *m.backward(*part(rows), *part(rows), g, g, pos)), near):
        assert torch.equal(a, b)
    m.forward(*part(rows), g, g, pos, in_place=True)
    assert torch.equal(part(rows)[0], near[0]) and torch.equal(part(rows)[1], near[1])


@pytest.mark.parametrize("cols", [256, 253])
def test_dropout(cols):
    from paper_2606_29758_gb300 import RowDropout
    N = 70000
    rows, packed = _apart(N, cols, 32768, torch.bfloat16)
    traj = torch.arange(N, device="cuda", dtype=torch.int32) // 100
    pos = (torch.arange(N, device="cuda", dtype=torch.int32) % 100) + 1
    d = RowDropout(0.2)
    want = d.forward(packed, traj, pos, 1, 2, res=packed)
    assert torch.equal(d.forward(rows, traj, pos, 1, 2, res=rows, out=rows), want)


def test_ffn():
    from paper_2606_29758_gb300 import FFNShape, GatedFFN
    N, d, F = 140, 64, 136
    rows, packed = _apart(N, d, 1 << 24, torch.bfloat16)
    g = torch.Generator(device="cuda").manual_seed(4)
    w = [(torch.randn(*s, device="cuda", generator=g) * 0.2).to(torch.bfloat16) for s in ((F, d), (F, d), (d, F))]
    m = GatedFFN(FFNShape(N, d, F))
    y = m.forward(packed, *w).clone()
    grads = [t.clone() for t in m.backward(packed, packed, *w)]
    assert torch.equal(m.forward(rows, *w), y)
    for a, b in zip(m.backward(rows, rows, *w), grads):
        assert torch.equal(a, b)
