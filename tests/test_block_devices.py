"""Tensors of the block operators on another device than the launch: refused by name, before the library is called. (The devices
are made up: none of these calls reaches a GPU.)"""
import pytest
import torch

BF, I32 = torch.bfloat16, torch.int32
HERE, OTHER = torch.device("cuda", 0), torch.device("cuda", 1)


class Rows:
    """What the holders look at of a contiguous tensor on `device`."""
    is_cuda = True

    def __init__(self, shape, dtype=BF, device=HERE):
        self.shape, self.dtype, self.device = torch.Size(shape), dtype, device

    def dim(self):
        return len(self.shape)

    def stride(self):
        return (self.shape[1], 1) if len(self.shape) == 2 else (1,)

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 1 << 20

    def __getitem__(self, rows):
        return self


@pytest.fixture()
def block(monkeypatch):
    from paper_2606_29758_gb300 import _build, block
    _build.build()
    monkeypatch.setattr(block, "_device", lambda: 0)
    monkeypatch.setattr(block, "_stream", lambda: 0)
    return block


class Call:
    """In a library entry's place."""
    def __init__(self):
        self.made = 0

    def __call__(self, *a):
        self.made += 1
        return 0


def _holders(block, at):
    """(name, entry, the call with one tensor's device changed, the names of its tensors) of each operator with buffers on `at`."""
    N, d, F, D = 3, 16, 24, 16
    ffn = block.GatedFFN(block.FFNShape(4, d, F), device="cpu")
    qk = block.QKNormRope(block.QKShape(4, 2, 1, D, 0), None, device="cpu")
    drop = block.RowDropout(0.5)
    ffn._at = qk._at = at
    ffn._fwd, ffn._bwd, qk._fwd, qk._bwd, drop._call = (Call() for _ in range(5))

    def on(names, which, device):
        return {n: Rows(s, t, device if n == which else at) for n, (s, t) in names.items()}
    block_in = dict(X=((N, d), BF), Wg=((F, d), BF), Wu=((F, d), BF), Wd=((d, F), BF))
    qk_in = dict(q=((N, 2 * D), BF), k=((N, D), BF), gq=((D,), BF), gk=((D,), BF))
    drop_in = dict(x=((N, d), BF), row_traj=((N,), I32), row_pos=((N,), I32), res=((N, d), BF), out=((N, d), BF))

    def ffn_fwd(which=None, device=None):
        t = on(dict(block_in, out=((N, d), BF)), which, device)
        return ffn.forward(t["X"], t["Wg"], t["Wu"], t["Wd"], out=t["out"])

    def ffn_bwd(which=None, device=None):
        t = on(dict(block_in, dY=((N, d), BF)), which, device)
        ffn.stored = N
        return ffn.backward(t["dY"], t["X"], t["Wg"], t["Wu"], t["Wd"])

    def qk_fwd(which=None, device=None):
        t = on(qk_in, which, device)
        return qk.forward(t["q"], t["k"], t["gq"], t["gk"], None)

    def qk_bwd(which=None, device=None):
        t = on(dict(qk_in, dq_out=((N, 2 * D), BF), dk_out=((N, D), BF)), which, device)
        return qk.backward(t["dq_out"], t["dk_out"], t["q"], t["k"], t["gq"], t["gk"], None)

    def dropout(which=None, device=None):
        t = on(drop_in, which, device)
        return drop.forward(t["x"], t["row_traj"], t["row_pos"], 1, 1, res=t["res"], out=t["out"])
    return [("ffn forward", ffn._fwd, ffn_fwd, [*block_in, "out"]), ("ffn backward", ffn._bwd, ffn_bwd, [*block_in, "dY"]),
            ("qk forward", qk._fwd, qk_fwd, list(qk_in)), ("qk backward", qk._bwd, qk_bwd, [*qk_in, "dq_out", "dk_out"]),
            ("dropout", drop._call, dropout, list(drop_in))]


def test_a_tensor_on_another_device(block):
    for name, entry, call, tensors in _holders(block, HERE):
        call()
        assert entry.made == 1, name
        for t in tensors:
            with pytest.raises(ValueError):
                call(t, OTHER)
            assert entry.made == 1, (name, t)


def test_everything_on_a_device_that_is_not_current(block):
    """The launch would go to the current device's stream."""
    for name, entry, call, _ in _holders(block, OTHER):
        with pytest.raises(ValueError):
            call()
        assert entry.made == 0, name


@pytest.mark.gpu
def test_small_calls_leave_another_device_to_the_holder():
    """Plans that name another device than the tensors' (their buffers' addresses are 0: nothing could be launched)."""
    from paper_2606_29758_gb300 import _binding
    c = _binding.calls()
    z = lambda *s, dt=BF: torch.zeros(*s, dtype=dt, device="cuda")  # noqa: E731
    q, x = z(3, 16), z(3, 8)
    here = torch.cuda.current_device()
    for at in (here + 1, -1):
        qk = c.qk_plan(4, 1, 1, 16, 0, 0, 0, 0, 1e-6, *[0] * 9, at)
        ffn = c.ffn_plan(4, 8, 8, 0, 0, 0, *[0] * 11, at)
        assert c.qk_fwd(qk, q, q, None, None, None, 1, False) is None
        assert c.qk_bwd(qk, q, q, q, q, None, None, None, 1, False) is None
        assert c.ffn_fwd(ffn, x, z(8, 8), z(8, 8), z(8, 8), None) is None
    qk = c.qk_plan(4, 1, 1, 16, 0, 0, 0, 0, 1e-6, *[0] * 9, here)
    assert c.qk_fwd(qk, q, q, None, None, None, 1, False) == _binding.PS_ERR_INVALID_ARG      # (the library's refusal)
