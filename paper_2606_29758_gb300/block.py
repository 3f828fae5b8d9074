"""Row-wise operators of a policy block over packed rows, with buffers held in torch.

GatedFFN, QKNormRope and RowDropout run the library's calls of the same names on the current stream. Their
rows are those of a packed batch (UpdatePass.pack: src_row, row_traj, row_pos, cu_seqlens), so they carry the
head's dH into the policy's body and prepare its rows for the head. Each call takes the first N = x.shape[0] rows
of the buffers it was built for; the tensors it returns are views of those buffers, overwritten by its next call.
Every tensor of a call is on the current device, where the holder's buffers are.
"""
from __future__ import annotations

from dataclasses import dataclass
from typing import Optional

import torch

from . import _binding as B


# the current stream's raw handle; the tensors that a call was given are on the device already, so torch is set up
_raw_stream, _device = (getattr(torch._C, n, None) for n in ("_cuda_getCurrentRawStream", "_cuda_getDevice"))
_device = _device or torch.cuda.current_device
_stream = (lambda: _raw_stream(_device())) if _raw_stream else B._stream

_CODE = {torch.bfloat16: B.PS_DTYPE_BF16, torch.float32: B.PS_DTYPE_F32}


# The checks of a call's ordinary way, before a pointer is taken: one comparison of what a right call has, and the reason after
# it fails. (Calls in order go by B.calls(), which compares the same on the tensors themselves.) `at`: the device that the
# call's buffers, and so its launches, are on.
def _pitch(name: str, t: torch.Tensor, n: int, cols: int, dtype: torch.dtype, at: torch.device) -> int:
    """The row pitch of a tensor of n rows of cols elements that lie side by side."""
    st = t.stride()
    if t.shape != (n, cols) or t.dtype is not dtype or not t.is_cuda or t.device != at or (st[1] != 1 and cols > 1 and n > 0):
        if t.dim() != 2 or t.shape != (n, cols):
            raise ValueError(f"{name}: need [{n}][{cols}], got {tuple(t.shape)}")
        _placed(name, t, dtype, at)
        raise ValueError(f"{name}: the elements of a row must lie side by side (stride {st[1]})")
    return st[0] if n > 1 else cols      # (a single row's stride says nothing)


def _whole(name: str, t: torch.Tensor, shape, dtype: torch.dtype, at: torch.device) -> int:
    """The address of a contiguous tensor."""
    if t.shape != shape or t.dtype is not dtype or not t.is_cuda or t.device != at or not t.is_contiguous():
        _placed(name, t, dtype, at)
        raise ValueError(f"{name}: need a contiguous {tuple(shape)}, got {tuple(t.shape)}, strides {t.stride()}")
    return t.data_ptr()


def _placed(name: str, t: torch.Tensor, dtype: torch.dtype, at: torch.device):
    if t.dtype is not dtype:
        raise TypeError(f"{name}: need {dtype}, got {t.dtype}")
    if not t.is_cuda:
        raise ValueError(f"{name}: not on a GPU ({t.device})")
    if t.device != at:
        raise ValueError(f"{name}: on {t.device}, the call's other buffers are on {at}")


def _launched_on(at: torch.device):
    """The current stream, which has to be one of the call's device."""
    if _device() != at.index:
        raise ValueError(f"the call's buffers are on {at}, the current device is cuda:{_device()}")
    return _stream()


def _row_count(name: str, t: torch.Tensor, most: int) -> int:
    if t.dim() != 2 or t.shape[0] > most:
        raise ValueError(f"{name}: {tuple(t.shape)}, built for {most} rows")
    return t.shape[0]


def _first(t: torch.Tensor, n: int) -> torch.Tensor:
    return t if t.shape[0] == n else t[:n]


def _index(at: torch.device) -> int:
    return -1 if at.index is None else at.index


def _status(what: str, ws):
    rc, bits = B.ps_workspace_status(ws)
    if rc != B.PS_OK:
        raise B.PsppoError(rc, f"{what} (device bits {bits:#x})")


@dataclass
class FFNShape:
    rows: int                     # most rows of a call
    d: int
    F: int
    act: int = B.PS_ACT_SILU
    train: bool = True            # keep what the backward needs (6.1 bytes per row and column of F)
    dx_dtype: torch.dtype = torch.bfloat16
    dw_dtype: torch.dtype = torch.float32    # bf16: rounded once from the f32 sums, not accumulated over calls


class GatedFFN:
    """Y = (s(X Wg^T) * (X Wu^T)) Wd^T and its gradients (ps_gated_ffn_fwd, ps_gated_ffn_bwd), bf16."""

    def __init__(self, shape: FFNShape, device: str = "cuda"):
        s = shape
        self.s, self.device = s, device
        L = B.lib()
        self._fwd, self._bwd = L.ps_gated_ffn_fwd, L.ps_gated_ffn_bwd
        bf16 = dict(dtype=torch.bfloat16, device=device)
        u8 = dict(dtype=torch.uint8, device=device)   # zeroed: a status word never written reads clear
        self.Y = torch.empty(s.rows, s.d, **bf16)
        self._at = self.Y.device
        self.ws_fwd = torch.zeros(B.ps_gated_ffn_fwd_workspace_size(s.rows, s.d, s.F, s.train), **u8)
        self._fwd_tail = (None, 0, self.ws_fwd.data_ptr(), self.ws_fwd.numel())
        self.store = self.ws_bwd = None
        self.stored = -1              # rows of the last forward, until its backward has used the store
        if s.train:
            self.store = torch.empty(B.ps_gated_ffn_store_size(s.rows, s.F), **u8)
            self.ws_bwd = torch.zeros(B.ps_gated_ffn_bwd_workspace_size(s.rows, s.d, s.F), **u8)
            self.dX = torch.empty(s.rows, s.d, dtype=s.dx_dtype, device=device)
            self.dWg, self.dWu = (torch.empty(s.F, s.d, dtype=s.dw_dtype, device=device) for _ in range(2))
            self.dWd = torch.empty(s.d, s.F, dtype=s.dw_dtype, device=device)
            kept = (self.store.data_ptr(), self.store.numel())
            self._fwd_tail = kept + self._fwd_tail[2:]
            self._bwd_tail = kept + (self.dX.data_ptr(), s.d, B.dtype_code(self.dX), self.dWg.data_ptr(),
                                     self.dWu.data_ptr(), self.dWd.data_ptr(), B.dtype_code(self.dWd))
            self._bwd_ws = (self.ws_bwd.data_ptr(), self.ws_bwd.numel())
        self._w1, self._w2 = (s.F, s.d), (s.d, s.F)
        calls = B.calls()
        self._fast_fwd, self._fast_bwd = calls.ffn_fwd, calls.ffn_bwd
        at = lambda t: 0 if t is None else t.data_ptr()  # noqa: E731
        size = lambda t: 0 if t is None else t.numel()  # noqa: E731
        grads = (self.dX, self.dWg, self.dWu, self.dWd) if s.train else [None] * 4
        self._plan = calls.ffn_plan(s.rows, s.d, s.F, s.act, *(self._bwd_tail[4], self._bwd_tail[8]) if s.train else (0, 0),
                                    *map(at, (self.Y, self.store, self.ws_fwd, self.ws_bwd, *grads)),
                                    *map(size, (self.store, self.ws_fwd, self.ws_bwd)), _index(self._at))

    def _inputs(self, X, Wg, Wu, Wd):
        N, t, at = X.shape[0], torch.bfloat16, self._at
        return (X.data_ptr(), _pitch("X", X, N, self.s.d, t, at), _whole("Wg", Wg, self._w1, t, at),
                _whole("Wu", Wu, self._w1, t, at), _whole("Wd", Wd, self._w2, t, at))

    def forward(self, X, Wg, Wu, Wd, out=None):
        """Y [N][d] (in `out` if given)."""
        s = self.s
        rc = self._fast_fwd(self._plan, X, Wg, Wu, Wd, out)
        N = _row_count("X", X, s.rows)
        Y = _first(self.Y, N) if out is None else out
        if rc is None:
            inputs = self._inputs(X, Wg, Wu, Wd)
            rc = self._fwd(N, s.d, s.F, B.PS_DTYPE_BF16, s.act, *inputs, Y.data_ptr(),
                           s.d if out is None else _pitch("out", out, N, s.d, torch.bfloat16, self._at), *self._fwd_tail,
                           _launched_on(self._at))
        self.stored = N if s.train and rc == B.PS_OK else -1
        if rc:
            B._check(rc, "ps_gated_ffn_fwd")
        return Y

    def backward(self, dY, X, Wg, Wu, Wd, dw_accumulate: bool = False):
        """(dX, dWg, dWu, dWd) of the last forward, which must have been given the same X and weights: one
        backward per forward (it turns the store into dG and dU in place)."""
        s = self.s
        N = _row_count("X", X, s.rows)
        if self.stored != N:
            self._inputs(X, Wg, Wu, Wd)
            raise RuntimeError("backward needs a forward of the same rows before it (train=True, one backward each)")
        rc = self._fast_bwd(self._plan, dY, X, Wg, Wu, Wd, dw_accumulate)
        if rc is None:
            inputs = self._inputs(X, Wg, Wu, Wd)
            rc = self._bwd(N, s.d, s.F, B.PS_DTYPE_BF16, dY.data_ptr(), _pitch("dY", dY, N, s.d, torch.bfloat16, self._at),
                           *inputs, *self._bwd_tail, B.PS_DW_ACCUMULATE if dw_accumulate else 0, *self._bwd_ws,
                           _launched_on(self._at))
        self.stored = -1
        if rc:
            B._check(rc, "ps_gated_ffn_bwd")
        return _first(self.dX, N), self.dWg, self.dWu, self.dWd

    def check_status(self):
        """Raise PsppoError if a workspace reports a device-side error."""
        _status("ffn forward", self.ws_fwd)
        if self.ws_bwd is not None:
            _status("ffn backward", self.ws_bwd)


def rope_table(T: int, R: int, theta: float = 10000.0, device: str = "cuda") -> torch.Tensor:
    """The table of QKNormRope: f32 [T][R/2][2], (cos, sin) of t theta^(-2i/R) (ps_rope_table)."""
    table = torch.empty(T, R // 2, 2, dtype=torch.float32, device=device)
    B.ps_rope_table(T, R, theta, table)
    return table


@dataclass
class QKShape:
    rows: int
    Hq: int
    Hk: int
    D: int
    R: int                        # rotated dims of a head (0: norms only)
    dtype: torch.dtype = torch.bfloat16
    interleaved: bool = False     # pairs (2i, 2i + 1) instead of (i, i + R/2)
    eps: float = 1e-6
    train: bool = True


class QKNormRope:
    """Norms of queries and keys per head and their rotary positions in one pass, and the gradients
    (ps_qk_norm_rope_fwd, ps_qk_norm_rope_bwd). q and k are [N][H * D] with any row pitch of whole 16 bytes, so
    they may be column ranges of one projection's output; `pos` is row_pos of the packed rows with pos_base = 1."""

    def __init__(self, shape: QKShape, table: Optional[torch.Tensor], device: str = "cuda"):
        s = shape
        if s.R > 0:
            if table is None or table.dim() != 3:
                raise ValueError("a table [T][R/2][2] is needed (rope_table)")
            _whole("table", table, (table.shape[0], s.R // 2, 2), torch.float32, torch.empty(0, device=device).device)
        self.s, self.table, self.device = s, table if s.R > 0 else None, device
        L = B.lib()
        self._fwd, self._bwd = L.ps_qk_norm_rope_fwd, L.ps_qk_norm_rope_bwd
        code = B.dtype_code(torch.empty(0, dtype=s.dtype))
        self._head = (s.Hq, s.Hk, s.D, s.R, code, B.PS_ROPE_EVEN if s.interleaved else B.PS_ROPE_HALF)
        self._table = (table.shape[0], table.data_ptr()) if s.R > 0 else (0, None)
        self._wq, self._wk = s.Hq * s.D, s.Hk * s.D
        t = dict(dtype=s.dtype, device=device)
        self.q, self.k = torch.empty(s.rows, self._wq, **t), torch.empty(s.rows, self._wk, **t)
        self._at = self.q.device
        size = B.ps_qk_norm_rope_workspace_size(s.D) if s.train else 256
        self.ws = torch.zeros(max(size, 256), dtype=torch.uint8, device=device)
        self._ws = (self.ws.data_ptr(), self.ws.numel())
        self._out = (self.q.data_ptr(), self._wq, self.k.data_ptr(), self._wk)
        if s.train:
            self.dq, self.dk = torch.empty(s.rows, self._wq, **t), torch.empty(s.rows, self._wk, **t)
            self.dgq, self.dgk = (torch.empty(s.D, dtype=torch.float32, device=device) for _ in range(2))
            self._grads = (self.dq.data_ptr(), self._wq, self.dk.data_ptr(), self._wk, self.dgq.data_ptr(),
                           self.dgk.data_ptr())
        calls = B.calls()
        self._fast_fwd, self._fast_bwd = calls.qk_fwd, calls.qk_bwd
        grads = [t.data_ptr() for t in (self.dq, self.dk, self.dgq, self.dgk)] if s.train else [0] * 4
        self._plan = calls.qk_plan(s.rows, *self._head, self._table[0], s.eps, self._table[1] or 0, self.q.data_ptr(),
                                   self.k.data_ptr(), *self._ws, *grads, _index(self._at))

    def _inputs(self, N, q, k, gq, gk, pos, pos_base):
        s = self.s
        t, gain, at = s.dtype, (s.D,), self._at
        return (q.data_ptr(), _pitch("q", q, N, self._wq, t, at), k.data_ptr(), _pitch("k", k, N, self._wk, t, at),
                None if gq is None else _whole("gq", gq, gain, t, at), None if gk is None else _whole("gk", gk, gain, t, at),
                s.eps, _whole("pos", pos, (N,), torch.int32, at) if s.R > 0 else None, pos_base, *self._table)

    def forward(self, q, k, gq, gk, pos, pos_base: int = 1, in_place: bool = False):
        """(q, k) normed and rotated; in_place writes over the inputs (serving: no backward follows)."""
        rc = self._fast_fwd(self._plan, q, k, gq, gk, pos, pos_base, in_place)
        N = _row_count("q", q, self.s.rows)
        if rc is None:
            inputs = self._inputs(N, q, k, gq, gk, pos, pos_base)
            rc = self._fwd(N, *self._head, *inputs, *(inputs[:4] if in_place else self._out), *self._ws,
                           _launched_on(self._at))
        if rc:
            B._check(rc, "ps_qk_norm_rope_fwd")
        return (q, k) if in_place else (_first(self.q, N), _first(self.k, N))

    def backward(self, dq_out, dk_out, q, k, gq, gk, pos, pos_base: int = 1, dw_accumulate: bool = False):
        """(dq, dk, dgq, dgk) from the gradients of the forward's outputs and its inputs."""
        s = self.s
        rc = self._fast_bwd(self._plan, dq_out, dk_out, q, k, gq, gk, pos, pos_base, dw_accumulate)
        N = _row_count("q", q, s.rows)
        if rc is None:
            if not s.train:
                raise RuntimeError("built without a backward (train=False)")
            rc = self._bwd(N, *self._head, dq_out.data_ptr(), _pitch("dq_out", dq_out, N, self._wq, s.dtype, self._at),
                           dk_out.data_ptr(), _pitch("dk_out", dk_out, N, self._wk, s.dtype, self._at),
                           *self._inputs(N, q, k, gq, gk, pos, pos_base), *self._grads,
                           B.PS_DW_ACCUMULATE if dw_accumulate else 0, *self._ws, _launched_on(self._at))
        if rc:
            B._check(rc, "ps_qk_norm_rope_bwd")
        return _first(self.dq, N), _first(self.dk, N), self.dgq, self.dgk

    def check_status(self):
        _status("q/k norm and rotation", self.ws)


class RowDropout:
    """Dropout of a branch's rows added to the residual rows (ps_dropout_rows). The mask is a function of
    (seed, step, site, completion, position, column): it is never stored, and a token keeps it whatever the
    cutoffs, the packing or the shard (traj_base: the global index of the shard's first completion)."""

    def __init__(self, p: float, site: int = 0):
        self.p, self.site = float(p), int(site)
        self._call, self._fast = B.lib().ps_dropout_rows, B.calls().dropout_rows

    def _run(self, x, row_traj, row_pos, seed, step, res, traj_base, out):
        y = self._fast(x, row_traj, row_pos, seed, step, res, traj_base, out, self.p, self.site)
        if y is not None:
            if type(y) is int:
                B._check(y, "ps_dropout_rows")
            return y
        N, d = x.shape
        t, at = x.dtype, x.device
        pitch = _pitch("x", x, N, d, t, at)
        y = torch.empty_like(x) if out is None else out
        rc = self._call(N, d, _CODE[t] if t in _CODE else B.dtype_code(x), x.data_ptr(), pitch,
                        None if res is None else res.data_ptr(), 0 if res is None else _pitch("res", res, N, d, t, at),
                        _whole("row_traj", row_traj, (N,), torch.int32, at),
                        _whole("row_pos", row_pos, (N,), torch.int32, at), traj_base, self.p, seed & (2**64 - 1),
                        step & (2**64 - 1), self.site, y.data_ptr(), d if out is None else _pitch("out", out, N, d, t, at),
                        _launched_on(at))
        B._check(rc, "ps_dropout_rows")
        return y

    def forward(self, x, row_traj, row_pos, seed: int, step: int, res=None, traj_base: int = 0, out=None):
        """res + x where kept, scaled by the inverse survival; `out` may be x or res."""
        return self._run(x, row_traj, row_pos, seed, step, res, traj_base, out)

    def backward(self, dy, row_traj, row_pos, seed: int, step: int, traj_base: int = 0, out=None):
        """The gradient of x (that of res is dy itself)."""
        return self._run(dy, row_traj, row_pos, seed, step, None, traj_base, out)
