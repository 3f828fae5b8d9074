"""Row-wise operators of a policy block over packed rows, with buffers held in torch.

GatedFFN, QKNormRope and RowDropout run the library's calls of the same names on the current stream. Their
rows are those of a packed batch (UpdatePass.pack: src_row, row_traj, row_pos, cu_seqlens), so they carry the
head's dH into the policy's body and prepare its rows for the head. Each call takes the first N = x.shape[0] rows
of the buffers it was built for; the tensors it returns are views of those buffers, overwritten by its next call.
"""
from __future__ import annotations

from dataclasses import dataclass
from typing import Optional

import torch

from . import _binding as B


def _rows(name: str, t: torch.Tensor, n: Optional[int], cols: int, dtype: torch.dtype) -> torch.Tensor:
    """A 2-D tensor of n rows (any number: None) whose elements lie side by side, checked before its pointer is taken."""
    if t.dim() != 2 or t.shape[1] != cols or (n is not None and t.shape[0] != n):
        raise ValueError(f"{name}: need [{'N' if n is None else n}][{cols}], got {tuple(t.shape)}")
    if t.dtype != dtype:
        raise TypeError(f"{name}: need {dtype}, got {t.dtype}")
    if cols > 1 and t.numel() > 0 and t.stride(1) != 1:
        raise ValueError(f"{name}: the elements of a row must lie side by side (stride {t.stride(1)})")
    return t


def _whole(name: str, t: torch.Tensor, shape, dtype: torch.dtype) -> torch.Tensor:
    if tuple(t.shape) != tuple(shape) or not t.is_contiguous():
        raise ValueError(f"{name}: need a contiguous {tuple(shape)}, got {tuple(t.shape)}")
    if t.dtype != dtype:
        raise TypeError(f"{name}: need {dtype}, got {t.dtype}")
    return t


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
        bf16 = dict(dtype=torch.bfloat16, device=device)
        u8 = dict(dtype=torch.uint8, device=device)   # zeroed: a status word never written reads clear
        self.Y = torch.empty(s.rows, s.d, **bf16)
        self.ws_fwd = torch.zeros(B.ps_gated_ffn_fwd_workspace_size(s.rows, s.F, s.train), **u8)
        self.store = self.ws_bwd = None
        self.stored = -1              # rows of the last forward, until its backward has used the store
        if s.train:
            self.store = torch.empty(B.ps_gated_ffn_store_size(s.rows, s.F), **u8)
            self.ws_bwd = torch.zeros(B.ps_gated_ffn_bwd_workspace_size(), **u8)
            self.dX = torch.empty(s.rows, s.d, dtype=s.dx_dtype, device=device)
            self.dWg, self.dWu = (torch.empty(s.F, s.d, dtype=s.dw_dtype, device=device) for _ in range(2))
            self.dWd = torch.empty(s.d, s.F, dtype=s.dw_dtype, device=device)
            self._dx, self._dw = (B.dtype_code(t) for t in (self.dX, self.dWd))

    def _inputs(self, X, Wg, Wu, Wd) -> int:
        s, t = self.s, torch.bfloat16
        _rows("X", X, None, s.d, t)
        if X.shape[0] > s.rows:
            raise ValueError(f"X: {X.shape[0]} rows, built for {s.rows}")
        _whole("Wg", Wg, (s.F, s.d), t)
        _whole("Wu", Wu, (s.F, s.d), t)
        _whole("Wd", Wd, (s.d, s.F), t)
        return X.shape[0]

    def forward(self, X, Wg, Wu, Wd, out=None):
        """Y [N][d] (in `out` if given)."""
        s, N = self.s, self._inputs(X, Wg, Wu, Wd)
        Y = self.Y[:N] if out is None else _rows("out", out, N, s.d, torch.bfloat16)
        B.ps_gated_ffn_fwd(N, s.d, s.F, B.PS_DTYPE_BF16, s.act, X, Wg, Wu, Wd, Y, self.store, self.ws_fwd)
        self.stored = N if s.train else -1
        return Y

    def backward(self, dY, X, Wg, Wu, Wd, dw_accumulate: bool = False):
        """(dX, dWg, dWu, dWd) of the last forward, which must have been given the same X and weights: one
        backward per forward (it turns the store into dG and dU in place)."""
        s, N = self.s, self._inputs(X, Wg, Wu, Wd)
        if self.stored != N:
            raise RuntimeError("backward needs a forward of the same rows before it (train=True, one backward each)")
        _rows("dY", dY, N, s.d, torch.bfloat16)
        B.ps_gated_ffn_bwd(N, s.d, s.F, B.PS_DTYPE_BF16, dY, X, Wg, Wu, Wd, self.store, self.dX[:N], self._dx, self.dWg,
                           self.dWu, self.dWd, self._dw, B.PS_DW_ACCUMULATE if dw_accumulate else 0, self.ws_bwd)
        self.stored = -1
        return self.dX[:N], self.dWg, self.dWu, self.dWd

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
            _whole("table", table, (table.shape[0], s.R // 2, 2), torch.float32)
        self.s, self.table, self.device = s, table, device
        self.code = B.dtype_code(torch.empty(0, dtype=s.dtype))
        self.layout = B.PS_ROPE_EVEN if s.interleaved else B.PS_ROPE_HALF
        t = dict(dtype=s.dtype, device=device)
        self.q, self.k = torch.empty(s.rows, s.Hq * s.D, **t), torch.empty(s.rows, s.Hk * s.D, **t)
        size = B.ps_qk_norm_rope_workspace_size(s.D) if s.train else 256
        self.ws = torch.zeros(max(size, 256), dtype=torch.uint8, device=device)
        if s.train:
            self.dq, self.dk = torch.empty(s.rows, s.Hq * s.D, **t), torch.empty(s.rows, s.Hk * s.D, **t)
            self.dgq, self.dgk = (torch.empty(s.D, dtype=torch.float32, device=device) for _ in range(2))

    def _inputs(self, q, k, gq, gk, pos) -> int:
        s, N = self.s, q.shape[0]
        if N > s.rows:
            raise ValueError(f"q: {N} rows, built for {s.rows}")
        _rows("q", q, N, s.Hq * s.D, s.dtype)
        _rows("k", k, N, s.Hk * s.D, s.dtype)
        for name, g in (("gq", gq), ("gk", gk)):
            if g is not None:
                _whole(name, g, (s.D,), s.dtype)
        if s.R > 0:
            _whole("pos", pos, (N,), torch.int32)
        return N

    def _rope(self, pos, pos_base):
        return (pos, pos_base, self.table.shape[0], self.table) if self.s.R > 0 else (None, 0, 0, None)

    def forward(self, q, k, gq, gk, pos, pos_base: int = 1, in_place: bool = False):
        """(q, k) normed and rotated; in_place writes over the inputs (serving: no backward follows)."""
        s, N = self.s, self._inputs(q, k, gq, gk, pos)
        qo, ko = (q, k) if in_place else (self.q[:N], self.k[:N])
        B.ps_qk_norm_rope_fwd(N, s.Hq, s.Hk, s.D, s.R, self.code, self.layout, q, k, gq, gk, s.eps,
                              *self._rope(pos, pos_base), qo, ko, self.ws)
        return qo, ko

    def backward(self, dq_out, dk_out, q, k, gq, gk, pos, pos_base: int = 1, dw_accumulate: bool = False):
        """(dq, dk, dgq, dgk) from the gradients of the forward's outputs and its inputs."""
        s, N = self.s, self._inputs(q, k, gq, gk, pos)
        if not s.train:
            raise RuntimeError("built without a backward (train=False)")
        _rows("dq_out", dq_out, N, s.Hq * s.D, s.dtype)
        _rows("dk_out", dk_out, N, s.Hk * s.D, s.dtype)
        B.ps_qk_norm_rope_bwd(N, s.Hq, s.Hk, s.D, s.R, self.code, self.layout, dq_out, dk_out, q, k, gq, gk, s.eps,
                              *self._rope(pos, pos_base), self.dq[:N], self.dk[:N], self.dgq, self.dgk,
                              B.PS_DW_ACCUMULATE if dw_accumulate else 0, self.ws)
        return self.dq[:N], self.dk[:N], self.dgq, self.dgk

    def check_status(self):
        _status("q/k norm and rotation", self.ws)


class RowDropout:
    """Dropout of a branch's rows added to the residual rows (ps_dropout_rows). The mask is a function of
    (seed, step, site, completion, position, column): it is never stored, and a token keeps it whatever the
    cutoffs, the packing or the shard (traj_base: the global index of the shard's first completion)."""

    def __init__(self, p: float, site: int = 0):
        self.p, self.site = float(p), int(site)

    def _run(self, x, row_traj, row_pos, seed, step, res, traj_base, out):
        N, d = x.shape
        _rows("x", x, None, d, x.dtype)
        code = B.dtype_code(x)
        _whole("row_traj", row_traj, (N,), torch.int32)
        _whole("row_pos", row_pos, (N,), torch.int32)
        if res is not None:
            _rows("res", res, N, d, x.dtype)
        y = torch.empty(N, d, dtype=x.dtype, device=x.device) if out is None else _rows("out", out, N, d, x.dtype)
        B.ps_dropout_rows(N, d, code, x, res, row_traj, row_pos, traj_base, self.p, seed, step, self.site, y)
        return y

    def forward(self, x, row_traj, row_pos, seed: int, step: int, res=None, traj_base: int = 0, out=None):
        """res + x where kept, scaled by the inverse survival; `out` may be x or res."""
        return self._run(x, row_traj, row_pos, seed, step, res, traj_base, out)

    def backward(self, dy, row_traj, row_pos, seed: int, step: int, traj_base: int = 0, out=None):
        """The gradient of x (that of res is dy itself)."""
        return self._run(dy, row_traj, row_pos, seed, step, None, traj_base, out)
