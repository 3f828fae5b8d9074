"""Keys and values of a policy block in sampling, in pages, and the attention of a new token over them.

PagedCache holds the pages of every layer, the table that says which pages a sequence has, and the sequences' lengths;
DecodeAttention runs one new token a sequence over a layer of it. A step of sampling is, per layer: the new rows' q, k
and v (QKNormRope in place), PagedCache.append, DecodeAttention.forward; and PagedCache.lengths counts the new tokens
before the first layer's attention. All of that is ordered on the current stream and may be captured in a CUDA graph;
reserve, share and release, which hand out pages, run between the steps.
"""
from __future__ import annotations

from dataclasses import dataclass
from typing import Optional

import torch

from . import _binding as B
from .block import _first, _index, _launched_on, _pitch, _row_count, _status, _whole


@dataclass
class CacheShape:
    seqs: int                     # sequences (completions) at a time
    pages: int                    # pages of a layer
    page: int                     # positions a page, a power of two
    Hk: int
    D: int
    max_len: int                  # longest sequence that the table can name
    layers: int = 1
    dtype: torch.dtype = torch.bfloat16


class PagedCache:
    """k and v [layers][pages][Hk][page][D], table [seqs][max_len / page] and lengths [seqs] on the device (ps_paged_append).

    The table and the lengths may be written by the caller, in place; or reserve() gives sequences pages, share() lets completions
    have their prompt's pages without a copy, and release() takes a finished sequence's back."""

    def __init__(self, shape: CacheShape, device: str = "cuda"):
        s = shape
        if s.page < 1 or s.page & (s.page - 1):
            raise ValueError(f"page: a power of two, got {s.page}")
        self.s, self.device = s, device
        self.width = -(-s.max_len // s.page)
        t, i32 = dict(dtype=s.dtype, device=device), dict(dtype=torch.int32, device=device)
        self._k, self._v = (torch.empty(s.layers, s.pages, s.Hk, s.page, s.D, **t) for _ in range(2))
        self._table = torch.full((s.seqs, self.width), -1, **i32)
        self._lengths = torch.zeros(s.seqs, **i32)
        self.ws = torch.zeros(256, dtype=torch.uint8, device=device)
        self._at = self.k.device
        self._layers = [(k.data_ptr(), v.data_ptr()) for k, v in zip(self.k, self.v)]
        self._append = B.lib().ps_paged_append
        self._code = B.dtype_code(self.k)
        self._free = list(range(s.pages - 1, -1, -1))
        self._users = [0] * s.pages          # sequences that have a page
        self._own = [[] for _ in range(s.seqs)]
        calls = B.calls()
        self._fast = calls.append
        self._plan = calls.cache_plan(s.seqs, s.Hk, s.D, self._code, s.layers, s.pages, s.page, self.width,
                                      self.k.stride(0) * self.k.element_size(),
                                      *(t.data_ptr() for t in (self.k, self.v, self.table, self.lengths, self.ws)),
                                      self.ws.numel(), _index(self._at))

    # (written in place: the calls have their addresses)
    k = property(lambda self: self._k)
    v = property(lambda self: self._v)
    table = property(lambda self: self._table)
    lengths = property(lambda self: self._lengths)

    def _layer(self, layer: int):
        if not 0 <= layer < self.s.layers:
            raise IndexError(f"layer {layer} of {self.s.layers}")
        return self._layers[layer]

    def append(self, layer: int, k, v, row_seq, row_pos, pos_base: int = 1):
        """Rows of k and v [N][Hk * D] to positions row_pos - pos_base of sequences row_seq (-1: the row is passed by)."""
        rc = self._fast(self._plan, layer, k, v, row_seq, row_pos, pos_base)
        if rc is None:
            if not -2 ** 31 <= pos_base < 2 ** 31:
                raise ValueError(f"pos_base: {pos_base}, beyond 32 bits")
            s, at = self.s, self._at
            if k.dim() != 2:
                raise ValueError(f"k: need [N][{s.Hk * s.D}], got {tuple(k.shape)}")
            N, w = k.shape[0], s.Hk * s.D
            rc = self._append(N, s.seqs, s.Hk, s.D, self._code, k.data_ptr(), _pitch("k", k, N, w, s.dtype, at), v.data_ptr(),
                              _pitch("v", v, N, w, s.dtype, at), _whole("row_seq", row_seq, (N,), torch.int32, at),
                              _whole("row_pos", row_pos, (N,), torch.int32, at), pos_base, self.table.data_ptr(), self.width,
                              s.pages, s.page, *self._layer(layer), self.ws.data_ptr(), self.ws.numel(), _launched_on(at))
        if rc:
            B._check(rc, "ps_paged_append")

    # ------------------------------------------------------------------ pages
    def _publish(self, own):
        """The pages own[b] of sequences b to the table, wherever it is (before they are taken or given back: a call that fails
        here leaves the cache as it was)."""
        rows = torch.full((len(own), self.width), -1, dtype=torch.int32)
        for i, pages in enumerate(own.values()):
            rows[i, :len(pages)] = torch.tensor(pages, dtype=torch.int32)
        self.table[torch.tensor(list(own), device=self.table.device)] = rows.to(self.table.device)

    def _seq(self, seq: int) -> int:
        if not 0 <= seq < self.s.seqs:
            raise IndexError(f"sequence {seq} of {self.s.seqs}")
        return int(seq)

    def reserve(self, seq: int, n: int):
        """Pages for the first n positions of a sequence (those it has stay)."""
        s, seq = self.s, self._seq(seq)
        need = -(-n // s.page)
        if not 0 <= need <= self.width:
            raise ValueError(f"{n} positions, built for {s.max_len}")
        own = self._own[seq]
        if need - len(own) > len(self._free):
            raise B.PsppoError(B.PS_ERR_CAPACITY, f"PagedCache.reserve: {need - len(own)} pages wanted, {len(self._free)} free")
        more = need - len(own)
        if more > 0:
            new = self._free[:-more - 1:-1]
            self._publish({seq: own + new})
            del self._free[-more:]
            for p in new:
                self._users[p] = 1
            own += new

    def share(self, src: int, dst, n: int):
        """The first n positions of `src` for the sequences `dst`, which have none: whole pages are shared, a begun one is copied."""
        s, whole = self.s, n // self.s.page
        src, dst = self._seq(src), [self._seq(b) for b in dst]
        if any(self._own[b] for b in dst) or src in dst or len(set(dst)) != len(dst):
            raise ValueError("share: the sequences must be different ones without pages")
        if not 0 <= n <= len(self._own[src]) * s.page:
            raise ValueError(f"share: sequence {src} has pages for {len(self._own[src]) * s.page} positions, not {n}")
        begun = n % s.page != 0
        if begun and len(dst) > len(self._free):
            raise B.PsppoError(B.PS_ERR_CAPACITY, f"PagedCache.share: {len(dst)} pages wanted, {len(self._free)} free")
        if not dst:
            return
        shared, new = self._own[src][:whole], self._free[:-len(dst) - 1:-1] if begun else []
        for p in new:
            for c in (self.k, self.v):
                c[:, p].copy_(c[:, self._own[src][whole]])
        own = {b: shared + new[i:i + 1] for i, b in enumerate(dst)}
        self._publish(own)
        del self._free[len(self._free) - len(new):]
        for p in shared:
            self._users[p] += len(dst)
        for p in new:
            self._users[p] = 1
        for b in dst:
            self._own[b] = own[b]

    def release(self, seq: int):
        """A sequence's pages back, except those that others still have; its length becomes 0."""
        seq = self._seq(seq)
        self._publish({seq: []})
        self.lengths[seq] = 0
        for p in reversed(self._own[seq]):
            self._users[p] -= 1
            if self._users[p] == 0:
                self._free.append(p)
        self._own[seq] = []

    def check_status(self):
        """Raise PsppoError if the last append reports a device-side error."""
        _status("append", self.ws)


@dataclass
class DecodeShape:
    seqs: int
    Hq: int
    Hk: int
    D: int
    dtype: torch.dtype = torch.bfloat16
    window: int = 0               # a query sees the last `window` keys (0: all)
    scale: Optional[float] = None  # D ** -0.5


class DecodeAttention:
    """Attention of one new token a sequence over a layer of a PagedCache (ps_paged_decode): row b of q is sequence b's, whose
    length counts the new token. One holder serves all layers of a policy, one call after another."""

    def __init__(self, shape: DecodeShape, device: str = "cuda"):
        s = shape
        self.s, self.device = s, device
        self._call = B.lib().ps_paged_decode
        self._scale = s.D ** -0.5 if s.scale is None else float(s.scale)
        self.o = torch.empty(s.seqs, s.Hq * s.D, dtype=s.dtype, device=device)
        self._at = self.o.device
        self._code = B.dtype_code(self.o)
        self.ws = torch.zeros(max(256, B.ps_paged_decode_workspace_size(s.D)), dtype=torch.uint8, device=device)
        calls = B.calls()
        self._fast = calls.decode
        self._plan = calls.decode_plan(s.seqs, s.Hq, s.Hk, s.D, self._code, s.window, self._scale, self.o.data_ptr(),
                                       self.ws.data_ptr(), self.ws.numel(), _index(self._at))

    def forward(self, q, cache: PagedCache, layer: int = 0, out=None, lse=None):
        """o [n][Hq * D] (in `out` if given; it may be q) of the first n = q.shape[0] sequences; lse f32 [n][Hq] is written if
        given. A sequence of length 0 gives zeros."""
        rc = self._fast(self._plan, cache._plan, layer, q, out, lse)
        if rc is None:
            rc = self._forward(q, cache, layer, out, lse)
        if rc:
            B._check(rc, "ps_paged_decode")
        return _first(self.o, q.shape[0]) if out is None else out

    def _forward(self, q, cache, layer, out, lse):
        s, c, at = self.s, cache.s, self._at
        if (c.Hk, c.D, c.dtype) != (s.Hk, s.D, s.dtype):
            raise ValueError(f"the cache holds {c.Hk} heads of {c.D} in {c.dtype}, built for {s.Hk} of {s.D} in {s.dtype}")
        if cache._at != at:
            raise ValueError(f"the cache is on {cache._at}, the call's other buffers are on {at}")
        n, w = _row_count("q", q, min(s.seqs, c.seqs)), s.Hq * s.D
        o = _first(self.o, n) if out is None else out
        return self._call(n, s.Hq, s.Hk, s.D, self._code, q.data_ptr(), _pitch("q", q, n, w, s.dtype, at), *cache._layer(layer),
                          c.pages, c.page, cache.table.data_ptr(), cache.width, cache.lengths.data_ptr(), s.window, self._scale,
                          o.data_ptr(), w if out is None else _pitch("out", out, n, w, s.dtype, at),
                          None if lse is None else _whole("lse", lse, (n, s.Hq), torch.float32, at), self.ws.data_ptr(),
                          self.ws.numel(), _launched_on(at))

    def check_status(self):
        """Raise PsppoError if the last call reports a device-side error."""
        _status("decode", self.ws)
