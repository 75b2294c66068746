"""Buffer management around the three C-ABI calls: upload, allocate, call, download.

Nothing here computes a step of the layer; it strings l2a_route_compact, l2a_attn_fwd and
l2a_attn_bwd together the way a framework integration would, for the tests, the smoke check
and the benchmark.
"""
from __future__ import annotations

from dataclasses import dataclass
from typing import Optional

import numpy as np
import torch

from . import binding as B
from .inputs import f32_to_bf16_bits


def to_device(x: np.ndarray, dtype: str, device="cuda") -> torch.Tensor:
    """fp32 host array -> device tensor of the workload's element type (bf16 values must be exact)."""
    if dtype == "bf16":
        bits = torch.from_numpy(f32_to_bf16_bits(x).view(np.int16))
        return bits.to(device).view(torch.bfloat16)
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(device)


def to_host(t: torch.Tensor) -> np.ndarray:
    return t.detach().to(torch.float64).cpu().numpy()


class GuardedAllocator:
    """torch.empty with a guard band of a known byte pattern on both sides of every buffer.  The tests
    allocate all outputs and workspaces of a layer through one of these and call check() after the
    kernels ran: a store outside a buffer's bounds shows as a changed guard byte."""
    BAND = 4096          # bytes on each side; keeps the 256-byte alignment of what torch returns
    PATTERN = 0xA5

    def __init__(self):
        self.bands = []  # (name, raw uint8 buffer, payload bytes)

    def __call__(self, shape, dtype=torch.float32, device="cuda"):
        shape = (shape,) if isinstance(shape, int) else tuple(shape)
        n = 1
        for d in shape:
            n *= int(d)
        nbytes = n * torch.empty((), dtype=dtype).element_size()
        pad = (-nbytes) % 256
        raw = torch.full((self.BAND + nbytes + pad + self.BAND,), self.PATTERN, dtype=torch.uint8, device=device)
        self.bands.append((f"buffer {len(self.bands)} {shape} {dtype}", raw, nbytes))
        return raw[self.BAND:self.BAND + nbytes].view(dtype).view(shape)

    def check(self):
        """Raises if any guard byte differs from the pattern."""
        for name, raw, nbytes in self.bands:
            lo, hi = raw[:self.BAND], raw[self.BAND + nbytes:]
            if not (bool((lo == self.PATTERN).all()) and bool((hi == self.PATTERN).all())):
                nlo, nhi = int((lo != self.PATTERN).sum()), int((hi != self.PATTERN).sum())
                raise AssertionError(f"{name}: {nlo} guard bytes before and {nhi} after the buffer were overwritten")
        return len(self.bands)


@dataclass
class Layer:
    """Device buffers of one layer call."""
    p: B.l2a_params
    q: torch.Tensor
    k: torch.Tensor
    v: torch.Tensor
    mask: Optional[torch.Tensor]
    qg: Optional[torch.Tensor] = None
    kg: Optional[torch.Tensor] = None
    vg: Optional[torch.Tensor] = None
    alloc: Optional[GuardedAllocator] = None   # tests: every output and workspace between guard bands

    def __post_init__(self):
        p, dev = self.p, self.q.device
        self.qg = self.q if self.qg is None else self.qg
        self.kg = self.k if self.kg is None else self.kg
        self.vg = self.v if self.vg is None else self.vg
        self.dense = bool(p.flags & B.L2A_FLAG_DENSE)
        if self.dense:
            self.row_idx = self.count = self.first = self.route_ws = None
        else:
            self.row_idx, self.count, self.first, self.route_ws = B.alloc_route(p, dev, self.alloc)
        self.O, self.lse_l, self.lse_g, self.S, self.A = B.alloc_fwd(p, dev, alloc=self.alloc)
        self.fwd_ws = B.alloc_fwd_workspace(p, dev, self.alloc)
        self.dq = self.dk = self.dv = self.bwd_ws = None
        self.dqg = self.dkg = self.dvg = None
        self.delta_g = None

    # ---- the hot path, in order
    def route(self):
        if not self.dense:
            B.l2a_route_compact(self.p, self.mask, self.row_idx, self.count, self.first, self.route_ws)

    def forward(self, save_branches: bool = True):
        B.l2a_attn_fwd(self.p, self.q, self.k, self.v, self.qg, self.kg, self.vg, self.row_idx, self.count,
                       self.first, self.O, self.lse_l, self.lse_g, self.S if save_branches else None,
                       self.A if save_branches else None, self.fwd_ws)

    def backward(self, dO: torch.Tensor, separate: bool = False, want_delta: bool = False):
        if self.dq is None:
            self.dq, self.dk, self.dv, self.bwd_ws = B.alloc_bwd(self.p, self.q.device, self.alloc)
            if separate:
                self.dqg, self.dkg, self.dvg, _ = B.alloc_bwd(self.p, self.q.device, self.alloc)
            if want_delta:
                self.delta_g = (self.alloc or torch.empty)(tuple(self.lse_g.shape), dtype=torch.float32,
                                                           device=self.q.device)
        g = (self.dqg, self.dkg, self.dvg) if separate else (self.dq, self.dk, self.dv)
        B.l2a_attn_bwd(self.p, dO, self.q, self.k, self.v, self.qg, self.kg, self.vg, self.row_idx, self.count,
                       self.first, self.S, self.A, self.lse_l, self.lse_g, self.dq, self.dk, self.dv, g[0], g[1],
                       g[2], self.delta_g, self.bwd_ws)


def layer_from_numpy(q, k, v, mask, W, dtype="bf16", flags=0, scale=None, qg=None, kg=None, vg=None,
                     device="cuda", guard: bool = False) -> Layer:
    Bn, T, Hq, D = q.shape
    Hkv = k.shape[2]
    Hm = 1 if mask is None else mask.shape[1]
    p = B.make_params(Bn, T, Hq, Hkv, D, W, Hm, B.L2A_BF16 if dtype == "bf16" else B.L2A_FP32, flags, scale)
    up = lambda x: None if x is None else to_device(x, dtype, device)
    m = None if mask is None else torch.from_numpy(np.array(mask, dtype=np.uint8, order="C", copy=True)).to(device)
    return Layer(p, up(q), up(k), up(v), m, up(qg), up(kg), up(vg), GuardedAllocator() if guard else None)


class PagedCache:
    """A paged KV cache for `p.B` sequences (p: make_params' sizes of the layer; a copy is kept as .p, whose T every step sets) and the bookkeeping around it: pages
    are handed out as sequences grow and taken back when they end.  The pool, the table and the steps' index arrays are on the GPU, what decides
    about them on the host.  A step uploads the table and its index arrays, which waits for the stream's earlier work, and allocates its output (and
    its workspace, where none is given).  Steps of one cache are ordered, on one stream or by the caller."""

    def __init__(self, p: B.l2a_params, pages: int, page_size: int, max_pages: int, fp8: bool = False, device="cuda"):
        self.p, self.page_size = B.l2a_params.from_buffer_copy(p), page_size
        self.cache = B.alloc_cache(p, pages, page_size, max_pages, fp8, device)
        self.table = np.full((p.B, max_pages), -1, dtype=np.int32)
        self.length = np.zeros(p.B, dtype=np.int32)
        self.free = list(range(pages - 1, -1, -1))

    def _upload(self, x: np.ndarray) -> torch.Tensor:
        return torch.from_numpy(np.ascontiguousarray(x)).to(self.cache.tensors[4].device)

    def _check_not_captured(self):
        if torch.cuda.is_initialized() and torch.cuda.is_current_stream_capturing():
            raise RuntimeError("steps upload their indices from the host and cannot be captured; capture l2a_cache_write and l2a_attn_extend with index "
                               "arrays at fixed addresses")

    def begin_step(self, new):
        """Room for new[b] tokens of every sequence, which count as theirs from here on.  -> (seq_start, pos) on the GPU; the params' T is their
        number."""
        self._check_not_captured()
        new = np.asarray(new)
        if new.shape != (self.p.B,):
            raise ValueError(f"a step has a number of new tokens for each of the {self.p.B} sequences; got {new.tolist()}")
        if new.dtype.kind not in "biuf" or (new.dtype.kind == "f" and not (new == np.floor(new)).all()) or (new == np.inf).any():
            raise ValueError(f"numbers of new tokens are whole numbers; got {new.tolist()}")
        # (compared as they came: what does not fit into 32 bits does not fit into the table either)
        if (new < 0).any() or (new > self.table.shape[1] * self.page_size - self.length.astype(np.int64)).any():
            raise ValueError("no room for the step's tokens")
        new = new.astype(np.int32)
        need = -(-(self.length + new) // self.page_size)
        have = -(-self.length // self.page_size)
        if int((need - have).sum()) > len(self.free):
            raise ValueError("no room for the step's tokens")
        before, self.length = self.length, self.length + new
        try:
            for b in np.nonzero(need > have)[0]:
                for i in range(have[b], need[b]):
                    self.table[b, i] = self.free.pop()
            self.cache.tensors[4].copy_(torch.from_numpy(self.table))
            start, pos = self._upload(np.concatenate([[0], np.cumsum(new)]).astype(np.int32)), self._upload(before)
        except BaseException:
            self._take_back(before)
            raise
        self.p.T = int(new.sum())
        return start, pos

    def _take_back(self, length: np.ndarray):
        """The sequences are as long as they were: what lies behind is free again, the pages that were handed out last first."""
        used, have = -(-length // self.page_size), -(-self.length // self.page_size)
        for b in np.nonzero(have > used)[0][::-1]:
            for i in reversed(range(used[b], have[b])):
                if self.table[b, i] >= 0:
                    self.free.append(int(self.table[b, i]))
                    self.table[b, i] = -1
        self.length = length

    def extend(self, new, q, k, v, mask, **outs):
        """Writes the packed new tokens' k, v and attends: q [T,Hq,D], k, v [T,Hkv,D], mask [mask_heads,T] -> o [T,Hq,D].  Where a call is
        refused, the sequences are what they were before."""
        before = self.length
        start, pos = self.begin_step(new)
        try:
            O = torch.empty_like(q)
            if self.p.T == 0:
                if q.numel() or k.numel() or v.numel():
                    raise ValueError("the step has no new tokens, but rows")
                return O
            B.l2a_cache_write(self.p, self.cache, k, v, start, pos)
            B.l2a_attn_extend(self.p, self.cache, q, start, pos, mask, max(int(max(new)), 1), O, **outs)
        except BaseException:
            self._take_back(before)
            raise
        return O

    def read(self, b: int):
        """-> k, v [length, Hkv, D] of sequence b, as bf16."""
        b = range(self.p.B)[b]  # (-1: the last one)
        self._check_not_captured()
        n = int(self.length[b])
        size = np.where(np.arange(self.p.B) == b, n, 0)
        k, v = (torch.empty(n, self.p.Hkv, self.p.D, dtype=torch.bfloat16, device=self.cache.tensors[4].device) for _ in range(2))
        if n == 0:
            return k, v
        self.p.T = n
        B.l2a_cache_read(self.p, self.cache, self._upload(np.concatenate([[0], np.cumsum(size)]).astype(np.int32)),
                         self._upload(np.zeros(self.p.B, dtype=np.int32)), k, v)
        return k, v

    def end(self, b: int):
        """Sequence b is over: its pages are free."""
        b = range(self.p.B)[b]  # (-1: the last one)
        used = -(-int(self.length[b]) // self.page_size)
        self.free.extend(int(x) for x in self.table[b, :used])
        self.table[b], self.length[b] = -1, 0
