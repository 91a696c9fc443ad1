"""Several questions on one video: attention of their new tokens over the video's cache, read once for all of them, and
over every question's own slots.

``PrefixPlan`` marshals arguments for sttm_prefix_attend and holds its buffers; ``sttm_prefix_attend`` is a single call.
All work is enqueued on the current stream, nothing synchronises; conditions found on the device are OR-ed into the plan's ``status``,
which it never clears.  A plan's buffers serve one call after the other: use it on one stream, or order the
streams.  There is no fallback.
"""
from __future__ import annotations

import ctypes as C
import math
from dataclasses import dataclass
from typing import Optional

import torch

from . import binding
from .binding import _check
from .cache import PagedCache, _device, _heads, _ints, _raw_stream, _want


class PrefixParams(C.Structure):
    _fields_ = [("q", C.c_void_p), ("q_row", C.c_longlong), ("q_head", C.c_longlong), ("rows", C.c_longlong), ("q_heads", C.c_int),
                ("seqs", C.c_int), ("row_offsets", C.c_void_p), ("seq_offsets", C.c_void_p), ("prefix_lengths", C.c_void_p),
                ("lengths", C.c_void_p), ("max_prefix", C.c_int), ("max_own", C.c_int), ("scale", C.c_float), ("out", C.c_void_p),
                ("lse", C.c_void_p), ("device_status", C.c_void_p), ("fine", C.c_int)]


@dataclass
class PrefixOutput:
    out: torch.Tensor                # [rows, q_heads, dim]
    lse: torch.Tensor                # [rows, q_heads] float32: log of the sum of the exponentials
    status: torch.Tensor


class PrefixPlan:
    """Repeated sttm_prefix_attend calls.  ``prefix``: a table row per prefix; ``own``: one per sequence (None: new tokens see their
    prefix only).  ``max_rows``: new tokens of a call at most; ``max_prefix``, ``max_own``: slots at most (None: what the tables have room for).
    ``fine``: attention weights are not rounded to the cache's type before they meet the values, as in AttendPlan; closer, and slower."""

    def __init__(self, prefix: PagedCache, q_heads: int, own: Optional[PagedCache] = None, max_rows: int = 1, scale: Optional[float] = None,
                 max_prefix: Optional[int] = None, max_own: Optional[int] = None, seqs: Optional[int] = None, fine: bool = False):
        _want(own is None or own.device == prefix.device, "both caches must be on one device")
        _want(own is not None or seqs is not None, "seqs is wanted where there are no own slots")
        self.prefix, self.own, self.q_heads, self.max_rows = prefix, own, q_heads, max_rows
        self.seqs = own.seqs if own is not None else int(seqs)
        self.out = torch.empty((max_rows, q_heads, prefix.dim), dtype=prefix.dtype, device=prefix.device)
        self.lse = torch.empty((max_rows, q_heads), dtype=torch.float32, device=prefix.device)
        self.status = torch.zeros(1, dtype=torch.int32, device=prefix.device)
        p = self.params = PrefixParams()
        p.rows, p.q_heads, p.seqs, p.fine = max_rows, q_heads, self.seqs, int(fine)
        p.max_prefix = prefix.width * prefix.page if max_prefix is None else int(max_prefix)
        if own is not None:
            p.max_own = own.width * own.page if max_own is None else int(max_own)
        p.scale = 1.0 / math.sqrt(prefix.dim) if scale is None else scale
        p.lse, p.device_status = self.lse.data_ptr(), self.status.data_ptr()
        lib = binding.load_library()
        self.at, self.call, self.own_at = C.byref(p), lib.sttm_prefix_attend, None if own is None else own.at
        p.seq_offsets = self.status.data_ptr()                   # (several prefixes want some; the size does not depend on them)
        # (0: the call itself names the reason)
        self.ws = torch.empty(max(int(lib.sttm_prefix_workspace_bytes(prefix.at, self.own_at, self.at)), 256), dtype=torch.uint8, device=prefix.device)
        self.ws_at = self.ws.data_ptr(), self.ws.numel()
        self.last = (-1, None)

    def run(self, q: torch.Tensor, row_offsets: torch.Tensor, prefix_lengths: torch.Tensor, lengths: Optional[torch.Tensor] = None,
            seq_offsets: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None) -> PrefixOutput:
        """``q`` ``[rows, q_heads, dim]`` (any row and head strides); ``row_offsets`` int64 ``[seqs + 1]``; ``prefix_lengths`` int32
        ``[prefixes]``; ``lengths`` int32 ``[seqs]``: own slots, the new tokens' among them; ``seq_offsets`` int32 ``[prefixes + 1]``: the sequences of
        every prefix (None: all of the only one); ``out``: contiguous, instead of the plan's buffer."""
        c, p, n = self.prefix, self.params, q.shape[0]
        index = c.index
        if self.last[0] != n:
            if n > self.max_rows:
                raise ValueError("%d rows: the plan has room for %d" % (n, self.max_rows))
            self.last = n, PrefixOutput(self.out[:n], self.lse[:n], self.status)
        output = self.last[1]
        p.q, p.q_row, p.q_head = _heads(q, (n, self.q_heads, c.dim), c.dtype, index, "q")
        p.rows = n
        o = row_offsets
        if o.dtype is not torch.int64 or o.shape != (self.seqs + 1,) or o.get_device() != index or not o.is_contiguous():
            raise ValueError("row_offsets must be a contiguous int64 tensor [seqs + 1] on the cache's device")
        p.row_offsets = o.data_ptr()
        p.seq_offsets = None if seq_offsets is None else _ints(seq_offsets, (c.seqs + 1,), "seq_offsets", index)
        p.prefix_lengths = _ints(prefix_lengths, (c.seqs,), "prefix_lengths", index)
        if self.own is not None:
            _want(lengths is not None, "lengths are wanted where there are own slots")
            p.lengths = _ints(lengths, (self.seqs,), "lengths", index)
        if out is None:
            p.out = self.out.data_ptr()
        elif out.dtype is not c.dtype or out.shape != q.shape or out.get_device() != index or not out.is_contiguous():
            raise ValueError("out must be contiguous [rows, q_heads, dim] of the cache's type")
        else:
            p.out = out.data_ptr()
        if _device() != index:
            c.other_device()
        code = self.call(c.at, self.own_at, self.at, self.ws_at[0], self.ws_at[1], _raw_stream(index))
        if code:
            _check(code, "sttm_prefix_attend")
        return output if out is None else PrefixOutput(out, output.lse, self.status)


def sttm_prefix_attend(prefix: PagedCache, q: torch.Tensor, row_offsets: torch.Tensor, prefix_lengths: torch.Tensor, own: Optional[PagedCache] = None,
                       lengths: Optional[torch.Tensor] = None, seq_offsets: Optional[torch.Tensor] = None, scale: Optional[float] = None, fine: bool = False) -> PrefixOutput:
    """Attention of new tokens over a shared prefix and their own slots; see PrefixPlan and PrefixPlan.run."""
    plan = PrefixPlan(prefix, q.shape[1], own, q.shape[0], scale, seqs=row_offsets.shape[0] - 1, fine=fine)
    return plan.run(q, row_offsets, prefix_lengths, lengths, seq_offsets)
