"""The merged tokens inside a language model: a paged key-value cache of theirs.

``AppendPlan`` (norm of queries and keys, rotation by position ids, cache entry), ``AttendPlan``
(attention of one new token per sequence) and ``EvictPlan`` (keeps the slots that received most
attention) marshal arguments for sttm_cache_append, sttm_cache_attend and sttm_cache_evict; a plan
holds buffers and parameters for repeated calls on one cache.  The functions of those names are
single calls.  All work is enqueued on the current stream, nothing synchronises; conditions found
on the device are OR-ed into a plan's ``status``, which it never clears.  A plan's buffers serve one call after
the other: use it on one stream, or order the streams.  There is no fallback.
"""
from __future__ import annotations

import ctypes as C
import math
from dataclasses import dataclass
from typing import Optional, Sequence

import torch

from . import binding
from .binding import _check

# Current device, and the current stream's handle alone: torch.cuda.current_stream() makes a stream object, which takes as
# long as a small call does.
_device, _raw_stream = torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream
_DTYPES = {torch.bfloat16: 0, torch.float16: 2}


class SttmCache(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("pages", C.c_longlong), ("heads", C.c_int), ("page", C.c_int),
                ("dim", C.c_int), ("page_stride", C.c_longlong), ("head_stride", C.c_longlong),
                ("slot_stride", C.c_longlong), ("table", C.c_void_p), ("table_stride", C.c_longlong),
                ("table_width", C.c_int), ("seqs", C.c_int), ("dtype", C.c_int)]


class AppendParams(C.Structure):
    _fields_ = [("q", C.c_void_p), ("k", C.c_void_p), ("v", C.c_void_p), ("q_row", C.c_longlong), ("q_head", C.c_longlong),
                ("k_row", C.c_longlong), ("k_head", C.c_longlong), ("v_row", C.c_longlong), ("v_head", C.c_longlong),
                ("q_out", C.c_void_p), ("rows", C.c_longlong), ("q_heads", C.c_int), ("row_offsets", C.c_void_p),
                ("lengths", C.c_void_p), ("new_lengths", C.c_void_p), ("positions", C.c_void_p), ("positions_f32", C.c_int),
                ("axes", C.c_int), ("axis_stride", C.c_longlong), ("sections", C.c_int * 3), ("inv_freq", C.c_void_p),
                ("rot", C.c_int), ("interleaved", C.c_int), ("q_norm", C.c_void_p), ("k_norm", C.c_void_p),
                ("eps", C.c_float), ("device_status", C.c_void_p)]


class AttendParams(C.Structure):
    _fields_ = [("q", C.c_void_p), ("q_seq", C.c_longlong), ("q_head", C.c_longlong), ("q_heads", C.c_int),
                ("lengths", C.c_void_p), ("max_len", C.c_int), ("scale", C.c_float), ("mask", C.c_void_p),
                ("mask_stride", C.c_longlong), ("scores", C.c_void_p), ("score_seq", C.c_longlong),
                ("score_head", C.c_longlong), ("decay", C.c_float), ("out", C.c_void_p), ("lse", C.c_void_p),
                ("device_status", C.c_void_p)]


class EvictParams(C.Structure):
    _fields_ = [("lengths", C.c_void_p), ("max_len", C.c_int), ("keep", C.c_void_p), ("first", C.c_int), ("last", C.c_int),
                ("scores", C.c_void_p), ("score_seq", C.c_longlong), ("score_head", C.c_longlong), ("kept_width", C.c_int),
                ("new_lengths", C.c_void_p), ("kept", C.c_void_p), ("new_scores", C.c_void_p), ("device_status", C.c_void_p)]


def _want(ok: bool, text: str) -> None:
    if not ok:
        raise ValueError(text)


def _ints(t: torch.Tensor, shape: tuple, what: str, index: int) -> int:
    if t.dtype is not torch.int32 or t.shape != shape or t.get_device() != index or not t.is_contiguous():
        raise ValueError("%s must be a contiguous int32 tensor [%d] on the cache's device" % (what, shape[0]))
    return t.data_ptr()


def _heads(t: Optional[torch.Tensor], shape: tuple, dtype: torch.dtype, index: int, what: str):
    """Address, row stride and head stride of [rows, heads, dim] (any strides of the first two axes)."""
    if t is None or t.dtype is not dtype or t.shape != shape or t.get_device() != index:
        raise ValueError("%s must be a %s tensor %s on the cache's device" % (what, dtype, list(shape)))
    row, head, channel = t.stride()
    if channel != 1 and shape[0] > 0:
        raise ValueError("%s must have contiguous channels" % what)
    # (the stride of an axis of length one says nothing)
    return t.data_ptr(), row if shape[0] > 1 else 0, head if shape[1] > 1 else 0


class PagedCache:
    """Pools of keys and values and a page table.  ``k`` and ``v``: ``[pages, heads, page, dim]`` bf16 or
    fp16 CUDA tensors with contiguous channels (a pool laid out slot by slot is passed as
    ``pool.transpose(1, 2)``); ``table``: int32 ``[seqs, width]``, the page of every stretch of ``page`` slots."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, table: torch.Tensor):
        _want(k.dim() == 4 and k.shape == v.shape and k.stride() == v.stride() and k.dtype == v.dtype and k.dtype in _DTYPES
              and k.is_cuda and v.device == k.device and k.stride(3) == 1,
              "k and v must be bf16 or fp16 CUDA tensors [pages, heads, page, dim], alike, with contiguous channels")
        _want(table.dim() == 2 and table.dtype == torch.int32 and table.device == k.device and table.stride(1) == 1,
              "table must be an int32 CUDA tensor [seqs, width] with contiguous rows")
        self.k, self.v, self.table, self.device, self.dtype = k, v, table, k.device, k.dtype
        self.index = k.get_device()
        self.pages, self.heads, self.page, self.dim = k.shape
        self.seqs, self.width = table.shape
        self.struct = SttmCache(k.data_ptr(), v.data_ptr(), self.pages, self.heads, self.page, self.dim, k.stride(0),
                                k.stride(1), k.stride(2), table.data_ptr(), table.stride(0), self.width, self.seqs,
                                _DTYPES[k.dtype])
        self.at = C.byref(self.struct)

    def other_device(self) -> None:
        raise ValueError("the cache is not on the current CUDA device")


def empty_cache(seqs: int, max_len: int, heads: int, dim: int, page: int = 64, dtype: torch.dtype = torch.bfloat16,
                device="cuda") -> PagedCache:
    """A cache with pages of its own for ``max_len`` slots of every sequence."""
    width = -(-max_len // page)
    k, v = (torch.empty((seqs * width, heads, page, dim), dtype=dtype, device=device) for _ in range(2))
    return PagedCache(k, v, torch.arange(seqs * width, dtype=torch.int32, device=k.device).view(seqs, width))


@dataclass
class Rotary:
    """Rotation by position: ``inv_freq`` float32 ``[rot / 2]`` on the device.  Pairs are channels (i, i + rot / 2), or
    (2 i, 2 i + 1) when ``interleaved``.  ``sections``: pairs turned by each of three positions (time, row, column), which
    the caller makes of a merge's survived ids: ``id // (H * W)``, ``id % (H * W) // W`` and ``id % W``."""
    inv_freq: torch.Tensor
    interleaved: bool = False
    sections: Optional[Sequence[int]] = None


@dataclass
class AppendOutput:
    q: Optional[torch.Tensor]        # [rows, q_heads, dim]: queries, normed and rotated
    new_lengths: torch.Tensor        # [seqs] int32
    status: torch.Tensor


class AppendPlan:
    """Repeated sttm_cache_append calls on one cache."""

    def __init__(self, cache: PagedCache, q_heads: int, rotary: Optional[Rotary] = None, q_norm: Optional[torch.Tensor] = None,
                 k_norm: Optional[torch.Tensor] = None, eps: float = 1e-6):
        self.cache, self.q_heads, self.rotary, self.keep = cache, q_heads, rotary, (q_norm, k_norm)
        # three of them: a call writes neither what the call before it wrote nor what it reads
        n = cache.seqs
        ints = torch.zeros(3 * n + 1, dtype=torch.int32, device=cache.device)
        self.new_lengths, self.status = [ints[i * n:(i + 1) * n] for i in range(3)], ints[3 * n:]
        self.new_at, self.written = [t.data_ptr() for t in self.new_lengths], 2
        p = self.params = AppendParams()
        self.at, self.call = C.byref(p), binding.load_library().sttm_cache_append
        self.axes = 1 if rotary is None or rotary.sections is None else 3
        p.q_heads, p.eps, p.axes = q_heads, eps, 1
        p.device_status = self.status.data_ptr()
        if rotary is not None:
            f = rotary.inv_freq
            _want(f.dtype == torch.float32 and f.dim() == 1 and f.is_contiguous() and f.device == cache.device,
                  "inv_freq must be a contiguous float32 tensor [rot / 2] on the cache's device")
            p.inv_freq, p.rot, p.interleaved = f.data_ptr(), 2 * f.shape[0], int(rotary.interleaved)
            if rotary.sections is not None:
                _want(len(rotary.sections) == 3, "sections must be three numbers")
                p.axes = 3
                p.sections[:] = [int(x) for x in rotary.sections]
        for name, w in (("q_norm", q_norm), ("k_norm", k_norm)):
            if w is not None:
                _want(w.dtype == torch.float32 and tuple(w.shape) == (cache.dim,) and w.is_contiguous() and w.device == cache.device,
                      "%s must be a contiguous float32 tensor [dim] on the cache's device" % name)
                setattr(p, name, w.data_ptr())

    def run(self, q: Optional[torch.Tensor], k: torch.Tensor, v: torch.Tensor, row_offsets: torch.Tensor,
            lengths: Optional[torch.Tensor] = None, positions: Optional[torch.Tensor] = None,
            q_out: Optional[torch.Tensor] = None) -> AppendOutput:
        """``q`` ``[rows, q_heads, dim]``, ``k``, ``v`` ``[rows, heads, dim]`` (any row and head strides, views of one
        projection for instance); ``row_offsets`` int64 ``[seqs + 1]``; ``lengths`` int32 ``[seqs]`` (None: an empty cache);
        ``positions`` int32 or float32 ``[rows]`` or ``[axes, rows]``.  The ``new_lengths`` that it returns stand until the call after
        the next, whatever lengths either is given."""
        c, p = self.cache, self.params
        dim, dtype, index, rows = c.dim, c.dtype, c.index, k.shape[0]
        if self.q_heads > 0:
            p.q, p.q_row, p.q_head = _heads(q, (rows, self.q_heads, dim), dtype, index, "q")
            if q_out is None:
                q_out = torch.empty((rows, self.q_heads, dim), dtype=dtype, device=c.device)
            elif q_out.dtype is not dtype or q_out.shape != q.shape or q_out.get_device() != index or not q_out.is_contiguous():
                raise ValueError("q_out must be contiguous [rows, q_heads, dim] of the cache's type")
            p.q_out = q_out.data_ptr()
        p.k, p.k_row, p.k_head = _heads(k, (rows, c.heads, dim), dtype, index, "k")
        p.v, p.v_row, p.v_head = _heads(v, (rows, c.heads, dim), dtype, index, "v")
        o = row_offsets
        if o.dtype is not torch.int64 or o.shape != (c.seqs + 1,) or o.get_device() != index or not o.is_contiguous():
            raise ValueError("row_offsets must be a contiguous int64 tensor [seqs + 1] on the cache's device")
        p.row_offsets, p.rows = row_offsets.data_ptr(), rows
        p.lengths = at = None if lengths is None else _ints(lengths, (c.seqs,), "lengths", index)
        which = (self.written + 1) % 3
        if at == self.new_at[which]:
            which = (which + 1) % 3
        p.new_lengths = self.new_at[which]
        if self.rotary is not None:
            floats = positions is not None and positions.dtype is torch.float32
            shape = None if positions is None else positions.shape
            if (shape is None or not (floats or positions.dtype is torch.int32) or positions.get_device() != index
                    or shape != (self.axes, rows) and (self.axes > 1 or shape != (rows,)) or rows > 1 and positions.stride()[-1] != 1):
                raise ValueError("positions must be int32 or float32 [axes, rows] on the cache's device")
            p.positions, p.positions_f32 = positions.data_ptr(), floats
            if self.axes > 1:
                p.axis_stride = positions.stride()[0]
        if _device() != index:
            c.other_device()
        code = self.call(c.at, self.at, _raw_stream(index))
        if code:
            _check(code, "sttm_cache_append")
        self.written = which
        return AppendOutput(q_out, self.new_lengths[which], self.status)


@dataclass
class AttendOutput:
    out: torch.Tensor                # [seqs, q_heads, dim]
    lse: torch.Tensor                # [seqs, q_heads] float32: log of the sum of the exponentials
    status: torch.Tensor


class AttendPlan:
    """Repeated sttm_cache_attend calls on one cache; ``out`` and ``lse`` are the plan's own buffers."""

    def __init__(self, cache: PagedCache, q_heads: int, scale: Optional[float] = None, max_len: Optional[int] = None,
                 decay: float = 1.0):
        self.cache, self.q_heads, self.shape = cache, q_heads, (cache.seqs, q_heads, cache.dim)
        self.max_len = cache.width * cache.page if max_len is None else int(max_len)
        self.out = torch.empty((cache.seqs, q_heads, cache.dim), dtype=cache.dtype, device=cache.device)
        self.lse = torch.empty((cache.seqs, q_heads), dtype=torch.float32, device=cache.device)
        self.status = torch.zeros(1, dtype=torch.int32, device=cache.device)
        p = self.params = AttendParams()
        p.q_heads, p.max_len, p.decay = q_heads, self.max_len, decay
        p.scale = 1.0 / math.sqrt(cache.dim) if scale is None else scale
        p.out, p.lse, p.device_status = self.out.data_ptr(), self.lse.data_ptr(), self.status.data_ptr()
        self.ws = {}
        self.at, self.call = C.byref(p), binding.load_library().sttm_cache_attend
        self.output = AttendOutput(self.out, self.lse, self.status)

    def _workspace(self, scored: bool):
        n = int(binding.load_library().sttm_attend_workspace_bytes(C.byref(self.cache.struct), C.byref(self.params)))
        # (0: the call itself names the reason)
        ws = torch.empty(max(n, 256), dtype=torch.uint8, device=self.cache.device)
        self.ws[scored] = ws.data_ptr(), ws.numel(), ws
        return self.ws[scored]

    def run(self, q: torch.Tensor, lengths: torch.Tensor, mask: Optional[torch.Tensor] = None,
            scores: Optional[torch.Tensor] = None) -> AttendOutput:
        """``q`` ``[seqs, q_heads, dim]``; ``lengths`` int32 ``[seqs]``; ``mask`` bool or uint8 ``[seqs, >= max_len]``,
        false: slot left out; ``scores`` float32 ``[seqs, heads, >= max_len]``, updated in place."""
        c, p = self.cache, self.params
        p.q, p.q_seq, p.q_head = _heads(q, self.shape, c.dtype, c.index, "q")
        p.lengths = _ints(lengths, (c.seqs,), "lengths", c.index)
        if mask is None:
            p.mask = None
        else:
            stride = mask.stride()
            if not (mask.dtype in (torch.bool, torch.uint8) and mask.dim() == 2 and mask.shape[0] == c.seqs
                    and mask.shape[1] >= self.max_len and stride[1] == 1 and mask.get_device() == c.index):
                raise ValueError("mask must be bool or uint8 [seqs, >= max_len] with contiguous rows, on the cache's device")
            p.mask, p.mask_stride = mask.data_ptr(), stride[0]
        if scores is None:
            p.scores = None
        else:
            p.scores, p.score_seq, p.score_head = _scores(scores, c, self.max_len)
        ws = self.ws.get(scores is not None) or self._workspace(scores is not None)
        if _device() != c.index:
            c.other_device()
        code = self.call(c.at, self.at, ws[0], ws[1], _raw_stream(c.index))
        if code:
            _check(code, "sttm_cache_attend")
        return self.output


def _scores(t: torch.Tensor, c: PagedCache, max_len: int):
    """Address, sequence stride and head stride of float32 [seqs, heads, >= max_len]."""
    shape, stride = t.shape, t.stride()
    if not (len(shape) == 3 and shape[0] == c.seqs and shape[1] == c.heads and shape[2] >= max_len and t.dtype is torch.float32
            and stride[2] == 1 and t.get_device() == c.index):
        raise ValueError("scores must be float32 [seqs, heads, >= max_len] with contiguous slots, on the cache's device")
    return t.data_ptr(), stride[0], stride[1]


@dataclass
class EvictOutput:
    new_lengths: torch.Tensor        # [seqs] int32
    kept: torch.Tensor               # [seqs, heads, kept_width] int32: slots of the source, then -1
    new_scores: torch.Tensor         # [seqs, heads, kept_width] float32: their scores, then 0
    status: torch.Tensor


class EvictPlan:
    """Repeated sttm_cache_evict calls from one cache to another (pages of its own); outputs are the plan's buffers."""

    def __init__(self, src: PagedCache, dst: PagedCache, kept_width: int, first: int = 0, last: int = 0,
                 max_len: Optional[int] = None):
        _want(dst.device == src.device, "both caches must be on one device")
        self.src, self.dst = src, dst
        self.max_len = src.width * src.page if max_len is None else int(max_len)
        shape = (src.seqs, src.heads, kept_width)
        self.new_lengths = torch.zeros(src.seqs, dtype=torch.int32, device=src.device)
        self.kept = torch.empty(shape, dtype=torch.int32, device=src.device)
        self.new_scores = torch.empty(shape, dtype=torch.float32, device=src.device)
        self.status = torch.zeros(1, dtype=torch.int32, device=src.device)
        p = self.params = EvictParams()
        self.at, self.call = C.byref(p), binding.load_library().sttm_cache_evict
        self.output = EvictOutput(self.new_lengths, self.kept, self.new_scores, self.status)
        p.max_len, p.first, p.last, p.kept_width = self.max_len, first, last, kept_width
        p.new_lengths, p.kept, p.new_scores = self.new_lengths.data_ptr(), self.kept.data_ptr(), self.new_scores.data_ptr()
        p.device_status = self.status.data_ptr()

    def run(self, lengths: torch.Tensor, keep: torch.Tensor, scores: torch.Tensor) -> EvictOutput:
        """``lengths``, ``keep`` int32 ``[seqs]``; ``scores`` float32 ``[seqs, heads, >= max_len]``."""
        c, p = self.src, self.params
        p.lengths = _ints(lengths, (c.seqs,), "lengths", c.index)
        p.keep = _ints(keep, (c.seqs,), "keep", c.index)
        p.scores, p.score_seq, p.score_head = _scores(scores, c, self.max_len)
        if _device() != c.index:
            c.other_device()
        code = self.call(c.at, self.dst.at, self.at, _raw_stream(c.index))
        if code:
            _check(code, "sttm_cache_evict")
        return self.output


def _room(cache: PagedCache, max_len: Optional[int], *per_slot) -> int:
    return min([cache.width * cache.page] + [t.shape[-1] for t in per_slot if t is not None]) if max_len is None else max_len


def sttm_cache_append(cache: PagedCache, q, k, v, row_offsets, lengths=None, positions=None, rotary: Optional[Rotary] = None,
                      q_norm=None, k_norm=None, eps: float = 1e-6) -> AppendOutput:
    """Norm, rotation and cache entry of new tokens; see AppendPlan.run."""
    return AppendPlan(cache, 0 if q is None else q.shape[1], rotary, q_norm, k_norm, eps).run(q, k, v, row_offsets, lengths, positions)


def sttm_cache_attend(cache: PagedCache, q, lengths, mask=None, scores=None, scale: Optional[float] = None,
                      max_len: Optional[int] = None, decay: float = 1.0) -> AttendOutput:
    """Attention of one new token per sequence; see AttendPlan.run.  ``max_len`` None: what the table, and the mask and
    the scores, have room for."""
    max_len = _room(cache, max_len, mask, scores)
    return AttendPlan(cache, q.shape[1], scale, max_len, decay).run(q, lengths, mask, scores)


def sttm_cache_evict(src: PagedCache, dst: PagedCache, lengths, keep, scores, kept_width: int, first: int = 0, last: int = 0,
                     max_len: Optional[int] = None) -> EvictOutput:
    """Keeps the highest-scored slots; see EvictPlan.run.  ``max_len`` None: what the table and the scores have room for."""
    max_len = _room(src, max_len, scores)
    return EvictPlan(src, dst, kept_width, first, last, max_len).run(lengths, keep, scores)
