"""The rest of a decoder layer: norms before and after a block with its gate and residual, rows in 8 bits, and
matrix products of them.

``NormPlan`` (sttm_block_norm), ``QuantizePlan`` (sttm_quantize_rows) and ``MatmulPlan`` (sttm_quant_matmul)
marshal arguments; a plan holds buffers for up to ``max_rows`` rows and what does not change from call to call.  The functions
of the C names are single calls.  All work is enqueued on the current stream, nothing synchronises; conditions found on the device are
OR-ed into a plan's ``status``, which it never clears.  A plan's outputs are its own buffers unless the call is given others: they stand until its next call, so use a plan on one stream, or order the
streams.  There is no fallback.
"""
from __future__ import annotations

import ctypes as C
from dataclasses import dataclass
from typing import Optional

import torch

from . import binding
from .binding import _check
from .cache import _device, _raw_stream, _want

_TYPES = {torch.bfloat16: 0, torch.float32: 1, torch.float16: 2}


class NormParams(C.Structure):
    _fields_ = [("x", C.c_void_p), ("residual", C.c_void_p), ("gate_rows", C.c_void_p), ("x_row", C.c_longlong),
                ("residual_row", C.c_longlong), ("gate_row", C.c_longlong), ("rows", C.c_longlong), ("dim", C.c_int), ("dtype", C.c_int),
                ("post_norm", C.c_void_p), ("gate", C.c_void_p), ("pre_norm", C.c_void_p), ("residual_scale", C.c_float), ("eps", C.c_float),
                ("sum", C.c_void_p), ("out", C.c_void_p), ("sum_row", C.c_longlong), ("out_row", C.c_longlong),
                ("q", C.c_void_p), ("q_row", C.c_longlong), ("q_scale", C.c_void_p), ("device_status", C.c_void_p)]


class QuantizeParams(C.Structure):
    _fields_ = [("x", C.c_void_p), ("x_row", C.c_longlong), ("rows", C.c_longlong), ("dim", C.c_int), ("dtype", C.c_int), ("gated", C.c_int),
                ("q", C.c_void_p), ("q_row", C.c_longlong), ("scale", C.c_void_p), ("device_status", C.c_void_p)]


class MatmulParams(C.Structure):
    _fields_ = [("x", C.c_void_p), ("x_row", C.c_longlong), ("x_scale", C.c_void_p), ("rows", C.c_longlong), ("w", C.c_void_p),
                ("w_row", C.c_longlong), ("w_scale", C.c_void_p), ("inner", C.c_int), ("outer", C.c_int), ("bias", C.c_void_p),
                ("out", C.c_void_p), ("out_row", C.c_longlong), ("out_dtype", C.c_int), ("device_status", C.c_void_p)]


def _rows(t: torch.Tensor, rows: int, width: int, dtype: torch.dtype, index: int, what: str):
    """Address and row stride of [rows, width] (the call itself wants a row stride of at least width, more rows than one)."""
    if t.dtype is not dtype or t.shape != (rows, width) or t.get_device() != index:
        raise ValueError("%s must be a %s tensor %s on the plan's device" % (what, dtype, [rows, width]))
    row, col = t.stride()
    if col != 1 and width > 1 and rows > 0:
        raise ValueError("%s must have contiguous channels" % what)
    return t.data_ptr(), row


def _weights(t: Optional[torch.Tensor], dim: int, index: int, what: str) -> Optional[int]:
    if t is None:
        return None
    _want(t.dtype is torch.float32 and t.shape == (dim,) and t.is_contiguous() and t.get_device() == index,
          "%s must be a contiguous float32 tensor [%d] on the plan's device" % (what, dim))
    return t.data_ptr()


def _index(device) -> int:
    device = torch.device(device)
    _want(device.type == "cuda", "a plan's device must be a CUDA device")
    return _device() if device.index is None else device.index


def _on(index: int) -> int:
    if _device() != index:
        raise ValueError("the plan's device is not the current CUDA device")
    return _raw_stream(index)


@dataclass
class QuantRows:
    """Rows in 8 bits: ``q`` int8 ``[rows, dim]`` (row stride a multiple of 16, 16-byte aligned), ``scale`` float32 ``[rows]``."""
    q: torch.Tensor
    scale: torch.Tensor

    def dequantized(self) -> torch.Tensor:
        return self.q.float() * self.scale.unsqueeze(1)


def empty_quant_rows(rows: int, dim: int, device="cuda") -> QuantRows:
    q = torch.empty((rows, -(-dim // 16) * 16), dtype=torch.int8, device=device)[:, :dim]
    return QuantRows(q, torch.empty(rows, dtype=torch.float32, device=device))


@dataclass
class NormOutput:
    sum: Optional[torch.Tensor]      # [rows, dim] the residual stream
    out: Optional[torch.Tensor]      # [rows, dim] its norm
    rows: Optional[QuantRows]        # the same in 8 bits


class NormPlan:
    """Repeated sttm_block_norm calls: ``sum = residual_scale * residual + gate * norm(x; post_norm)`` and
    ``out = norm(sum; pre_norm)``, in 8 bits instead when ``quantize``.  ``post_norm``, ``gate``, ``pre_norm``: float32 ``[dim]`` or
    None (no norm, a gate of 1).  Without ``pre_norm`` and ``quantize`` there is no ``out``."""

    def __init__(self, dim: int, dtype: torch.dtype, max_rows: int, post_norm: Optional[torch.Tensor] = None, gate: Optional[torch.Tensor] = None,
                 residual_scale: float = 1.0, pre_norm: Optional[torch.Tensor] = None, eps: float = 1e-6, quantize: bool = False, device="cuda"):
        _want(dtype in _TYPES and dim >= 1 and max_rows >= 0, "rows must be bf16, fp16 or fp32, of at least one channel")
        self.index, self.dim, self.dtype, self.max_rows, self.quantize = _index(device), dim, dtype, max_rows, quantize
        self.normed, self.keep = pre_norm is not None and not quantize, (post_norm, gate, pre_norm)
        device = torch.device("cuda", self.index)
        self.sum = torch.empty((max_rows, dim), dtype=dtype, device=device)
        self.out = torch.empty((max_rows, dim), dtype=dtype, device=device) if self.normed else None
        self.rows = empty_quant_rows(max_rows, dim, device) if quantize else None
        self.status = torch.zeros(1, dtype=torch.int32, device=device)
        p = self.params = NormParams()
        p.device_status = self.status.data_ptr()
        p.dim, p.dtype, p.residual_scale, p.eps = dim, _TYPES[dtype], residual_scale, eps
        p.post_norm, p.gate, p.pre_norm = (_weights(t, dim, self.index, n) for t, n in ((post_norm, "post_norm"), (gate, "gate"), (pre_norm, "pre_norm")))
        self.at, self.call = C.byref(p), binding.load_library().sttm_block_norm
        self.last = (-1, None)

    def _outputs(self, n: int) -> NormOutput:
        """The first n rows of the plan's buffers (the views of the last number of rows are kept: making them takes longer than a small call)."""
        if self.last[0] != n:
            if n > self.max_rows:
                raise ValueError("%d rows: the plan has room for %d" % (n, self.max_rows))
            self.last = n, NormOutput(self.sum[:n], self.out[:n] if self.normed else None,
                                      QuantRows(self.rows.q[:n], self.rows.scale[:n]) if self.quantize else None)
        return self.last[1]

    def run(self, x: torch.Tensor, residual: Optional[torch.Tensor] = None, gate: Optional[torch.Tensor] = None, sum: Optional[torch.Tensor] = None) -> NormOutput:
        """``x``, ``residual``, ``gate`` (a gate for every row) ``[rows, dim]`` with any row strides of at least ``dim``; ``sum``: where the residual
        stream goes instead of the plan's buffer, ``residual`` itself for instance."""
        p, n, index = self.params, x.shape[0], self.index
        mine = self._outputs(n)
        p.x, p.x_row = _rows(x, n, self.dim, self.dtype, index, "x")
        p.residual, p.residual_row = (None, 0) if residual is None else _rows(residual, n, self.dim, self.dtype, index, "residual")
        p.gate_rows, p.gate_row = (None, 0) if gate is None else _rows(gate, n, self.dim, self.dtype, index, "gate")
        p.sum, p.sum_row = (self.sum.data_ptr(), self.dim) if sum is None else _rows(sum, n, self.dim, self.dtype, index, "sum")
        p.rows = n
        if self.normed:
            p.out, p.out_row = self.out.data_ptr(), self.dim
        if self.quantize:
            p.q, p.q_row, p.q_scale = self.rows.q.data_ptr(), self.rows.q.stride(0), self.rows.scale.data_ptr()
        code = self.call(self.at, _on(index))
        if code:
            _check(code, "sttm_block_norm")
        return mine if sum is None else NormOutput(sum, mine.out, mine.rows)


class QuantizePlan:
    """Repeated sttm_quantize_rows calls.  ``gated``: rows are ``[a | b]`` of ``2 dim`` channels and ``silu(a) * b`` is quantized.  More than
    16384 channels, up to 32768, want rows of whole 16-byte words."""

    def __init__(self, dim: int, dtype: torch.dtype, max_rows: int, gated: bool = False, device="cuda"):
        _want(dtype in _TYPES and dim >= 1 and max_rows >= 0, "rows must be bf16, fp16 or fp32, of at least one channel")
        self.index, self.width, self.dtype, self.max_rows = _index(device), 2 * dim if gated else dim, dtype, max_rows
        self.rows = empty_quant_rows(max_rows, dim, torch.device("cuda", self.index))
        self.status = torch.zeros(1, dtype=torch.int32, device=self.rows.q.device)
        p = self.params = QuantizeParams()
        p.device_status = self.status.data_ptr()
        p.dim, p.dtype, p.gated = dim, _TYPES[dtype], int(gated)
        p.q, p.q_row, p.scale = self.rows.q.data_ptr(), self.rows.q.stride(0), self.rows.scale.data_ptr()
        self.at, self.call = C.byref(p), binding.load_library().sttm_quantize_rows
        self.last = (-1, None)

    def run(self, x: torch.Tensor) -> QuantRows:
        """``x`` ``[rows, dim]`` (``[rows, 2 dim]`` when gated) with any row stride of at least that."""
        p, n = self.params, x.shape[0]
        if self.last[0] != n:
            if n > self.max_rows:
                raise ValueError("%d rows: the plan has room for %d" % (n, self.max_rows))
            self.last = n, QuantRows(self.rows.q[:n], self.rows.scale[:n])
        p.x, p.x_row = _rows(x, n, self.width, self.dtype, self.index, "x")
        p.rows = n
        code = self.call(self.at, _on(self.index))
        if code:
            _check(code, "sttm_quantize_rows")
        return self.last[1]


def _quant_rows(r: QuantRows, rows: int, dim: int, index: int, what: str):
    q, s = r.q, r.scale
    if (q.dtype is not torch.int8 or q.shape != (rows, dim) or q.get_device() != index or s.dtype is not torch.float32 or s.shape != (rows,)
            or s.get_device() != index or not s.is_contiguous()):
        raise ValueError("%s must be int8 [%d, %d] with float32 scales, on the plan's device" % (what, rows, dim))
    row, col = q.stride()
    if col != 1 and dim > 1 and rows > 0:
        raise ValueError("%s must have contiguous channels" % what)
    return q.data_ptr(), row if rows > 1 else -(-dim // 16) * 16, s.data_ptr()


class MatmulPlan:
    """Repeated sttm_quant_matmul calls with one weight: ``weight`` its output channels as QuantRows ``[outer, inner]``, ``bias`` float32
    ``[outer]`` or None; outputs are ``dtype``."""

    def __init__(self, weight: QuantRows, dtype: torch.dtype, max_rows: int, bias: Optional[torch.Tensor] = None):
        _want(dtype in _TYPES and weight.q.dim() == 2 and weight.q.is_cuda and max_rows >= 0,
              "weight must be rows in 8 bits on a CUDA device, outputs bf16, fp16 or fp32")
        self.index, self.dtype, self.max_rows, self.keep = weight.q.get_device(), dtype, max_rows, (weight, bias)
        self.outer, self.inner = weight.q.shape
        device = weight.q.device
        self.out = torch.empty((max_rows, self.outer), dtype=dtype, device=device)
        self.status = torch.zeros(1, dtype=torch.int32, device=device)
        p = self.params = MatmulParams()
        p.w, p.w_row, p.w_scale = _quant_rows(weight, self.outer, self.inner, self.index, "weight")
        p.inner, p.outer, p.out_dtype, p.device_status = self.inner, self.outer, _TYPES[dtype], self.status.data_ptr()
        p.bias = _weights(bias, self.outer, self.index, "bias")
        self.at, self.call = C.byref(p), binding.load_library().sttm_quant_matmul
        self.last = (-1, None)

    def run(self, x: QuantRows, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """``x`` ``[rows, inner]``; returns ``[rows, outer]``, ``out`` if it is given (any row stride of at least ``outer``)."""
        p, n = self.params, x.q.shape[0]
        p.x, p.x_row, p.x_scale = _quant_rows(x, n, self.inner, self.index, "x")
        if out is None:
            if self.last[0] != n:
                if n > self.max_rows:
                    raise ValueError("%d rows: the plan has room for %d" % (n, self.max_rows))
                self.last = n, self.out[:n]
            p.out, p.out_row = self.out.data_ptr(), self.outer
            out = self.last[1]
        else:
            p.out, p.out_row = _rows(out, n, self.outer, self.dtype, self.index, "out")
        p.rows = n
        code = self.call(self.at, _on(self.index))
        if code:
            _check(code, "sttm_quant_matmul")
        return out


def sttm_block_norm(x: torch.Tensor, residual: Optional[torch.Tensor] = None, post_norm: Optional[torch.Tensor] = None, gate: Optional[torch.Tensor] = None,
                    residual_scale: float = 1.0, pre_norm: Optional[torch.Tensor] = None, eps: float = 1e-6, quantize: bool = False) -> NormOutput:
    """One NormPlan.run; ``gate`` float32 ``[dim]`` or ``[rows, dim]`` of the rows' type."""
    rows = gate is not None and gate.dim() == 2
    plan = NormPlan(x.shape[1], x.dtype, x.shape[0], post_norm, None if rows else gate, residual_scale, pre_norm, eps, quantize, x.device)
    return plan.run(x, residual, gate if rows else None)


def sttm_quantize_rows(x: torch.Tensor, gated: bool = False) -> QuantRows:
    """Rows in 8 bits, a weight's output channels for instance; see QuantizePlan."""
    _want(x.dim() == 2 and not (gated and x.shape[1] % 2), "x must be [rows, dim], [rows, 2 dim] when gated")
    return QuantizePlan(x.shape[1] // 2 if gated else x.shape[1], x.dtype, x.shape[0], gated, x.device).run(x)


def sttm_quant_matmul(x: QuantRows, weight: QuantRows, dtype: torch.dtype, bias: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Product of 8-bit rows; see MatmulPlan."""
    return MatmulPlan(weight, dtype, x.q.shape[0], bias).run(x)
