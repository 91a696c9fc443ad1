"""Calls of a decoder layer on no rows at all: nothing to do, whatever the addresses (empty tensors have none)."""
import ctypes as C

import pytest
import torch

from paper_2507_07990_b200 import binding, cache, layer, prefix


def make(struct, **kw):
    p = struct()
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def test_of_the_library():
    lib = binding.load_library()
    norm = dict(rows=0, dim=64, dtype=0, residual_scale=1.0, eps=1e-6)
    assert lib.sttm_block_norm(C.byref(make(layer.NormParams, **norm)), None) == 0
    assert lib.sttm_block_norm(C.byref(make(layer.NormParams, **{**norm, "eps": -1.0})), None) == 1
    assert lib.sttm_quantize_rows(C.byref(make(layer.QuantizeParams, rows=0, dim=64, dtype=0)), None) == 0


@pytest.mark.gpu
def test_of_the_plans():
    none = torch.empty((0, 64), dtype=torch.bfloat16, device="cuda")
    ones = torch.ones(64, device="cuda")
    for kw in (dict(), dict(pre_norm=ones), dict(quantize=True), dict(residual=none, post_norm=ones)):
        got = layer.sttm_block_norm(none, **kw)
        assert got.sum.shape == (0, 64) and (got.out is None or got.out.shape == (0, 64))
    rows = layer.sttm_quantize_rows(none)
    w = layer.sttm_quantize_rows(torch.randn((48, 64), device="cuda"))
    assert layer.sttm_quant_matmul(rows, w, torch.bfloat16).shape == (0, 48)
    pool = cache.empty_cache(1, 32, 2, 64)
    ints = lambda *x, t=torch.int32: torch.tensor(x, dtype=t, device="cuda")  # noqa: E731
    got = prefix.sttm_prefix_attend(pool, torch.empty((0, 4, 64), dtype=torch.bfloat16, device="cuda"), ints(0, 0, t=torch.int64), ints(5))
    assert got.out.shape == (0, 4, 64) and int(got.status) == 0
