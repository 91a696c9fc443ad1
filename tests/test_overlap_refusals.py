"""Outputs that share memory with anything else that a decoder layer's call reads or writes are refused, before anything reaches a GPU."""
import ctypes as C

import pytest

from paper_2507_07990_b200 import binding, cache, layer, prefix

ARG = 1
BUF = (C.c_char * (1 << 17))()
AT = (C.addressof(BUF) + 255) // 256 * 256


def make(struct, **kw):
    p = struct()
    for k, v in kw.items():
        setattr(p, k, v)
    return p


# where every array lies, and its bytes: 4 rows of 64
NORM = dict(x=512, residual=512, gate_rows=512, post_norm=256, gate=256, pre_norm=256, sum=512, out=512, q=256, q_scale=16, device_status=4)
QUANTIZE = dict(x=1024, q=256, scale=16, device_status=4)
MATMUL = dict(x=256, x_scale=16, w=32 * 64, w_scale=128, bias=128, out=4 * 32 * 2, device_status=4)
# 5 rows, 4 heads of 64 channels, 3 sequences, 2 prefixes
PREFIX = dict(q=2560, row_offsets=32, seq_offsets=12, prefix_lengths=8, lengths=12, out=2560, lse=80, device_status=4)


def places(sizes):
    return {name: AT + 4096 * i for i, name in enumerate(sizes)}


def refused(call, sizes, outputs, free=()):
    for out in outputs:
        step = {"q": 1, "sum": 2}.get(out, 4)
        for other in sizes:
            if other == out or (out, other) in free or (other, out) in free:
                continue
            at = places(sizes)
            for shift in (-sizes[out] + step, sizes[other] - step):          # their first, their last bytes
                at[out] = at[other] + shift // step * step
                assert call(at) == ARG, (out, other, shift)


@pytest.mark.parametrize("dtype", [0, 2])
def test_norms(dtype):
    lib = binding.load_library()
    call = lambda at: lib.sttm_block_norm(C.byref(make(  # noqa: E731
        layer.NormParams, x_row=64, residual_row=64, gate_row=64, rows=4, dim=64, dtype=dtype, residual_scale=1.0, eps=1e-6, sum_row=64, out_row=64, q_row=64,
        **at)), None)
    refused(call, NORM, ["sum", "out", "q", "q_scale"])


def test_8_bit_rows():
    lib = binding.load_library()
    call = lambda at: lib.sttm_quantize_rows(C.byref(make(layer.QuantizeParams, x_row=128, rows=4, dim=64, dtype=0, gated=1, q_row=64, **at)), None)  # noqa: E731
    refused(call, QUANTIZE, ["q", "scale"])


def test_products():
    lib = binding.load_library()
    call = lambda at: lib.sttm_quant_matmul(C.byref(make(layer.MatmulParams, x_row=64, rows=4, w_row=64, inner=64, outer=32, out_row=32, out_dtype=0, **at)), None)  # noqa: E731
    refused(call, MATMUL, ["out"])


def test_prefix_attention():
    lib = binding.load_library()
    pool = lambda seqs: cache.SttmCache(AT + 65536, AT + 65536, 10, 2, 16, 64, 2 * 16 * 64, 16 * 64, 64, AT + 65536, 4, 4, seqs, 0)  # noqa: E731
    pre, own = pool(2), pool(3)

    def call(at, ws=AT + 8 * 4096, at_ws=None):
        p = make(prefix.PrefixParams, q_row=256, q_head=64, rows=5, q_heads=4, seqs=3, max_prefix=64, max_own=64, scale=1.0, **at)
        need = lib.sttm_prefix_workspace_bytes(C.byref(pre), C.byref(own), C.byref(p))
        return lib.sttm_prefix_attend(C.byref(pre), C.byref(own), C.byref(p), ws, need, None)

    # (queries have been read when outputs are written; 16-byte aligned outputs cannot begin at a shorter array's last word)
    refused(call, PREFIX, ["lse"], free=[("lse", "q")])
    for other in PREFIX:
        if other not in ("q", "out"):
            at = places(PREFIX)
            at["out"] = at[other] - 2544
            at[other] = at["out"] + 2560 - (8 if other == "row_offsets" else 4)
            assert call(at) == ARG, other
    for name in PREFIX:                                         # the workspace
        at = places(PREFIX)
        assert call(at, ws=at[name]) == ARG, name


def test_strides_whose_spans_pass_64_bits():
    lib = binding.load_library()
    args = dict(x_row=64, rows=4, w_row=64, inner=64, outer=32, out_row=32, out_dtype=0)
    for kw in (dict(x_row=2 ** 61), dict(w_row=2 ** 59), dict(out_row=2 ** 62)):
        assert lib.sttm_quant_matmul(C.byref(make(layer.MatmulParams, **{**args, **kw}, **places(MATMUL))), None) == ARG, kw
