"""Arguments that the calls of a decoder layer refuse, before anything reaches a GPU."""
import ctypes as C

from paper_2507_07990_b200 import binding, cache, layer, prefix

ARG, UNSUPPORTED, WORKSPACE = 1, 2, 3
BUF = (C.c_char * 65536)()
AT = (C.addressof(BUF) + 255) // 256 * 256


def make(struct, **kw):
    p = struct()
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def norm(**kw):
    return make(layer.NormParams, **{**dict(x=AT, residual=AT + 4096, x_row=64, residual_row=64, rows=4, dim=64, dtype=0, residual_scale=1.0, eps=1e-6,
                                            sum=AT + 8192, sum_row=64), **kw})


def quantize(**kw):
    return make(layer.QuantizeParams, **{**dict(x=AT, x_row=64, rows=4, dim=64, dtype=0, q=AT + 4096, q_row=64, scale=AT + 8192), **kw})


def matmul(**kw):
    return make(layer.MatmulParams, **{**dict(x=AT, x_row=64, x_scale=AT, rows=4, w=AT, w_row=64, w_scale=AT, inner=64, outer=32, out=AT + 16384, out_row=32,
                                              out_dtype=0), **kw})


def pool(**kw):
    c = cache.SttmCache(AT, AT, 10, 2, 16, 64, 2 * 16 * 64, 16 * 64, 64, AT, 4, 4, 1, 0)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def attend(**kw):
    return make(prefix.PrefixParams, **{**dict(q=AT, q_row=256, q_head=64, rows=5, q_heads=4, seqs=3, row_offsets=AT, prefix_lengths=AT, lengths=AT,
                                               max_prefix=64, max_own=64, scale=1.0, out=AT), **kw})


def test_bad_norm_arguments():
    lib = binding.load_library()
    inf, nan = float("inf"), float("nan")
    for kw, code in [(dict(rows=-1), ARG), (dict(dim=0), ARG), (dict(dtype=3), ARG), (dict(sum=None), ARG), (dict(x=None), ARG), (dict(q=AT), ARG),
                     (dict(q_scale=AT), ARG), (dict(residual_scale=nan), ARG), (dict(eps=-1.0), ARG), (dict(eps=nan), ARG), (dict(dim=16385), UNSUPPORTED),
                     (dict(x_row=63), ARG), (dict(residual_row=63), ARG), (dict(sum_row=63), ARG), (dict(x=AT + 1), ARG), (dict(residual_scale=inf), ARG),
                     (dict(pre_norm=AT + 2), ARG), (dict(sum=AT + 128), ARG), (dict(out=AT + 8192, out_row=64), ARG), (dict(sum=AT, sum_row=72), ARG),
                     (dict(q=AT, q_row=64, q_scale=AT + 32768), ARG), (dict(rows=2 ** 31), UNSUPPORTED), (dict(x_row=2 ** 62), ARG)]:
        assert lib.sttm_block_norm(C.byref(norm(**kw)), None) == code, kw
    assert lib.sttm_block_norm(None, None) == ARG
    assert lib.sttm_block_norm(C.byref(norm(rows=0)), None) == 0


def test_bad_quantize_arguments():
    lib = binding.load_library()
    for kw, code in [(dict(rows=-1), ARG), (dict(dim=0), ARG), (dict(dtype=5), ARG), (dict(x=None), ARG), (dict(q=None), ARG), (dict(scale=None), ARG),
                     (dict(scale=AT + 2), ARG), (dict(x=AT + 1), ARG), (dict(x_row=63), ARG), (dict(q_row=63), ARG), (dict(gated=1), ARG),
                     (dict(dim=16385), UNSUPPORTED), (dict(q=AT), ARG), (dict(q=AT + 64), ARG)]:
        assert lib.sttm_quantize_rows(C.byref(quantize(**kw)), None) == code, kw
    assert lib.sttm_quantize_rows(None, None) == ARG
    assert lib.sttm_quantize_rows(C.byref(quantize(rows=0)), None) == 0


def test_bad_matmul_arguments():
    lib = binding.load_library()
    for kw, code in [(dict(rows=-1), ARG), (dict(inner=0), ARG), (dict(outer=0), ARG), (dict(out_dtype=7), ARG), (dict(x=None), ARG), (dict(w=None), ARG),
                     (dict(x_scale=None), ARG), (dict(w_scale=None), ARG), (dict(out=None), ARG), (dict(x=AT + 8), ARG), (dict(w=AT + 8), ARG),
                     (dict(x_row=72), ARG), (dict(w_row=72), ARG), (dict(x_row=48), ARG), (dict(w_row=48), ARG), (dict(out_row=31), ARG),
                     (dict(out=AT + 1), ARG), (dict(bias=AT + 2), ARG), (dict(out=AT), ARG), (dict(out=AT + 1024), ARG), (dict(inner=131057, x_row=131072, w_row=131072), UNSUPPORTED)]:
        assert lib.sttm_quant_matmul(C.byref(matmul(**kw)), None) == code, kw
    assert lib.sttm_quant_matmul(None, None) == ARG
    assert lib.sttm_quant_matmul(C.byref(matmul(rows=0)), None) == 0


def test_bad_prefix_arguments():
    lib = binding.load_library()
    pre, own = pool(), pool(seqs=3)
    need = lib.sttm_prefix_workspace_bytes(C.byref(pre), C.byref(own), C.byref(attend()))
    assert need > lib.sttm_prefix_workspace_bytes(C.byref(pre), None, C.byref(attend())) > 0
    call = lambda p, a=pre, b=own, ws=AT, n=need: lib.sttm_prefix_attend(C.byref(a), C.byref(b) if b is not None else None, C.byref(p), ws, n, None)  # noqa: E731
    nan = float("nan")
    for kw, code in [(dict(q=None), ARG), (dict(out=None), ARG), (dict(row_offsets=None), ARG), (dict(prefix_lengths=None), ARG), (dict(lengths=None), ARG),
                     (dict(rows=-1), ARG), (dict(seqs=0), ARG), (dict(seqs=2), ARG), (dict(q_heads=3), ARG), (dict(q_heads=0), ARG), (dict(max_prefix=0), ARG),
                     (dict(max_prefix=65), ARG), (dict(max_own=0), ARG), (dict(max_own=65), ARG), (dict(scale=0.0), ARG), (dict(scale=-1.0), ARG),
                     (dict(scale=nan), ARG), (dict(q=AT + 8), ARG), (dict(out=AT + 8), ARG), (dict(q_row=252), ARG), (dict(q_head=60), ARG), (dict(q_row=8), ARG),
                     (dict(row_offsets=AT + 4), ARG), (dict(lse=AT + 2), ARG), (dict(q_heads=130), UNSUPPORTED), (dict(rows=2 ** 31), UNSUPPORTED)]:
        assert call(attend(**kw)) == code, kw
    for kw, code in [(dict(dim=96), UNSUPPORTED), (dict(page=12), UNSUPPORTED), (dict(table=None), ARG), (dict(seqs=2), ARG), (dict(dtype=1), UNSUPPORTED)]:
        assert call(attend(), a=pool(**kw)) == code, kw          # (two prefixes want seq_offsets)
    for kw in [dict(heads=1), dict(dim=128, slot_stride=128), dict(dtype=2), dict(seqs=2)]:
        assert call(attend(), b=pool(**{**dict(seqs=3), **kw})) == ARG, kw
    assert call(attend(), ws=None) == ARG and call(attend(), ws=AT + 128) == ARG and call(attend(), n=need - 1) == WORKSPACE
    assert lib.sttm_prefix_attend(None, None, C.byref(attend()), AT, need, None) == ARG
    assert lib.sttm_prefix_attend(C.byref(pre), None, None, AT, need, None) == ARG
    assert call(attend(rows=0)) == 0
