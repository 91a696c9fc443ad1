"""Arrays that lie directly beside each other in memory, without overlapping, in the calls of a decoder layer: as an allocator may place them, or a
program that cuts one buffer up.  Same results as in buffers of their own; one byte closer is refused."""
import ctypes as C

import pytest
import torch

from paper_2507_07990_b200 import binding, layer
from tests.test_gpu_prefix import plan_of, problem, run

pytestmark = pytest.mark.gpu

ARG = 1
CODES = {torch.bfloat16: 0, torch.float32: 1, torch.float16: 2}


def call(name, struct, **kw):
    p = struct()
    for k, v in kw.items():
        setattr(p, k, v.data_ptr() if isinstance(v, torch.Tensor) else v)
    return getattr(binding.load_library(), name)(C.byref(p), torch.cuda.current_stream().cuda_stream)


def cut(flat, at, rows, width, dtype):
    """[rows, width] out of a buffer of bytes, and where it ends."""
    end = at + rows * width * dtype.itemsize
    return flat[at:end].view(dtype).view(rows, width), end


@pytest.mark.parametrize("dtype", list(CODES))
@pytest.mark.parametrize("rows,dim", [(1, 14336), (1, 3584), (3, 1024), (1200, 512), (2, 333)])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("q_first", [True, False])
def test_8_bit_rows_beside_their_input(q_first, gated, rows, dim, dtype):
    gen = torch.Generator().manual_seed(dim)
    x = torch.randn((rows, 2 * dim if gated else dim), generator=gen).to(dtype).cuda()
    want = layer.sttm_quantize_rows(x, gated)
    scale = torch.empty(rows, device="cuda")
    flat = torch.zeros(rows * dim + x.numel() * x.itemsize + 16, dtype=torch.int8, device="cuda")
    gap = -rows * dim % dtype.itemsize if q_first else 0
    if q_first:
        q, at = cut(flat, 0, rows, dim, torch.int8)
        xs, _ = cut(flat, at + gap, rows, x.shape[1], dtype)
    else:
        xs, at = cut(flat, 0, rows, x.shape[1], dtype)
        q, _ = cut(flat, at, rows, dim, torch.int8)
    xs.copy_(x)
    args = dict(x=xs, x_row=x.shape[1], rows=rows, dim=dim, dtype=CODES[dtype], gated=int(gated), q=q, q_row=dim, scale=scale)
    assert call("sttm_quantize_rows", layer.QuantizeParams, **args) == 0
    assert torch.equal(q, want.q) and torch.equal(scale, want.scale) and torch.equal(xs, x)
    closer = q.data_ptr() + gap + 1 if q_first else q.data_ptr() - 1
    assert call("sttm_quantize_rows", layer.QuantizeParams, **{**args, "q": closer}) == ARG


@pytest.mark.parametrize("dtype", list(CODES))
@pytest.mark.parametrize("rows,dim", [(1, 3584), (3, 1024), (1500, 512), (2, 333)])
@pytest.mark.parametrize("beside", ["x", "residual", "gate_rows", "sum", "out"])
@pytest.mark.parametrize("q_first", [True, False])
def test_a_norms_8_bit_rows_beside_its_other_arrays(q_first, beside, rows, dim, dtype):
    gen = torch.Generator().manual_seed(dim + 1)
    x, residual, gate = (torch.randn((rows, dim), generator=gen).to(dtype).cuda() for _ in range(3))
    pre = torch.ones(dim, device="cuda")
    arrays = dict(x=x, residual=residual, gate_rows=gate, sum=torch.empty_like(x), out=torch.empty_like(x))
    scale = torch.empty(rows, device="cuda")
    args = dict(x_row=dim, residual_row=dim, gate_row=dim, sum_row=dim, out_row=dim, rows=rows, dim=dim, dtype=CODES[dtype], residual_scale=0.5, eps=1e-6,
                pre_norm=pre, q_row=dim, q_scale=scale)
    q = torch.empty((rows, dim), dtype=torch.int8, device="cuda")
    assert call("sttm_block_norm", layer.NormParams, q=q, **arrays, **args) == 0
    want = [t.clone() for t in (q, scale, arrays["sum"], arrays["out"])]
    flat = torch.zeros(rows * dim * (1 + x.itemsize) + 16, dtype=torch.int8, device="cuda")
    gap = -rows * dim % dtype.itemsize if q_first else 0
    if q_first:
        q, at = cut(flat, 0, rows, dim, torch.int8)
        moved, _ = cut(flat, at + gap, rows, dim, dtype)
    else:
        moved, at = cut(flat, 0, rows, dim, dtype)
        q, _ = cut(flat, at, rows, dim, torch.int8)
    moved.copy_(arrays[beside])
    arrays[beside] = moved
    scale.zero_()
    assert call("sttm_block_norm", layer.NormParams, q=q, **arrays, **args) == 0
    for got, w in zip((q, scale, arrays["sum"], arrays["out"]), want):
        assert torch.equal(got, w)
    closer = q.data_ptr() + gap + 1 if q_first else q.data_ptr() - 1
    assert call("sttm_block_norm", layer.NormParams, q=closer, **arrays, **args) == ARG


@pytest.mark.parametrize("rows", [1, 40, 500])
def test_a_products_arrays_beside_each_other(rows):
    gen = torch.Generator().manual_seed(rows)
    x, w = (layer.sttm_quantize_rows(torch.randn((n, 1024), generator=gen).cuda()) for n in (rows, 336))
    bias = torch.randn(336, generator=gen).cuda()
    want = layer.sttm_quant_matmul(x, w, torch.bfloat16, bias)
    flat = torch.zeros(rows * (1024 + 4 + 672) + 336 * (1024 + 8) + 256, dtype=torch.int8, device="cuda")
    for order in (["out", "x", "w", "x_scale", "w_scale", "bias"], ["x", "out", "w_scale", "bias", "w", "x_scale"]):
        at, placed = 0, {}
        for name in order:
            data = dict(x=x.q, w=w.q, x_scale=x.scale.unsqueeze(1), w_scale=w.scale.unsqueeze(1), bias=bias.unsqueeze(1), out=torch.zeros_like(want))[name]
            at = -(-at // 16) * 16
            placed[name], at = cut(flat, at, data.shape[0], data.shape[1], data.dtype)
            placed[name].copy_(data)
        assert call("sttm_quant_matmul", layer.MatmulParams, x_row=1024, w_row=1024, rows=rows, inner=1024, outer=336, out_row=336, out_dtype=0, **placed) == 0
        assert torch.equal(placed["out"], want)


@pytest.mark.parametrize("length,new", [(300, (1, 2)), (3000, (70, 41))])
def test_attention_written_where_the_queries_lie(length, new):
    p = problem(3, q_heads=8, heads=2, lens=(length,), groups=(2,), new=new, held=(3, 0), spare=0)
    p["q"] = p["q"].contiguous()
    plan = plan_of(p)
    want = run(p, plan).out.clone()
    assert torch.equal(run(p, plan, out=p["q"]).out, want) and torch.equal(p["q"], want)
