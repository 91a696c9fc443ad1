"""Block norms, 8-bit rows and their products (sttm_block_norm, sttm_quantize_rows, sttm_quant_matmul) on the GPU against the
definition in 64 bits.

Tolerances.  Norms: one rounding to the type (half a step, ROUNDING), and fp32 arithmetic: a sum of squares of at most 16384 elements in
partial sums of 32 and a tree (below 2^-17 of it, 2^-18 of the factor), a root, three products and a sum: 2^-16 of what is added.
8 bits: the step and the value divided by it are off by 2^-16 relatively, so q is off by half a step and 127 * 2^-16 of one.
Products: sums are whole numbers and exact; three fp32 operations (2^-22) and one rounding."""
import math

import pytest
import torch

from paper_2507_07990_b200 import binding, layer

pytestmark = pytest.mark.gpu

ROUNDING = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
TYPES = [torch.bfloat16, torch.float16, torch.float32]


def rows_of(gen, rows, width, dtype, stride=None, shift=0):
    """[rows, width] with a row stride and a shifted start."""
    stride = stride or width
    flat = torch.randn(rows * stride + shift, generator=gen).to(dtype).cuda()
    return flat[shift:].view(rows, stride)[:, :width] if rows else flat[:0].view(0, width)


def rms(x, w, eps):
    return x if w is None else x / (x.pow(2).mean(-1, keepdim=True) + eps).sqrt() * w.double()


def expect(x, residual, post, gates, scale, pre, eps):
    y = rms(x.double(), post, eps)
    for g in gates:
        y = y * g.double()
    r = y + (scale * residual.double() if residual is not None else 0.0)
    size = y.abs() + (abs(scale) * residual.double().abs() if residual is not None else 0.0)
    return r, size, rms(r, pre, eps)


def check_norm(got, x, residual, post, gates, scale, pre, eps, quantize):
    dtype = x.dtype
    r, size, t = expect(x, residual, post, gates, scale, pre, eps)
    tiny = 2.0 ** -25 if dtype is torch.float16 else 1e-37
    assert not ((got.sum.double() - r).abs() > ROUNDING[dtype] * r.abs() + 2.0 ** -16 * size + tiny).any()
    # an element of the sum that is off by 2^-16 of what was added is off by as much times the norm's factor
    ratio = t.abs() / r.abs().clamp(min=1e-300) if pre is not None else torch.ones_like(t)
    off = 2.0 ** -16 * t.abs() + 2.0 ** -16 * size * torch.where(r == 0, 0.0, ratio)
    if got.out is not None:
        assert not ((got.out.double() - t).abs() > ROUNDING[dtype] * t.abs() + off + tiny).any()
    if quantize:
        step = t.abs().amax(1, keepdim=True) / 127
        assert not ((got.rows.scale.double() - step[:, 0]).abs() > 2.0 ** -15 * step[:, 0]).any()
        assert not ((got.rows.dequantized().double() - t).abs() > step * (0.5 + 127 * 2.0 ** -14) + off).any()
        assert int(got.rows.q.abs().max()) == 127


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,width", [(1, 3584), (5, 8), (7, 1), (3, 1157), (9, 1024), (2, 16384), (2, 16383), (131, 256), (3, 4104), (3, 8192), (3, 2052)])
def test_block_norm(dtype, rows, width):
    gen = torch.Generator().manual_seed(rows * 20000 + width)
    w = [(1 + 0.3 * torch.randn(width, generator=gen)).cuda() for _ in range(3)]
    x, residual, gate = (rows_of(gen, rows, width, dtype) for _ in range(3))
    for kw, g in [(dict(post_norm=w[0], gate=w[1], pre_norm=w[2], residual_scale=0.7), None), (dict(pre_norm=w[2]), None), (dict(post_norm=w[0]), gate),
                  (dict(gate=w[1], pre_norm=w[2], quantize=True), gate), (dict(quantize=True), None)]:
        plan = layer.NormPlan(width, dtype, rows + 2, eps=1e-5, **kw)
        got = plan.run(x, residual, gate=g)
        gates = [t for t in (kw.get("gate"), g) if t is not None]
        check_norm(got, x, residual, kw.get("post_norm"), gates, kw.get("residual_scale", 1.0), kw.get("pre_norm"), 1e-5, kw.get("quantize"))
    got = layer.NormPlan(width, dtype, rows, pre_norm=w[2], eps=1e-5).run(x)        # no residual: the stream is x
    check_norm(got, x, None, None, [], 1.0, w[2], 1e-5, False)


@pytest.mark.parametrize("dtype", TYPES)
def test_block_norm_strides_and_in_place(dtype):
    gen = torch.Generator().manual_seed(3)
    width = 512
    for stride, shift in [(width + 8, 0), (width + 3, 0), (width, 1), (3 * width, 8)]:
        x, residual = rows_of(gen, 6, width, dtype, stride, shift), rows_of(gen, 6, width, dtype, stride, shift)
        plan = layer.NormPlan(width, dtype, 6, pre_norm=torch.ones(width).cuda(), eps=1e-5)
        check_norm(plan.run(x, residual), x, residual, None, [], 1.0, torch.ones(width).cuda(), 1e-5, False)
        want = plan.sum.clone(), plan.out.clone()
        before = residual.clone()
        got = plan.run(x, residual, sum=residual)
        assert got.sum is residual and torch.equal(residual, want[0]) and torch.equal(got.out, want[1]) and not torch.equal(before, want[0])
    zeros = torch.zeros((2, width), dtype=dtype).cuda()
    got = layer.NormPlan(width, dtype, 2, pre_norm=torch.ones(width).cuda(), quantize=True).run(zeros)
    assert not got.sum.any() and not got.rows.q.any() and not got.rows.scale.any()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("width,stride,shift", [(3584, 3584, 0), (1157, 1157, 0), (96, 104, 8), (67, 67, 3), (1000, 1003, 1), (2048, 2056, 0)])
def test_many_rows(dtype, width, stride, shift):
    # a warp to a row, out of shared memory; rows that share 16-byte words with their neighbours, in place too
    gen = torch.Generator().manual_seed(width)
    rows = 1301
    w = [(1 + 0.3 * torch.randn(width, generator=gen)).cuda() for _ in range(3)]
    x, residual, gate = (rows_of(gen, rows, width, dtype, stride, shift) for _ in range(3))
    for kw, g in [(dict(post_norm=w[0], gate=w[1], pre_norm=w[2], residual_scale=0.7), None), (dict(pre_norm=w[2]), gate),
                  (dict(post_norm=w[0], pre_norm=w[2], quantize=True), gate)]:
        plan = layer.NormPlan(width, dtype, rows, eps=1e-5, **kw)
        got = plan.run(x, residual, gate=g)
        gates = [t for t in (kw.get("gate"), g) if t is not None]
        check_norm(got, x, residual, kw.get("post_norm"), gates, kw.get("residual_scale", 1.0), w[2], 1e-5, kw.get("quantize"))
        want, mine = got.sum.clone(), residual.clone()
        room = rows_of(gen, rows, width, dtype, stride, shift)
        room.copy_(mine)
        assert torch.equal(plan.run(x, room, gate=g, sum=room).sum, want) and int(plan.status) == 0
    got = layer.NormPlan(width, dtype, rows, pre_norm=w[2], eps=1e-5).run(x)
    check_norm(got, x, None, None, [], 1.0, w[2], 1e-5, False)
    for gated in (False, True):
        z = rows_of(gen, rows, 2 * width, dtype, 2 * stride, shift) if gated else x
        y = z.double()
        if gated:
            y = y[:, :width] * torch.sigmoid(y[:, :width]) * y[:, width:]
        q = layer.sttm_quantize_rows(z, gated)
        step = y.abs().amax(1, keepdim=True) / 127
        assert not ((q.scale.double() - step[:, 0]).abs() > 2.0 ** -18 * step[:, 0]).any()
        assert not ((q.dequantized().double() - y).abs() > step * (0.5 + 127 * 2.0 ** -17)).any()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("width,starts", [(1157, (0, 1, 0)), (1157, (1, 1, 1)), (334, (1, 1, 0)), (65, (1, 0, 1))])
def test_many_rows_that_begin_in_different_halves_of_a_word(dtype, width, starts):
    gen = torch.Generator().manual_seed(width + starts[1])
    rows = 1301
    w = [(1 + 0.3 * torch.randn(width, generator=gen)).cuda() for _ in range(2)]
    x, residual, gate = (rows_of(gen, rows, width, dtype, width + (i & 1), s) for i, s in enumerate(starts))
    for quantize in (False, True):
        got = layer.NormPlan(width, dtype, rows, eps=1e-5, post_norm=w[0], pre_norm=w[1], residual_scale=0.7, quantize=quantize).run(x, residual, gate=gate)
        check_norm(got, x, residual, w[0], [gate], 0.7, w[1], 1e-5, quantize)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,width", [(1, 14336), (33, 64), (5, 1157), (4, 3584), (3, 1), (2, 16384)])
@pytest.mark.parametrize("gated", [False, True])
def test_quantize_rows(dtype, rows, width, gated):
    gen = torch.Generator().manual_seed(width)
    x = rows_of(gen, rows, 2 * width if gated else width, dtype, shift=8 if width % 8 == 0 else 1)
    y = x.double()
    if gated:
        y = y[:, :width] * torch.sigmoid(y[:, :width]) * y[:, width:]
    got = layer.sttm_quantize_rows(x, gated)
    step = y.abs().amax(1, keepdim=True) / 127
    assert not ((got.scale.double() - step[:, 0]).abs() > 2.0 ** -18 * step[:, 0]).any()
    assert not ((got.dequantized().double() - y).abs() > step * (0.5 + 127 * 2.0 ** -17)).any()
    assert got.q.stride(0) % 16 == 0


def test_rows_that_are_not_numbers():
    x = torch.randn((6, 320)).cuda()
    x[1, 5], x[2, 300], x[3, 7] = math.inf, math.nan, -math.inf
    x[4] = 1e-33
    x[5] = 0.0
    r = layer.sttm_quantize_rows(x)
    assert torch.isnan(r.scale[1:4]).all() and not r.q[1:6].any() and not r.scale[4:].any()
    w = layer.sttm_quantize_rows(torch.randn((40, 320)).cuda())
    out = layer.sttm_quant_matmul(r, w, torch.bfloat16, bias=torch.ones(40).cuda())
    assert torch.isfinite(out[0]).all() and torch.isnan(out[1:4]).all() and (out[4:] == 1.0).all()
    got = layer.sttm_block_norm(x.bfloat16(), pre_norm=torch.ones(320).cuda(), quantize=True)
    assert torch.isnan(got.rows.scale[1:4]).all() and torch.isfinite(got.rows.scale[0])


def quant(gen, rows, inner, pad=0):
    width = -(-(inner + pad) // 16) * 16
    q = torch.randint(-127, 128, (max(rows, 1), width), generator=gen).to(torch.int8).cuda()[:rows, :inner]
    return layer.QuantRows(q, (0.5 + torch.rand(rows, generator=gen)).cuda() / 100)


def check_matmul(x, w, bias, out):
    want = x.q.double() @ w.q.double().t()
    want = want * x.scale.double().unsqueeze(1) * w.scale.double()
    size = want.abs()
    if bias is not None:
        want, size = want + bias.double(), size + bias.double().abs()
    tiny = 2.0 ** -25 if out.dtype is torch.float16 else 0.0
    assert not ((out.double() - want).abs() > ROUNDING[out.dtype] * want.abs() + 2.0 ** -22 * size + tiny).any(), float(((out.double() - want).abs() / size.clamp(min=1e-9)).max())


@pytest.mark.parametrize("rows", [1, 2, 16, 17, 33, 64, 100, 128, 200, 256, 257, 300, 513, 1025])
@pytest.mark.parametrize("inner,outer", [(3584, 4608), (64, 16), (1157, 333), (200, 1), (128, 1000), (1, 130)])
def test_quant_matmul(rows, inner, outer):
    gen = torch.Generator().manual_seed(rows * 7 + inner)
    x, w = quant(gen, rows, inner, 5), quant(gen, outer, inner, 40)
    bias = torch.randn(outer, generator=gen).cuda()
    for dtype in TYPES:
        plan = layer.MatmulPlan(w, dtype, rows, bias)
        check_matmul(x, w, bias, plan.run(x))
        assert int(plan.status) == 0
    check_matmul(x, w, None, layer.sttm_quant_matmul(x, w, torch.bfloat16))


@pytest.mark.parametrize("rows,inner,outer", [(20, 256, 50001), (3, 3584, 40000), (700, 384, 20000)])
def test_more_tiles_than_blocks(rows, inner, outer):
    # blocks go from tile to tile
    gen = torch.Generator().manual_seed(outer)
    x, w = quant(gen, rows, inner), quant(gen, outer, inner)
    check_matmul(x, w, None, layer.sttm_quant_matmul(x, w, torch.bfloat16))


def test_the_largest_sums_are_exact():
    inner = 131056
    x = layer.QuantRows(torch.full((3, inner), -128, dtype=torch.int8).cuda(), torch.ones(3).cuda())
    w = layer.QuantRows(torch.full((5, inner), -128, dtype=torch.int8).cuda(), torch.ones(5).cuda())
    assert (layer.sttm_quant_matmul(x, w, torch.float32) == float(128 * 128 * inner)).all()
    x = layer.QuantRows(x.q[:1].expand(300, inner).contiguous(), torch.ones(300).cuda())
    assert (layer.sttm_quant_matmul(x, w, torch.float32) == float(128 * 128 * inner)).all()


@pytest.mark.parametrize("rows", [3, 300])
def test_outputs_with_strides_and_rows_behind_them(rows):
    gen = torch.Generator().manual_seed(4)
    x, w = quant(gen, rows, 500), quant(gen, 72, 500)
    for stride, shift in [(80, 0), (75, 0), (72, 1)]:
        flat = torch.full((rows * stride + shift + 8,), 9.0, dtype=torch.bfloat16).cuda()
        out = flat[shift:shift + rows * stride].view(rows, stride)[:, :72]
        plan = layer.MatmulPlan(w, torch.bfloat16, 0)
        assert plan.run(x, out) is out
        check_matmul(x, w, None, out)
        assert (flat[:shift] == 9.0).all() and (flat[shift + rows * stride:] == 9.0).all()
        assert (flat[shift:shift + rows * stride].view(rows, stride)[:, 72:] == 9.0).all()


def test_a_layers_calls_captured_on_another_stream():
    gen = torch.Generator().manual_seed(6)
    width = 512
    x, residual = rows_of(gen, 9, width, torch.bfloat16), rows_of(gen, 9, width, torch.bfloat16)
    norm = layer.NormPlan(width, torch.bfloat16, 9, pre_norm=torch.ones(width).cuda(), quantize=True)
    up = layer.MatmulPlan(quant(gen, 768, width), torch.bfloat16, 9)
    act = layer.QuantizePlan(384, torch.bfloat16, 9, gated=True)
    down = layer.MatmulPlan(quant(gen, width, 384), torch.bfloat16, 9)
    call = lambda: down.run(act.run(up.run(norm.run(x, residual).rows)))  # noqa: E731
    want = call().clone()
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        with torch.cuda.graph(graph, stream=stream):
            out = call()
    torch.cuda.synchronize()
    out.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)
    x.copy_(-x)
    graph.replay()
    torch.cuda.synchronize()
    assert not torch.equal(out, want)
    check_matmul(act.rows, down.keep[0], None, out)


def test_refusals_of_the_plans():
    gen = torch.Generator().manual_seed(7)
    x = rows_of(gen, 4, 64, torch.bfloat16)
    plan = layer.NormPlan(64, torch.bfloat16, 4, pre_norm=torch.ones(64).cuda())
    for bad in [dict(x=x.float()), dict(x=x[:, :32]), dict(x=torch.cat([x, x])), dict(x=x, residual=x[:2]), dict(x=x, gate=x.float()), dict(x=x.t().contiguous().t())]:
        with pytest.raises(ValueError):
            plan.run(**bad)
    flat = torch.zeros(1000, dtype=torch.bfloat16).cuda()
    with pytest.raises(binding.SttmError):                      # overlapping, but not in place
        plan.run(flat[:256].view(4, 64), None, sum=flat[64:320].view(4, 64))
    with pytest.raises(ValueError):
        layer.NormPlan(64, torch.bfloat16, 4, pre_norm=torch.ones(32).cuda())
    with pytest.raises(binding.SttmError):
        layer.NormPlan(16385, torch.bfloat16, 1).run(torch.zeros((1, 16385), dtype=torch.bfloat16).cuda())
    w = quant(gen, 10, 64)
    mat = layer.MatmulPlan(w, torch.bfloat16, 4)
    for bad in [quant(gen, 4, 48), quant(gen, 5, 64), layer.QuantRows(w.q.float(), w.scale), layer.QuantRows(w.q[:4], w.scale)]:
        with pytest.raises(ValueError):
            mat.run(bad)
    odd = torch.zeros(4 * 72 + 8, dtype=torch.int8).cuda()
    with pytest.raises(binding.SttmError):                      # rows that are no multiple of 16 bytes apart, or start off one
        mat.run(layer.QuantRows(odd[:288].view(4, 72)[:, :64], w.scale[:4].contiguous()))
    with pytest.raises(binding.SttmError):
        mat.run(layer.QuantRows(odd[8:264].view(4, 64), w.scale[:4].contiguous()))
    assert mat.run(quant(gen, 0, 64)).shape == (0, 10) and plan.run(x[:0]).out.shape == (0, 64)


def test_offsets_beyond_32_bits():
    # more than 2^31 elements; the last rows are looked at
    rows, width = 2 ** 31 // 4096 + 300, 4096
    x = torch.empty((rows, width), dtype=torch.bfloat16, device="cuda").fill_(0.5)
    gen = torch.Generator().manual_seed(9)
    x[-3:] = torch.randn((3, width), generator=gen).bfloat16().cuda()
    w = (1 + 0.3 * torch.randn(width, generator=gen)).cuda()
    plan = layer.NormPlan(width, torch.bfloat16, rows, pre_norm=w, eps=1e-5)
    got = plan.run(x, x)
    last = layer.NormOutput(got.sum[-3:], got.out[-3:], None)
    check_norm(last, x[-3:], x[-3:], None, [], 1.0, w, 1e-5, False)
    q = layer.sttm_quantize_rows(x)
    y = x[-3:].double()
    step = y.abs().amax(1, keepdim=True) / 127
    assert not ((layer.QuantRows(q.q[-3:], q.scale[-3:]).dequantized().double() - y).abs() > step * (0.5 + 127 * 2.0 ** -17)).any()
    del plan, got, x
    out = layer.sttm_quant_matmul(q, layer.QuantRows(torch.ones((4100, width), dtype=torch.int8, device="cuda"), torch.ones(4100, device="cuda")), torch.bfloat16)
    assert out.numel() > 2 ** 31
    want = layer.QuantRows(q.q[-3:], q.scale[-3:]).dequantized().double().sum(1, keepdim=True)
    assert not ((out[-3:].double() - want).abs() > 2.0 ** -8 * want.abs() + 1e-4).any() and not ((out[:3] - out[3]).abs() > 0).any()


def test_plans_on_two_streams():
    gen = torch.Generator().manual_seed(10)
    rows = [40, 2000]
    xs = [rows_of(gen, n, 1024, torch.bfloat16) for n in rows]
    w = quant(gen, 512, 1024)
    plans = [(layer.QuantizePlan(1024, torch.bfloat16, n), layer.MatmulPlan(w, torch.bfloat16, n)) for n in rows]
    streams = [torch.cuda.Stream() for _ in rows]
    torch.cuda.synchronize()
    for _ in range(20):
        for x, (quantize, product), stream in zip(xs, plans, streams):
            with torch.cuda.stream(stream):
                product.run(quantize.run(x))
    torch.cuda.synchronize()
    for n, (quantize, product) in zip(rows, plans):
        check_matmul(quantize.rows, w, None, product.out)
        assert int(quantize.status) == int(product.status) == 0
