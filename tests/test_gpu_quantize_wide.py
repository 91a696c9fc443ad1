"""Rows of more than 16384 channels in 8 bits: the inner widths of large gated blocks (18944, 29568), as they come, out of a gated activation, and
into a product.

Tolerances: the largest magnitude is exact for rows as they are; silu takes an exponential, an addition, a division and a product in 32 bits (2 + 0.5 + 0.5
ulp for sigmoid's parts, half a step for the product: below 2^-21 of the value), the scale one more product: 2^-20 together.  A value divided by its step is off by as much,
of at most 127 steps."""
import math

import pytest
import torch

from paper_2507_07990_b200 import binding, layer

pytestmark = pytest.mark.gpu

TYPES = [torch.bfloat16, torch.float16, torch.float32]


def check(got, x, gated):
    y = x.double()
    if gated:
        width = y.shape[1] // 2
        y = y[:, :width] / (1 + torch.exp(-y[:, :width])) * y[:, width:]
    step = y.abs().amax(1, keepdim=True) / 127
    assert not ((got.scale.double() - step[:, 0]).abs() > 2.0 ** -20 * step[:, 0]).any()
    assert not ((got.dequantized().double() - y).abs() > step * (0.5 + 127 * 2.0 ** -19)).any()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("width", [16392, 18944, 29568, 32768])
@pytest.mark.parametrize("rows", [1, 5, 400])
@pytest.mark.parametrize("gated", [False, True])
def test_wide_rows(gated, rows, width, dtype):
    gen = torch.Generator(device="cuda").manual_seed(width + rows)
    most = 2 * width if gated else width
    flat = torch.randn((rows, most + 16), generator=gen, device="cuda").to(dtype)
    for x in (flat[:, :most].contiguous(), flat[:, 8:most + 8]):
        plan = layer.QuantizePlan(width, dtype, rows + 1, gated)
        plan.rows.q.fill_(55)
        got = plan.run(x)
        check(got, x, gated)
        assert (plan.rows.q[rows:] == 55).all() and int(plan.status) == 0
        first = got.q.clone()
        assert torch.equal(plan.run(x).q, first)


def test_rows_that_are_not_numbers():
    x = torch.randn((5, 18944), device="cuda")
    x[1, 18943], x[2, 0], x[3] = math.inf, math.nan, 0.0
    got = layer.sttm_quantize_rows(x)
    assert torch.isnan(got.scale[1:3]).all() and not got.q[1:4].any() and got.scale[3] == 0 and torch.isfinite(got.scale[[0, 4]]).all()


@pytest.mark.parametrize("rows,inner,outer", [(1, 18944, 3584), (40, 29568, 512)])
def test_a_last_product_of_these_widths(rows, inner, outer):
    gen = torch.Generator(device="cuda").manual_seed(rows)
    x = torch.randn((rows, 2 * inner), generator=gen, device="cuda").bfloat16()
    w = torch.randn((outer, inner), generator=gen, device="cuda") * inner ** -0.5
    xq, wq = layer.sttm_quantize_rows(x, gated=True), layer.sttm_quantize_rows(w)
    check(xq, x, True)
    check(wq, w, False)
    got = layer.sttm_quant_matmul(xq, wq, torch.bfloat16).double()
    # sums of whole numbers, exact; two products in 32 bits and one rounding
    want = (xq.q.double() @ wq.q.double().t()) * xq.scale.double().unsqueeze(1) * wq.scale.double()
    assert not ((got - want).abs() > (2.0 ** -8 + 2.0 ** -22) * want.abs()).any()


def test_refusals():
    zeros = lambda width, shift=0: torch.zeros(4 * width + shift, dtype=torch.bfloat16, device="cuda")[shift:].view(4, width)  # noqa: E731
    for width, shift in ((18945, 0), (18948, 0), (18944, 1), (32776, 0)):
        with pytest.raises(binding.SttmError) as e:
            layer.sttm_quantize_rows(zeros(width, shift))
        assert e.value.code == 2, (width, shift)
