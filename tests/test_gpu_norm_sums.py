"""The longest sums of squares of the norms: wide rows that a warp takes, one element at a time, with the terms that lose most.

Bound.  A lane adds its n = ceil(width / 32) squares up in two chains of ceil(n / 2) in 32 bits, joins them and takes five steps with the other
lanes: each addition is off by at most 2^-24 of the sum, all terms being positive.  The norm's factor is off by half of that and by rsqrtf's two ulp
(2^-22), the scale by three roundings more: (ceil(n / 2) + 6) / 2 + 4 + 3 times 2^-24.
Rows: one element of 1 for every lane, then values whose squares are just below half an ulp of 1, which a single chain loses all: n - 1 times 2^-24."""
import pytest
import torch

from paper_2507_07990_b200 import layer

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,width", [(torch.float16, 8127), (torch.bfloat16, 8127), (torch.float32, 4301)])
@pytest.mark.parametrize("shift", [0, 1])
def test_small_terms_behind_large_ones(dtype, width, shift):
    rows = 3600
    row = torch.full((width,), 2.0 ** -12 * (1 - torch.finfo(dtype).eps / 2), dtype=torch.float64)
    row[:32] = 1.0
    assert torch.equal(row.to(dtype).double(), row)
    x = row.to(dtype).cuda().repeat(rows, 1)
    residual = torch.zeros(rows * width + 1, dtype=dtype, device="cuda")[shift:shift + rows * width].view(rows, width)
    got = layer.NormPlan(width, dtype, rows, pre_norm=torch.ones(width, device="cuda"), eps=0.0, quantize=True).run(x, residual)
    want = 1 / float(row.square().mean().sqrt()) / 127
    chain = (-(-width // 32) + 1) // 2
    off = (got.rows.scale.double() / want - 1).abs().max()
    assert float(off) <= ((chain + 6) / 2 + 7) * 2.0 ** -24, float(off) * 2 ** 24
