"""8-bit products whose last tile holds any number of tokens and channels: lanes of a warp without a token of their own, between loads that are
the whole warp's.  Bits are those of the same tokens among others (sums are exact, and one rounding follows)."""
import pytest
import torch

from paper_2507_07990_b200 import layer

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("outer", [3584, 3600, 1111])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_any_number_of_tokens(outer, dtype):
    gen = torch.Generator().manual_seed(outer)
    most = 1600
    q = torch.randint(-127, 128, (most, 512), generator=gen).to(torch.int8).cuda()
    scale = (0.5 + torch.rand(most, generator=gen)).cuda()
    w = layer.QuantRows(torch.randint(-127, 128, (outer, 512), generator=gen).to(torch.int8).cuda(), torch.rand(outer, generator=gen).cuda())
    bias = torch.randn(outer, generator=gen).cuda()
    plan = layer.MatmulPlan(w, dtype, most, bias)
    whole = plan.run(layer.QuantRows(q, scale)).clone()
    # (the definition, in whole numbers below 2^24 * 2^9: exact in 64 bits)
    want = (q.double() @ w.q.double().t()) * scale.double().unsqueeze(1) * w.scale.double() + bias.double()
    half_step = torch.finfo(dtype).eps / 2
    size = (want - bias.double()).abs() + bias.double().abs()
    assert not ((whole.double() - want).abs() > half_step * want.abs() + 2.0 ** -22 * size).any()
    for rows in list(range(1, 40)) + list(range(1281, 1281 + 40)) + list(range(1400, 1600, 7)):
        plan.out.fill_(3.0)
        got = plan.run(layer.QuantRows(q[:rows], scale[:rows]))
        assert torch.equal(got, whole[:rows]) and (plan.out[rows:] == 3.0).all(), rows
    assert int(plan.status) == 0
