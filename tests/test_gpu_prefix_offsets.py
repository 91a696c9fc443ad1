"""Offsets that sttm_prefix_attend finds wrong on the device."""
import pytest
import torch

from paper_2507_07990_b200 import cache, prefix
from tests.test_gpu_prefix import plan_of, problem, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("own", [False, True])
@pytest.mark.parametrize("seqs", [4, 900])
def test_offsets_that_decrease_inside_a_prefix(seqs, own):
    p = problem(71, q_heads=4, heads=2, dim=64, lens=(100,), groups=(seqs,), new=[2] * seqs, held=[0] * seqs, own=own, page=16)
    p["row_offsets"][seqs // 2] -= 3                            # below the one before; the prefix's first and last are in order
    plan = plan_of(p)
    plan.out.fill_(7.0)
    plan.lse.fill_(7.0)
    r = run(p, plan)
    assert int(r.status) == 2 and (r.out == 7.0).all() and (r.lse == 7.0).all()


@pytest.mark.parametrize("held", [0, 150])
def test_offsets_beyond_the_rows(held):
    # a sequence's new tokens are those that are there, which is also what sttm_cache_append counts
    p = problem(72, lens=(60,), groups=(2,), new=(2, 3), held=(4, held), spare=0)
    q, k, v = p["q"].contiguous(), torch.randn((5, 2, 128), device="cuda").bfloat16(), torch.randn((5, 2, 128), device="cuda").bfloat16()
    before = torch.tensor([4, held], dtype=torch.int32, device="cuda")
    own = cache.PagedCache(*p["mine"])
    beyond = torch.tensor([0, 2, 9], device="cuda")
    entered = cache.AppendPlan(own, 4).run(q, k, v, beyond, before, None)
    assert entered.new_lengths.tolist() == [6, held + 3] and int(entered.status) == 16
    outs = []
    for offsets, status in ((beyond, 16), (p["row_offsets"], 0)):
        plan = prefix.PrefixPlan(cache.PagedCache(*p["pre"]), 4, own, 5)
        r = plan.run(q, offsets, p["prefix_lengths"], entered.new_lengths)
        assert int(r.status) == status
        outs.append((r.out.clone(), r.lse.clone()))
    for a, b in zip(*outs):
        assert torch.equal(a, b)
