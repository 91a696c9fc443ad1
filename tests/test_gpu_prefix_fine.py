"""sttm_prefix_attend with weights that are not rounded to the cache's type.

Tolerance: that of the rounded form (see test_gpu_prefix.py) with a weight off by half a step squared instead of half a step: the remainder of the rounding,
at most half a step of the weight, is itself rounded by half a step of it."""
import pytest
import torch

from paper_2507_07990_b200 import cache, prefix
from tests import cache_reference as ref
from tests.test_gpu_prefix import CASES, expect, plan_of, problem, run

pytestmark = pytest.mark.gpu


def check(p, r):
    out, lse, bound, lse_bound, used = expect(p)
    # sum of w |v|: the output for the values' magnitudes
    sizes = dict(p, **{name: None if p[name] is None else [p[name][0], p[name][1].abs(), p[name][2]] for name in ("pre", "mine")})
    half = ref.ROUNDING[p["dtype"]]
    bound = bound - (half - half * half) * expect(sizes)[0]
    assert int(r.status) == 0 and torch.isfinite(r.out[used]).all()
    err = (r.out.double() - out).abs()
    assert not (err > bound)[used].any(), float((err / bound.clamp(min=1e-30))[used].max())
    empty = lse == -float("inf")
    assert torch.equal((r.lse == -float("inf"))[used], empty[used]) and not (((r.lse.double() - lse).abs() > lse_bound) & ~empty)[used].any()


@pytest.mark.parametrize("kw", CASES, ids=range(len(CASES)))
def test_against_the_definition(kw):
    p = problem(61 + len(str(kw)), **kw)
    plan = plan_of(p, fine=True)
    plan.out.fill_(7.0)
    check(p, run(p, plan))
    first = plan.out.clone()
    assert torch.equal(run(p, plan).out, first)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("new,length", [(1, 20000), (40, 3000), (150, 700)])
def test_long_caches_and_logits_that_rise(new, length, dim, dtype):
    for ramp in (0.0, 6.0):
        p = problem(62, dtype=dtype, dim=dim, q_heads=8, heads=2, page=64, lens=(length,), groups=(2,), new=(new, 1), held=(70, 0), scale=2.0 if ramp else 1.0, ramp=ramp)
        check(p, run(p, plan_of(p, fine=True)))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("new", [1, 64])
def test_as_close_as_one_token_at_a_time(dtype, new):
    """Errors against 64 bits are those of the output's rounding, a third of a step squared on average; rounded weights add about as much."""
    p = problem(63, dtype=dtype, q_heads=8, heads=2, page=64, lens=(5000,), groups=(1,), new=(new,), held=(0,), own=False, spare=0)
    out = expect(p)[0]
    ideal = float((out.to(p["q"].dtype).double() - out).norm())
    rounded, fine = (float((run(p, plan_of(p, fine=f)).out.double() - out).norm()) for f in (False, True))
    # (1.1: fp32 arithmetic beside the rounding)
    assert fine < 1.1 * ideal < rounded
    one = prefix.sttm_prefix_attend(cache.PagedCache(*p["pre"]), p["q"], p["row_offsets"], p["prefix_lengths"], seq_offsets=p["seq_offsets"], fine=True)
    assert torch.equal(one.out, run(p, plan_of(p, fine=True)).out)
