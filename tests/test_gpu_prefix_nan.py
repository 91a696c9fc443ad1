"""Queries and keys that are not numbers in sttm_prefix_attend: the rows that meet them, and no others, give NaN in `out` and in `lse`, however
the work is cut into pieces.  Nothing is compared but NaN with NaN and bits with bits."""
import math

import pytest
import torch

from tests.test_gpu_prefix import problem, run, slots

pytestmark = pytest.mark.gpu

# one tile and fewer, pieces of one tile each, pieces of several tiles
LENGTHS = [1, 200, 2600, 20000, 54736]


def results(p):
    r = run(p)
    assert int(r.status) == 0
    return r.out.clone(), r.lse.clone()


def compare(got, want, lost):
    """NaN where `lost` [rows, heads] says so, and the same bits as without it elsewhere."""
    for g, w in zip(got, want):
        each = g.isnan().all(-1) if g.dim() == 3 else g.isnan()
        assert torch.equal(each, lost)
        assert torch.equal(g[~lost], w[~lost])


@pytest.mark.parametrize("dtype,dim", [("bf16", 128), ("f16", 64), ("bf16", 256)])
@pytest.mark.parametrize("new,held", [(1, None), (1, 0), (1, 700), (40, None), (40, 700)])
@pytest.mark.parametrize("length", LENGTHS)
def test_queries_that_are_not_numbers(length, new, held, dtype, dim):
    p = problem(31, dtype=dtype, dim=dim, q_heads=8, heads=4, page=64, lens=(length,), groups=(2,), new=(new, 1), held=(held or 0, 3), own=held is not None, spare=0)
    want = results(p)
    lost = torch.zeros(want[1].shape, dtype=torch.bool, device="cuda")
    for row, head in ((0, 0), (0, 1), (new // 2, 5), (new, 7)):
        p["q"][row, head, 3] = math.nan
        lost[row, head] = True
    compare(results(p), want, lost)


@pytest.mark.parametrize("dtype,dim", [("bf16", 128), ("f16", 64), ("bf16", 256)])
@pytest.mark.parametrize("new,held", [(1, None), (40, 300)])
@pytest.mark.parametrize("length", LENGTHS)
def test_keys_that_are_not_numbers(length, new, held, dtype, dim):
    p = problem(32, dtype=dtype, dim=dim, q_heads=8, heads=4, page=64, lens=(length,), groups=(2,), new=(new, 1), held=(held or 0, 3), own=held is not None, spare=0)
    want = results(p)
    # a key of the prefix, of KV head 2: all rows of its two query heads
    k, _, table = p["pre"]
    for slot in {0, length // 2, length - 1}:
        at = (int(table[0, slot // 64]), 2, slot % 64, 5)
        was, k[at] = k[at].clone(), math.nan
        lost = torch.zeros(want[1].shape, dtype=torch.bool, device="cuda")
        lost[:, 4:6] = True
        compare(results(p), want, lost)
        k[at] = was
    if held is None:
        return
    # an own key: the rows of its sequence that see it (token i sees slots up to held + i)
    k, _, table = p["mine"]
    for slot in (7, held, held + new // 2):
        at = (int(table[0, slot // 64]), 1, slot % 64, 0)
        was, k[at] = k[at].clone(), math.nan
        lost = torch.zeros(want[1].shape, dtype=torch.bool, device="cuda")
        lost[max(0, slot - held):new, 2:4] = True
        compare(results(p), want, lost)
        k[at] = was


@pytest.mark.parametrize("dtype,dim", [("bf16", 128), ("f16", 64)])
def test_a_whole_cache_that_is_not_a_number(dtype, dim):
    for length in LENGTHS:
        p = problem(33, dtype=dtype, dim=dim, q_heads=8, heads=4, page=64, lens=(length,), groups=(2,), new=(1, 1), held=(0, 0), own=False, spare=0)
        p["pre"][0].fill_(math.nan)
        out, lse = results(p)
        assert out.isnan().all() and lse.isnan().all()
        assert slots(p["pre"], 0, length)[0].isnan().all()


@pytest.mark.parametrize("dtype,dim", [("bf16", 128), ("f16", 64), ("bf16", 256)])
@pytest.mark.parametrize("new", [1, 40])
@pytest.mark.parametrize("length", [130, 20000])
def test_logits_of_minus_infinity(length, new, dtype, dim):
    # keys at -inf in a channel where queries are 1: slots that weigh nothing, some or all of them
    p = problem(34, dtype=dtype, dim=dim, q_heads=8, heads=4, page=64, lens=(length,), groups=(2,), new=(new, 1), held=(0, 0), own=False, spare=0)
    p["q"][:, :, 0] = 1.0
    p["pre"][0][..., 0] = 0.0
    half = dict(p, lens=(length // 2,), prefix_lengths=p["prefix_lengths"] // 2)
    k, _, table = p["pre"]
    behind = torch.arange(length // 2, length, device="cuda")
    k[table[0].long()[behind // 64], :, behind % 64, 0] = -math.inf
    out, lse = results(p)
    want, want_lse = results(half)
    # the same weights, cut into other pieces: sums in 32 bits in another order, weights rounded against another reference, half a step each
    step = 2.0 ** -7 if dtype == "bf16" else 2.0 ** -10
    assert float((out.double() - want.double()).norm() / want.double().norm()) < step and float((lse - want_lse).abs().max()) < 2.0 ** -15 * 20
    k[..., 0] = -math.inf
    out, lse = results(p)
    assert not out.any() and (lse == -math.inf).all()
