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
