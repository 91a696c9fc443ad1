"""The ways in which a cache call is split over CTAs, each reached for certain (tests/cache_plans.py) and compared with
the definition in 64 bits.  (The longer rows of test_gpu_cache.test_attend_a_cta_per_row all go to clusters of one CTA, and the sizes of
test_gpu_cache.test_evict_long_rows to clusters of 4 and 8: the other splits are here.)

Tolerances: those of tests/test_gpu_cache.py, and for rows of thousands of slots the order of fp32 additions besides.  A lane adds up at
most n / 4 of a row's n weights one after the other and an output takes n / 16 products, each rounded to 2^-24 of the
running sum or truncated to 2^-23 of it: together below n 2^-25 of the sum (of the largest |v|)."""
import math

import numpy as np
import pytest
import torch

from paper_2507_07990_b200 import cache
from tests import cache_plans as plans
from tests import cache_reference as ref
from tests import test_gpu_cache as base

pytestmark = pytest.mark.gpu


def sms():
    return torch.cuda.get_device_properties(0).multi_processor_count


def split_of(p):
    return plans.attend_split(p["lens"], p["k_pages"].shape[1], p["q"].shape[2], p["max_len"], p["scores"] is not None, p["mask"] is not None, sms())


def gathered(pool, table, b, n):
    """[heads, n, dim] of sequence b's first n slots, in 64 bits on the device."""
    at = torch.arange(n, device=pool.device)
    return pool[table[b].long()[at // pool.shape[2]], :, at % pool.shape[2]].transpose(0, 1).double()


def check_rows(p, out, before, decay=0.75):
    heads, dim, tol = p["k_pages"].shape[1], p["q"].shape[2], ref.ROUNDING[p["dtype"]]
    group, scale = p["q"].shape[1] // heads, p["q"].shape[2] ** -0.5
    below = lambda got, want, allow: bool(((got - want).abs() <= allow).all())
    for b, n in enumerate(p["lens"]):
        on = torch.ones(n, dtype=torch.bool, device="cuda") if p["mask"] is None else p["mask"][b, :n]
        k, v = (gathered(p[x], p["table"], b, n) for x in ("k_pages", "v_pages"))
        q = p["q"][b].double().view(heads, group, dim)
        got, lse = out.out[b].double().view(heads, group, dim), out.lse[b].double().view(heads, group)
        w = torch.zeros((heads, group, n), dtype=torch.float64, device="cuda")
        f = torch.zeros((heads, group), dtype=torch.float64, device="cuda")
        order = n * 2.0 ** -25
        if not bool(on.any()):
            assert not got.any() and bool((lse == -math.inf).all())
        else:
            k, v = k[:, on], v[:, on]
            a = q @ k.transpose(1, 2) * scale
            w[:, :, on] = a.softmax(-1)
            f = 2.0 ** -19 * (q.abs() @ k.abs().transpose(1, 2)).amax(-1) * scale
            want, factor = w[:, :, on] @ v, f + 2.0 ** -17 + 2.0 ** -20
            most = v.abs().amax((1, 2)).view(heads, 1, 1)
            assert below(got, want, tol * want.abs() + (2 * factor.unsqueeze(2) + order) * most + 2.0 ** -24), b
            assert below(lse, a.logsumexp(-1), factor + order + 2.0 ** -21 * a.logsumexp(-1).abs()), b
        if p["scores"] is not None:
            after, was, add = p["scores"][b].double(), before[b].double(), w.sum(1)
            allow = (2 * f.amax(1, keepdim=True) + 2.0 ** -18 + order) * add + 2.0 ** -22 * was[:, :n].abs() + 2.0 ** -40
            assert below(after[:, :n], decay * was[:, :n] + add, allow), b
            assert torch.equal(after[:, n:], was[:, n:])
    assert int(out.status) == 0


def runs_masked(p, seed, none=None):
    """Half of the slots left out, in runs of 37; all of sequence `none`."""
    S, most = len(p["lens"]), p["max_len"]
    runs = torch.rand((S, most // 37 + 1), generator=torch.Generator().manual_seed(seed)) < 0.5
    p["mask"] = runs.cuda().repeat_interleave(37, 1)[:, :most].contiguous()
    if none is not None:
        p["mask"][none] = False


def between(seed, lo, hi, n):
    return [int(x) for x in np.random.RandomState(seed).randint(lo, hi, n)]


# lengths, KV heads, dim; every one of them is cut into shares of more tiles than a CTA's ring has stages
LONG = {
    "ragged64": ([3000] + between(1, 2200, 3000, 17), 8, 64),
    "forty128": ([0, 4200] + between(2, 3500, 4200, 20) + [0] * 9 + between(3, 3500, 4200, 18) + [0], 1, 128),
    "uneven128": ([130000, 0, 3, 20000], 2, 128),
    "uneven256": ([40000, 0, 20000, 20011], 1, 256),
    "two256": ([0, 15000, 9000], 2, 256),
}


@pytest.mark.parametrize("scored", [False, True])
@pytest.mark.parametrize("name,group,dtype", [("ragged64", 2, "bf16"), ("ragged64", 17, "f16"), ("forty128", 7, "bf16"), ("forty128", 20, "bf16"),
                                              ("uneven128", 1, "f16"), ("uneven128", 9, "bf16"), ("uneven256", 5, "bf16"), ("uneven256", 16, "f16"),
                                              ("two256", 24, "bf16"), ("two256", 40, "bf16")])
def test_attend_shares_that_end_with_their_rows(name, group, dtype, scored):
    lens, heads, dim = LONG[name]
    p = base.attend_problem(71, lens, dtype=dtype, q_heads=group * heads, heads=heads, dim=dim, page=32, scored=scored)
    split = split_of(p)
    assert split["cluster"] == 0 and split["with_rows"] and split["each"] > plans.stages(dim)
    before = None if not scored else p["scores"].clone()
    check_rows(p, base.run_attend(p), before)


@pytest.mark.parametrize("scored", [False, True])
@pytest.mark.parametrize("name,group,dtype", [("ragged64", 2, "bf16"), ("ragged64", 17, "f16"), ("ragged64", 40, "bf16"), ("forty128", 7, "bf16"), ("forty128", 20, "bf16"),
                                              ("uneven128", 9, "bf16"), ("uneven256", 5, "bf16"), ("uneven256", 16, "f16"), ("two256", 24, "bf16"),
                                              ("two256", 40, "bf16")])
def test_attend_shares_that_run_on_under_a_mask(name, group, dtype, scored):
    # a share goes on from a row into the next, the ring of stages with it
    lens, heads, dim = LONG[name]
    p = base.attend_problem(72, lens, dtype=dtype, q_heads=group * heads, heads=heads, dim=dim, page=24, order="slots", scored=scored)
    runs_masked(p, 5, none=len(lens) - 2)
    split = split_of(p)
    assert split["cluster"] == 0 and not split["with_rows"] and split["each"] > plans.stages(dim)
    before = None if not scored else p["scores"].clone()
    check_rows(p, base.run_attend(p), before)


@pytest.mark.parametrize("dim,group", [(64, 7), (128, 7), (128, 33)])
def test_attend_long_shares_of_rows_that_do_not_fit_them(dim, group):
    # without a mask, where shares cannot end with their rows for a sixth more
    lens = [0, 3000, 0] + between(4, 1500, 3000, 33)
    p = base.attend_problem(73, lens, q_heads=4 * group, heads=4, dim=dim, page=16)
    split = split_of(p)
    assert split["cluster"] == 0 and not split["with_rows"] and split["each"] > plans.stages(dim)
    check_rows(p, base.run_attend(p), None)


@pytest.mark.parametrize("scored", [False, True])
@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("dim,group,page", [(256, 3, 8), (256, 20, 64), (128, 40, 32), (64, 9, 128)])
def test_attend_a_long_row_to_one_cta(dim, group, page, masked, scored):
    # rows enough to fill the GPU, each of up to 16 tiles through one CTA's ring
    most = 16 * 8192 // dim
    lens = [most, 0, 1, most - 1] + between(6, most // 2, most, 16)
    heads = 16 if dim < 256 else 8
    p = base.attend_problem(74, lens, q_heads=group * heads, heads=heads, dim=dim, page=page, scored=scored)
    if masked:
        runs_masked(p, 7, none=4)
    assert split_of(p) == {"cluster": 1, "each": 16}
    before = None if not scored else p["scores"].clone()
    check_rows(p, base.run_attend(p), before)


@pytest.mark.parametrize("dim,size", [(64, 16), (128, 16), (256, 8)])
@pytest.mark.parametrize("group", [7, 20, 64])
def test_attend_large_clusters_at_their_longest(dim, size, group):
    most = size * 6 * 8192 // dim
    p = base.attend_problem(75, [most, 0, most - 3, 40], q_heads=group, dim=dim, page=48)
    assert split_of(p) == {"cluster": size, "each": 6}
    check_rows(p, base.run_attend(p), None)
    runs_masked(p, 8, none=2)
    check_rows(p, base.run_attend(p), None)


def attend_launches(rows, n, dim):
    plan = cache.AttendPlan(cache.empty_cache(1, n, rows, dim, 32), rows, max_len=n)
    q, lengths = torch.zeros((1, rows, dim), dtype=torch.bfloat16, device="cuda"), torch.tensor([n], dtype=torch.int32, device="cuda")
    return plans.launches(lambda: plan.run(q, lengths))


@pytest.mark.parametrize("rows,n", [(4, 1024), (8, 1024), (16, 1024), (16, 512), (18, 700), (36, 300)])
def test_attend_clusters_have_to_fit_at_once(rows, n):
    """A cluster lies in one group of SMs, whose number it need not divide.  Where a CTA of 256 channels takes an SM, rows whose
    clusters are not all resident would run in two goes."""
    made = attend_launches(rows, n, 256)
    size = made[0].grid[0] // rows if len(made) == 1 else 0
    assert size > 1 or rows > 8
    assert size <= 1 or (made[0].grid[0] == rows * size and plans.resident_clusters(made[0], size) >= rows)
    p = base.attend_problem(77, [n, n - 3], q_heads=3 * rows // 2, heads=rows // 2, dim=256, page=32)
    check_rows(p, base.run_attend(p), None)


@pytest.mark.parametrize("dim,rows,n,size", [(64, 1, 4096, 16), (128, 4, 6144, 16), (128, 9, 3000, 16), (128, 18, 2000, 8), (64, 37, 2000, 4),
                                             (256, 4, 1536, 8), (256, 80, 512, 1), (128, 4, 7000, 0), (64, 160, 4000, 0)])
def test_attend_launches_the_split_that_is_worked_out(dim, rows, n, size):
    made = attend_launches(rows, n, dim)
    assert plans.attend_split([n], rows, dim, n, False, False, sms())["cluster"] == size
    if size:
        assert len(made) == 1 and made[0].grid[0] == rows * size
    else:
        assert len(made) == 2 and made[0].grid[0] == min(sms() * (1 if dim == 256 else 2), rows * -(-n // (8192 // dim)))


def test_attend_gives_the_same_bits_every_time():
    for name, group, masked in (("forty128", 7, False), ("forty128", 7, True), ("uneven256", 20, False)):
        lens, heads, dim = LONG[name]
        p = base.attend_problem(76, lens, q_heads=group * heads, heads=heads, dim=dim, page=32, scored=True)
        if masked:
            runs_masked(p, 9)
        seen = []
        for _ in range(3):
            again = {**p, "scores": p["scores"].clone()}
            out = base.run_attend(again)
            seen.append((out.out.clone(), out.lse.clone(), again["scores"]))
        for other in seen[1:]:
            assert all(torch.equal(a, b) for a, b in zip(seen[0], other))


# ---------------------------------------------------------------- evict

def kept_slots(scores, keep, first, last):
    """The definition of tests/cache_reference.py's evict, sorted by numpy: [slots that stay] of one row."""
    n = len(scores)
    slot = np.arange(n)
    nan = np.isnan(scores)
    rank = np.where((slot < first) | (slot >= n - last), 0, np.where(nan, 2, 1))
    order = np.lexsort((slot, np.where(rank == 1, -scores.astype(np.float64), 0.0), rank))
    return np.sort(order[:max(0, min(keep, n))])


def check_selection(p, first, last):
    src, dst, keep = p["src"], p["dst"], p["keep"]
    dev = lambda x: torch.tensor(x, dtype=torch.int32).cuda()
    out = cache.sttm_cache_evict(src, dst, dev(p["lens"]), dev(keep), p["scores"], p["kept_width"], first, last, p["max_len"])
    scores, kept, new = p["scores"].cpu().numpy(), out.kept.cpu().numpy(), out.new_scores.cpu().numpy()
    assert int(out.status) == 0
    for b, n in enumerate(p["lens"]):
        for h in range(src.heads):
            at = kept_slots(scores[b, h, :n], keep[b], first, last)
            assert int(out.new_lengths[b]) == len(at)
            np.testing.assert_array_equal(kept[b, h], np.concatenate([at, np.full(p["kept_width"] - len(at), -1)]))
            np.testing.assert_array_equal(new[b, h], np.concatenate([scores[b, h, at], np.zeros(p["kept_width"] - len(at), np.float32)]))
        at = torch.from_numpy(kept[b, :, :int(out.new_lengths[b])]).long().cuda()
        to = torch.arange(at.shape[1], device="cuda")
        for was, now in ((src.k, dst.k), (src.v, dst.v)):
            for h in range(src.heads):
                a = was[src.table[b].long()[at[h] // src.page], h, at[h] % src.page]
                c = now[dst.table[b].long()[to // dst.page], h, to % dst.page]
                assert torch.equal(a, c)


def test_the_sorted_definition_is_the_plain_one():
    for kind in ("weights", "ties", "odd"):
        p = base.evict_problem(80, (77, 300), (31, 200), kind=kind)
        for row, keep in ((p["scores"][0, 0, :77], 31), (p["scores"][1, 1], 200), (p["scores"][1, 0], 300)):
            row = row.cpu().numpy()
            for ends in ((0, 0), (4, 9)):
                assert kept_slots(row, keep, *ends).tolist() == ref.evict(row, keep, *ends)


@pytest.mark.parametrize("kind", ["weights", "ties", "odd"])
@pytest.mark.parametrize("seqs,heads,n,split", [
    (25, 3, 3000, (1, 3)), (25, 3, 9000, (1, 9)), (16, 8, 16421, (1, 17)), (25, 3, 25000, (1, 25)), (25, 3, 33000, (1, 33)),
    (2, 1, 6144, (2, 3)), (2, 1, 3073, (2, 3)), (20, 2, 9000, (2, 9)), (20, 2, 25000, (2, 17)), (14, 2, 50001, (4, 17)), (20, 2, 70000, (4, 25)),
    (1, 2, 25001, (8, 9)), (2, 1, 130000, (8, 17)), (1, 2, 199999, (8, 25)), (1, 2, 270000, (8, 33)),
], ids=str)
def test_evict_every_split(seqs, heads, n, split, kind):
    lens = [n, n - 1, n // 3, 0, 1][:seqs] + between(seqs, n // 2, n, max(0, seqs - 5))
    keep = [max(1, int(m * x)) for m, x in zip(lens, np.random.RandomState(n).rand(seqs))]
    p = base.evict_problem(81, lens, keep, heads=heads, page=64, dst_page=32, kind=kind)
    assert plans.select_split(seqs * heads, n, sms()) == split
    check_selection(p, 4, 64)


def select_launch(rows, n):
    src, dst = cache.empty_cache(1, n, rows, 64, 64), cache.empty_cache(1, 40, rows, 64, 64)
    plan = cache.EvictPlan(src, dst, 40, max_len=n)
    ints = lambda x: torch.tensor([x], dtype=torch.int32, device="cuda")
    lengths, keep, scores = ints(n), ints(40), torch.rand((1, rows, n), device="cuda")
    select, move = plans.launches(lambda: plan.run(lengths, keep, scores))
    return select


@pytest.mark.parametrize("rows,n", [(1, 6144), (15, 30000), (32, 30000), (40, 25000), (75, 9000), (2, 270000)])
def test_evict_launches_the_split_that_is_worked_out(rows, n):
    assert select_launch(rows, n).grid[0] == rows * plans.select_split(rows, n, sms())[0]


@pytest.mark.parametrize("rows,n", [(16, 25000), (18, 55788), (17, 130000), (34, 25000), (37, 55788), (16, 16421)])
def test_evict_clusters_have_to_fit_at_once(rows, n):
    """A cluster lies in one group of SMs, whose number it need not divide: rows whose clusters are not all resident would be
    selected from in two goes."""
    select = select_launch(rows, n)
    size = select.grid[0] // rows
    assert size >= 2 and select.grid[0] == rows * size and plans.resident_clusters(select, size) >= rows


@pytest.mark.parametrize("kind", ["weights", "ties", "odd"])
@pytest.mark.parametrize("n,keep", [(270337, 100000), (450001, 1000), (450001, 225003), (450001, 450000)])
def test_evict_rows_beyond_registers(n, keep, kind):
    # equal scores all through the row: their order over warps, goes and CTAs decides
    p = base.evict_problem(82, (n, n // 2), (keep, keep // 2), heads=1, page=64, kind=kind)
    assert plans.select_split(2, n, sms()) == (8, 0)
    check_selection(p, 1, 30)
    check_selection(p, 0, 0)
