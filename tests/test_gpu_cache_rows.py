"""Which rows an append takes, what it says about the others, and how long its outputs stand."""
import pytest
import torch

from paper_2507_07990_b200 import binding, cache
from tests import test_gpu_cache as base

pytestmark = pytest.mark.gpu
CAPACITY = 1 << 4


def offsets(*values):
    return torch.tensor(values, dtype=torch.int64, device="cuda")


@pytest.mark.parametrize("ends,real", [((3, 3, 12), (3, 0, 7)), ((3, 11, 15), (3, 7, 0)), ((10, 10, 11), (10, 0, 0)), ((30, 40, 50), (10, 0, 0))],
                         ids=str)
def test_append_counts_only_rows_that_are_there(ends, real):
    """Offsets may end beyond the rows (a merge whose output buffer was too small counts what it had no room for): the rows
    that are there are cached, the lengths count no others, and the status says so."""
    p, want = (base.append_problem(61, rows=(4, 4, 2), held=(0, 2, 20), spare=0, page=32) for _ in range(2))
    want["offsets"] = offsets(0, real[0], real[0] + real[1], 10)
    p["offsets"] = offsets(0, *ends)
    expected, got = base.run_append(want), base.run_append(p)
    assert got.new_lengths.tolist() == expected.new_lengths.tolist() == [h + r for h, r in zip((0, 2, 20), real)]
    assert int(got.status) == CAPACITY and int(expected.status) == 0
    assert torch.equal(got.q, expected.q)
    for name in ("k_pages", "v_pages"):
        assert torch.equal(p[name].view(torch.int16), want[name].view(torch.int16))


def test_append_of_no_rows_with_offsets_that_name_some():
    p = base.append_problem(62, rows=(2, 2), held=(5, 7), spare=0)
    before = p["k_pages"].clone()
    for name in ("q", "k", "v"):
        p[name] = p[name][:0]
    p["pos"] = p["pos"][:, :0]
    p["offsets"] = offsets(0, 3, 3)
    out = base.run_append(p)
    assert out.new_lengths.tolist() == [5, 7] and int(out.status) == CAPACITY
    assert torch.equal(p["k_pages"].view(torch.int16), before.view(torch.int16))


def test_append_of_a_merge_whose_buffer_was_too_small():
    from paper_2507_07990_b200 import inputs
    from tests import helpers
    video = helpers.to_torch(inputs.make_video(helpers.small_spec(61, 6, 13, 13, 64, p_static=0.8)))
    whole = binding.sttm_merge_ex(video, 0.97, 0.9)
    n = int(whole.out_count[0])
    m = binding.sttm_merge_ex(video, 0.97, 0.9, capacity=n - 5)
    assert int(m.out_offsets[1]) == n and m.out_feats.shape[0] == n - 5
    pool = cache.empty_cache(1, n, 1, 64)
    x = m.out_feats.view(-1, 1, 64)
    out = cache.sttm_cache_append(pool, None, x, x, m.out_offsets)
    assert out.new_lengths.tolist() == [n - 5] and int(out.status) == CAPACITY


@pytest.mark.parametrize("first", [1, 2, 9])
def test_append_leaves_rows_before_the_first_offset_alone(first):
    """Offsets of a window into a longer buffer: neither the slots in use nor the queries of the rows before it change."""
    p = base.append_problem(63, rows=(4, 0, 6), held=(12, 3, 30), spare=0)
    ends = [first, max(first, 4), max(first, 4), 10]
    p["offsets"] = offsets(*ends)
    before_k, before_v = p["k_pages"].clone(), p["v_pages"].clone()
    q_out = torch.full_like(p["q"].contiguous(), 7.0)
    out = base.run_append(p, q_out)
    assert torch.equal(q_out[:first], torch.full_like(q_out[:first], 7.0)) and not (q_out[first:] == 7.0).all()
    rows = [b - a for a, b in zip(ends, ends[1:])]
    assert out.new_lengths.tolist() == [h + r for h, r in zip((12, 3, 30), rows)] and int(out.status) == 0
    touched = torch.zeros(before_k.shape[0], 16, dtype=torch.bool)
    for b, (h, r) in enumerate(zip((12, 3, 30), rows)):
        for i in range(r):
            pg, place = int(p["table"][b, (h + i) // 16]), (h + i) % 16
            touched[pg, place] = True
            assert torch.equal(p["v_pages"][pg, :, place], p["v"][ends[b] + i])
    touched = touched.cuda()
    for now, was in ((p["k_pages"], before_k), (p["v_pages"], before_v)):
        same = (now.view(torch.int16) == was.view(torch.int16)).all(3).all(1)
        assert same[~touched].all()


def test_append_lengths_outlive_the_next_call():
    """A call's new lengths are written again by the call after the next, whatever lengths either is given."""
    p = base.append_problem(64, rows=(1, 1), held=(3, 9), spare=0, page=32)
    plan = cache.AppendPlan(cache.PagedCache(p["k_pages"], p["v_pages"], p["table"]), 4, cache.Rotary(p["freq"]))
    step = lambda lengths: plan.run(p["q"], p["k"], p["v"], p["offsets"], lengths, p["pos"])
    older, latest = step(p["lengths"]).new_lengths, step(None).new_lengths
    # a caller's lengths, none, the plan's latest, the plan's latest but one: every order of two of them
    for kind in "ccnnclpnplcplnlppccpnncl":
        lengths = {"c": p["lengths"], "n": None, "l": latest, "p": older}[kind]
        given, was = [0, 0] if lengths is None else lengths.tolist(), latest.tolist()
        new = step(lengths).new_lengths
        assert new.tolist() == [n + 1 for n in given], kind
        assert latest.tolist() == was, kind
        assert lengths is None or lengths.tolist() == given, kind
        older, latest = latest, new
    assert int(plan.status) == 0


def test_append_outputs_of_two_calls_are_two_objects():
    p = base.append_problem(65, rows=(1,), held=(3,), spare=0)
    plan = cache.AppendPlan(cache.PagedCache(p["k_pages"], p["v_pages"], p["table"]), 4, cache.Rotary(p["freq"]))
    first = plan.run(p["q"], p["k"], p["v"], p["offsets"], p["lengths"], p["pos"])
    q, new = first.q, first.new_lengths
    second = plan.run(p["q"], p["k"], p["v"], p["offsets"], first.new_lengths, p["pos"])
    assert first.q is q and first.new_lengths is new and second.new_lengths is not new
    assert first.new_lengths.tolist() == [4] and second.new_lengths.tolist() == [5]
