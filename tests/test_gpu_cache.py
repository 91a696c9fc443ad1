"""The cache operators (sttm_cache_append, sttm_cache_attend, sttm_cache_evict) on the GPU against the
definition in 64 bits.

Tolerances.  append: one rounding to the type (half a unit in the last place) and fp32 arithmetic on
the pair: a norm factor (sum of <= 256 squares, a square root, a division: below 2^-20), a product by the weight, cos
and sin to 2^-22, two products and a sum: below 2^-19 of the pair's length.  attend: a logit is an fp32 sum of at most
256 products, off by at most 2^-19 of the sum of the products' magnitudes (tensor-core sums truncate: an ulp for each of 16
steps); a weight is off by that factor plus 2^-17 (its two 16-bit parts) plus 2^-20 (exponential, sum), and an output by that share of
the largest |v|, plus one rounding.  evict: exact."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from paper_2507_07990_b200 import binding, cache
from tests import cache_reference as ref

pytestmark = pytest.mark.gpu


# ---------------------------------------------------------------- append

def append_problem(seed, dtype="bf16", q_heads=4, heads=2, dim=64, page=16, order="heads", rows=(3, 0, 5), held=(0, 2, 30), spare=2,
                   norm=True, axes=1, mean=False, interleaved=False, rot=None, fused=True, base=0):
    gen = torch.Generator().manual_seed(seed)
    rot = dim if rot is None else rot
    width = max(-(-(r + h) // page) for r, h in zip(rows, held)) or 1
    table = ref.make_table(gen, len(rows), width)
    k_pages, v_pages = ref.make_pool(gen, len(rows) * width + 2, heads, page, dim, dtype, order)
    n = sum(rows) + spare
    dt = ref.DTYPES[dtype]
    if fused:
        x = torch.randn((n, q_heads + 2 * heads, dim), generator=gen).to(dt).cuda()
        q, k, v = x[:, :q_heads], x[:, q_heads:q_heads + heads], x[:, q_heads + heads:]
    else:
        # heads outermost: a row's heads are far apart
        q, k, v = (torch.randn((h, n, dim), generator=gen).to(dt).cuda().transpose(0, 1) for h in (q_heads, heads, heads))
    pos = base + torch.randint(0, 5000, (axes, n), generator=gen)
    pos = (pos.float() + torch.rand(pos.shape, generator=gen)) if mean else pos.to(torch.int32)
    half = rot // 2
    freq = (1e6 ** (-torch.arange(half, dtype=torch.float64) / max(half, 1))).float()
    sections = (half // 4, half - half // 4 - half // 2, half // 2) if axes == 3 else None
    q_norm, k_norm = ((1 + 0.3 * torch.randn(dim, generator=gen)).cuda() if norm else None for _ in range(2))
    return dict(dtype=dtype, q=q, k=k, v=v, pos=pos.cuda(), freq=freq.cuda(), sections=sections, interleaved=interleaved,
                q_norm=q_norm, k_norm=k_norm, k_pages=k_pages, v_pages=v_pages, table=table, rows=rows, held=held, page=page,
                offsets=torch.tensor([0] + list(np.cumsum(rows)), dtype=torch.int64).cuda(),
                lengths=torch.tensor(held, dtype=torch.int32).cuda(), rot=rot)


def run_append(p, q_out=None):
    pool = cache.PagedCache(p["k_pages"], p["v_pages"], p["table"])
    rotary = cache.Rotary(p["freq"], p["interleaved"], p["sections"]) if p["rot"] else None
    plan = cache.AppendPlan(pool, p["q"].shape[1], rotary, p["q_norm"], p["k_norm"], eps=1e-5)
    return plan.run(p["q"], p["k"], p["v"], p["offsets"], p["lengths"], p["pos"] if p["rot"] else None, q_out)


def expect_head(p, x, weight, row):
    half = p["rot"] // 2
    s = p["sections"] or (half, 0, 0)
    axis = [0] * s[0] + [1] * s[1] + [2] * s[2]
    pos = ref.f64(p["pos"].reshape(-1, p["q"].shape[0]))[:, row]
    return ref.turn(ref.f64(x), None if weight is None else ref.f64(weight), 1e-5, pos, ref.f64(p["freq"]), axis, p["interleaved"])


def check_append(p, out, before_k, before_v):
    tol = ref.ROUNDING[p["dtype"]]
    page, want_k, want_v = p["page"], before_k.copy(), before_v.copy()
    got_q, touched = ref.f64(out.q), np.zeros(before_k.shape[:1] + before_k.shape[2:3], dtype=bool)
    close = lambda got, want: np.testing.assert_array_less(
        np.abs(got - want), tol * np.abs(want) + 2.0 ** -19 * np.abs(want).max() + 2.0 ** -24)
    row = 0
    for b, (r, h) in enumerate(zip(p["rows"], p["held"])):
        for i in range(r):
            for hd in range(p["q"].shape[1]):
                close(got_q[row, hd], expect_head(p, p["q"][row, hd], p["q_norm"], row))
            slot = h + i
            pg, place = int(p["table"][b, slot // page]), slot % page
            touched[pg, place] = True
            for hd in range(p["k"].shape[1]):
                close(ref.f64(p["k_pages"][pg, hd, place]), expect_head(p, p["k"][row, hd], p["k_norm"], row))
                np.testing.assert_array_equal(ref.f64(p["v_pages"][pg, hd, place]), ref.f64(p["v"][row, hd]))
            row += 1
        assert int(out.new_lengths[b]) == h + r
    # nothing else moved
    for got, was in ((p["k_pages"], before_k), (p["v_pages"], before_v)):
        g = ref.f64(got).transpose(0, 2, 1, 3)[~touched]
        np.testing.assert_array_equal(g, was.transpose(0, 2, 1, 3)[~touched])
    assert int(out.status) == 0


@pytest.mark.parametrize("case", [
    dict(), dict(dtype="f16", dim=128, page=8, order="slots"), dict(dim=256, q_heads=3, heads=1, page=24, fused=False),
    dict(norm=False, interleaved=True), dict(rot=32), dict(rot=32, interleaved=True, dim=128, norm=False, dtype="f16"),
    dict(axes=3, dim=128), dict(axes=3, mean=True, fused=False, order="slots"), dict(rot=0), dict(mean=True, base=170000, dim=128),
    dict(base=2000000, dtype="f16"), dict(rows=(1,) * 7, held=(0, 1, 15, 16, 17, 47, 100), spare=0, q_heads=28, heads=4, dim=128),
    dict(rows=(1,), held=(0,), spare=0, q_heads=14, heads=2), dict(rows=(0, 0, 41), held=(3, 0, 7), spare=5, q_heads=7, heads=7),
    dict(rows=(70,), held=(0,), axes=3, interleaved=True, dim=256, q_heads=2, heads=1),
    dict(rows=tuple(int(x) for x in np.random.RandomState(0).randint(0, 3, 75)), held=(5,) * 75, q_heads=1, heads=1, spare=0),
], ids=str)
def test_append(case):
    p = append_problem(11, **case)
    before = ref.f64(p["k_pages"]), ref.f64(p["v_pages"])
    check_append(p, run_append(p), *before)


def test_append_many_rows():
    # enough rows that one warp takes a whole row, several sequences per block
    p = append_problem(5, rows=(2500, 1, 2900), held=(0, 7, 3), q_heads=1, heads=1, dim=64, page=64)
    before = ref.f64(p["k_pages"]), ref.f64(p["v_pages"])
    check_append(p, run_append(p), *before)


def test_append_in_place_queries_and_rows_beyond_the_count():
    p = append_problem(3, fused=False, spare=4)
    p["q"] = p["q"].contiguous()
    kept = p["q"].clone()
    out = run_append(p, q_out=p["q"])
    apart = append_problem(3, fused=False, spare=4)
    want = run_append(apart)
    n = sum(p["rows"])
    assert torch.equal(p["q"][:n], want.q[:n])
    assert torch.equal(p["q"][n:], kept[n:])            # rows that are no tokens stay as they were
    assert int(out.status) == 0


def test_append_without_queries():
    p, whole = append_problem(4), append_problem(4)
    run_append(whole)
    pool = cache.PagedCache(p["k_pages"], p["v_pages"], p["table"])
    out = cache.sttm_cache_append(pool, None, p["k"], p["v"], p["offsets"], p["lengths"], p["pos"], cache.Rotary(p["freq"]),
                                  k_norm=p["k_norm"], eps=1e-5)
    assert out.q is None and torch.equal(p["k_pages"], whole["k_pages"]) and torch.equal(p["v_pages"], whole["v_pages"])


def test_append_drops_what_has_no_place():
    p = append_problem(9, rows=(4, 3), held=(14, 0), page=16, spare=0)
    p["table"] = p["table"][:, :1].clone()              # 16 slots per sequence: rows 2 and 3 of sequence 0 have none
    p["table"][1, 0] = 999                              # and sequence 1's page does not exist
    before_k = p["k_pages"].clone()
    out = run_append(p)
    assert int(out.status) == (1 << 4) | (1 << 1)
    pg = int(p["table"][0, 0])
    assert not torch.equal(p["k_pages"][pg, :, 14:], before_k[pg, :, 14:])
    before_k[pg, :, 14:] = p["k_pages"][pg, :, 14:]
    assert torch.equal(p["k_pages"], before_k)
    assert torch.isfinite(out.q.float()).all()


def test_append_takes_what_the_merge_leaves():
    """out_offsets and out_pos of a merge go in as they are; the buffer is sized for all of the video's tokens."""
    from paper_2507_07990_b200 import inputs
    from tests import helpers
    video = inputs.make_video(helpers.small_spec(61, 6, 13, 13, 64, p_static=0.8))
    m = binding.sttm_merge_ex(helpers.to_torch(video), 0.97, 0.9)
    n = int(m.out_count[0])
    pool = cache.empty_cache(1, 6 * 169, 1, 64)
    pool.k.zero_()
    x = m.out_feats.view(-1, 1, 64)
    freq = (1e4 ** (-torch.arange(32).float() / 32)).cuda()
    out = cache.sttm_cache_append(pool, x, x, x, m.out_offsets, None, m.out_pos, cache.Rotary(freq))
    assert 0 < n < 6 * 169 and int(out.new_lengths[0]) == n and int(out.status) == 0
    flat = pool.k[:, 0].reshape(-1, 64)
    assert torch.equal(flat[:n], out.q[:n, 0]) and not flat[n:].any()
    assert torch.equal(pool.v[:, 0].reshape(-1, 64)[:n], x[:n, 0])


# ---------------------------------------------------------------- attend

def attend_problem(seed, lens, dtype="bf16", q_heads=7, heads=1, dim=64, page=16, order="heads", masked=None, scored=False, size=1.0,
                   max_len=None):
    gen = torch.Generator().manual_seed(seed)
    most = max(max(lens), 1) if max_len is None else max_len
    width = -(-most // page)
    table = ref.make_table(gen, len(lens), width)
    k_pages, v_pages = ref.make_pool(gen, len(lens) * width + 2, heads, page, dim, dtype, order)
    q = (torch.randn((len(lens), q_heads, dim), generator=gen) * size).to(ref.DTYPES[dtype]).cuda()
    mask = (torch.rand((len(lens), most), generator=gen) >= masked).cuda() if masked is not None else None
    scores = torch.rand((len(lens), heads, most), generator=gen).cuda() if scored else None
    return dict(dtype=dtype, q=q, k_pages=k_pages, v_pages=v_pages, table=table, lens=list(lens), mask=mask, scores=scores, max_len=most,
                lengths=torch.tensor(list(lens), dtype=torch.int32).cuda())


def run_attend(p, decay=0.75, scale=None):
    pool = cache.PagedCache(p["k_pages"], p["v_pages"], p["table"])
    return cache.AttendPlan(pool, p["q"].shape[1], scale=scale, max_len=p["max_len"], decay=decay).run(p["q"], p["lengths"], p["mask"], p["scores"])


def check_attend(p, out, scores_before=None, decay=0.75, scale=None):
    dim, heads = p["q"].shape[2], p["k_pages"].shape[1]
    scale = dim ** -0.5 if scale is None else scale
    got, lse = ref.f64(out.out), ref.f64(out.lse)
    for b, n in enumerate(p["lens"]):
        k, v, q = ref.slots_of(p["k_pages"], p["table"], b, n), ref.slots_of(p["v_pages"], p["table"], b, n), ref.f64(p["q"][b])
        mask = None if p["mask"] is None else p["mask"][b].cpu().numpy()[:n]
        want, want_lse, w = ref.attend(q, k, v, mask, scale)
        group = q.shape[0] // heads
        on = np.ones(n, dtype=bool) if mask is None else mask
        for i in range(q.shape[0]):
            if not on.any():
                assert not got[b, i].any() and lse[b, i] == -math.inf
                continue
            kk, vv = k[i // group][on], v[i // group][on]
            factor = 2.0 ** -19 * (np.abs(kk) @ np.abs(q[i])).max() * abs(scale) + 2.0 ** -17 + 2.0 ** -20
            allow = ref.ROUNDING[p["dtype"]] * np.abs(want[i]) + 2 * factor * np.abs(vv).max() + 2.0 ** -24
            np.testing.assert_array_less(np.abs(got[b, i] - want[i]), allow)
            assert abs(lse[b, i] - want_lse[i]) <= factor + 2.0 ** -21 * abs(want_lse[i])
        if p["scores"] is not None:
            after, before = ref.f64(p["scores"][b]), ref.f64(scores_before[b])
            for h in range(heads):
                f = max([0.0] + [2.0 ** -19 * (np.abs(k[h][on]) @ np.abs(q[h * group + g])).max() * abs(scale) for g in range(group) if on.any()])
                want_s = decay * before[h, :n] + w[h * group:(h + 1) * group].sum(0)
                allow = (2 * f + 2.0 ** -18) * w[h * group:(h + 1) * group].sum(0) + 2.0 ** -22 * np.abs(before[h, :n]) + 2.0 ** -40
                np.testing.assert_array_less(np.abs(after[h, :n] - want_s), allow)
                np.testing.assert_array_equal(after[h, n:], before[h, n:])
    assert int(out.status) == 0


LENS = (0, 1, 2, 15, 16, 17, 63, 64, 65, 130, 255)


@pytest.mark.parametrize("case", [
    dict(), dict(dtype="f16", dim=128, q_heads=28, heads=4, page=64), dict(dim=256, q_heads=8, heads=2, page=8), dict(dim=256, q_heads=20, heads=2, page=32, dtype="f16"),
    dict(q_heads=9, page=24, order="slots"), dict(q_heads=16, dim=128, page=128), dict(q_heads=40, heads=2, dim=128), dict(q_heads=33, dtype="f16"),
    dict(q_heads=64, page=40), dict(q_heads=3, heads=3, dim=128, order="slots", page=48),
    dict(masked=0.5), dict(masked=0.95, q_heads=12, dim=128, dtype="f16"), dict(scored=True), dict(scored=True, masked=0.6, q_heads=20, heads=2),
    dict(scored=True, q_heads=40, page=8, dim=128, dtype="f16"),
], ids=str)
@pytest.mark.parametrize("long", [False, True], ids=["short", "long"])
def test_attend(case, long):
    # long: rows beyond what one CTA takes whole, some of them in several CTAs' shares
    p = attend_problem(21, LENS + ((1000, 0, 700) if long else ()), **case)
    before = None if p["scores"] is None else p["scores"].clone()
    check_attend(p, run_attend(p), before)


@pytest.mark.parametrize("case", [dict(q_heads=7, dim=128), dict(q_heads=7, dim=128, scored=True, masked=0.3), dict(q_heads=2, heads=2, dim=64, dtype="f16"),
                                  dict(q_heads=24, dim=256, page=64)], ids=str)
def test_attend_one_long_sequence(case):
    # one row in hundreds of shares
    p = attend_problem(22, (20011,), **case)
    before = None if p["scores"] is None else p["scores"].clone()
    check_attend(p, run_attend(p), before)


@pytest.mark.parametrize("case", [dict(q_heads=7, dim=128), dict(q_heads=20, heads=1, dtype="f16"), dict(q_heads=40, dim=128, order="slots", page=48)], ids=str)
def test_attend_rows_joined_in_large_clusters(case):
    # clusters of 16 CTAs, under a mask of whole stretches (copies left out) whose rows begin at odd addresses
    p = attend_problem(34, (4003, 2999, 100), masked=0.0, **case)
    p["mask"] &= (torch.rand((3, 4003 // 37 + 1), generator=torch.Generator().manual_seed(1)) < 0.5).cuda().repeat_interleave(37, 1)[:, :4003]
    check_attend(p, run_attend(p))
    p["scores"] = torch.rand((3, 1, 4003), device="cuda")
    before = p["scores"].clone()
    check_attend(p, run_attend(p), before)


@pytest.mark.parametrize("scored", [False, True])
def test_attend_a_cta_per_row(scored):
    # rows enough to fill the GPU: whole rows to single CTAs; and longer ones in shares that end with rows
    rng = np.random.RandomState(5)
    for most, heads in ((700, 8), (1500, 8)):
        lens = [most] + [int(x) for x in rng.randint(most // 2, most, 21)]
        p = attend_problem(35, lens, q_heads=16, heads=heads, dim=64, page=32, scored=scored)
        before = None if p["scores"] is None else p["scores"].clone()
        check_attend(p, run_attend(p), before)


def test_attend_more_sequences_than_a_warp_scans_at_once():
    rng = np.random.RandomState(3)
    lens = [int(x) for x in rng.randint(0, 400, 90)]
    lens[40:75] = [0] * 35                              # a whole stretch without a slot
    check_attend(*(lambda p: (p, run_attend(p)))(attend_problem(23, lens, q_heads=5)))


@pytest.mark.parametrize("lens", [(0,), (0, 0, 0), (1,)], ids=str)
@pytest.mark.parametrize("max_len", [64, 640])
def test_attend_nothing_or_one_slot(lens, max_len):
    p = attend_problem(24, lens, max_len=max_len)
    check_attend(p, run_attend(p))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("long", [False, True])
def test_attend_ignores_what_lies_in_slots_that_do_not_count(dtype, long):
    """NaN and infinities beyond a sequence's length and under the mask, in keys and in values."""
    lens = (5, 100, 1) + ((900,) if long else ())
    p = attend_problem(25, lens, dtype=dtype, masked=0.4, scored=True, q_heads=10)
    clean = {**p, "k_pages": p["k_pages"].clone(), "v_pages": p["v_pages"].clone(), "scores": p["scores"].clone()}
    used = torch.zeros(p["k_pages"].shape[0], 16, dtype=torch.bool)
    for b, n in enumerate(lens):
        for s in range(n):
            if p["mask"][b, s]:
                used[int(p["table"][b, s // 16]), s % 16] = True
    used = used.cuda()
    for name, bad in (("k_pages", float("nan")), ("v_pages", float("inf"))):
        x = p[name].transpose(1, 2)
        x[~used] = bad
        x[~used] *= torch.where(torch.rand(x[~used].shape, device="cuda") < 0.5, float("nan"), 1.0).to(x.dtype)
    a, b = run_attend(p), run_attend(clean)
    assert torch.equal(a.out, b.out) and torch.equal(a.lse, b.lse) and torch.equal(p["scores"], clean["scores"])
    assert torch.isfinite(a.out.float()).all()


def test_attend_large_logits_and_other_scales():
    # logits of some hundreds: the running maximum has to hold in every part and across parts
    for size, scale, dtype in ((40.0, None, "bf16"), (1.0, -3.0, "bf16"), (20.0, None, "f16"), (1.0, 0.0, "f16")):
        p = attend_problem(26, (700, 64, 3), q_heads=8, size=size, dtype=dtype)
        check_attend(p, run_attend(p, scale=scale), scale=scale)


def test_attend_a_maximum_that_grows_and_one_that_comes_first():
    p = attend_problem(27, (640,), q_heads=7, dim=64, max_len=640)
    direction = p["q"][0, 0].float() / p["q"][0, 0].float().norm()
    for grow in (1, -1):
        for s in range(640):
            p["k_pages"][int(p["table"][0, s // 16]), 0, s % 16] = (direction * grow * (s - 320) / 8).to(torch.bfloat16)
        check_attend(p, run_attend(p))


def test_attend_minus_infinity_and_nan_in_slots_that_count():
    p = attend_problem(28, (130, 130), q_heads=4, max_len=130)
    p["q"].abs_()
    pg = lambda b, s: (int(p["table"][b, s // 16]), s % 16)
    a = pg(0, 70)
    p["k_pages"][a[0], 0, a[1]] = -math.inf             # weight zero, as if the slot were masked
    b = pg(1, 3)
    p["k_pages"][b[0], 0, b[1]] = math.nan
    out = run_attend(p)
    p["mask"] = torch.ones((2, 130), dtype=torch.bool, device="cuda")
    p["mask"][0, 70] = False
    want = run_attend(p)
    assert torch.equal(out.out[0], want.out[0]) and torch.isnan(out.out[1]).all()


def test_attend_questions_share_the_pages_of_a_video():
    p = attend_problem(29, (300,), q_heads=7, dim=128)
    alone = run_attend(p).out.clone()
    shared = {**p, "table": p["table"].expand(5, -1).contiguous(), "q": p["q"].expand(5, -1, -1), "lens": [300] * 5,
              "lengths": p["lengths"].expand(5).contiguous()}
    out = run_attend(shared).out
    torch.testing.assert_close(out[3].float(), alone[0].float(), rtol=2.0 ** -8, atol=1e-6)


def test_attend_strides_and_repeated_calls():
    p = attend_problem(30, (90, 700, 33), q_heads=7, heads=1, scored=True, masked=0.2)
    wide = torch.randn((3, 9, 64), device="cuda").bfloat16()
    wide[:, 1:8] = p["q"]
    scores = torch.zeros((3, 2, 705), device="cuda")
    scores[:, :1, :700] = p["scores"]
    mask = torch.zeros((3, 777), dtype=torch.uint8, device="cuda")
    mask[:, :700] = p["mask"].to(torch.uint8) * 255      # any byte that is not zero counts
    pool = cache.PagedCache(p["k_pages"], p["v_pages"], p["table"])
    plan = cache.AttendPlan(pool, 7, max_len=700, decay=0.5)
    first = plan.run(wide[:, 1:8], p["lengths"], mask[:, :701], scores[:, :1])
    one = first.out.clone(), first.lse.clone()
    plan.run(wide[:, 1:8], p["lengths"])                 # a call of another kind in between
    again = plan.run(wide[:, 1:8], p["lengths"], mask[:, :701], scores[:, :1])
    assert torch.equal(again.out, one[0]) and torch.equal(again.lse, one[1])    # the same bits
    q = {**p, "scores": p["scores"].clone()}
    run_attend(q, decay=0.5)
    run_attend(q, decay=0.5)
    assert torch.equal(scores[:, :1, :700], q["scores"]) and not scores[:, 1].any()


def test_attend_lengths_and_pages_that_cannot_be():
    p = attend_problem(31, (40, 600, 40), q_heads=4, max_len=600)
    p["lengths"] = torch.tensor([-3, 100000, 40], dtype=torch.int32).cuda()
    out = run_attend(p)
    assert int(out.status) == 1 << 4
    p["lens"] = [0, 600, 40]
    out.status.zero_()
    check_attend(p, out)                                 # -3 counts as none, 100000 as max_len
    p["table"][2, 1] = -1
    p["table"][1, 5] = 2 ** 30
    out = run_attend(p)
    assert int(out.status) == (1 << 4) | (1 << 1) and torch.isfinite(out.out.float()).all()


def test_attend_on_a_side_stream_and_in_a_graph():
    p = attend_problem(32, (500, 70), q_heads=7, scored=True)
    want = run_attend({**p, "scores": p["scores"].clone()})
    pool = cache.PagedCache(p["k_pages"], p["v_pages"], p["table"])
    plan = cache.AttendPlan(pool, 7, max_len=500)
    scores = p["scores"].clone()
    plan.run(p["q"], p["lengths"], None, scores.clone())
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        plan.run(p["q"], p["lengths"], None, scores)
    plan.out.zero_()
    for _ in range(3):
        g.replay()
    torch.cuda.synchronize()
    assert torch.equal(plan.out, want.out) and torch.equal(plan.lse, want.lse)
    ref_scores = p["scores"].clone()
    for _ in range(3):
        plan.run(p["q"], p["lengths"], None, ref_scores)
    assert torch.equal(scores, ref_scores)


def test_attend_a_cache_of_more_than_2_to_the_31_elements():
    """Pages whose offset passes 32 bits: 4.4 G elements in each pool, the sequence's pages at both ends."""
    pages, page, dim = 4200, 8192, 128
    k, v = (torch.empty((pages, 1, page, dim), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    at = [0, pages - 1, 2047, 2048, 4095, 4096]
    gen = torch.Generator().manual_seed(3)
    small = [torch.randn((len(at), 1, page, dim), generator=gen).bfloat16().cuda() for _ in range(2)]
    for i, pg in enumerate(at):
        k[pg], v[pg] = small[0][i], small[1][i]
    n = 5 * page + 77
    lengths = torch.tensor([n], dtype=torch.int32, device="cuda")
    q = torch.randn((1, 4, dim), generator=gen).bfloat16().cuda()
    big = cache.sttm_cache_attend(cache.PagedCache(k, v, torch.tensor([at], dtype=torch.int32).cuda()), q, lengths)
    same = cache.sttm_cache_attend(cache.PagedCache(*small, torch.arange(len(at), dtype=torch.int32).view(1, -1).cuda()), q, lengths)
    assert torch.equal(big.out, same.out) and torch.equal(big.lse, same.lse)
    # append and evict there too
    x = torch.randn((2, 1, dim), generator=gen).bfloat16().cuda()
    pool = cache.PagedCache(k, v, torch.tensor([[4100]], dtype=torch.int32).cuda())
    cache.sttm_cache_append(pool, None, x, x, torch.tensor([0, 2]).cuda(), torch.tensor([8190], dtype=torch.int32).cuda())
    assert torch.equal(k[4100, 0, 8190:], x[:, 0])
    dst = cache.empty_cache(1, 2, 1, dim)
    out = cache.sttm_cache_evict(pool, dst, torch.tensor([8192], dtype=torch.int32).cuda(), torch.tensor([2], dtype=torch.int32).cuda(),
                                 torch.arange(8192.0, device="cuda").view(1, 1, -1), 2)
    assert out.kept.tolist() == [[[8190, 8191]]] and torch.equal(dst.k[0, 0, :2], x[:, 0])


# ---------------------------------------------------------------- evict

def evict_problem(seed, lens, keep, dtype="bf16", heads=2, dim=64, page=16, dst_page=16, order="heads", kind="weights", same_pool=False, max_len=None):
    gen = torch.Generator().manual_seed(seed)
    most = max(max(lens), 1) if max_len is None else max_len
    width, kept_width = -(-most // page), max(max(keep), 1)
    dst_width = -(-kept_width // dst_page)
    table = ref.make_table(gen, len(lens), width, spare=len(lens) * dst_width if same_pool else 2)
    pages = len(lens) * (width + (dst_width if same_pool else 0)) + 2
    k, v = ref.make_pool(gen, pages, heads, page, dim, dtype, order)
    if same_pool:
        free = torch.tensor(sorted(set(range(pages)) - set(table.flatten().tolist())), dtype=torch.int32)
        dst_k, dst_v, dst_table = k, v, free[:len(lens) * dst_width].view(len(lens), dst_width).cuda()
    else:
        dst_k, dst_v = ref.make_pool(gen, len(lens) * dst_width + 2, heads, dst_page, dim, dtype)
        dst_table = ref.make_table(gen, len(lens), dst_width)
    s = torch.randn((len(lens), heads, most), generator=gen)
    if kind == "ties":
        s = torch.randint(0, 3, s.shape, generator=gen).float() - 1
        s[..., ::5] = -0.0
    elif kind == "odd":
        x = torch.tensor([math.nan, math.inf, -math.inf, 0.0, -0.0, 1e-40, -1e-40, 3e38, -math.nan, 1.0])
        s = x[torch.randint(0, len(x), s.shape, generator=gen)]
    elif kind == "weights":
        s = torch.where(torch.rand(s.shape, generator=gen) < 0.2, torch.zeros(()), torch.exp(3 * s))
    return dict(src=cache.PagedCache(k, v, table), dst=cache.PagedCache(dst_k, dst_v, dst_table), lens=list(lens), keep=list(keep),
                scores=s.cuda(), kept_width=kept_width, max_len=most)


def check_evict(p, first=0, last=0):
    src, dst = p["src"], p["dst"]
    was_k, was_v = dst.k.clone(), dst.v.clone()
    dev = lambda x: torch.tensor(x, dtype=torch.int32).cuda()
    out = cache.sttm_cache_evict(src, dst, dev(p["lens"]), dev(p["keep"]), p["scores"], p["kept_width"], first, last, p["max_len"])
    scores, kept, new = p["scores"].cpu().numpy(), out.kept.cpu().numpy(), out.new_scores.cpu().numpy()
    want_k, want_v = was_k, was_v
    for b, n in enumerate(p["lens"]):
        m = min(n, max(p["keep"][b], 0))
        assert int(out.new_lengths[b]) == m
        for h in range(src.heads):
            at = ref.evict(scores[b, h, :n], p["keep"][b], first, last)
            assert kept[b, h].tolist() == at + [-1] * (p["kept_width"] - m)
            np.testing.assert_array_equal(new[b, h, :m], scores[b, h, at])
            assert not new[b, h, m:].any()
            to = torch.arange(m, device="cuda")
            at = torch.tensor(at, dtype=torch.long, device="cuda")
            dp, sp = dst.table[b].long()[to // dst.page], src.table[b].long()[at // src.page]
            want_k[dp, h, to % dst.page] = src.k[sp, h, at % src.page]
            want_v[dp, h, to % dst.page] = src.v[sp, h, at % src.page]
    assert torch.equal(dst.k, want_k) and torch.equal(dst.v, want_v)
    assert int(out.status) == 0


@pytest.mark.parametrize("kind", ["weights", "ties", "odd"])
@pytest.mark.parametrize("case", [
    dict(), dict(dtype="f16", dim=128, page=64, dst_page=8, order="slots"), dict(dim=256, heads=3, page=24), dict(same_pool=True, dim=128),
], ids=str)
def test_evict(kind, case):
    p = evict_problem(41, (0, 1, 2, 64, 100, 511, 513, 300, 77), (5, 1, 1, 64, 31, 200, 512, 0, 1000), kind=kind, **case)
    check_evict(p)
    check_evict(p, first=4, last=9)
    check_evict(p, first=0, last=2000)


@pytest.mark.parametrize("n,keep", [(8192, 4000), (8193, 1), (20001, 17000), (33000, 16000), (70001, 35000), (210000, 100001)])
@pytest.mark.parametrize("kind", ["weights", "ties"])
def test_evict_long_rows(n, keep, kind):
    # a cluster of 1, 2, 4 and 8 CTAs per row
    p = evict_problem(42, (n, n // 3), (keep, keep // 4), heads=1, kind=kind)
    check_evict(p, first=4, last=64)


def test_evict_rows_beyond_shared_memory():
    # more slots than a cluster holds as keys: the rest is read again from memory
    p = evict_problem(43, (450001,), (1000,), heads=1, page=64)
    check_evict(p, first=1, last=30)


def test_evict_says_what_does_not_fit():
    p = evict_problem(44, (100, 90), (50, 20))
    dev = lambda x: torch.tensor(x, dtype=torch.int32).cuda()
    small = cache.PagedCache(p["dst"].k, p["dst"].v, p["dst"].table[:, :2].contiguous())        # 32 slots
    out = cache.sttm_cache_evict(p["src"], small, dev([100, 90]), dev([50, 20]), p["scores"], 50, max_len=100)
    assert out.new_lengths.tolist() == [32, 20] and int(out.status) == 1 << 4
    assert out.kept[0, 0, :32].tolist() == ref.evict(p["scores"][0, 0, :100].cpu().numpy(), 32, 0, 0)
    out = cache.sttm_cache_evict(p["src"], p["dst"], dev([100, 90]), dev([50, 20]), p["scores"], 40, max_len=100)
    assert out.new_lengths.tolist() == [40, 20] and int(out.status) == 1 << 4
    p["dst"].table[1, 0] = 10 ** 6
    out = cache.sttm_cache_evict(p["src"], p["dst"], dev([100, 90]), dev([50, 20]), p["scores"], 50, max_len=100)
    assert int(out.status) == 1 << 1


def test_the_three_together():
    """A cache filled, read with scores and thinned: attention over what is kept equals attention under a mask of it."""
    p = append_problem(51, rows=(600,), held=(0,), spare=0, q_heads=7, heads=1, dim=64)
    run_append(p)
    pool = cache.PagedCache(p["k_pages"], p["v_pages"], p["table"])
    q = torch.randn((1, 7, 64), device="cuda").bfloat16()
    lengths = torch.tensor([600], dtype=torch.int32, device="cuda")
    scores = torch.zeros((1, 1, 600), device="cuda")
    cache.sttm_cache_attend(pool, q, lengths, scores=scores, max_len=600)
    assert abs(float(scores.sum()) - 7.0) < 1e-4
    thin = cache.empty_cache(1, 200, 1, 64)
    e = cache.sttm_cache_evict(pool, thin, lengths, torch.tensor([200], dtype=torch.int32, device="cuda"), scores, 200, 4, 32, max_len=600)
    mask = torch.zeros((1, 600), dtype=torch.bool, device="cuda")
    mask[0, e.kept[0, 0].long()] = True
    a = cache.sttm_cache_attend(thin, q, e.new_lengths)
    b = cache.sttm_cache_attend(pool, q, lengths, mask, max_len=600)
    torch.testing.assert_close(a.out.float(), b.out.float(), rtol=2.0 ** -7, atol=1e-5)
    torch.testing.assert_close(a.lse, b.lse, rtol=0, atol=1e-5)


# ---------------------------------------------------------------- refusals on the device's tensors

def test_wrong_tensors_are_refused():
    p = attend_problem(33, (40, 20), q_heads=4)
    pool = cache.PagedCache(p["k_pages"], p["v_pages"], p["table"])
    plan = cache.AttendPlan(pool, 4, max_len=40)
    for bad in (p["q"].float(), p["q"][:, :3], p["q"].cpu(), p["q"].transpose(1, 2).contiguous().transpose(1, 2)):
        with pytest.raises(ValueError):
            plan.run(bad, p["lengths"])
    with pytest.raises(ValueError):
        plan.run(p["q"], p["lengths"].long())
    with pytest.raises(ValueError):
        plan.run(p["q"], p["lengths"], mask=torch.ones((2, 39), dtype=torch.bool, device="cuda"))
    with pytest.raises(ValueError):
        plan.run(p["q"], p["lengths"], scores=torch.zeros((2, 1, 40), dtype=torch.float64, device="cuda"))
    with pytest.raises(ValueError):
        cache.PagedCache(p["k_pages"].float(), p["v_pages"].float(), p["table"])
    with pytest.raises(ValueError):
        cache.PagedCache(p["k_pages"], p["v_pages"], p["table"].long())
    unaligned = torch.randn(2 * 4 * 64 + 1, device="cuda").bfloat16()[1:].view(2, 4, 64)
    with pytest.raises(binding.SttmError) as e:
        plan.run(unaligned, p["lengths"])
    assert e.value.code == 1
    a = append_problem(34)
    ap = cache.AppendPlan(cache.PagedCache(a["k_pages"], a["v_pages"], a["table"]), 4, cache.Rotary(a["freq"]))
    with pytest.raises(ValueError):
        ap.run(a["q"], a["k"], a["v"], a["offsets"].int(), a["lengths"], a["pos"])
    with pytest.raises(ValueError):
        ap.run(a["q"], a["k"], a["v"], a["offsets"], a["lengths"], a["pos"].double())
    with pytest.raises(ValueError):
        ap.run(a["q"], a["k"], a["v"][1:], a["offsets"], a["lengths"], a["pos"])
    with pytest.raises(binding.SttmError):
        cache.AppendPlan(ap.cache, 4, cache.Rotary(a["freq"], sections=(1, 2, 3))).run(
            a["q"], a["k"], a["v"], a["offsets"], a["lengths"], a["pos"].expand(3, -1).contiguous())
