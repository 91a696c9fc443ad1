"""Attention over a shared prefix and own slots (sttm_prefix_attend) on the GPU against the definition in 64 bits.

Tolerance.  A logit is an fp32 sum of at most 256 products, off by at most 2^-19 of the sum of the products' magnitudes
(tensor-core sums truncate: an ulp for each of 16 steps) and by 2^-23 of itself in the multiplication by the scale; the exponential of the
difference to the reference m is off by that, by 2^-22 of itself, and by 2^-24 of the exponent (up to some 100).  A weight is then rounded to the
type (half a step, ROUNDING; in fp16, where it is taken 2^4 larger, by 2^-25 absolutely at least: 2^-29 of the largest), 32-bit
sums add 2^-16.  So an output is off by (ROUNDING + logit error + 2^-15) of sum w |v|, and by one rounding."""
import math

import pytest
import torch

from paper_2507_07990_b200 import binding, cache, prefix
from tests import cache_reference as ref

pytestmark = pytest.mark.gpu


def problem(seed, dtype="bf16", q_heads=4, heads=2, dim=128, page=16, order="heads", lens=(40,), groups=(2,), new=(1, 3), held=(0, 5), own=True,
            spare=2, lead=0, layout="fused", scale=1.0, ramp=0.0):
    """groups: sequences of every prefix; new, held: per sequence."""
    gen = torch.Generator().manual_seed(seed)
    dt, seqs, n = ref.DTYPES[dtype], len(new), lead + sum(new) + spare

    def one(counts):
        width = max(1, max(-(-c // page) for c in counts))
        k, v = ref.make_pool(gen, len(counts) * width + 2, heads, page, dim, dtype, order)
        return [k, v, ref.make_table(gen, len(counts), width)]

    pre, mine = one(lens), one([a + b for a, b in zip(new, held)]) if own else None
    for pool, counts in ((pre, lens), (mine, [a + b for a, b in zip(new, held)])):
        if pool is None:
            continue
        for b, c in enumerate(counts):                          # what lies behind a length is rubbish
            for s in range(c, pool[2].shape[1] * page):
                pool[0][int(pool[2][b, s // page]), :, s % page] = math.nan
                pool[1][int(pool[2][b, s // page]), :, s % page] = math.inf
            if ramp:                                            # keys that grow: the reference of the exponentials has to follow
                for s in range(c):
                    pool[0][int(pool[2][b, s // page]), :, s % page] *= ramp * s / max(1, c)
    if layout == "fused":
        q = torch.randn((n, q_heads + 3, dim), generator=gen).mul_(scale).to(dt).cuda()[:, 1:q_heads + 1]
    else:
        q = torch.randn((q_heads, n, dim), generator=gen).mul_(scale).to(dt).cuda().transpose(0, 1)
    ints = lambda x, t=torch.int32: torch.tensor(list(x), dtype=t).cuda()  # noqa: E731
    cum = lambda x, at=0: [at + sum(x[:i]) for i in range(len(x) + 1)]  # noqa: E731
    return dict(dtype=dtype, q=q, pre=pre, mine=mine, lens=lens, groups=groups, new=new, own=[a + b for a, b in zip(new, held)], lead=lead, page=page,
                row_offsets=ints(cum(list(new), lead), torch.int64), seq_offsets=ints(cum(list(groups))), prefix_lengths=ints(lens),
                lengths=ints(a + b for a, b in zip(new, held)))


def plan_of(p, rows=None, **kw):
    own = None if p["mine"] is None else cache.PagedCache(*p["mine"])
    return prefix.PrefixPlan(cache.PagedCache(*p["pre"]), p["q"].shape[1], own, rows or p["q"].shape[0], seqs=len(p["new"]), **kw)


def run(p, plan=None, **kw):
    plan = plan or plan_of(p)
    return plan.run(p["q"], p["row_offsets"], p["prefix_lengths"], p["lengths"], seq_offsets=p["seq_offsets"], **kw)


def slots(pool, row, n):
    k, v, table = pool
    at = torch.arange(n, device=table.device)
    pages = table[row].long()[at // k.shape[2]]
    return [t[pages, :, at % k.shape[2]].double().transpose(0, 1) for t in (k, v)]


def expect(p, scale=None):
    """out, lse, and bounds of both, rows of sequences only (dict row -> values)."""
    q = p["q"].double()
    rows, heads, dim = q.shape
    kv = p["pre"][0].shape[1]
    scale = dim ** -0.5 if scale is None else scale
    rnd = ref.ROUNDING[p["dtype"]]
    out, lse = torch.zeros_like(q), torch.full((rows, heads), -math.inf, dtype=torch.float64, device=q.device)
    bound, lse_bound, used = torch.zeros_like(q), torch.zeros_like(lse), torch.zeros(rows, dtype=torch.bool, device=q.device)
    at = p["lead"]
    starts = [sum(p["groups"][:i]) for i in range(len(p["groups"]) + 1)]
    for b, n in enumerate(p["new"]):
        parts = []
        which = next((g for g in range(len(p["groups"])) if starts[g] <= b < starts[g + 1]), None)
        if which is not None:
            parts.append(slots(p["pre"], which, p["lens"][which]))
        shared = parts[0][0].shape[1] if parts else 0
        m = p["own"][b] if p["mine"] is not None else 0
        if p["mine"] is not None:
            parts.append(slots(p["mine"], b, m))
        k, v = (torch.cat([x[i] for x in parts], 1).repeat_interleave(heads // kv, 0) for i in (0, 1)) if parts else (None, None)
        used[at:at + n] = True
        if n and parts and k.shape[1]:
            x = q[at:at + n].transpose(0, 1)
            a = x @ k.transpose(1, 2) * scale
            size = x.abs() @ k.abs().transpose(1, 2) * scale * 2.0 ** -19 + a.abs() * 2.0 ** -23
            last = shared + m - n + torch.arange(n, device=q.device) if p["mine"] is not None else torch.full((n,), shared, device=q.device)
            hidden = torch.arange(shared + m, device=q.device) > last.view(-1, 1)
            a = a.masked_fill(hidden, -math.inf)
            top = a.amax(-1, keepdim=True)
            w = torch.where(top == -math.inf, 0.0, (a - torch.where(top == -math.inf, 0.0, top)).exp())
            total = w.sum(-1, keepdim=True)
            w = w / total.clamp(min=1e-300)
            off = torch.where(hidden, 0.0, size).amax(-1, keepdim=True)
            out[at:at + n] = (w @ v).transpose(0, 1)
            lse[at:at + n] = torch.where(total == 0, -math.inf, total.log() + top)[..., 0].t()
            tiny = 2.0 ** -28 / total.clamp(min=1e-300) * torch.where(hidden, 0.0, 1.0) @ v.abs() if p["dtype"] == "f16" else 0.0
            bound[at:at + n] = ((rnd + 2 * off + 2.0 ** -15) * (w @ v.abs()) + tiny + rnd * (w @ v).abs()).transpose(0, 1)
            lse_bound[at:at + n] = (off[..., 0] + 2.0 ** -15).t()
        at += n
    return out, lse, bound, lse_bound, used


def check(p, r, scale=None, before=None):
    out, lse, bound, lse_bound, used = expect(p, scale)
    assert int(r.status) == 0
    err = (r.out.double() - out).abs()
    worst = (err - bound)[used]
    assert not (worst > 0).any() and torch.isfinite(r.out[used]).all(), float((err / bound.clamp(min=1e-30))[used].max())
    got = r.lse.double()
    empty = lse == -math.inf
    assert torch.equal((got == -math.inf)[used], empty[used])
    assert not (((got - lse).abs() > lse_bound) & ~empty)[used].any()
    if before is not None:
        assert torch.equal(r.out[~used], before[~used])


CASES = [
    dict(),
    dict(lens=(1,), groups=(1,), new=(1,), held=(0,)),
    dict(dtype="f16", dim=64, lens=(127,), groups=(3,), new=(1, 1, 1), held=(0, 1, 40)),
    dict(dim=256, lens=(129,), groups=(3,), new=(2, 0, 5), held=(63, 0, 0)),
    dict(dim=256, dtype="f16", q_heads=7, heads=1, lens=(700, 64), groups=(1, 2), new=(30, 1, 2), held=(0, 200, 0), page=64),
    dict(q_heads=28, heads=4, page=64, lens=(676,), groups=(2,), new=(1, 1), held=(13, 0)),
    dict(q_heads=28, heads=4, page=8, order="slots", lens=(300, 0, 65), groups=(2, 1, 3), new=(1, 9, 20, 0, 3, 1), held=(0, 0, 1, 5, 130, 128)),
    dict(q_heads=64, heads=1, lens=(257,), groups=(2,), new=(3, 2), held=(1, 0)),                  # 64 heads to a KV head: two tokens a block
    dict(q_heads=40, heads=2, page=24, lens=(95,), groups=(4,), new=(6, 7, 1, 13), held=(0, 9, 24, 0), layout="heads"),
    dict(q_heads=10, heads=10, dim=64, page=48, lens=(513,), groups=(2,), new=(129, 130), held=(0, 3)),   # two blocks and a bit, one query head each
    dict(q_heads=8, heads=1, page=128, lens=(4000,), groups=(3,), new=(100, 33, 17), held=(0, 0, 300)),
    dict(q_heads=14, heads=2, dim=64, lens=(1500, 900), groups=(2, 2), new=(40, 41, 1, 60), held=(0, 0, 0, 0), own=False),
    dict(lens=(0,), groups=(2,), new=(2, 1), held=(0, 0)),
    dict(lens=(0,), groups=(2,), new=(2, 1), held=(0, 0), own=False),                              # nothing to see at all
    dict(lens=(50,), groups=(1,), new=(2, 3, 1), held=(0, 4, 0)),                                  # two sequences without a prefix
    dict(lens=(60, 30), groups=(0, 3), new=(2, 3, 1), held=(0, 4, 0), lead=3),
]


@pytest.mark.parametrize("kw", CASES, ids=range(len(CASES)))
def test_against_the_definition(kw):
    p = problem(11 + len(str(kw)), **kw)
    plan = plan_of(p)
    plan.out.fill_(7.0)
    before = plan.out.clone()
    check(p, run(p, plan), before=before)
    first = plan.out.clone()
    assert torch.equal(run(p, plan).out, first)                 # every call repeats its bits


@pytest.mark.parametrize("dtype,dim", [("bf16", 128), ("f16", 64), ("f16", 256)])
@pytest.mark.parametrize("new", [1, 40])
def test_logits_that_rise_along_the_cache(dtype, dim, new):
    # keys up to 6 times as large at the end: the maximum rises by far more than 2^8 on the way
    p = problem(5, dtype=dtype, dim=dim, q_heads=8, heads=2, lens=(900,), groups=(2,), new=(new, new), held=(70, 0), scale=2.0, ramp=6.0)
    check(p, run(p))


def test_another_scale_and_shorter_limits():
    p = problem(6, lens=(200,), groups=(2,), new=(3, 1), held=(20, 0))
    check(p, run(p, plan_of(p, scale=0.03)), scale=0.03)
    r = run(p, plan_of(p, max_prefix=150))
    assert int(r.status) == 1 << 4                              # STTM_ERR_CAPACITY: cut
    p["lens"] = (150,)
    out = expect(p)[0]
    assert float((r.out.double() - out)[:4].abs().max()) < 0.05


def test_more_sequences_than_threads():
    n = 700
    new = [1 + i % 3 for i in range(n)]
    p = problem(8, q_heads=2, heads=1, dim=64, lens=(33,) * 350, groups=(2,) * 350, new=new, held=[i % 5 for i in range(n)])
    check(p, run(p))


@pytest.mark.parametrize("dtype,dim", [("bf16", 128), ("f16", 256)])
def test_many_pieces_of_every_kind_to_a_block(dtype, dim):
    # own slots of one tile, of several, of none, and new tokens of more than one block of rows, by turns
    n = 120
    new, held = [(1, 2, 40, 0)[b % 4] for b in range(n)], [(5, 150, 0, 0, 260)[b % 5] for b in range(n)]
    p = problem(21, dtype=dtype, dim=dim, q_heads=32, heads=8, page=16, lens=(130, 700), groups=(50, 70), new=new, held=held)
    check(p, run(p))


def test_hidden_values_do_not_matter_but_seen_ones_do():
    p = problem(9, lens=(100,), groups=(2,), new=(2, 2), held=(0, 0))
    p["mine"][1][int(p["mine"][2][0, 0]), :, 0] = math.nan      # sequence 0's first slot: seen by its tokens
    r = run(p)
    assert torch.isnan(r.out[:2]).all() and torch.isfinite(r.out[2:4]).all()


def test_conditions_found_on_the_device():
    p = problem(10, lens=(100,), groups=(2,), new=(2, 2), held=(0, 0))
    good = run(p).out.clone()
    p["row_offsets"][1], p["row_offsets"][2] = 3, 1             # decreasing: nothing is written
    plan = plan_of(p)
    plan.out.fill_(7.0)
    r = run(p, plan)
    assert int(r.status) & 2 and (r.out == 7.0).all()
    p["row_offsets"][1], p["row_offsets"][2] = 2, 9             # beyond the rows (6 of them)
    r = run(p)
    assert int(r.status) == 1 << 4
    p["row_offsets"][2] = 4
    p["pre"][2][0, 1] = 10 ** 6                                 # a page that is not there: zeros
    r = run(p)
    assert int(r.status) == 2 and torch.isfinite(r.out[:4]).all() and not torch.equal(r.out[:4], good[:4])
    p["seq_offsets"][1] = 3
    assert int(run(p).status) & 2


def test_captured_on_another_stream_and_replayed_with_new_lengths():
    p = problem(12, q_heads=28, heads=4, lens=(600,), groups=(2,), new=(2, 3), held=(9, 0))
    plan = plan_of(p)
    run(p, plan)
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        with torch.cuda.graph(graph, stream=stream):
            r = run(p, plan)
    for length in (600, 77, 0):
        p["lens"] = (length,)
        p["prefix_lengths"].fill_(length)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        check(p, r)


def test_one_call_and_refusals_of_the_plan():
    p = problem(13)
    r = prefix.sttm_prefix_attend(cache.PagedCache(*p["pre"]), p["q"], p["row_offsets"], p["prefix_lengths"], cache.PagedCache(*p["mine"]), p["lengths"])
    check(p, r)
    plan = plan_of(p)
    for kw in [dict(q=p["q"].float()), dict(q=p["q"][:, :3]), dict(row_offsets=p["row_offsets"].int()), dict(lengths=None),
               dict(lengths=p["lengths"][:1]), dict(prefix_lengths=p["prefix_lengths"].long()), dict(seq_offsets=p["row_offsets"]),
               dict(q=torch.cat([p["q"], p["q"]])), dict(out=p["q"])]:
        a = dict(q=p["q"], row_offsets=p["row_offsets"], prefix_lengths=p["prefix_lengths"], lengths=p["lengths"], seq_offsets=p["seq_offsets"])
        a.update(kw)
        with pytest.raises(ValueError):
            plan.run(**a)
    with pytest.raises(binding.SttmError):
        prefix.PrefixPlan(cache.PagedCache(*p["pre"]), 3, cache.PagedCache(*p["mine"]), 6).run(
            p["q"][:, :3], p["row_offsets"], p["prefix_lengths"], p["lengths"])
    nothing = plan.run(p["q"][:0], torch.zeros_like(p["row_offsets"]), p["prefix_lengths"], p["lengths"])
    assert nothing.out.shape[0] == 0


def test_offsets_beyond_32_bits():
    # pools of more than 2^31 elements; the sequences' pages lie at their ends
    gen = torch.Generator().manual_seed(14)
    p = problem(14, lens=(150,), groups=(2,), new=(2, 1), held=(20, 0), page=64)
    pages = 2 ** 31 // (2 * 64 * 128) + 40
    for name in ("pre", "mine"):
        k, v, table = p[name]
        big = [torch.empty((pages, 2, 64, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        where = pages - 1 - torch.randperm(30, generator=gen)[:k.shape[0]].cuda()
        for to, small in zip(big, (k, v)):
            to[where] = small
        p[name] = [*big, where[table.long()].to(torch.int32)]
        assert int(p[name][2].min()) * 2 * 64 * 128 > 2 ** 31
    check(p, run(p))


def test_two_plans_on_two_streams():
    a, b = problem(15, lens=(700,), new=(3, 9), held=(40, 0)), problem(16, dtype="f16", dim=64, lens=(900,), new=(30, 2), held=(0, 7))
    plans, streams = [plan_of(p) for p in (a, b)], [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(20):
        for p, plan, stream in zip((a, b), plans, streams):
            with torch.cuda.stream(stream):
                r = run(p, plan)
    torch.cuda.synchronize()
    for p, plan in zip((a, b), plans):
        check(p, prefix.PrefixOutput(plan.out[:p["q"].shape[0]], plan.lse[:p["q"].shape[0]], plan.status))
