"""Cases and plain forms of the cache operators: what an LLM does with a video's merged tokens.

  append  norm of queries and keys per head, rotation by the rows' positions, keys and values into a paged cache
  attend  attention of one new token per sequence over its paged cache; optionally adds each slot's weight to a running score
  evict   keeps a sequence's highest-scored slots: selection per KV head, and the kept rows copied to other pages

``own`` false: elementary torch operations in 32 bits, rounded once at the end.  ``own`` true: the
package's operators.  ``exact`` is the definition in 64 bits.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
THETA = 1e6                # base of the rotation's frequencies
CELLS = 169                # tokens of a 13 x 13 frame, the grid of most videos here
ROWS_OF_FRAME = 82         # what the merge leaves of such a frame at half the tokens
EPS = 1e-6
DECAY = 0.95               # what a running score keeps of itself per step


# ---------------------------------------------------------------- cases

def listed():
    """Head layouts: 28 query and 4 KV heads of 128 channels are a 7B model of 3584 channels, 64 and 8 a 72B
    one.  Row counts of videos are those the merge leaves: 5278 of 64 frames of 13 x 13 at half the tokens,
    15630 of 128 frames of 16 x 16 at half, 55724 of 1024 frames of 13 x 13 at three tenths."""
    base = {"dtype": "bf16", "q_heads": 28, "kv_heads": 4, "dim": 128, "page": 64, "order": "heads", "seqs": 1, "spread": 0.0}
    big = dict(base, q_heads=64, kv_heads=8)
    ap = dict(base, op="append", spare=0, held=0, norm=False, axes=1, mean=False, interleaved=False, rot=128, fused=True)
    at = dict(base, op="attend", masked=0.0, scored=False)
    ev = dict(base, op="evict", first=4, last=64)
    return [
        # one answer token of one user: latency
        dict(ap, name="append_one_token", rows=1, held=5330),
        # one answer token for each of 64 users of a batch, with norms, half precision, small pages
        dict(ap, name="append_64_tokens", q_heads=64, kv_heads=8, dtype="f16", page=16, seqs=64, rows=1, held=300, spread=0.5, norm=True),
        # a merged video enters the cache under (time, row, column) positions, out of a buffer sized for all its tokens
        dict(ap, name="append_video_3_axes", rows=15630, spare=17138, axes=3),
        # the longest video, under mean positions of merged tokens, with norms, pools slot by slot
        dict(ap, name="append_long_video_mean", rows=55724, norm=True, mean=True, fused=False, order="slots"),
        # an answer's first step after a short prompt: latency
        dict(at, name="attend_37", len=37),
        # one user's answer over a merged video and the question
        dict(at, name="attend_5338", len=5338),
        # the same over the longest video, collecting the weights for an eviction
        dict(at, name="attend_55788_scored", len=55788, scored=True),
        # questions on parts of videos: half of the frames masked, ragged lengths, 64-channel heads
        dict(at, name="attend_24_ragged_masked", dtype="f16", q_heads=14, kv_heads=2, dim=64, page=16, seqs=24, len=21013, spread=0.9, masked=0.5),
        # a full serving batch with weights collected
        dict(big, op="attend", name="attend_32_long_scored", seqs=32, len=32700, spread=0.1, masked=0.0, scored=True, page=32, order="slots"),
        # a short clip's cache is thinned before the answer: latency
        dict(ev, name="evict_1352", len=1352, keep=0.3, last=32),
        # the longest video's cache is halved
        dict(ev, name="evict_55788", len=55788, keep=0.5),
        # a batch's caches are cut to three tenths
        dict(big, op="evict", name="evict_16_ragged", dtype="f16", page=16, seqs=16, len=16421, spread=0.6, keep=0.3, first=4, last=100),
    ]


def draw(rng):
    def upto(lo, hi):                      # spread over the logarithm, odd values among them
        return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    most = max(work(c)["bytes"] for c in listed())
    while True:
        qh, kh = rng.choice([(28, 4), (64, 8), (14, 2), (10, 10), (40, 8), (20, 4), (8, 1), (40, 2)])
        c = {"dtype": rng.choice(["bf16", "f16"]), "q_heads": qh, "kv_heads": kh, "dim": rng.choice([64, 128, 128, 256]),
             "page": rng.choice([16, 32, 64, 128]), "order": rng.choice(["heads", "slots"]), "seqs": upto(1, 64),
             "spread": round(rng.choice([0.0, rng.random()]), 3), "op": rng.choice(["append", "attend", "evict"])}
        if c["op"] == "append":
            c.update(rows=rng.choice([1, upto(1, 55724)]), spare=rng.choice([0, upto(1, 5000)]), held=rng.choice([0, upto(1, 6000)]),
                     norm=rng.random() < 0.5, axes=rng.choice([1, 3]), mean=rng.random() < 0.5,
                     interleaved=rng.random() < 0.3, rot=rng.choice([c["dim"], c["dim"], c["dim"] // 2]), fused=rng.random() < 0.5)
        elif c["op"] == "attend":
            c.update(len=upto(1, 131000), masked=round(rng.choice([0.0, 0.0, rng.uniform(0.05, 0.95)]), 3), scored=rng.random() < 0.5)
        else:
            c.update(len=upto(64, 131000), keep=round(rng.uniform(0.05, 0.95), 3), first=rng.choice([0, 4]), last=rng.choice([0, upto(1, 64)]))
        # a drawn case stays below the largest listed one, its pools included
        slots = sum(held(c)) + sum(lengths(c)) + c.get("spare", 0)
        if max(work(c)["bytes"], 4 * slots * kh * c["dim"]) <= most:
            return c


def ragged(n, c, least):
    """n for the first sequence, down to (1 - spread) n for the last."""
    return [max(least, int(round(n * (1 - c["spread"] * b / max(1, c["seqs"] - 1))))) for b in range(c["seqs"])]


def lengths(c):
    """Per sequence: rows to append, or slots in the cache."""
    return ragged(c["rows"], c, 1) if c["op"] == "append" else ragged(c["len"], c, 1)


def held(c):
    """Per sequence: slots in use before the call (append)."""
    return ragged(c["held"], c, 0) if c["op"] == "append" else [0]


def kept(c):
    return [max(1, int(round(c["keep"] * n))) for n in lengths(c)]


def work(c):
    n, H, K, D = sum(lengths(c)), c["q_heads"], c["kv_heads"], c["dim"]
    if c["op"] == "append":                # every row's heads read and written once, its positions
        return {"bytes": n * ((H + 2 * K) * D * 4 + 4 * c["axes"]), "flops": n * (H + K) * D * (8 if c["norm"] else 4)}
    if c["op"] == "attend":                # keys and values of the attended slots, queries, outputs, scores
        seen = n * (1 - c["masked"])
        score = n * K * 8 if c["scored"] else 0
        return {"bytes": seen * K * D * 4 + c["seqs"] * H * (4 * D + 4) + (n if c["masked"] else 0) + score, "flops": 4 * seen * H * D}
    m = sum(kept(c))                       # all scores, the kept rows read and written, their indices and scores
    return {"bytes": n * K * 4 + m * K * (8 * D + 8), "flops": n * K}


# ---------------------------------------------------------------- inputs

def ids_of(n, gen, dev):
    """Position ids of n surviving tokens: increasing, two to three apart."""
    return torch.cumsum(torch.randint(1, 5, (n,), generator=gen, device=dev), 0) - 1


def pool(c, per_seq, gen, dev, fill):
    """Key and value pools [pages, heads, page, dim] and the table of a cache whose sequences hold per_seq slots."""
    width = max(-(-n // c["page"]) for n in per_seq)
    pages = c["seqs"] * width + 3
    table = torch.randperm(pages, generator=gen, device=dev)[:c["seqs"] * width].to(torch.int32).view(c["seqs"], width)
    inner = (c["kv_heads"], c["page"]) if c["order"] == "heads" else (c["page"], c["kv_heads"])
    both = []
    for _ in range(2):
        shape = (pages, *inner, c["dim"])
        p = torch.randn(shape, generator=gen, device=dev, dtype=DTYPES[c["dtype"]]) if fill else torch.zeros(shape, device=dev, dtype=DTYPES[c["dtype"]])
        both.append(p if c["order"] == "heads" else p.transpose(1, 2))
    return both[0], both[1], table


def prepare(c, seed):
    dev = "cuda"
    gen = torch.Generator(device=dev).manual_seed(int(seed) % (1 << 62))
    dt, H, K, D, S = DTYPES[c["dtype"]], c["q_heads"], c["kv_heads"], c["dim"], c["seqs"]
    n = lengths(c)
    s = {"case": c}
    if c["op"] == "append":
        before, rows = held(c), sum(n) + c["spare"]
        s["k_pages"], s["v_pages"], s["table"] = pool(c, [a + b for a, b in zip(before, n)], gen, dev, False)
        s["lengths"] = torch.tensor(before, dtype=torch.int32, device=dev)
        s["row_offsets"] = torch.cumsum(torch.tensor([0] + n, dtype=torch.int64, device=dev), 0)
        if c["fused"]:                     # views of one projection's output
            qkv = torch.randn((rows, H + 2 * K, D), generator=gen, device=dev, dtype=dt)
            s["q"], s["k"], s["v"] = qkv[:, :H], qkv[:, H:H + K], qkv[:, H + K:]
        else:
            s["q"], s["k"], s["v"] = (torch.randn((rows, h, D), generator=gen, device=dev, dtype=dt) for h in (H, K, K))
        ids = ids_of(rows, gen, dev)
        pos = torch.stack([ids // CELLS, ids % CELLS // 13, ids % 13]) if c["axes"] == 3 else ids.view(1, rows)
        if c["mean"]:                      # means of a few members' ids
            pos = pos.float() + torch.randint(0, 7, pos.shape, generator=gen, device=dev) / 7
        s["positions"] = pos.float() if c["mean"] else pos.to(torch.int32)
        half = c["rot"] // 2
        s["inv_freq"] = (THETA ** (-torch.arange(half, dtype=torch.float64, device=dev) / half)).float()
        a, b = (half // 4, half // 4 + (half - half // 4) // 2) if c["axes"] == 3 else (half, half)
        s["sections"] = (a, b - a, half - b) if c["axes"] == 3 else None
        i = torch.arange(half, device=dev)
        s["axis"] = (i >= a).long() + (i >= b).long()
        s["q_norm"], s["k_norm"] = ((1 + 0.2 * torch.randn(D, generator=gen, device=dev)) if c["norm"] else None for _ in range(2))
        s["q_out"] = torch.zeros((rows, H, D), device=dev, dtype=dt)
    elif c["op"] == "attend":
        s["k_pages"], s["v_pages"], s["table"] = pool(c, n, gen, dev, True)
        s["lengths"] = torch.tensor(n, dtype=torch.int32, device=dev)
        # unit-variance logits, with a few heads that look at little
        s["q"] = torch.randn((S, H, D), generator=gen, device=dev).mul_(torch.rand((S, H, 1), generator=gen, device=dev) * 2 + 0.3).to(dt)
        # a question on part of a video leaves out whole frames: runs of the rows that the merge leaves of one
        s["mask"] = None
        if c["masked"]:
            frames = torch.rand((S, max(n) // ROWS_OF_FRAME + 1), generator=gen, device=dev) >= c["masked"]
            s["mask"] = frames.repeat_interleave(ROWS_OF_FRAME, 1)[:, :max(n)].contiguous()
        s["scores"] = torch.rand((S, K, max(n)), generator=gen, device=dev) * 1e-2 if c["scored"] else None
    else:
        s["k_pages"], s["v_pages"], s["table"] = pool(c, n, gen, dev, True)
        m = kept(c)
        s["k_dst"], s["v_dst"], s["table_dst"] = pool(c, m, gen, dev, False)
        s["lengths"] = torch.tensor(n, dtype=torch.int32, device=dev)
        s["keep"] = torch.tensor(m, dtype=torch.int32, device=dev)
        s["keep_max"] = max(m)
        # sums of attention weights: heavy-tailed, and exactly zero where a slot was masked every time
        x = torch.randn((S, K, max(n)), generator=gen, device=dev)
        s["scores"] = torch.where(torch.rand(x.shape, generator=gen, device=dev) < 0.1, torch.zeros_like(x), torch.exp(1.5 * x) / c["len"])
    if own:
        s["plan"] = plan_of(c, s)
    return s


def plan_of(c, s):
    from paper_2507_07990_b200 import cache
    pages = cache.PagedCache(s["k_pages"], s["v_pages"], s["table"])
    if c["op"] == "append":
        rotary = cache.Rotary(s["inv_freq"], interleaved=c["interleaved"], sections=s["sections"])
        return cache.AppendPlan(pages, c["q_heads"], rotary, q_norm=s["q_norm"], k_norm=s["k_norm"], eps=EPS)
    if c["op"] == "attend":
        return cache.AttendPlan(pages, c["q_heads"], max_len=c["len"], decay=DECAY)
    return cache.EvictPlan(pages, cache.PagedCache(s["k_dst"], s["v_dst"], s["table_dst"]), s["keep_max"], first=c["first"], last=c["last"],
                           max_len=c["len"])


# ---------------------------------------------------------------- one pass

def run(s):
    op = s["case"]["op"]
    if op == "append":
        if own:
            r = s["plan"].run(s["q"], s["k"], s["v"], s["row_offsets"], s["lengths"], s["positions"], q_out=s["q_out"])
            return {"q": r.q, "k_pages": s["k_pages"], "v_pages": s["v_pages"], "lengths": r.new_lengths}
        return plain_append(s)
    if op == "attend":
        if own:
            r = s["plan"].run(s["q"], s["lengths"], mask=s["mask"], scores=s["scores"])
            return {"out": r.out, "lse": r.lse, "scores": s["scores"]}
        return plain_attend(s)
    if own:
        r = s["plan"].run(s["lengths"], s["keep"], s["scores"])
        return {"lengths": r.new_lengths, "kept": r.kept, "scores": r.new_scores, "k_pages": s["k_dst"], "v_pages": s["v_dst"]}
    return plain_evict(s)


def plain_rotate(x, w, cos, sin, interleaved):
    """Norm over a head's channels (w None: none), then the rotation of its first 2 * cos.shape[-1] channels."""
    y = x.float()
    if w is not None:
        y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + EPS) * w
    half = cos.shape[-1]
    r, rest = y[..., :2 * half], y[..., 2 * half:]
    if interleaved:
        a, b = r[..., 0::2], r[..., 1::2]
        r = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = r[..., :half], r[..., half:]
        r = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([r, rest], -1).to(x.dtype)


def plain_append(s):
    c, off = s["case"], s["row_offsets"]
    ang = s["positions"].float()[s["axis"]].t() * s["inv_freq"]
    cos, sin = ang.cos().unsqueeze(1), ang.sin().unsqueeze(1)
    q = plain_rotate(s["q"], s["q_norm"], cos, sin, c["interleaved"])
    k = plain_rotate(s["k"], s["k_norm"], cos, sin, c["interleaved"])
    # rows at or beyond the last offset are no tokens: they repeat the last token's write
    n = torch.arange(q.shape[0], device=q.device)
    real = torch.minimum(n, off[-1] - 1)
    seq = torch.searchsorted(off, real, right=True) - 1
    slot = s["lengths"][seq].long() + real - off[seq]
    page = s["table"][seq, slot // c["page"]].long()
    s["k_pages"][page, :, slot % c["page"]] = k[real]
    s["v_pages"][page, :, slot % c["page"]] = s["v"][real]
    s["q_out"].copy_(torch.where((n < off[-1]).view(-1, 1, 1), q, s["q_out"]))
    return {"q": s["q_out"], "k_pages": s["k_pages"], "v_pages": s["v_pages"], "lengths": s["lengths"] + (off[1:] - off[:-1]).int()}


def plain_gather(pages, table):
    """[seqs, heads, slots, dim] of a sequence's pages, in table order."""
    return pages[table.long()].transpose(1, 2).flatten(2, 3)


def plain_attend(s):
    c = s["case"]
    S, H, K, D = c["seqs"], c["q_heads"], c["kv_heads"], c["dim"]
    k, v = (plain_gather(s[x], s["table"])[:, :, :c["len"]].float() for x in ("k_pages", "v_pages"))
    within = torch.arange(c["len"], device=k.device) < s["lengths"].view(S, 1)
    seen = (within if s["mask"] is None else within & s["mask"]).view(S, 1, 1, -1)
    logits = torch.matmul(s["q"].float().view(S, K, H // K, D), k.transpose(2, 3)) / math.sqrt(D)
    logits = torch.where(seen, logits, -math.inf)
    top = logits.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    e = torch.exp(logits - top)
    total = e.sum(-1, keepdim=True)
    p = e / torch.where(total == 0, torch.ones_like(total), total)
    out = torch.matmul(p, torch.where(seen.view(S, 1, -1, 1), v, torch.zeros_like(v)))
    if c["scored"]:
        s["scores"].copy_(torch.where(within.unsqueeze(1), s["scores"] * DECAY + p.sum(2), s["scores"]))
    return {"out": out.view(S, H, D).to(s["q"].dtype), "lse": (torch.log(total) + top).view(S, H), "scores": s["scores"]}


def plain_evict(s):
    c = s["case"]
    S, K, L = s["scores"].shape
    slot = torch.arange(L, device=s["scores"].device)
    n = s["lengths"].view(S, 1, 1)
    new = torch.minimum(s["keep"], s["lengths"])
    key = torch.where((slot < c["first"]) | (slot >= n - c["last"]), math.inf, s["scores"])
    key = torch.where(slot < n, key, -math.inf)
    order = torch.sort(key, dim=-1, descending=True, stable=True).indices
    rank = torch.empty_like(order).scatter_(-1, order, slot.expand_as(order))
    at = torch.sort(torch.where(rank < new.view(S, 1, 1), slot, L), dim=-1).values[..., :s["keep_max"]]
    i = torch.arange(s["keep_max"], device=at.device)
    real = i < new.view(S, 1, 1)
    kept_at = torch.where(real, at, -1)
    # places beyond a sequence's new length repeat the write of its last kept slot
    i = torch.minimum(i.view(1, -1), new.view(S, 1).long() - 1)
    at = torch.gather(at, 2, i.unsqueeze(1).expand(S, K, -1))
    P, seq, head = c["page"], torch.arange(S, device=at.device).view(S, 1, 1), torch.arange(K, device=at.device).view(1, K, 1)
    src = s["table"][seq, at // P].long()
    dst = s["table_dst"][seq, (i // P).unsqueeze(1)].long()
    for_dst = (i % P).unsqueeze(1)
    s["k_dst"][dst, head, for_dst] = s["k_pages"][src, head, at % P]
    s["v_dst"][dst, head, for_dst] = s["v_pages"][src, head, at % P]
    scores = torch.where(real, torch.gather(s["scores"], 2, at), 0.0)
    return {"lengths": new, "kept": kept_at.int(), "scores": scores, "k_pages": s["k_dst"], "v_pages": s["v_dst"]}


# ---------------------------------------------------------------- the definition in 64 bits

def exact(c, seed):
    global own
    was, own = own, False
    try:
        s = prepare(c, seed)
    finally:
        own = was
    return {"append": exact_append, "attend": exact_attend, "evict": exact_evict}[c["op"]](c, s)


def exact_append(c, s):
    n, before, P = lengths(c), held(c), c["page"]
    kp, vp, q = s["k_pages"].double(), s["v_pages"].double(), s["q_out"].double()
    freq = s["inv_freq"].double()
    half, lo = len(freq), 0
    for b, rows in enumerate(n):
        for at in range(lo, lo + rows, 8192):
            r = slice(at, min(at + 8192, lo + rows))
            ang = torch.stack([s["positions"][int(s["axis"][j]), r].double() * freq[j] for j in range(half)], -1)
            turn = torch.polar(torch.ones_like(ang), ang).unsqueeze(1)
            new = []
            for x, w in ((s["q"], s["q_norm"]), (s["k"], s["k_norm"])):
                y = x[r].double()
                if w is not None:
                    y = y / (y.pow(2).sum(-1, keepdim=True) / c["dim"] + EPS).sqrt() * w.double()
                z = y[..., :2 * half]
                pair = z.unflatten(-1, (half, 2)) if c["interleaved"] else z.unflatten(-1, (2, half)).transpose(-1, -2)
                z = torch.view_as_real(torch.view_as_complex(pair.contiguous()) * turn)
                z = z.flatten(-2) if c["interleaved"] else z.transpose(-1, -2).flatten(-2)
                new.append(torch.cat([z, y[..., 2 * half:]], -1))
            q[r] = new[0]
            slot = before[b] + torch.arange(r.start - lo, r.stop - lo, device=q.device)
            page = s["table"][b].long()[slot // P]
            kp[page, :, slot % P] = new[1]
            vp[page, :, slot % P] = s["v"][r].double()
        lo += rows
    return {"q": q, "k_pages": kp, "v_pages": vp, "lengths": torch.tensor([a + b for a, b in zip(before, n)], dtype=torch.int32)}


def exact_attend(c, s):
    G = c["q_heads"] // c["kv_heads"]
    out, lse, scores = [], [], None if s["scores"] is None else s["scores"].double()
    for b, n in enumerate(lengths(c)):
        pages = s["table"][b].long()[:-(-n // c["page"])]
        for h in range(c["kv_heads"]):
            k, v = (s[x][pages, h].reshape(-1, c["dim"])[:n].double() for x in ("k_pages", "v_pages"))
            at = torch.arange(n, device=k.device) if s["mask"] is None else torch.nonzero(s["mask"][b, :n]).flatten()
            a = s["q"][b, h * G:(h + 1) * G].double() @ k[at].t() * c["dim"] ** -0.5
            if scores is not None:
                scores[b, h, :n] *= DECAY
            if len(at) == 0:
                out.append(torch.zeros((G, c["dim"]), dtype=torch.float64, device=k.device))
                lse.append(torch.full((G,), -math.inf, dtype=torch.float64, device=k.device))
                continue
            p = torch.softmax(a, -1)
            out.append(p @ v[at])
            lse.append(torch.logsumexp(a, -1))
            if scores is not None:
                scores[b, h, at] += p.sum(0)
    return {"out": torch.cat(out).view(c["seqs"], c["q_heads"], c["dim"]), "lse": torch.cat(lse).view(c["seqs"], -1), "scores": scores}


def exact_evict(c, s):
    P, n, m = c["page"], lengths(c), kept(c)
    kd, vd = s["k_dst"].double(), s["v_dst"].double()
    scores = torch.zeros((c["seqs"], c["kv_heads"], s["keep_max"]), dtype=torch.float64, device=kd.device)
    for b in range(c["seqs"]):
        to = torch.arange(min(m[b], n[b]), device=kd.device)
        dst = s["table_dst"][b].long()[to // P]
        for h in range(c["kv_heads"]):
            x = s["scores"][b, h, :n[b]].double().clone()
            x[:c["first"]] = math.inf
            x[max(0, n[b] - c["last"]):] = math.inf
            # the threshold, all above it, and of those at it the first
            least = torch.topk(x, len(to)).values[-1]
            tied = torch.nonzero(x == least).flatten()[:len(to) - int((x > least).sum())]
            at = torch.cat([torch.nonzero(x > least).flatten(), tied]).sort().values
            src = s["table"][b].long()[at // P]
            kd[dst, h, to % P] = s["k_pages"][src, h, at % P].double()
            vd[dst, h, to % P] = s["v_pages"][src, h, at % P].double()
            scores[b, h, :len(to)] = s["scores"][b, h, at].double()
    return {"lengths": None, "kept": None, "scores": scores, "k_pages": kd, "v_pages": vd}
