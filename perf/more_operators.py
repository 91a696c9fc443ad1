"""Cases and plain forms of the operators of a decoder layer that answers several questions on one video.

  prefix  attention of new tokens of several sequences over a cache that they share (a merged video) and over their own slots
  norm    a block's output normed, gated and added to the scaled residual stream, and the norm before the next block
  matmul  matrix product in 8-bit integers with a scale per token and per output channel; the tokens are quantized on the way:
          as they come, out of a norm (which returns the residual stream too), or out of a gated activation

``own`` false: elementary torch operations in 32 bits, rounded once at the end.  ``own`` true: the
package's operators.  ``exact`` is the definition in 64 bits.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
EPS = 1e-6


# ---------------------------------------------------------------- cases

def listed():
    """28 query and 4 KV heads of 128 channels and tokens of 3584 channels are a 7B model, 64 and 8 heads a 72B one.  Row counts
    of videos are those the merge leaves: 5278 of 64 frames of 13 x 13 at half the tokens, 15630 of 128 frames of
    16 x 16 at half, 55724 of 1024 frames of 13 x 13 at three tenths."""
    pre = {"op": "prefix", "dtype": "bf16", "q_heads": 28, "kv_heads": 4, "dim": 128, "page": 64, "order": "heads", "prefixes": 1, "spread": 0.0}
    norm = {"op": "norm", "dtype": "bf16", "post": True, "gate": "channel", "scale": 1.0, "pre": True}
    mat = {"op": "matmul", "dtype": "bf16", "inner": 3584, "bias": False, "after": "rows"}
    return [
        # the first answer token of two questions on a short clip: latency
        dict(pre, name="prefix_2_answers", len=676, seqs=2, new=1, held=13),
        # one answer token of 16 questions on the longest video
        dict(pre, name="prefix_16_answers_long", len=55724, seqs=16, new=1, held=61, spread=0.7),
        # 8 questions on an ordinary video are read in one go
        dict(pre, name="prefix_8_questions", len=5278, seqs=8, new=29, held=0, spread=0.5),
        # a serving batch: answer tokens of 96 questions on 6 videos, small pages
        dict(pre, name="prefix_96_answers_6_videos", dtype="f16", q_heads=64, kv_heads=8, page=16, order="slots", prefixes=6, len=15630,
             seqs=96, new=1, held=300, spread=0.6),
        # 16 long questions (choices, subtitles) on the longest video are read in one go
        dict(pre, name="prefix_16_questions_long", len=55724, seqs=16, new=53, held=0, spread=0.2),
        # between two blocks of a layer, one answer token: latency
        dict(norm, name="norm_one_token", rows=1, width=3584, post=False, gate="none"),
        # the same for all rows of the longest video, with norms on both sides
        dict(norm, name="norm_long_video", rows=55724, width=3584),
        # a width that fills no whole vectors, gates of every token, a damped residual stream
        dict(norm, name="norm_odd_gated_rows", dtype="f16", rows=15630, width=1157, gate="row", scale=0.5),
        # queries, keys and values of one answer token: latency
        dict(mat, name="matmul_one_token_qkv", rows=1, outer=4608, bias=True, after="norm"),
        # the last product of 16 answer tokens' layer
        dict(mat, name="matmul_16_tokens_down", rows=16, inner=14336, outer=3584, after="gated"),
        # an ordinary video's rows through the layer's widest product
        dict(mat, name="matmul_video_up", rows=5278, outer=28672, after="norm"),
        # the longest video's rows through the attention's output product
        dict(mat, name="matmul_long_video_out", rows=55724, outer=3584),
    ]


def draw(rng):
    def upto(lo, hi):                      # spread over the logarithm, odd values among them
        return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    op = rng.choice(["prefix", "norm", "matmul"])
    most = {k: max(work(c)[k] for c in listed() if c["op"] == op) for k in ("bytes", "flops")}
    while True:
        if op == "prefix":
            qh, kh = rng.choice([(28, 4), (64, 8), (14, 2), (10, 10), (40, 8), (20, 4), (8, 1), (40, 2)])
            p = rng.choice([1, 1, upto(1, 8)])
            c = {"op": op, "dtype": rng.choice(["bf16", "f16"]), "q_heads": qh, "kv_heads": kh, "dim": rng.choice([64, 128, 128, 256]),
                 "page": rng.choice([16, 32, 64, 128]), "order": rng.choice(["heads", "slots"]), "prefixes": p, "spread": round(rng.choice([0.0, rng.random()]), 3),
                 "len": upto(1, 60000), "seqs": p * upto(1, 32), "new": rng.choice([1, 1, upto(1, 200)]), "held": rng.choice([0, upto(1, 600)])}
            # (what a plain form keeps: logits of the prefix and of the sequences' own slots)
            fits = c["q_heads"] * c["new"] * c["seqs"] * (c["len"] + c["new"] + c["held"]) <= 28 * 53 * 16 * 55777
        elif op == "norm":
            c = {"op": op, "dtype": rng.choice(["bf16", "bf16", "f16", "f32"]), "rows": upto(1, 55724),
                 "width": rng.choice([3584, 8192, 1024, 256, upto(64, 8192)]), "post": rng.random() < 0.6, "gate": rng.choice(["none", "channel", "row"]),
                 "scale": rng.choice([1.0, round(rng.uniform(0.2, 1.5), 3)]), "pre": rng.random() < 0.8}
            fits = True
        else:
            c = {"op": op, "dtype": rng.choice(["bf16", "f16"]), "rows": upto(1, 55724), "inner": rng.choice([3584, 1024, 8192, upto(64, 14336)]),
                 "outer": rng.choice([3584, 4608, 1024, upto(16, 28672)]), "bias": rng.random() < 0.5, "after": rng.choice(["rows", "norm", "gated"])}
            fits = c["rows"] * c["inner"] <= 55724 * 3584
        w = work(c)
        if fits and all(w[k] <= most[k] for k in most):
            return c


def ragged(n, c, least):
    """n for the first sequence, down to (1 - spread) n for the last."""
    return [max(least, int(round(n * (1 - c["spread"] * b / max(1, c["seqs"] - 1))))) for b in range(c["seqs"])]


def new_tokens(c):
    return ragged(c["new"], c, 1)


def own_slots(c):
    """Per sequence: its own slots, the new tokens' among them."""
    return [a + b for a, b in zip(ragged(c["held"], c, 0), new_tokens(c))]


def prefix_lengths(c):
    """len for the first video, down to (1 - spread) len for the last."""
    return [max(1, int(round(c["len"] * (1 - c["spread"] * p / max(1, c["prefixes"] - 1))))) for p in range(c["prefixes"])]


def work(c):
    if c["op"] == "prefix":                # every prefix and own slot once, queries, outputs and their statistics; products with both
        n, own_n, pre, each = new_tokens(c), own_slots(c), prefix_lengths(c), c["seqs"] // c["prefixes"]
        slots = sum(pre) + sum(own_n)
        seen = sum(a * pre[b // each] + a * m - a * (a - 1) / 2 for b, (a, m) in enumerate(zip(n, own_n)))
        return {"bytes": slots * c["kv_heads"] * c["dim"] * 4 + sum(n) * c["q_heads"] * (c["dim"] * 4 + 4), "flops": 4.0 * seen * c["q_heads"] * c["dim"]}
    if c["op"] == "norm":                  # block's output, residual, gates; the new residual and its norm
        e, n = DTYPES[c["dtype"]].itemsize, c["rows"] * c["width"]
        return {"bytes": n * e * (3 + (1 if c["pre"] else 0) + (1 if c["gate"] == "row" else 0)), "flops": 8.0 * n}
    # matmul: weights and their scales, the tokens as they come, the outputs, a norm's residual read and written
    x = c["rows"] * c["inner"] * 2 * {"rows": 1, "gated": 2, "norm": 3}[c["after"]]
    return {"bytes": c["outer"] * (c["inner"] + 4) + x + c["rows"] * c["outer"] * 2, "flops": 2.0 * c["rows"] * c["inner"] * c["outer"]}


# ---------------------------------------------------------------- inputs

def pool(c, per_seq, gen, dev):
    """Key and value pools [pages, heads, page, dim] and the table of a cache whose sequences hold per_seq slots."""
    width = max(1, max(-(-n // c["page"]) for n in per_seq))
    pages = len(per_seq) * width + 3
    table = torch.randperm(pages, generator=gen, device=dev)[:len(per_seq) * width].to(torch.int32).view(len(per_seq), width)
    inner = (c["kv_heads"], c["page"]) if c["order"] == "heads" else (c["page"], c["kv_heads"])
    both = [torch.randn((pages, *inner, c["dim"]), generator=gen, device=dev, dtype=DTYPES[c["dtype"]]) for _ in range(2)]
    return [p if c["order"] == "heads" else p.transpose(1, 2) for p in both] + [table]


def offsets(counts, dev, dtype):
    return torch.cumsum(torch.tensor([0] + list(counts), device=dev), 0).to(dtype)


def prepare(c, seed):
    dev = "cuda"
    gen = torch.Generator(device=dev).manual_seed(int(seed) % (1 << 62))
    dt = DTYPES[c["dtype"]]
    normal = lambda *shape: torch.randn(shape, generator=gen, device=dev)  # noqa: E731
    # a residual stream and a block's output: tokens of several magnitudes, a few channels much larger than the others
    def stream(rows, width):
        x = normal(rows, width).mul_(torch.exp(0.5 * normal(rows, 1)))
        return x.mul_(torch.where(torch.rand(width, generator=gen, device=dev) < 0.004, 12.0, 1.0)).to(dt)

    s = {"case": c}
    if c["op"] == "prefix":
        n, H, D = sum(new_tokens(c)), c["q_heads"], c["dim"]
        s["k"], s["v"], s["table"] = pool(c, prefix_lengths(c), gen, dev)
        s["own_k"], s["own_v"], s["own_table"] = pool(c, own_slots(c), gen, dev)
        s["prefix_lengths"] = torch.tensor(prefix_lengths(c), dtype=torch.int32, device=dev)
        s["lengths"] = torch.tensor(own_slots(c), dtype=torch.int32, device=dev)
        s["row_offsets"] = offsets(new_tokens(c), dev, torch.int64)
        s["seq_offsets"] = offsets([c["seqs"] // c["prefixes"]] * c["prefixes"], dev, torch.int32)
        # unit-variance logits, with a few heads that look at little
        s["q"] = normal(n, H, D).mul_(torch.rand((n, H, 1), generator=gen, device=dev) * 2 + 0.3).to(dt)
    else:
        width = c["width"] if c["op"] == "norm" else c["inner"]
        s["x"] = stream(c["rows"], 2 * width if c.get("after") == "gated" else width)
        if c["op"] == "norm" or c["after"] == "norm":
            s["residual"] = stream(c["rows"], width)
            s["post_w"] = 1 + 0.2 * normal(width) if c.get("post") else None
            s["pre_w"] = 1 + 0.2 * normal(width) if c.get("pre", True) else None
            s["gate_c"] = 0.3 * normal(width) if c.get("gate") == "channel" else None
            s["gate_r"] = (0.3 * normal(c["rows"], width)).to(dt) if c.get("gate") == "row" else None
    if c["op"] == "matmul":
        # a program quantizes its weights once: [outer, inner] in rows of whole 16 bytes, a scale per output channel
        w = normal(c["outer"], c["inner"]).mul_(c["inner"] ** -0.5)
        s["w_scale"] = w.abs().amax(1) / 127
        s["w"] = torch.zeros((c["outer"], -(-c["inner"] // 16) * 16), dtype=torch.int8, device=dev)[:, :c["inner"]]
        s["w"].copy_(torch.round(w / s["w_scale"].unsqueeze(1)))
        s["bias"] = 0.1 * normal(c["outer"]) if c["bias"] else None
    if own:
        plans(c, s)
    return s


def plans(c, s):
    from paper_2507_07990_b200 import cache, layer, prefix
    dt = DTYPES[c["dtype"]]
    if c["op"] == "prefix":
        s["plan"] = prefix.PrefixPlan(cache.PagedCache(s["k"], s["v"], s["table"]), c["q_heads"], own=cache.PagedCache(s["own_k"], s["own_v"], s["own_table"]),
                                      max_rows=s["q"].shape[0], max_prefix=c["len"])
        return
    if c["op"] == "norm":
        s["norm"] = layer.NormPlan(c["width"], dt, c["rows"], post_norm=s["post_w"], gate=s["gate_c"], residual_scale=c["scale"], pre_norm=s["pre_w"], eps=EPS)
        return
    if c["after"] == "norm":
        s["norm"] = layer.NormPlan(c["inner"], dt, c["rows"], pre_norm=s["pre_w"], eps=EPS, quantize=True)
    else:
        s["quantize"] = layer.QuantizePlan(c["inner"], dt, c["rows"], gated=c["after"] == "gated")
    s["plan"] = layer.MatmulPlan(layer.QuantRows(s["w"], s["w_scale"]), dt, c["rows"], bias=s["bias"])


# ---------------------------------------------------------------- one pass

def run(s):
    c = s["case"]
    if c["op"] == "prefix":
        if own:
            r = s["plan"].run(s["q"], s["row_offsets"], s["prefix_lengths"], s["lengths"], seq_offsets=s["seq_offsets"])
            return {"out": r.out, "lse": r.lse}
        return plain_prefix(s)
    if c["op"] == "norm":
        if own:
            r = s["norm"].run(s["x"], s["residual"], gate=s["gate_r"])
            return {"sum": r.sum, "out": r.out}
        total, y = plain_norm(s, s["post_w"], s["gate_c"] if s["gate_r"] is None else s["gate_r"], c["scale"])
        return {"sum": total.to(s["x"].dtype), "out": None if s["pre_w"] is None else y.to(s["x"].dtype)}
    if own:
        if c["after"] == "norm":
            r = s["norm"].run(s["x"], s["residual"])
            return {"sum": r.sum, "out": s["plan"].run(r.rows)}
        return {"sum": None, "out": s["plan"].run(s["quantize"].run(s["x"]))}
    return plain_matmul(s)


def plain_gather(pages, table, width):
    """[seqs, heads, width, dim] of a sequence's pages, in table order."""
    return pages[table.long()].transpose(1, 2).flatten(2, 3)[:, :, :width].float()


def plain_part(q, k, v, seen):
    """Largest logit, sum of the exponentials and sum of the values, for q [n, heads, rows, dim] over k, v [n, heads, slots, dim]."""
    logits = torch.matmul(q, k.transpose(2, 3)) / math.sqrt(q.shape[-1])
    logits = torch.where(seen.unsqueeze(1), logits, -math.inf)
    top = logits.amax(-1, keepdim=True)
    e = torch.exp(logits - torch.where(top == -math.inf, 0.0, top))
    return top.squeeze(-1), e.sum(-1), torch.matmul(e, v)


def plain_prefix(s):
    c, off = s["case"], s["row_offsets"]
    H, K, D, P, S = c["q_heads"], c["kv_heads"], c["dim"], c["prefixes"], c["seqs"]
    n, G = s["q"].shape[0], H // K
    row = torch.arange(n, device=off.device)
    seq = torch.searchsorted(off, row, right=True) - 1
    # rows in boxes [box, rows of a box]: by prefix, and by sequence
    at = torch.searchsorted(s["seq_offsets"], seq.int(), right=True) - 1
    starts = off[s["seq_offsets"].long()]
    q = s["q"].float().view(n, K, G, D)

    def boxed(box, within, boxes, most):
        x = torch.zeros((boxes, most, K, G, D), device=off.device)
        x[box, within] = q
        return x.permute(0, 2, 1, 3, 4).reshape(boxes, K, most * G, D)

    def rows_of(x, box, within, most):
        return x.view(x.shape[0], K, most, G, -1).permute(0, 2, 1, 3, 4)[box, within]

    def part(box, within, boxes, most, keys, values, table, width, limit):
        # limit [boxes, most]: slots that a row sees
        seen = torch.arange(width, device=off.device) < limit.repeat_interleave(G, 1).unsqueeze(2)
        return [rows_of(x, box, within, most) for x in plain_part(boxed(box, within, boxes, most), plain_gather(keys, table, width), plain_gather(values, table, width), seen)]

    # (each prefix's and sequence's rows are at most these; the sizes come from the case, nothing is read back)
    each, counts = S // P, new_tokens(c)
    most = max(sum(counts[p * each:(p + 1) * each]) for p in range(P))
    shared = part(at, row - starts[at], P, most, s["k"], s["v"], s["table"], c["len"], s["prefix_lengths"].view(P, 1).expand(P, most))
    i = torch.arange(c["new"], device=off.device)
    limit = s["lengths"].view(S, 1) - (off[1:] - off[:-1]).view(S, 1) + 1 + i
    mine = part(seq, row - off[seq], S, c["new"], s["own_k"], s["own_v"], s["own_table"], max(own_slots(c)), torch.minimum(limit, s["lengths"].view(S, 1)))
    top = torch.maximum(shared[0], mine[0])
    a, b = torch.exp(shared[0] - top), torch.exp(mine[0] - top)
    total = a * shared[1] + b * mine[1]
    out = (a * shared[2] + b * mine[2]) / total
    return {"out": out.reshape(n, H, D).to(s["q"].dtype), "lse": (torch.log(total) + top).reshape(n, H)}


def plain_rms(x, w):
    return x if w is None else x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * w


def plain_norm(s, post_w, gate, scale):
    y = plain_rms(s["x"].float(), post_w)
    total = scale * s["residual"].float() + (y if gate is None else y * gate.float())
    return total, plain_rms(total, s["pre_w"])


def plain_matmul(s):
    c = s["case"]
    total = None
    if c["after"] == "norm":
        total, y = plain_norm(s, None, None, 1.0)
        total = total.to(s["x"].dtype)
    elif c["after"] == "gated":
        a, b = s["x"].float().chunk(2, -1)
        y = a * torch.sigmoid(a) * b
    else:
        y = s["x"].float()
    top = y.abs().amax(1, keepdim=True)
    q = torch.round(y * (127 / top))
    out = torch.matmul(q, s["w"].float().t())
    out = out * (top / 127) * s["w_scale"]
    if s["bias"] is not None:
        out = out + s["bias"]
    return {"sum": total, "out": out.to(s["x"].dtype)}


# ---------------------------------------------------------------- the definition in 64 bits

def exact(c, seed):
    global own
    was, own = own, False
    try:
        s = prepare(c, seed)
    finally:
        own = was
    return {"prefix": exact_prefix, "norm": exact_norm, "matmul": exact_matmul}[c["op"]](c, s)


def exact_prefix(c, s):
    K, D, G, page = c["kv_heads"], c["dim"], c["q_heads"] // c["kv_heads"], c["page"]
    out = torch.empty(s["q"].shape, dtype=torch.float64, device=s["q"].device)
    lse = torch.empty(s["q"].shape[:2], dtype=torch.float64, device=s["q"].device)
    each, at = c["seqs"] // c["prefixes"], 0
    for b, (n, m) in enumerate(zip(new_tokens(c), own_slots(c))):
        p = b // each
        shared = prefix_lengths(c)[p]
        for h in range(K):
            k, v = (torch.cat([s[x][s["table"][p].long(), h].reshape(-1, D)[:shared], s["own_" + x][s["own_table"][b].long(), h].reshape(-1, D)[:m]]).double()
                    for x in ("k", "v"))
            for lo in range(0, n, 16):
                hi = min(n, lo + 16)
                a = torch.einsum("tgd,sd->tgs", s["q"][at + lo:at + hi, h * G:(h + 1) * G].double(), k) * D ** -0.5
                # token i of n sees the prefix and its own slots up to itself
                last = shared + m - n + torch.arange(lo, hi, device=k.device)
                a.masked_fill_((torch.arange(shared + m, device=k.device) > last.view(-1, 1)).unsqueeze(1), -math.inf)
                out[at + lo:at + hi, h * G:(h + 1) * G] = torch.softmax(a, -1) @ v
                lse[at + lo:at + hi, h * G:(h + 1) * G] = torch.logsumexp(a, -1)
        at += n
    return {"out": out, "lse": lse}


def exact_normed(x, w):
    return x if w is None else x / (x.pow(2).sum(-1, keepdim=True) / x.shape[-1] + EPS).sqrt() * w.double()


def exact_stream(c, s):
    y = exact_normed(s["x"].double(), s["post_w"])
    for g in (s["gate_c"], s["gate_r"]):
        if g is not None:
            y = y * g.double()
    return y + s["residual"].double() * c.get("scale", 1.0)


def exact_norm(c, s):
    total = exact_stream(c, s)
    return {"sum": total, "out": None if s["pre_w"] is None else exact_normed(total, s["pre_w"])}


def exact_matmul(c, s):
    total = None
    if c["after"] == "norm":
        total = exact_stream(c, s)
        y = exact_normed(total, s["pre_w"])
    elif c["after"] == "gated":
        a, b = s["x"][:, :c["inner"]].double(), s["x"][:, c["inner"]:].double()
        y = a / (1 + torch.exp(-a)) * b
    else:
        y = s["x"].double()
    out = torch.empty((c["rows"], c["outer"]), dtype=torch.float64, device=y.device)
    w = s["w"].double().t()
    for lo in range(0, c["rows"], 8192):
        r = y[lo:lo + 8192]
        step = r.abs().max(1, keepdim=True).values / 127
        out[lo:lo + 8192] = (r / step).round() @ w * step * s["w_scale"].double()
    if s["bias"] is not None:
        out += s["bias"].double()
    return {"sum": total, "out": out}
