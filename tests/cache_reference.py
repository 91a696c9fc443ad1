"""The cache operators written out in 64 bits, one sequence and one head at a time (numpy), and random
problems for them.  Shares no code with the package."""
import math

import numpy as np
import torch

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
# half a unit in the last place, relative: one rounding to the type
ROUNDING = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11}


def f64(t):
    return t.detach().to(torch.float64).cpu().numpy()


def make_pool(gen, pages, heads, page, dim, dtype, order="heads", fill=True):
    """Pools [pages, heads, page, dim] in the given memory order; random, or NaN when not filled."""
    out = []
    for _ in range(2):
        shape = (pages, heads, page, dim) if order == "heads" else (pages, page, heads, dim)
        t = torch.randn(shape, generator=gen) if fill else torch.full(shape, float("nan"))
        t = t.to(DTYPES[dtype]).cuda()
        out.append(t if order == "heads" else t.transpose(1, 2))
    return out


def make_table(gen, seqs, width, spare=2):
    return torch.randperm(seqs * width + spare, generator=gen)[:seqs * width].to(torch.int32).view(seqs, width).cuda()


def slots_of(pool, table, b, n):
    """[heads, n, dim] of sequence b's first n slots."""
    page = pool.shape[2]
    rows = [pool[int(table[b, s // page]), :, s % page] for s in range(n)]
    return np.stack([f64(r) for r in rows], 1) if rows else np.zeros((pool.shape[1], 0, pool.shape[3]))


def attend(q, k, v, mask, scale):
    """One sequence: q [q_heads, dim], k, v [heads, n, dim], mask [n] or None -> out, lse, weights [q_heads, n]."""
    heads, n, dim = k.shape
    group = q.shape[0] // heads
    out, lse, w = np.zeros_like(q), np.full(q.shape[0], -math.inf), np.zeros((q.shape[0], n))
    for i in range(q.shape[0]):
        at = [s for s in range(n) if mask is None or mask[s]]
        if not at:
            continue
        a = k[i // group][at] @ q[i] * scale
        top = a.max()
        if top == -math.inf:
            continue
        e = np.exp(a - top)
        w[i, at] = e / e.sum()
        out[i] = w[i, at] @ v[i // group][at]
        lse[i] = top + math.log(e.sum())
    return out, lse, w


def turn(x, weight, eps, pos, freq, axis, interleaved):
    """One head of one row: norm (weight None: none), then the rotation.  pos: one number per axis."""
    y = np.array(x, dtype=np.float64)
    if weight is not None:
        y = y / math.sqrt((y * y).mean() + eps) * weight
    half = len(freq)
    for i in range(half):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        t = pos[axis[i]] * freq[i]
        y[a], y[b] = y[a] * math.cos(t) - y[b] * math.sin(t), y[b] * math.cos(t) + y[a] * math.sin(t)
    return y


def evict(scores, keep, first, last):
    """One row: slots that stay.  Protected first, then by score, equal ones and NaN by slot."""
    n = len(scores)
    def rank(s):
        if s < first or s >= n - last:
            return (0, 0.0, s)
        x = float(scores[s])
        return (2, 0.0, s) if math.isnan(x) else (1, -x, s)
    return sorted(sorted(range(n), key=rank)[:max(0, min(keep, n))])
