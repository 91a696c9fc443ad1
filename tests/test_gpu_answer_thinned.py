"""Answers from thinned caches, against 64 bits: which slots the question's attention leaves, and the logits that the next token
gets from them."""
import pytest
import torch

from paper_2507_07990_b200 import answer, binding, inputs
from tests import helpers

pytestmark = pytest.mark.gpu


class Wide:
    """The decoder's layers in 64 bits, one token sequence at a time."""

    def __init__(self, model):
        self.m, self.c = model, model.cfg

    def rms(self, x, w):
        return x / (x.pow(2).mean(-1, keepdim=True) + 1e-6).sqrt() * w.double()

    def qkv(self, layer, x, pos):
        c, ang = self.c, pos[:, None] * self.m.rotary.inv_freq.double()
        cos, sin = ang.cos()[:, None], ang.sin()[:, None]
        y = (self.rms(x, layer["norm1"]) @ layer["qkv"].double()).view(len(x), -1, c.dim)

        def turn(y, w):
            a, b = self.rms(y, w).chunk(2, -1)
            return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)

        q, k, v = y.split([c.q_heads, c.kv_heads, c.kv_heads], 1)
        return turn(q, layer["q_norm"]), turn(k, layer["k_norm"]), v

    def rest(self, layer, x, attended):
        x = x + attended.reshape(len(x), -1) @ layer["out"].double()
        gate, up = (self.rms(x, layer["norm2"]) @ layer["up"].double()).chunk(2, -1)
        return x + (torch.nn.functional.silu(gate) * up) @ layer["down"].double()

    def logits(self, x):
        return self.rms(x, self.m.norm) @ self.m.head.double()


@pytest.mark.parametrize("kv_heads,q_heads,keep", [(1, 7, 40), (2, 6, 33)])
def test_thinned_answers(monkeypatch, kv_heads, q_heads, keep):
    video = helpers.to_torch(inputs.make_video(helpers.small_spec(71, 8, 13, 13, 256, p_static=0.3)))
    model = answer.Answerer(answer.Config(kv_heads=kv_heads, q_heads=q_heads))
    rows = model.watch(video, 0.97, 0.9)
    assert rows > 2 * keep
    merged = binding.sttm_merge_ex(video, 0.97, 0.9)
    length, first, last = 9, 4, 9
    questions = torch.randint(0, model.cfg.vocab, (3, length), generator=torch.Generator().manual_seed(2)).cuda()
    kept, evict = [], answer.cache.sttm_cache_evict

    def spy(*args, **kw):
        out = evict(*args, **kw)
        kept.append(out.kept.clone())
        return out

    monkeypatch.setattr(answer.cache, "sttm_cache_evict", spy)
    answers = model.ask(questions, 2, keep=keep)
    assert len(kept) == model.cfg.layers and kept[0].shape == (3, kv_heads, keep)
    wide, c, group = Wide(model), model.cfg, q_heads // kv_heads
    for i in range(3):
        x = torch.cat([merged.out_feats[:rows].double(), model.embed[questions[i]].double()])
        pos = torch.cat([merged.out_pos[:rows].double(), model.next_position + torch.arange(length, device="cuda").double()])
        n = len(x)
        new, new_pos = model.embed[answers[i, :1]].double(), torch.tensor([model.next_position + length], device="cuda").double()
        causal = torch.ones((n, n), dtype=torch.bool, device="cuda").tril()
        for layer, at in zip(model.layers, kept):
            q, k, v = wide.qkv(layer, x, pos)
            kk, vv = k.repeat_interleave(group, 1), v.repeat_interleave(group, 1)
            p = torch.where(causal, torch.einsum("qhd,khd->hqk", q, kk) / c.dim ** 0.5, -torch.inf).softmax(-1)
            x = wide.rest(layer, x, torch.einsum("hqk,khd->qhd", p, vv).reshape(n, -1))
            # What the question's tokens gave every slot.  The decoder's own activations are bf16: a row is off by some ten
            # roundings of 2^-8, queries and keys (of length 8) by 4 % of theirs, a logit by 8 * 8 / 8 * 0.08 = 0.64, a weight by less than
            # a factor of 2.
            score = p[:, rows:].sum(1).view(kv_heads, group, n).sum(1)
            q2, k2, v2 = wide.qkv(layer, new, new_pos)
            attended = []
            for h in range(kv_heads):
                on = at[i, h].long()
                assert bool((on[1:] > on[:-1]).all()) and on[:first].tolist() == list(range(first)) and on[-last:].tolist() == list(range(n - last, n))
                off = torch.ones(n, dtype=torch.bool, device="cuda")
                off[on] = False
                assert float(score[h, on[first:-last]].min()) > float(score[h, off].max()) / 2
                a = q2[0, h * group:(h + 1) * group] @ torch.cat([k[on, h], k2[:, h]]).t() / c.dim ** 0.5
                attended.append(a.softmax(-1) @ torch.cat([v[on, h], v2[:, h]]))
            new = wide.rest(layer, new, torch.cat(attended).view(1, -1))
        want = wide.logits(new)[0]
        got = model.logits[i].double()
        assert float((got - want).norm() / want.norm()) < 20 * 2.0 ** -8
