"""The cache operators together: answers read from the cache, token by token, against the whole sequence
recomputed without a cache."""
import pytest
import torch

from paper_2507_07990_b200 import answer, binding, inputs
from tests import cache_reference as ref
from tests import helpers

pytestmark = pytest.mark.gpu


def recompute(model, video_rows, positions, tokens):
    """Logits after the last of ``tokens`` (one question), every layer over the whole sequence in 64 bits."""
    c = model.cfg
    f = lambda t: t.double()
    rms = lambda x, w: x / (x.pow(2).mean(-1, keepdim=True) + 1e-6).sqrt() * f(w)
    x = torch.cat([f(video_rows), f(model.embed[tokens])])
    pos = torch.cat([positions.double(), model.next_position + torch.arange(len(tokens), device=x.device).double()])
    ang = pos[:, None] * f(model.rotary.inv_freq)
    cos, sin = ang.cos()[:, None], ang.sin()[:, None]

    def turn(y, w):
        y = rms(y, w)
        a, b = y.chunk(2, -1)
        return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)

    n = x.shape[0]
    causal = torch.ones((n, n), dtype=torch.bool, device=x.device).tril()
    for layer in model.layers:
        y = (rms(x, layer["norm1"]) @ f(layer["qkv"])).view(n, -1, c.dim)
        q, k, v = y[:, :c.q_heads], y[:, c.q_heads:c.q_heads + c.kv_heads], y[:, c.q_heads + c.kv_heads:]
        q, k = turn(q, layer["q_norm"]), turn(k, layer["k_norm"])
        k, v = (t.repeat_interleave(c.q_heads // c.kv_heads, 1) for t in (k, v))
        a = torch.einsum("qhd,khd->hqk", q, k) / c.dim ** 0.5
        p = torch.where(causal, a, -torch.inf).softmax(-1)
        x = x + torch.einsum("hqk,khd->qhd", p, v).reshape(n, -1) @ f(layer["out"])
        gate, up = (rms(x, layer["norm2"]) @ f(layer["up"])).chunk(2, -1)
        x = x + (torch.nn.functional.silu(gate) * up) @ f(layer["down"])
    return (rms(x, model.norm) @ f(model.head))[-1]


@pytest.fixture(scope="module")
def watched():
    video = helpers.to_torch(inputs.make_video(helpers.small_spec(71, 8, 13, 13, 256, p_static=0.8)))
    model = answer.Answerer(answer.Config(kv_heads=1, q_heads=7))
    rows = model.watch(video, 0.97, 0.9)
    merged = binding.sttm_merge_ex(video, 0.97, 0.9)
    questions = torch.randint(0, model.cfg.vocab, (3, 9), generator=torch.Generator().manual_seed(2)).cuda()
    return model, merged.out_feats[:rows], merged.out_pos[:rows], questions


def test_cached_answers_match_the_recomputed_sequence(watched):
    model, rows, positions, questions = watched
    model.ask(questions, 1)
    got = model.logits.double()
    for i in range(questions.shape[0]):
        want = recompute(model, rows, positions, questions[i])
        # bf16 activations through two layers: some twenty roundings of 2^-8 relative to a row's norm, partly adding up
        assert float((got[i] - want).norm() / want.norm()) < 20 * 2.0 ** -8


def test_keeping_every_slot_changes_nothing_and_half_of_them_little(watched):
    model, rows, positions, questions = watched
    whole = model.ask(questions, 1)
    full = model.logits.clone()
    same = model.ask(questions, 1, keep=10 ** 6)
    # the logits that the first answer token comes from were there before the eviction
    assert torch.equal(same, whole) and torch.equal(model.logits, full)
    whole = model.ask(questions, 2)
    full = model.logits.clone()
    same = model.ask(questions, 2, keep=10 ** 6)
    # the second's come from the same keys and values in other pages, the shares of the work cut otherwise (see above)
    assert torch.equal(same[:, 0], whole[:, 0])
    assert float((model.logits - full).norm() / full.norm()) < 20 * 2.0 ** -8
    thin = model.ask(questions, 3, keep=len(rows) // 2)
    assert thin.shape == (3, 3) and torch.isfinite(model.logits).all()


def test_the_command_runs(capsys):
    answer.main()
    assert "rows in the cache" in capsys.readouterr().out
