"""Block norms, shared-prefix attention and 8-bit products together: questions of several lengths answered at once from one video's cache,
against the whole sequences recomputed in 64 bits without a cache."""
import pytest
import torch

from paper_2507_07990_b200 import answer, binding, inputs
from tests import helpers
from tests.test_gpu_answer import recompute

pytestmark = pytest.mark.gpu

# bf16 activations through two layers: some twenty roundings of 2^-8 relative to a row's norm, partly adding up
NEAR = 20 * 2.0 ** -8
# Eight products in 8 bits: steps of max / 127 on either side, with max some four times the root mean square: errors of 4 / 127 / sqrt(12) = 0.9 %
# of either, 1.3 % of a product, at most adding up, in the video's rows and in the questions': 16 of them
NEAR8 = NEAR + 16 * 0.013


def watch(**kw):
    video = helpers.to_torch(inputs.make_video(helpers.small_spec(71, 8, 13, 13, 256, p_static=0.8)))
    model = answer.Answerer(answer.Config(**kw))
    rows = model.watch(video, 0.97, 0.9)
    merged = binding.sttm_merge_ex(video, 0.97, 0.9)
    return model, merged.out_feats[:rows], merged.out_pos[:rows]


def lines(model, lengths=(9, 1, 4, 6)):
    gen = torch.Generator().manual_seed(2)
    return [torch.randint(0, model.cfg.vocab, (n,), generator=gen).cuda() for n in lengths]


@pytest.mark.parametrize("kw", [dict(), dict(kv_heads=2, q_heads=6), dict(dim=128, q_heads=2, page=64)])
def test_answers_match_the_recomputed_sequences(kw):
    model, rows, positions = watch(**kw)
    questions = lines(model)
    first = model.ask_together(questions, 1)
    logits = model.logits.double()
    answers = model.ask_together(questions, 3)
    assert torch.equal(answers[:, :1], first)
    for i, q in enumerate(questions):
        want = recompute(model, rows, positions, q)
        assert float((logits[i] - want).norm() / want.norm()) < NEAR
        want = recompute(model, rows, positions, torch.cat([q, answers[i, :2]]))
        assert float((model.logits[i].double() - want).norm() / want.norm()) < NEAR


def test_projections_in_8_bits():
    model, rows, positions = watch(int8=True)
    questions = lines(model)
    model.ask_together(questions, 1)
    for i, q in enumerate(questions):
        want = recompute(model, rows, positions, q)
        assert float((model.logits[i].double() - want).norm() / want.norm()) < NEAR8
    model.ask(torch.stack([q[:1] for q in questions]), 2)       # token by token, with the same weights
    assert torch.isfinite(model.logits).all()


def test_as_token_by_token():
    model, rows, positions = watch()
    questions = torch.stack(lines(model, (7, 7, 7)))
    model.ask(questions, 1)
    want = model.logits.clone()
    model.ask_together(list(questions), 1)
    assert float((model.logits - want).norm() / want.norm()) < 2 * NEAR


@pytest.mark.parametrize("int8", [False, True])
def test_what_the_calls_report_is_raised(int8):
    model, _, _ = watch(int8=int8)
    questions = lines(model)
    model.ask_together(questions, 2)
    model.pools[1].table[0, 0] = 10 ** 6
    with pytest.raises(binding.SttmError) as e:
        model.ask_together(questions, 2)
    assert e.value.code == 1
