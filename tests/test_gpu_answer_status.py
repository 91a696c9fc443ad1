"""What the calls on the cache say about themselves reaches the caller of the example decoder."""
import pytest
import torch

from paper_2507_07990_b200 import answer, binding, inputs
from tests import helpers

pytestmark = pytest.mark.gpu


def watch():
    video = helpers.to_torch(inputs.make_video(helpers.small_spec(71, 8, 13, 13, 256, p_static=0.8)))
    model = answer.Answerer(answer.Config())
    model.watch(video, 0.97, 0.9)
    return model


def questions(model):
    return torch.randint(0, model.cfg.vocab, (3, 4), generator=torch.Generator().manual_seed(2)).cuda()


@pytest.mark.parametrize("keep", [None, 20])
def test_a_page_that_is_not_there(keep):
    model = watch()
    assert model.ask(questions(model), 2, keep).shape == (3, 2)
    model.pools[1].table[0, 0] = 10 ** 6
    with pytest.raises(binding.SttmError) as e:
        model.ask(questions(model), 2, keep)
    assert e.value.code == 1


def test_a_video_that_its_cache_has_no_room_for(monkeypatch):
    real = answer.cache.empty_cache
    monkeypatch.setattr(answer.cache, "empty_cache", lambda seqs, n, *more: real(seqs, n - 16, *more))
    with pytest.raises(binding.SttmError) as e:
        watch()
    assert e.value.code == 4


def test_a_video_that_failed_leaves_nothing_to_ask(monkeypatch):
    model = watch()
    real = answer.cache.empty_cache
    monkeypatch.setattr(answer.cache, "empty_cache", lambda seqs, n, *more: real(seqs, n - 16, *more))
    video = helpers.to_torch(inputs.make_video(helpers.small_spec(72, 8, 13, 13, 256, p_static=0.8)))
    with pytest.raises(binding.SttmError):
        model.watch(video, 0.97, 0.9)
    with pytest.raises(ValueError):
        model.ask(questions(model), 1)
