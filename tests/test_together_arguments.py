"""Arguments that answering questions together refuses before it touches a GPU."""
import pytest
import torch

from paper_2507_07990_b200 import answer


@pytest.mark.parametrize("shapes,tokens", [([], 4), ([(3,), (0,)], 4), ([(3,)], 0), ([(2, 3)], 4)])
def test_questions_without_tokens_and_answers_of_none(shapes, tokens):
    model = answer.Answerer(answer.Config(), device="cpu")
    model.rows, model.pools = 10, [None]
    with pytest.raises(ValueError, match="at least"):
        model.ask_together([torch.zeros(s, dtype=torch.long) for s in shapes], tokens)


def test_questions_before_the_video():
    with pytest.raises(ValueError, match="watched"):
        answer.Answerer(answer.Config(), device="cpu").ask_together([torch.zeros(2, dtype=torch.long)], 1)
