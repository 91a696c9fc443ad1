"""Arguments that the example decoder refuses before it touches a GPU."""
import pytest
import torch

from paper_2507_07990_b200 import answer


@pytest.mark.parametrize("shape,tokens,keep", [((3, 0), 4, None), ((0, 5), 4, None), ((3, 5), 0, None), ((3, 5), 4, 0), ((3, 5), 4, -2), ((5,), 4, None)])
def test_questions_without_tokens_and_answers_of_none(shape, tokens, keep):
    model = answer.Answerer(answer.Config(), device="cpu")
    model.rows, model.pools = 10, []
    with pytest.raises(ValueError, match="at least"):
        model.ask(torch.zeros(shape, dtype=torch.long), tokens, keep)


def test_a_question_before_the_video():
    with pytest.raises(ValueError, match="watched"):
        answer.Answerer(answer.Config(), device="cpu").ask(torch.zeros((1, 2), dtype=torch.long), 1)
