"""Questions read at once with projections in 8 bits, within what independent errors add up to.

Bound.  A product in 8 bits is off by 1.3 % of its norm (steps of max / 127 with max some four times the root mean square: 0.9 % of either operand, the two
independent of each other).  Errors of different products are independent too, so their squares add up: 16 products (two layers of four, in the video's rows
and in the question's) give 4 * 1.3 %.  bf16 activations: some twenty roundings of 2^-8 that partly add up, as without 8 bits."""
import pytest

from tests.test_gpu_answer import recompute
from tests.test_gpu_together import NEAR, lines, watch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kw", [dict(), dict(kv_heads=2, q_heads=6), dict(dim=128, q_heads=2, page=64)])
def test_logits(kw):
    model, rows, positions = watch(int8=True, **kw)
    questions = lines(model)
    model.ask_together(questions, 1)
    for i, q in enumerate(questions):
        want = recompute(model, rows, positions, q)
        assert float((model.logits[i].double() - want).norm() / want.norm()) < NEAR + 4 * 0.013
