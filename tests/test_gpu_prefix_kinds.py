"""Types and channels that the other tests of sttm_prefix_attend leave out: pieces of every kind to a block, and logits that rise along the cache."""
import pytest

from tests.test_gpu_prefix import check, problem, run

pytestmark = pytest.mark.gpu

KINDS = [("bf16", 256), ("bf16", 64), ("f16", 128), ("f16", 64), ("f16", 256)]


@pytest.mark.parametrize("dtype,dim", KINDS)
@pytest.mark.parametrize("seed", [51, 52])
def test_many_pieces_of_every_kind_to_a_block(dtype, dim, seed):
    n = 120
    new, held = [(1, 2, 40, 0)[b % 4] for b in range(n)], [(5, 150, 0, 0, 260)[b % 5] for b in range(n)]
    p = problem(seed, dtype=dtype, dim=dim, q_heads=32, heads=8, page=16 if seed == 51 else 64, order="heads" if seed == 51 else "slots", lens=(130, 700),
                groups=(50, 70), new=new, held=held)
    check(p, run(p))


@pytest.mark.parametrize("dtype,dim", KINDS)
@pytest.mark.parametrize("new,length", [(1, 20000), (40, 3000)])
def test_logits_that_rise_along_a_long_cache(dtype, dim, new, length):
    p = problem(53, dtype=dtype, dim=dim, q_heads=8, heads=2, page=64, lens=(length,), groups=(2,), new=(new, new), held=(70, 0), scale=2.0, ramp=6.0)
    check(p, run(p))
