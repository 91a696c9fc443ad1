"""Arguments at the edges of what the calls on the paged cache can hold, refused before anything reaches a GPU."""
import ctypes as C

from paper_2507_07990_b200 import binding
from tests.test_cache_refusals import AT, UNSUPPORTED, attend, pool


def test_a_grid_that_only_the_second_launch_could_not_have():
    """Rows x query heads just fit a grid; with the blocks that update the scores they no longer do: refused before the first launch."""
    lib = binding.load_library()
    seqs, n = (2 ** 31 - 1) // 64, 33 * 64
    c = pool(page=64, table_width=33, table_stride=33, heads=1, seqs=seqs)
    plain, scored = attend(q_heads=64, max_len=n), attend(q_heads=64, max_len=n, scores=AT, score_seq=n)
    assert lib.sttm_attend_workspace_bytes(C.byref(c), C.byref(plain)) > 0
    assert lib.sttm_attend_workspace_bytes(C.byref(c), C.byref(scored)) == 0
    assert lib.sttm_cache_attend(C.byref(c), C.byref(scored), AT, 1 << 60, None) == UNSUPPORTED
