"""Arguments at the edges of what the calls on the paged cache can hold, refused before anything reaches a GPU."""
import ctypes as C

from paper_2507_07990_b200 import binding
from tests.test_cache_refusals import ARG, AT, UNSUPPORTED, append, attend, evict, pool

WIDTH = (2 ** 31 - 1) // 8              # pages of 8 slots: the longest table there is


def test_lengths_whose_slots_cannot_be_counted_in_steps():
    """The kernels step over a row's slots in 32-bit integers, up to 606208 at a time."""
    lib = binding.load_library()
    c = pool(page=8, table_width=WIDTH, table_stride=WIDTH, heads=1, seqs=1)
    for n in (8 * WIDTH, 2 ** 31 - 2 ** 20):
        for kw in (dict(), dict(scores=AT), dict(mask=AT, mask_stride=n)):
            p = attend(max_len=n, q_heads=1, **kw)
            assert lib.sttm_attend_workspace_bytes(C.byref(c), C.byref(p)) == 0, (n, kw)
            assert lib.sttm_cache_attend(C.byref(c), C.byref(p), AT, 1 << 60, None) == UNSUPPORTED, (n, kw)
        assert lib.sttm_cache_evict(C.byref(c), C.byref(pool(heads=1, seqs=1)), C.byref(evict(max_len=n)), None) == UNSUPPORTED, n
        assert lib.sttm_cache_evict(C.byref(pool()), C.byref(pool()), C.byref(evict(kept_width=n)), None) == UNSUPPORTED, n
    # (bytes of a workspace, no call) the longest that is taken
    assert lib.sttm_attend_workspace_bytes(C.byref(c), C.byref(attend(max_len=2 ** 31 - 2 ** 20 - 1, q_heads=1))) > 0


def test_a_grid_that_only_the_second_launch_could_not_have():
    """Rows x query heads just fit a grid; with the blocks that update the scores they no longer do: refused before the first launch."""
    lib = binding.load_library()
    seqs, n = (2 ** 31 - 1) // 64, 33 * 64
    c = pool(page=64, table_width=33, table_stride=33, heads=1, seqs=seqs)
    plain, scored = attend(q_heads=64, max_len=n), attend(q_heads=64, max_len=n, scores=AT, score_seq=n)
    assert lib.sttm_attend_workspace_bytes(C.byref(c), C.byref(plain)) > 0
    assert lib.sttm_attend_workspace_bytes(C.byref(c), C.byref(scored)) == 0
    assert lib.sttm_cache_attend(C.byref(c), C.byref(scored), AT, 1 << 60, None) == UNSUPPORTED


def test_arrays_of_numbers_at_odd_addresses():
    """A kernel that read them there would end with a misaligned address."""
    lib = binding.load_library()
    for table in (AT + 2, AT + 1):
        bad = pool(table=table)
        assert lib.sttm_cache_attend(C.byref(bad), C.byref(attend()), AT, 1 << 30, None) == ARG
        assert lib.sttm_cache_append(C.byref(bad), C.byref(append()), None) == ARG
        assert lib.sttm_cache_evict(C.byref(pool()), C.byref(bad), C.byref(evict()), None) == ARG
    for off in (1, 2, 3):
        at = AT + 2048 + off
        for kw in [dict(lengths=at), dict(lse=at), dict(device_status=at), dict(scores=at, score_seq=256, score_head=64)]:
            assert lib.sttm_cache_attend(C.byref(pool()), C.byref(attend(**kw)), AT, 1 << 30, None) == ARG, kw
        for kw in [dict(lengths=at), dict(new_lengths=at), dict(positions=at), dict(inv_freq=at), dict(device_status=at), dict(row_offsets=at),
                   dict(row_offsets=AT + 4)]:
            assert lib.sttm_cache_append(C.byref(pool()), C.byref(append(**kw)), None) == ARG, kw
        for kw in [dict(lengths=at), dict(keep=at), dict(scores=at), dict(new_lengths=at), dict(kept=at), dict(new_scores=at), dict(device_status=at)]:
            assert lib.sttm_cache_evict(C.byref(pool()), C.byref(pool()), C.byref(evict(**kw)), None) == ARG, kw


def test_scores_whose_rows_overlap_cannot_be_updated():
    """Every row of scores is read and written by a call; rows that share memory would be updated in any order."""
    lib = binding.load_library()
    need = lib.sttm_attend_workspace_bytes(C.byref(pool()), C.byref(attend(scores=AT, score_seq=128, score_head=64)))
    assert need > 0
    # (3 sequences, 2 heads, 64 slots)
    for seq, head in ((0, 64), (128, 0), (128, 63), (64, 64), (127, 64), (64, 191), (64, 64 * 2), (-128, 64), (128, -64)):
        p = attend(scores=AT, score_seq=seq, score_head=head)
        assert lib.sttm_cache_attend(C.byref(pool()), C.byref(p), AT, 1 << 30, None) == ARG, (seq, head)
    # either axis may lie inside the other, and the stride of an axis of length one says nothing: these get as far as the workspace
    for seqs, heads, seq, head in ((3, 2, 128, 64), (3, 2, 200, 70), (3, 2, 64, 192), (1, 2, 0, 64), (3, 1, 64, 0), (1, 1, 0, 0)):
        c = pool(seqs=seqs, heads=heads)
        p = attend(scores=AT, score_seq=seq, score_head=head)
        assert lib.sttm_cache_attend(C.byref(c), C.byref(p), AT, 0, None) == 3, (seqs, heads, seq, head)
    # an eviction only reads them: one row of scores may serve all sequences and heads (this one is refused for its widths alone)
    assert lib.sttm_cache_evict(C.byref(pool()), C.byref(pool()), C.byref(evict(score_seq=0, score_head=0, kept_width=0)), None) == ARG
