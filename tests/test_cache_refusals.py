"""Arguments that the calls on the paged cache refuse, before anything reaches a GPU."""
import ctypes as C

from paper_2507_07990_b200 import binding, cache

ARG, UNSUPPORTED, WORKSPACE = 1, 2, 3
BUF = (C.c_char * 8192)()
AT = (C.addressof(BUF) + 255) // 256 * 256


def pool(**kw):
    c = cache.SttmCache(AT, AT, 10, 2, 16, 64, 2 * 16 * 64, 16 * 64, 64, AT, 4, 4, 3, 0)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def attend(**kw):
    p = cache.AttendParams()
    p.q, p.q_seq, p.q_head, p.q_heads = AT, 256, 64, 4
    p.lengths, p.max_len, p.scale, p.out = AT, 64, 1.0, AT
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def append(**kw):
    p = cache.AppendParams()
    p.q = p.k = p.v = p.q_out = p.row_offsets = p.positions = p.inv_freq = AT
    p.q_row = p.k_row = p.v_row = 512
    p.q_head = p.k_head = p.v_head = 64
    p.rows, p.q_heads, p.axes, p.rot = 5, 4, 1, 64
    for k, v in kw.items():
        if k == "sections":
            p.sections[:] = v
        else:
            setattr(p, k, v)
    return p


def evict(**kw):
    p = cache.EvictParams()
    p.lengths, p.keep, p.scores = AT, AT + 256, AT + 512
    p.new_lengths, p.kept, p.new_scores = AT + 768, AT + 1024, AT + 1280
    p.max_len, p.kept_width = 64, 16
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def test_bad_caches():
    lib = binding.load_library()
    for kw, code in [(dict(k=None), ARG), (dict(v=None), ARG), (dict(table=None), ARG), (dict(pages=0), ARG), (dict(heads=0), ARG),
                     (dict(seqs=0), ARG), (dict(dtype=1), UNSUPPORTED), (dict(dim=96), UNSUPPORTED), (dict(dim=0), ARG),
                     (dict(page=12), UNSUPPORTED), (dict(page=0), ARG), (dict(k=AT + 2), ARG), (dict(slot_stride=68), ARG),
                     (dict(slot_stride=8), ARG), (dict(head_stride=1020), ARG), (dict(table_stride=3), ARG),
                     (dict(table_width=2 ** 30), UNSUPPORTED)]:
        c = pool(**kw)
        assert lib.sttm_cache_attend(C.byref(c), C.byref(attend()), AT, 8192, None) == code, kw
        assert lib.sttm_attend_workspace_bytes(C.byref(c), C.byref(attend())) == 0, kw
        assert lib.sttm_cache_append(C.byref(c), C.byref(append()), None) == code, kw
        assert lib.sttm_cache_evict(C.byref(c), C.byref(pool()), C.byref(evict()), None) == code, kw
        assert lib.sttm_cache_evict(C.byref(pool()), C.byref(c), C.byref(evict()), None) == code, kw


def test_bad_attend_arguments():
    lib = binding.load_library()
    c = pool()
    need = lib.sttm_attend_workspace_bytes(C.byref(c), C.byref(attend()))
    assert need > 0 and lib.sttm_attend_workspace_bytes(C.byref(c), C.byref(attend(scores=AT))) > need
    for kw in [dict(q=None), dict(out=None), dict(lengths=None), dict(q_heads=3), dict(q_heads=0), dict(max_len=0), dict(max_len=65),
               dict(q=AT + 8), dict(q_head=60), dict(q_seq=4), dict(scale=float("nan")), dict(mask=AT, mask_stride=63)]:
        assert lib.sttm_cache_attend(C.byref(c), C.byref(attend(**kw)), AT, 1 << 30, None) == ARG, kw
    assert lib.sttm_cache_attend(C.byref(c), C.byref(attend(q_heads=130)), AT, 1 << 30, None) == UNSUPPORTED
    assert lib.sttm_cache_attend(C.byref(c), C.byref(attend()), None, 1 << 30, None) == ARG
    assert lib.sttm_cache_attend(C.byref(c), C.byref(attend()), AT + 128, 1 << 30, None) == ARG
    assert lib.sttm_cache_attend(C.byref(c), C.byref(attend()), AT, need - 1, None) == WORKSPACE
    assert lib.sttm_cache_attend(None, C.byref(attend()), AT, need, None) == ARG
    assert lib.sttm_cache_attend(C.byref(c), None, AT, need, None) == ARG


def test_bad_append_arguments():
    lib = binding.load_library()
    c = pool()
    for kw in [dict(q=None), dict(k=None), dict(v=None), dict(q_out=None), dict(row_offsets=None), dict(rows=-1), dict(q_heads=-1),
               dict(positions=None), dict(inv_freq=None), dict(rot=72), dict(rot=80), dict(rot=-16), dict(axes=2), dict(k=AT + 8),
               dict(q_row=4), dict(v_head=4), dict(q_norm=AT + 4), dict(lengths=AT, new_lengths=AT),
               dict(axes=3, sections=(10, 10, 10)), dict(axes=3, sections=(40, -8, 0))]:
        assert lib.sttm_cache_append(C.byref(c), C.byref(append(**kw)), None) == ARG, kw
    assert lib.sttm_cache_append(C.byref(c), None, None) == ARG


def test_bad_evict_arguments():
    lib = binding.load_library()
    c = pool()
    for kw in [dict(lengths=None), dict(keep=None), dict(scores=None), dict(new_lengths=None), dict(kept=None), dict(new_scores=None),
               dict(max_len=0), dict(max_len=65), dict(kept_width=0), dict(first=-1), dict(last=-1), dict(new_lengths=AT),
               dict(new_scores=AT + 512)]:
        assert lib.sttm_cache_evict(C.byref(c), C.byref(pool()), C.byref(evict(**kw)), None) == ARG, kw
    for kw in [dict(heads=1), dict(dim=128, slot_stride=128), dict(dtype=2), dict(seqs=2)]:
        assert lib.sttm_cache_evict(C.byref(c), C.byref(pool(**kw)), C.byref(evict()), None) == ARG, kw
