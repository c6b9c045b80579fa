"""Argument checks of the decode operators at the C interface: refused before any device work (no GPU needed)."""
import ctypes
import math

import pytest

P = ctypes.c_void_p
EINVAL = -1
FAKE = 1 << 20      # an aligned address that is never read


@pytest.fixture(scope="module")
def lc():
    import paper_2608_01718_amd as m
    return m


def kv(lc, **kw):
    c = lc._KV(FAKE, FAKE, 0, 0, 10, 64, 2, 64, lc.KV_BF16)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def seqs(lc, **kw):
    c = lc._Seqs(FAKE, FAKE, FAKE, 2, 3)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def rot(lc, **kw):
    c = lc._Rotary(FAKE, 100, 64, 0)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


BAD_KV = [dict(page=48), dict(page=16), dict(page=512), dict(heads=0), dict(d=0), dict(d=60), dict(d=264), dict(type=0),
          dict(type=4), dict(n_pages=-1), dict(k=0), dict(v=0), dict(k=FAKE + 8), dict(v=FAKE + 2),
          dict(type=2), dict(type=3, k_scale=FAKE), dict(type=3, k_scale=FAKE, v_scale=FAKE + 4)]
BAD_SEQS = [dict(n_seq=-1), dict(max_pages=-1), dict(start=0), dict(lens=0), dict(pages=0)]
BAD_ROT = [dict(table=0), dict(table=FAKE + 4), dict(n_pos=0), dict(rot=0), dict(rot=63), dict(rot=66), dict(style=2)]


def ref(c):
    return ctypes.byref(c) if c is not None else None


def append(lc, c=None, s=None, r=None, **kw):
    a = dict(k=FAKE, v=FAKE, dtype=1, rows=2, k_row=128, v_row=128, q=FAKE, q_out=FAKE, q_heads=4, q_row=256, max_new=1)
    a.update(kw)
    return lc.raw_library().lacache_kv_append(ref(c), ref(s), a["k"], a["v"], a["dtype"], a["rows"], a["k_row"],
                                              a["v_row"], a["q"], a["q_out"], a["q_heads"], a["q_row"], ref(r),
                                              a["max_new"], None)


def attend(lc, c=None, s=None, **kw):
    a = dict(q=FAKE, dtype=1, rows=2, q_heads=4, q_row=256, max_new=1, scale=0.1, window=0, out=FAKE, lse=FAKE,
             workspace=FAKE, bytes=1 << 40)
    a.update(kw)
    return lc.raw_library().lacache_kv_attend(ref(c), ref(s), a["q"], a["dtype"], a["rows"], a["q_heads"], a["q_row"],
                                              a["max_new"], a["scale"], a["window"], a["out"], a["lse"], a["workspace"],
                                              a["bytes"], None)


def test_descriptions_are_checked(lc):
    lib = lc.raw_library()
    for bad in BAD_KV:
        c = kv(lc, **bad)
        assert append(lc, c, seqs(lc), rot(lc)) == EINVAL, bad
        assert attend(lc, c, seqs(lc)) == EINVAL, bad
        assert lib.lacache_kv_read(ref(c), ref(seqs(lc)), FAKE, FAKE, 1, 2, 1, None) == EINVAL, bad
    for bad in BAD_SEQS:
        assert append(lc, kv(lc), seqs(lc, **bad), rot(lc)) == EINVAL, bad
        assert attend(lc, kv(lc), seqs(lc, **bad)) == EINVAL, bad
        assert lib.lacache_kv_read(ref(kv(lc)), ref(seqs(lc, **bad)), FAKE, FAKE, 1, 2, 1, None) == EINVAL, bad
    for bad in BAD_ROT:
        assert append(lc, kv(lc), seqs(lc), rot(lc, **bad)) == EINVAL, bad
        assert lib.lacache_rope(FAKE, FAKE, 1, 2, 1, 64, 64, 64, 64, 64, FAKE, ref(rot(lc, **bad)), 0, None) == EINVAL, bad
    assert append(lc, None, seqs(lc), rot(lc)) == append(lc, kv(lc), None, rot(lc)) == EINVAL
    assert attend(lc, None, seqs(lc)) == attend(lc, kv(lc), None) == EINVAL
    assert lib.lacache_kv_read(None, ref(seqs(lc)), FAKE, FAKE, 1, 2, 1, None) == EINVAL
    assert lib.lacache_kv_read(ref(kv(lc)), None, FAKE, FAKE, 1, 2, 1, None) == EINVAL


def test_arguments_are_checked(lc):
    lib = lc.raw_library()
    good = kv(lc), seqs(lc), rot(lc)
    for bad in (dict(k=0), dict(v=0), dict(k=FAKE + 1), dict(v=FAKE + 1), dict(dtype=2), dict(dtype=7), dict(rows=-1),
                dict(rows=1 << 31), dict(k_row=-1), dict(v_row=-1), dict(q_row=-1), dict(q=0), dict(q_out=0),
                dict(q=FAKE + 1), dict(q_out=FAKE + 1), dict(q_heads=0), dict(q_heads=1 << 17), dict(max_new=-1),
                dict(dtype=0, k=FAKE + 2)):
        assert append(lc, *good, **bad) == EINVAL, bad
    assert append(lc, good[0], good[1], None) == EINVAL                                   # queries without a table
    for bad in (dict(q=0), dict(out=0), dict(q=FAKE + 1), dict(out=FAKE + 1), dict(lse=FAKE + 2), dict(dtype=2),
                dict(rows=-1), dict(rows=1 << 31), dict(q_heads=0), dict(q_heads=3), dict(q_heads=1 << 17),
                dict(q_row=-1), dict(max_new=-1), dict(scale=math.nan), dict(scale=math.inf), dict(window=-1),
                dict(bytes=-1)):
        assert attend(lc, good[0], good[1], **bad) == EINVAL, bad
    for out in ((FAKE + 1, FAKE), (FAKE, FAKE + 1)):
        assert lib.lacache_kv_read(ref(good[0]), ref(good[1]), *out, 1, 2, 1, None) == EINVAL
    assert lib.lacache_kv_read(ref(good[0]), ref(good[1]), FAKE, FAKE, 2, 2, 1, None) == EINVAL
    assert lib.lacache_kv_read(ref(good[0]), ref(good[1]), FAKE, FAKE, 1, -2, 1, None) == EINVAL
    r = ref(good[2])
    for bad in ((0, FAKE, 1, 2, 1, 64), (FAKE, 0, 1, 2, 1, 64), (FAKE, FAKE, 2, 2, 1, 64), (FAKE, FAKE, 1, -1, 1, 64),
                (FAKE, FAKE, 1, 2, 0, 64), (FAKE, FAKE, 1, 2, 1, 63), (FAKE, FAKE, 1, 2, 1, 4097),
                (FAKE + 1, FAKE, 1, 2, 1, 64), (FAKE, FAKE + 2, 0, 2, 1, 64)):
        assert lib.lacache_rope(*bad, 64, 64, 64, 64, FAKE, r, 0, None) == EINVAL, bad
    assert lib.lacache_rope(FAKE, FAKE, 1, 2, 1, 64, 64, 64, 64, 64, None, r, 0, None) == EINVAL
    assert lib.lacache_rope(FAKE, FAKE, 1, 2, 1, 64, 64, 64, 64, 64, FAKE, None, 0, None) == EINVAL
    assert lib.lacache_rope(FAKE, FAKE, 1, 2, 1, 64, -64, 64, 64, 64, FAKE, r, 0, None) == EINVAL
    for bad in (dict(table=0), dict(table=FAKE + 4), dict(first=-1), dict(n=-1), dict(rot=0), dict(rot=3), dict(rot=258),
                dict(base=1.0), dict(base=math.nan), dict(factor=0.5), dict(factor=math.inf), dict(original=-1.0),
                dict(low=-1.0), dict(low=32.0), dict(high=math.inf), dict(magnitude=math.nan)):
        a = dict(table=FAKE, first=0, n=4, rot=8, base=1e4, factor=1.0, original=0.0, low=1.0, high=32.0, magnitude=1.0)
        a.update(bad)
        assert lib.lacache_rope_table(*a.values(), None) == EINVAL, bad


def test_calls_without_work(lc):
    """No rows or no sequences: done, and no pointer is needed."""
    lib = lc.raw_library()
    empty = seqs(lc, start=0, lens=0, pages=0, n_seq=0)
    assert append(lc, kv(lc), empty, None, k=0, v=0, q=0, q_out=0, rows=0) == 0
    assert attend(lc, kv(lc), empty, q=0, out=0, lse=0, rows=0, workspace=0, bytes=0) == 0
    assert lib.lacache_kv_read(ref(kv(lc)), ref(empty), None, None, 1, 0, 0, None) == 0
    assert lib.lacache_rope(None, None, 1, 0, 1, 64, 64, 64, 64, 64, None, ref(rot(lc)), 0, None) == 0
    assert lib.lacache_rope_table(None, 0, 0, 8, 1e4, 1.0, 0.0, 1.0, 32.0, 1.0, None) == 0


def test_workspace_refuses(lc):
    ask = lc.raw_library().lacache_kv_attend_workspace
    for bad in (dict(page=48), dict(type=9), dict(d=12)):
        assert ask(ref(kv(lc, **bad)), 1, 2, 4, 1) == EINVAL
    for a in ((2, 2, 4, 1), (1, -1, 4, 1), (1, 2, 0, 1), (1, 2, 3, 1), (1, 2, 4, -1)):
        assert ask(ref(kv(lc)), *a) == EINVAL
    assert ask(None, 1, 2, 4, 1) == EINVAL
