"""Limits of the decode operators that the C interface checks before any device work (no GPU needed)."""
import ctypes

import pytest

EINVAL = -1
FAKE = 1 << 20      # an aligned address that is never read


@pytest.fixture(scope="module")
def lc():
    import paper_2608_01718_amd as m
    return m


def ref(c):
    return ctypes.byref(c)


@pytest.mark.parametrize("rows,n_seq,heads,q_heads", [(1 << 20, 1 << 20, 1024, 1024), (1 << 20, 1 << 30, 1025, 1025),
                                                      ((1 << 31) - 1, 1, 64, 64), (1 << 15, 1 << 15, 32768, 32768)])
def test_attention_of_more_row_groups_than_are_counted(lc, rows, n_seq, heads, q_heads):
    """The row groups of all sequences and heads are counted in 32 bits: a call that could have more is refused."""
    kv = lc._KV(FAKE, FAKE, 0, 0, 1, 32, heads, 8, lc.KV_BF16)
    seqs = lc._Seqs(FAKE, FAKE, FAKE, n_seq, 1)
    assert lc.raw_library().lacache_kv_attend(ref(kv), ref(seqs), FAKE, 1, rows, q_heads, 8 * q_heads, 1, 1.0, 0, FAKE, None,
                                              FAKE, 1 << 40, None) == EINVAL


@pytest.mark.parametrize("kw", [dict(d=20), dict(d=4), dict(d=260), dict(heads=0), dict(heads=65536), dict(heads=-1),
                                dict(n_pages=-1), dict(n_pages=1 << 31), dict(page=96), dict(type=4)])
def test_a_cache_that_no_call_would_take_is_not_allocated(lc, kw):
    with pytest.raises(ValueError):
        lc.KVCache(**{**dict(n_pages=4, heads=2, d=64, page=64, type=lc.KV_BF16), **kw})


@pytest.mark.parametrize("x,y,strides", [(FAKE, 2 * FAKE, (512, 128, 0, 128)), (FAKE, 2 * FAKE, (512, 128, 512, 0)),
                                         (FAKE, 2 * FAKE, (512, 128, 127, 1024)), (FAKE, 2 * FAKE, (512, 128, 512, 64)),
                                         (FAKE, FAKE, (512, 128, 1024, 128)), (FAKE, FAKE, (512, 128, 512, 256)),
                                         (FAKE, FAKE, (0, 128, 0, 128))])
def test_rotated_rows_that_would_overlap_are_refused(lc, x, y, strides):
    """Rows or heads of the result that share elements, and a result over the input in another order."""
    rope = lc._Rotary(FAKE, 100, 64, 0)
    turn = lc.raw_library().lacache_rope
    assert turn(x, y, 1, 3, 4, 128, *strides, FAKE, ref(rope), 0, None) == EINVAL
