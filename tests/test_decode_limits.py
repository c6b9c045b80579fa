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
