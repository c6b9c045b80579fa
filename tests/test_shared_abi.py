"""Argument checks of attention over shared prefixes at the C interface: refused before any device work (no GPU needed)."""
import math

from tests.test_decode_abi import BAD_KV, BAD_SEQS, EINVAL, FAKE, kv, lc, ref, seqs  # noqa: F401


def prefixes(lc, **kw):
    c = lc._Prefixes(FAKE, FAKE, 2)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def attend(lc, c, s, p, **kw):
    a = dict(q=FAKE, dtype=1, rows=2, q_heads=4, q_row=256, max_new=1, scale=0.1, window=0, out=FAKE, lse=FAKE, workspace=FAKE,
             bytes=1 << 40, stream=None)
    a.update(kw)
    return lc.raw_library().lacache_kv_attend_shared(ref(c), ref(s), ref(p), *a.values())


def test_refuses(lc):
    for bad in BAD_KV:
        assert attend(lc, kv(lc, **bad), seqs(lc), prefixes(lc)) == EINVAL, bad
    for bad in [*BAD_SEQS, dict(n_seq=(1 << 20) + 1)]:
        assert attend(lc, kv(lc), seqs(lc, **bad), prefixes(lc)) == EINVAL, bad
    for bad in (dict(group=0), dict(len=0), dict(group=FAKE + 2), dict(len=FAKE + 1), dict(n_groups=-1), dict(n_groups=(1 << 20) + 1)):
        assert attend(lc, kv(lc), seqs(lc), prefixes(lc, **bad)) == EINVAL, bad
    assert attend(lc, kv(lc), seqs(lc), None) == EINVAL
    for bad in (dict(dtype=3), dict(rows=-1), dict(rows=1 << 31), dict(q_heads=0), dict(q_heads=5), dict(q_row=-1), dict(max_new=-1),
                dict(scale=math.inf), dict(scale=math.nan), dict(window=-1), dict(q=0), dict(q=FAKE + 1), dict(out=0),
                dict(out=FAKE + 1), dict(lse=FAKE + 2), dict(bytes=-1), dict(rows=1 << 30, q_heads=8)):
        assert attend(lc, kv(lc), seqs(lc), prefixes(lc), **bad) == EINVAL, bad
    assert attend(lc, kv(lc), seqs(lc), prefixes(lc), rows=0) == attend(lc, kv(lc), seqs(lc, n_seq=0), prefixes(lc)) == 0


def test_workspace_refuses(lc):
    f = lc.raw_library().lacache_kv_attend_shared_workspace
    for bad in ((2, 1, 1, 1, 4, 0), (1, -1, 1, 1, 4, 0), (1, 1, -1, 1, 4, 0), (1, 1, 1, -1, 4, 0), (1, 1, 1, 1, 3, 0),
                (1, 1, 1, 1, 4, -1), (1, 1, 1, (1 << 20) + 1, 4, 0)):
        assert f(ref(kv(lc)), *bad) == EINVAL, bad
