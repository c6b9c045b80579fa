"""Argument checks of the choice of pages at the C interface: refused before any device work (no GPU needed)."""
import ctypes
import math

import pytest
import torch

from tests import select_ref as sel
from tests.test_decode_abi import BAD_KV, BAD_SEQS, EINVAL, FAKE, kv, lc, ref, seqs  # noqa: F401


def bounds(lc, **kw):
    c = lc._Bounds(FAKE, FAKE)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def bound(lc, c, b, s, **kw):
    a = dict(rows=2, max_new=1, stream=None)
    a.update(kw)
    return lc.raw_library().lacache_kv_bound(ref(c), ref(b), ref(s), *a.values())


def select(lc, c, b, s, **kw):
    a = dict(q=FAKE, dtype=1, rows=2, q_heads=4, q_row=256, n=3, first=1, last=1, max_new=1, blocks=FAKE, workspace=FAKE,
             bytes=1 << 40, stream=None)
    a.update(kw)
    return lc.raw_library().lacache_kv_select(ref(c), ref(b), ref(s), *a.values())


def attend(lc, c, s, **kw):
    a = dict(q=FAKE, dtype=1, rows=2, q_heads=4, q_row=256, blocks=FAKE, n=3, scale=0.1, out=FAKE, lse=FAKE, workspace=FAKE,
             bytes=1 << 40, stream=None)
    a.update(kw)
    return lc.raw_library().lacache_kv_attend_blocks(ref(c), ref(s), *a.values())


BAD_BOUNDS = [dict(code=0), dict(scale=0), dict(code=FAKE + 8), dict(scale=FAKE + 2)]


def test_bound_refuses(lc):
    for bad in BAD_KV:
        assert bound(lc, kv(lc, **bad), bounds(lc), seqs(lc)) == EINVAL, bad
    for bad in [*BAD_SEQS, dict(n_seq=(1 << 20) + 1), dict(max_pages=(1 << 20) + 1)]:
        assert bound(lc, kv(lc), bounds(lc), seqs(lc, **bad)) == EINVAL, bad
    for bad in BAD_BOUNDS:
        assert bound(lc, kv(lc), bounds(lc, **bad), seqs(lc)) == EINVAL, bad
    for bad in (dict(rows=-1), dict(max_new=-1), dict(rows=1 << 31)):
        assert bound(lc, kv(lc), bounds(lc), seqs(lc), **bad) == EINVAL, bad
    assert bound(lc, None, bounds(lc), seqs(lc)) == bound(lc, kv(lc), None, seqs(lc)) == bound(lc, kv(lc), bounds(lc), None) == EINVAL
    assert bound(lc, kv(lc), bounds(lc), seqs(lc), rows=0) == bound(lc, kv(lc), bounds(lc), seqs(lc, n_seq=0)) == 0


def test_read_refuses(lc):
    def read(c, b, pages=FAKE, n=2, most=FAKE, least=FAKE):
        return lc.raw_library().lacache_kv_bounds_read(ref(c), ref(b), pages, n, most, least, None)
    for bad in BAD_BOUNDS:
        assert read(kv(lc), bounds(lc, **bad)) == EINVAL, bad
    for bad in (dict(pages=0), dict(pages=FAKE + 2), dict(n=-1), dict(most=FAKE + 1), dict(least=FAKE + 2), dict(n=1 << 31)):
        assert read(kv(lc), bounds(lc), **bad) == EINVAL, bad
    assert read(kv(lc, d=12), bounds(lc)) == read(None, bounds(lc)) == EINVAL
    assert read(kv(lc), bounds(lc), n=0, pages=0) == read(kv(lc), bounds(lc), most=0, least=0) == 0


def test_select_refuses(lc):
    for bad in (dict(dtype=2), dict(rows=-1), dict(q_heads=0), dict(q_heads=3), dict(q_heads=65536), dict(q_row=-1), dict(n=0),
                dict(n=(1 << 20) + 1), dict(first=-1), dict(last=-1), dict(first=2, last=2), dict(max_new=-1), dict(q=0),
                dict(q=FAKE + 1), dict(blocks=0), dict(blocks=FAKE + 2), dict(workspace=0), dict(workspace=FAKE + 4),
                dict(bytes=100), dict(bytes=-1), dict(first=2 ** 31 - 1, last=2 ** 31 - 1)):
        assert select(lc, kv(lc), bounds(lc), seqs(lc), **bad) == EINVAL, bad
    for bad in BAD_BOUNDS:
        assert select(lc, kv(lc), bounds(lc, **bad), seqs(lc)) == EINVAL, bad
    for bad in [*BAD_SEQS, dict(n_seq=(1 << 20) + 1), dict(max_pages=(1 << 20) + 1)]:
        assert select(lc, kv(lc), bounds(lc), seqs(lc, **bad)) == EINVAL, bad
    assert select(lc, kv(lc, page=16), bounds(lc), seqs(lc)) == EINVAL
    assert select(lc, kv(lc), bounds(lc), seqs(lc), rows=0) == 0


def test_attend_refuses(lc):
    for bad in BAD_KV:
        assert attend(lc, kv(lc, **bad), seqs(lc)) == EINVAL, bad
    for bad in [*BAD_SEQS, dict(n_seq=(1 << 20) + 1), dict(max_pages=(1 << 20) + 1)]:
        assert attend(lc, kv(lc), seqs(lc, **bad)) == EINVAL, bad
    for bad in (dict(dtype=3), dict(rows=-1), dict(rows=1 << 23), dict(q_heads=0), dict(q_heads=5), dict(q_row=-1), dict(n=0),
                dict(n=(1 << 20) + 1), dict(scale=math.inf), dict(scale=math.nan), dict(q=0), dict(q=FAKE + 1), dict(out=0),
                dict(out=FAKE + 1), dict(lse=FAKE + 2), dict(blocks=0), dict(blocks=FAKE + 1), dict(bytes=-1)):
        assert attend(lc, kv(lc), seqs(lc), **bad) == EINVAL, bad
    assert attend(lc, kv(lc), seqs(lc), rows=0) == attend(lc, kv(lc), seqs(lc, n_seq=0)) == 0


def test_workspaces(lc):
    f = lc.raw_library().lacache_kv_select_workspace
    assert f(ref(kv(lc)), 2, 3) == 4 * 2 * 2 * 64
    for bad in ((-1, 3), (2, -1), (2, (1 << 20) + 1), (1 << 31, 1)):
        assert f(ref(kv(lc)), *bad) == EINVAL
    g = lc.raw_library().lacache_kv_attend_blocks_workspace
    for bad in ((-1, 4, 1), (1, 3, 1), (1, 0, 1), (1, 4, 0), (1, 4, (1 << 20) + 1), (1 << 31, 4, 1)):
        assert g(ref(kv(lc)), *bad) == EINVAL


def test_reference_bounds_hold():
    """The reference's own: a bound is no less than any key, and a score no less than the products of rounded queries."""
    g = torch.Generator().manual_seed(0)
    keys, q = torch.randn((40, 24), generator=g).double(), torch.randn((1, 3, 24), generator=g)
    code, scale = sel.bounds(keys)
    hi, lo = code.double() * scale.double()
    assert bool((keys <= hi + 1e-6).all()) and bool((keys >= lo - 1e-6).all())
    s = sel.scores(q, code[None, None], scale.view(1, 1))
    unit = q.abs().amax(2) * torch.tensor(1 / 127)
    rounded = (q / unit[..., None]).round() * unit[..., None]
    assert float((rounded.double() @ keys.T).max()) <= float(s) * (1 + 1e-5)
    assert ctypes.sizeof(ctypes.c_void_p) == 8


def test_workspaces_beyond_64_bits(lc):
    """2^31 rows of 65,535 heads have 2^67 scores of 2^20 pages: refused, not some number of bytes."""
    f, c = lc.raw_library().lacache_kv_select_workspace, kv(lc, heads=65535)
    for rows in ((1 << 31) - 1, 1 << 30, 1 << 29, 1 << 25):
        want = 4 * rows * 65535 * (1 << 20)
        assert f(ref(c), rows, 1 << 20) == (want if want < 1 << 63 else EINVAL), rows
        if want >= 1 << 63:
            assert select(lc, c, bounds(lc), seqs(lc, max_pages=1 << 20), rows=rows, q_heads=65535, bytes=(1 << 63) - 1) == EINVAL
    assert f(ref(c), (1 << 31) - 1, 0) == 0
