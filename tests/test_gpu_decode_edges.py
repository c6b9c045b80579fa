"""GPU tests of the decode operators' edges on every attention kernel: calls that bound their new tokens take the kernels of
up to 32 rows, calls that do not take the wide ones.  Results are held to bounds that charge each rounding what it is."""
from __future__ import annotations

import ctypes
import math

import pytest
import torch

from tests import decode_exact as ex
from tests import decode_ref as ref
from tests.test_gpu_decode import DEV, DTYPES, KINDS, Paged, check_attend, filled, lc, positions, same, say  # noqa: F401

pytestmark = pytest.mark.gpu

# new tokens, heads, query heads, d: the rows of a kv head, and so the kernel, go from 2 to 168
ROWS = [(1, 2, 4, 64), (2, 2, 8, 128), (3, 2, 16, 64), (7, 2, 16, 128), (21, 2, 16, 64), (21, 1, 8, 256), (30, 2, 4, 192)]


@pytest.fixture(autouse=True)
def tight(monkeypatch):
    monkeypatch.setattr(ref, "bounds", ex.bounds)


def queries(rows, Hq, d, dtype, seed=1, size=2):
    g = torch.Generator(DEV).manual_seed(seed)
    return torch.randn((rows, Hq, d), generator=g, device=DEV).mul_(size).to(dtype)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape", [*ROWS, (5, 2, 8, 96), (13, 2, 8, 128), (40, 2, 4, 192), (60, 2, 8, 256)])
@pytest.mark.parametrize("length", [700, 6000])
def test_weights_keep_their_bits(lc, kind, dtype, shape, length):
    """Values whose weighted sum cancels: what is left shows the roundings of the weights (16 bits, 24 with float32 rows)."""
    new, heads, Hq, d = shape
    if new * (Hq // heads) > d:
        new = d // (Hq // heads)
    say(f"[case] bits {kind} {dtype} {shape} {length}")
    g = torch.Generator(DEV).manual_seed(d + new)
    pg = Paged(lc, kind, heads, d, 32, 1, -(-length // 32), seed=d)
    whole = pg.seqs([length], [length])
    k = torch.randn((length, heads, d), generator=g, device=DEV)
    pg.cache.append(k, torch.zeros_like(k), whole)
    keys = pg.cache.read(whole, length, dtype=torch.float32)[0].double()
    q = ex.sparse_queries(new, Hq, d, seed=new)
    v = ex.cancelling_values(q.double(), keys.cpu(), length - new).float().to(DEV)
    pg.cache.append(k, v, whole)
    vals = pg.cache.read(whole, length, dtype=torch.float32)[1].double()
    q = q.to(dtype).to(DEV)
    seen = torch.arange(length, device=DEV)[None] <= torch.arange(length - new, length, device=DEV)[:, None]
    want = ref.attention(q.double(), keys, vals, seen, 1.0)
    b = ex.sparse_bounds(want, dtype == torch.float32)
    for max_new in (new, 0):
        o, _ = pg.cache.attend(q, pg.seqs([new], [length]), scale=1.0, max_new=max_new)
        worst = float(((o.double() - want[0]).abs() / b).max())
        say(f"[ok] {worst:.3f} of the bound")
        assert worst <= 1


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape", ROWS)
@pytest.mark.parametrize("longest", [1000, 5000])
def test_pages_that_are_not_there(lc, kind, dtype, shape, longest):
    """Pages given back, sequences without any, lengths beyond the page table; with windows; bounded calls and others."""
    new, heads, Hq, d = shape
    lens = [longest, 130, 64, 96]
    news = [new, 1, min(new, 64), 1]
    say(f"[case] pages {kind} {dtype} {shape} {longest}")
    pg, held = filled(lc, kind, heads, d, 32, lens, seed=13)
    table = pg.table.clone()
    table[0, :20] = -1
    table[0, 25] = pg.cache.n_pages
    table[1, 4] = -7
    table[2, :] = -1
    gone = [torch.zeros(n, dtype=torch.bool, device=DEV) for n in lens]
    gone[0][:640] = gone[0][800:832] = True
    gone[1][128:] = True
    gone[2][:] = True
    q = queries(sum(news), Hq, d, dtype)
    for max_new in (max(news), 0):
        for window in (0, 1, 33, 70, 400):
            check_attend(lc, pg, held, q, news, lens, table=table, gone=gone, window=window, max_new=max_new)
    cut = table[:, :3]
    gone = [torch.arange(n, device=DEV) >= 96 for n in lens]
    gone[0][:] = True
    gone[2][:] = True
    for max_new in (max(news), 0):
        check_attend(lc, pg, held, q, news, lens, table=cut, gone=gone, max_new=max_new)
        check_attend(lc, pg, held, q, news, lens, table=cut, gone=gone, max_new=max_new, window=50)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape", ROWS)
def test_scales_and_rows_before_the_first_position(lc, kind, dtype, shape):
    """Scores of hundreds, of zero, of either sign; more rows than a sequence has tokens, and a length below zero."""
    new, heads, Hq, d = shape
    say(f"[case] scales {kind} {dtype} {shape}")
    lens, news = [700, 65], [new, max(1, new - 1)]
    pg, held = filled(lc, kind, heads, d, 32, lens, seed=11, spread=4.0)
    q = queries(sum(news), Hq, d, dtype, seed=4, size=30)
    for scale in (1.0, 1e-3, 0.0, -0.125):
        check_attend(lc, pg, held, q, news, lens, scale=scale, max_new=new)
    lens, news = [max(1, new // 2), 40], [new, new]
    pg, held = filled(lc, kind, heads, d, 32, lens, seed=2)
    q = queries(sum(news), Hq, d, dtype)
    check_attend(lc, pg, held, q, news, lens, max_new=new)
    check_attend(lc, pg, [held[0], (held[1][0][:0], held[1][1][:0])], q, news, [lens[0], -3], max_new=new)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("shape", ROWS)
def test_strided_rows_and_repeats(lc, kind, shape):
    """Rows that start off a 16-byte boundary; the same call gives the same bits, with and without the sums' logarithms."""
    new, heads, Hq, d = shape
    say(f"[case] strided {kind} {shape}")
    lens, news = [900, 40], [new, min(new, 40)]
    pg, held = filled(lc, kind, heads, d, 64, lens, seed=6)
    for dtype in DTYPES:
        wide = torch.randn((sum(news), Hq * d + 24), device=DEV).to(dtype)
        for shift in (0, 8, 3):
            q = wide[:, shift:shift + Hq * d].unflatten(1, (Hq, d))
            check_attend(lc, pg, held, q, news, lens, max_new=new)
        q, seqs = wide[:, 8:8 + Hq * d].unflatten(1, (Hq, d)), pg.seqs(news, lens)
        first = pg.cache.attend(q, seqs, max_new=new)
        for _ in range(5):
            again = pg.cache.attend(q, seqs, max_new=new)
            assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])
        alone = torch.empty_like(first[0])
        code = lc.raw_library().lacache_kv_attend(
            pg.cache._ref, seqs._ref, q.data_ptr(), lc.F32 if dtype == torch.float32 else lc.BF16, q.shape[0], Hq, q.stride(0),
            new, d ** -0.5, 0, alone.data_ptr(), None, pg.cache._space.data_ptr(), pg.cache._space.numel(),
            ctypes.c_void_p(torch.cuda.current_stream().cuda_stream))
        assert code == lc.OK and torch.equal(alone, first[0])


@pytest.mark.parametrize("kind", ["bf16", "int8"])
@pytest.mark.parametrize("new", [1, 9])
def test_offsets_beyond_32_bits(lc, kind, new):
    """Pools of more than 2^32 elements, the sequence's pages at their end."""
    n_pages, heads, d, page = 36_000, 8, 128, 128
    last = lambda t, each: (n_pages - 1 - torch.arange(each))[None].to(torch.int32)  # noqa: E731
    pg, held = filled(lc, kind, heads, d, page, [1000], seed=8, n_pages=n_pages, table=last)
    check_attend(lc, pg, held, queries(new, 16, d, torch.bfloat16), [new], [1000], max_new=new)


@pytest.mark.parametrize("kind,dtype,new,Hq", [("fp8", torch.bfloat16, 1, 16), ("bf16", torch.bfloat16, 6, 64),
                                               ("int8", torch.float32, 2, 32), ("fp8", torch.bfloat16, 20, 32),
                                               ("bf16", torch.float32, 20, 16)])
def test_ranges_of_hundreds_of_tiles(lc, kind, dtype, new, Hq):
    """Ranges that are longer than the tiles whose pages a wave looks up together (256, or 64 in the wide kernels), whole
    stretches of them without pages.  The sequences share their pages, read alone."""
    n, length, heads, d = 64, 16_384, 16, 64
    say(f"[case] ranges {kind} {dtype} new={new} Hq={Hq}")
    pg, held = filled(lc, kind, heads, d, 32, [length], seed=3)
    table = pg.table.repeat(n, 1)
    lens = [length - 37 * (b % 5) - b for b in range(n)]
    gone = torch.zeros((n, length), dtype=torch.bool, device=DEV)
    for b in range(n):
        for lo, hi in ([], [(0, 300)], [(100, 420)], [(0, 511)])[b % 4]:
            table[b, lo:hi] = -1
            gone[b, 32 * lo:32 * hi] = True
    news = [new] * n
    q = queries(n * new, Hq, d, dtype)
    for window in (0, 9001):
        got = pg.cache.attend(q, pg.seqs(news, lens, table), max_new=new, window=window)
        for b in (0, 1, 2, 3, 30, 61, 62, 63):
            part = slice(b * new, (b + 1) * new)
            check_attend(lc, pg, held, q[part], [new], lens[b:b + 1], gone=[gone[b, :lens[b]]], window=window,
                         out=(got[0][part], got[1][part]))


@pytest.mark.parametrize("kind,dtype,n,new,heads,Hq,d", [
    ("bf16", torch.bfloat16, 700, 1, 1, 2, 64), ("int8", torch.float32, 1100, 1, 1, 2, 64), ("fp8", torch.bfloat16, 1100, 3, 1, 8, 64),
    ("bf16", torch.bfloat16, 1100, 7, 1, 8, 128), ("int8", torch.float32, 600, 9, 1, 4, 96), ("bf16", torch.bfloat16, 1100, 21, 1, 8, 256),
    ("fp8", torch.bfloat16, 600, 21, 1, 8, 128)])
def test_more_sequences_than_threads(lc, kind, dtype, n, new, heads, Hq, d):
    """Ragged sequences, more than a workgroup has threads, many without rows or tokens."""
    say(f"[case] sequences {kind} {dtype} {n} new={new} d={d}")
    lens = [i * 7 % 70 for i in range(n)]
    lens[n - 3], lens[300] = 900, 2000
    news = [0 if i % 5 == 0 and i != 300 else max(1, min(new, x)) for i, x in enumerate(lens)]
    pg, held = filled(lc, kind, heads, d, 32, [min(x, 96) for x in lens], seed=5)
    # the two long ones again and again over their first pages (shared, read alone)
    table = torch.full((n, 63), -1, dtype=torch.int32)
    table[:, :pg.table.shape[1]] = pg.table
    for b in (n - 3, 300):
        table[b] = pg.table[b, torch.arange(63) % 3]
        at = torch.arange(lens[b], device=DEV) % 96
        held[b] = tuple(x[at] for x in held[b])
    q = queries(sum(news), Hq, d, dtype)
    check_attend(lc, pg, held, q, news, lens, table=table, max_new=new)
    check_attend(lc, pg, held, q, news, lens, table=table, max_new=new, window=40)
    if n == 700:  # a page table of three pages: parts are joined in the launch
        short = [min(x, 96) for x in lens]
        held = [tuple(x[:m] for x in h) for h, m in zip(held, short)]
        check_attend(lc, pg, held, q, news, short, max_new=new)


@pytest.mark.parametrize("heads", [8, 64])
@pytest.mark.parametrize("dtype,new,group", [(torch.bfloat16, 1, 2), (torch.bfloat16, 3, 8), (torch.bfloat16, 21, 4), (torch.float32, 9, 4)])
def test_page_tables_of_millions_of_pages(lc, heads, dtype, new, group):
    """The pieces of work are counted in 32 bits: with page tables this long a piece is 16 to 128 tiles."""
    say(f"[case] long tables heads={heads} {dtype} new={new}")
    d, lens, news = 64, [5000, 70], [new, 1]
    pg, held = filled(lc, "bf16", heads, d, 256, lens, seed=17)
    table = torch.full((2, 1 << 26), -1, dtype=torch.int32, device=DEV)
    table[:, :pg.table.shape[1]] = pg.table.to(DEV)
    q = queries(sum(news), heads * group, d, dtype)
    for window in (0, 100, 3000):
        check_attend(lc, pg, held, q, news, lens, table=table, max_new=new, window=window)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("max_new", [0, 3000])
def test_append_and_read_of_a_prompt_among_single_tokens(lc, kind, dtype, max_new):
    """One launch for sequences of very different numbers of new tokens."""
    say(f"[case] mixed append {kind} {dtype} {max_new}")
    news = [1] * 120 + [3000] + [1, 0, 2] * 40
    lens = [n + 13 * i % 90 for i, n in enumerate(news)]
    heads, Hq, d, page = 2, 4, 64, 64
    table = torch.full((len(news), 50), -1, dtype=torch.int32)
    used, free = [-(-n // page) for n in lens], 0
    pg = Paged(lc, kind, heads, d, page, 1, 1, n_pages=sum(used))
    order = torch.randperm(sum(used), generator=torch.Generator().manual_seed(1)).to(torch.int32)
    for b, m in enumerate(used):
        table[b, :m] = order[free:free + m]
        free += m
    g = torch.Generator().manual_seed(2)
    T = sum(news)
    q, k, v = (torch.randn((T, h, d), generator=g).to(dtype) for h in (Hq, heads, heads))
    rows = ref.table64(max(lens), d).float()
    seqs = pg.seqs(news, lens, table)
    turned = pg.cache.append(k.to(DEV), v.to(DEV), seqs, q=q.to(DEV), rope=lc.Rope(rows.to(DEV)), max_new=max_new)
    at = rows[positions(news, lens)]
    assert same(turned, ref.turned(q, at, False).to(dtype))
    kb, vb = pg.cache.read(seqs, T, dtype=torch.float32, max_new=max_new)
    assert same(kb, ref.values(*ref.coded(ref.turned(k, at, False), kind)))
    assert same(vb, ref.values(*ref.coded(v.float(), kind)))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape", ROWS)
def test_keys_that_are_infinite(lc, dtype, shape):
    """A score of -infinity is the weight 0 (with float32 rows, whose queries are sums of terms, it may be a NaN too), one of
    +infinity makes the row NaN.  Rows that do not see the key are as if it were not there."""
    new, heads, Hq, d = shape
    say(f"[case] infinite keys {dtype} {shape}")
    length, at = 300, 300 - 1 - new // 2
    pg, held = filled(lc, "bf16", heads, d, 32, [length], seed=9)
    q = queries(new, Hq, d, dtype)
    q[..., 3] = q[..., 3].abs() + 1
    j, p = torch.arange(length, device=DEV)[None], torch.arange(length - new, length, device=DEV)[:, None]
    for bad in (-math.inf, math.inf):
        k, v = (x.float().clone() for x in held[0])
        k[at, :, 3] = bad
        pg.cache.append(k, v, pg.seqs([length], [length]))
        o, lse = pg.cache.attend(q, pg.seqs([new], [length]), max_new=new)
        without = (j <= p) & (j != at)
        want = ref.attention(q.double(), *held[0], without, d ** -0.5)
        eo, el = ex.bounds(want, d, dtype == torch.float32)
        near = ((o.double() - want[0]).abs() <= eo).all(2) & ((lse.double() - want[1]).abs() <= el)
        nan = o.isnan().all(2) & lse.isnan()
        sees = (p[:, 0] >= at)[:, None].expand_as(near)
        assert bool(near[~sees].all())
        if bad > 0:
            assert bool(nan[sees].all())
        else:
            assert bool((near | nan if dtype == torch.float32 else near)[sees].all())


def test_rows_whose_every_score_is_minus_infinity(lc):
    """They are as rows that see nothing."""
    pg, held = filled(lc, "bf16", 2, 64, 32, [70, 5000], seed=9)
    k, v = (torch.cat([h[i] for h in held]).float() for i in (0, 1))
    k[:, 0, 3] = -math.inf
    pg.cache.append(k, v, pg.seqs([70, 5000], [70, 5000]))
    for new in (1, 21):
        q = queries(2 * new, 4, 64, torch.bfloat16)
        q[..., 3] = q[..., 3].abs() + 1
        o, lse = pg.cache.attend(q, pg.seqs([new, new], [70, 5000]), max_new=new)
        assert bool((o[:, :2] == 0).all()) and bool((lse[:, :2] == -math.inf).all())
        assert bool(o[:, 2:].isfinite().all()) and bool(lse[:, 2:].isfinite().all())
