"""GPU tests of the choice of pages and the attention over them: bounds and lists bit for bit, attention against float64."""
from __future__ import annotations

import math

import pytest
import torch

from tests import decode_exact as ex
from tests import decode_ref as ref
from tests import select_ref as sel
from tests.test_gpu_decode import DEV, DTYPES, KINDS, Paged, filled, lc, positions, same, say  # noqa: F401

pytestmark = pytest.mark.gpu


def normals(shape, seed, dtype=torch.float32, size=1.0):
    return torch.randn(shape, generator=torch.Generator(DEV).manual_seed(seed), device=DEV).mul_(size).to(dtype)


def stored(k, kind):
    """What is stored of float32 keys [T, heads, d], exactly, in float64."""
    code, scale = ref.coded(k.cpu(), kind)
    return code.double() if scale is None else code.double() * scale.double()[..., None]


# ---- bounds ------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("heads,d,page,news,lens", [
    (1, 8, 32, [1], [1]), (2, 64, 32, [1, 1, 1, 1], [1, 32, 33, 70]), (3, 80, 64, [5, 0, 31, 70], [5, 17, 90, 133]),
    (4, 96, 128, [21, 21, 1], [21, 150, 128]), (2, 256, 256, [300, 2], [300, 257]), (1, 192, 32, [64, 32, 33], [96, 64, 65]),
    (8, 128, 64, [1] * 9, [1, 2, 31, 32, 63, 64, 65, 127, 128]), (1, 136, 64, [130], [200])])
def test_bounds(lc, kind, heads, d, page, news, lens):
    """The pages of the newest tokens, whatever memory holds behind a sequence's end; no other page's bounds change."""
    say(f"[case] bounds {kind} {heads} {d} {page} {news} {lens}")
    pg = Paged(lc, kind, heads, d, page, len(news), max(1, -(-max(lens) // page)), seed=d)
    k = normals((sum(lens), heads, d), d + page, size=3)
    whole = pg.seqs(lens, lens)
    pg.cache.append(k, k, whole)
    held = stored(k, kind).split(lens)
    for max_new in (max(news), 0, 1):
        b = lc.KVBounds(pg.cache)
        b.code.fill_(77)
        b.scale.fill_(-5)
        b.update(pg.seqs(news, lens), sum(news), max_new=max_new)
        code, scale = b.code.cpu(), b.scale.cpu()
        touched = set()
        for s, (n, length) in enumerate(zip(news, lens)):
            for j in range((length - n) // page, -(-length // page) if n else 0):
                at = int(pg.table[s, j])
                touched.add(at)
                for h in range(heads):
                    want, size = sel.bounds(held[s][j * page:(j + 1) * page, h])
                    assert torch.equal(code[at, h, :, :d], want) and scale[at, h] == size, (s, j, h)
                    assert bool((code[at, h, :, d:] == 0).all())
        rest = [i for i in range(pg.cache.n_pages) if i not in touched]
        assert bool((code[rest] == 77).all()) and bool((scale[rest] == -5).all())
    pages = torch.tensor([*sorted(touched), -1, pg.cache.n_pages], dtype=torch.int32, device=DEV)
    most, least = (x.cpu() for x in b.read(pages))
    for i, at in enumerate(sorted(touched)):
        back = code[at, :, :, :d].float() * scale[at][:, None, None]
        assert torch.equal(most[i], back[:, 0]) and torch.equal(least[i], back[:, 1])
    assert bool((most[-2:] == 0).all()) and bool((least[-2:] == 0).all())
    # the bounds hold, to the rounding of their scale
    for s, (n, length) in enumerate(zip(news, lens)):
        for j in range((length - n) // page, -(-length // page) if n else 0):
            i, keys = sorted(touched).index(int(pg.table[s, j])), held[s][j * page:(j + 1) * page]
            assert bool((keys <= most[i].double() + 2.0 ** -23 * most[i].abs()).all())
            assert bool((keys >= least[i].double() - 2.0 ** -23 * least[i].abs()).all())


@pytest.mark.parametrize("kind", KINDS)
def test_bounds_of_tokens_written_again(lc, kind):
    """A rejected draft's key leaves the bounds when the next token of its position is written."""
    pg = Paged(lc, kind, 2, 64, 32, 1, 4)
    k = normals((50, 2, 64), 1)
    pg.cache.append(k, k, pg.seqs([50], [50]))
    b = lc.KVBounds(pg.cache)
    b.update(pg.seqs([50], [50]), 50)
    drafts = normals((5, 2, 64), 2, size=9)
    pg.cache.append(drafts, drafts, pg.seqs([5], [55]))
    b.update(pg.seqs([5], [55]), 5)
    wide = b.scale.clone()
    again = normals((1, 2, 64), 3)
    pg.cache.append(again, again, pg.seqs([1], [51]))
    b.update(pg.seqs([1], [51]), 1)
    held = stored(torch.cat((k, again)), kind)
    at = int(pg.table[0, 1])
    for h in range(2):
        want, size = sel.bounds(held[32:51, h])
        assert torch.equal(b.code[at, h].cpu(), want) and b.scale[at, h] == size and size < wide[at, h]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_bounds_of_what_is_no_number(lc, kind, bad):
    pg = Paged(lc, kind, 2, 64, 32, 2, 2)
    k = normals((70, 2, 64), 4)
    k[40, 1, 5] = bad
    k[:32, 0] = 0.0                                       # a page of zeros
    k[64:, 0] = 2.0 ** -110                               # a page of next to nothing
    pg.cache.append(k, k, pg.seqs([64, 6], [64, 6]))
    b = lc.KVBounds(pg.cache)
    b.update(pg.seqs([64, 6], [64, 6]), 70)
    p0, p1, p2 = (int(pg.table[i, j]) for i, j in ((0, 0), (0, 1), (1, 0)))
    assert bool(b.scale[p1, 1].isnan()) and bool((b.code[p1, 1] == 0).all())
    assert not bool(b.scale[p1, 0].isnan()) and b.scale[p0, 0] == 0 and b.scale[p2, 0] == 0
    assert bool((b.code[p0, 0] == 0).all()) and bool((b.code[p2, 0] == 0).all()) and b.scale[p0, 1] > 0


def test_bounds_of_positions_that_do_not_exist(lc):
    """Empty slots, rows before position 0, pages that are not there, positions beyond the table."""
    pg = Paged(lc, "bf16", 1, 64, 32, 4, 2)
    k = normals((256, 1, 64), 1)
    pg.cache.append(k, k, pg.seqs([64] * 4, [64] * 4))
    table = pg.table.clone()
    table[2, 0], table[2, 1] = -1, pg.cache.n_pages
    b = lc.KVBounds(pg.cache)
    b.update(pg.seqs([3, 5, 40, 100], [0, 2, 40, 130], table), 148)
    written = {int(i) for i in b.scale[:, 0].nonzero()[:, 0]}
    assert written == {int(table[1, 0]), int(table[3, 0]), int(table[3, 1])}


# ---- lists -------------------------------------------------------------------------------------------------


def random_bounds(lc, cache, seed, spread=1.0):
    g = torch.Generator().manual_seed(seed)
    code = torch.randint(-127, 128, (cache.n_pages, cache.heads, 2, lc._padded(cache.d)), generator=g, dtype=torch.int8)
    code = code.sort(2, descending=True).values
    code[..., cache.d:] = 0
    scale = torch.rand((cache.n_pages, cache.heads), generator=g) * spread + 0.1
    return lc.KVBounds(cache, code=code.to(DEV), scale=scale.to(DEV))


def check_lists(lc, b, q, news, lens, table, n, first=1, last=1, max_new=0, got=None):
    c = b.cache
    seqs = lc.Sequences(torch.tensor([0, *news]).cumsum(0).to(torch.int32).to(DEV),
                        torch.tensor(lens, dtype=torch.int32, device=DEV), table.contiguous().to(DEV))
    got = b.select(q, seqs, n, first=first, last=last, max_new=max_new) if got is None else got
    assert got.dtype == torch.int32 and got.shape == (q.shape[0], c.heads, n)
    got, qc = got.cpu(), q.cpu()
    code, scale = b.code.cpu()[..., :c.d], b.scale.cpu()
    t = 0
    for s, (m, length) in enumerate(zip(news, lens)):
        there = (table[s] >= 0) & (table[s] < c.n_pages)
        at = torch.where(there, table[s], 0).long()
        for i in range(m):
            p = length - m + i
            if p < 0:
                assert bool((got[t] == -1).all())
            else:
                score = sel.scores(qc[t].view(c.heads, -1, c.d), code[at], scale[at])
                for h in range(c.heads):
                    want = sel.chosen(score[h], there, p // c.page, n, first, last)
                    assert got[t, h].tolist() == want, (s, i, h)
            t += 1


LISTS = [  # heads, q_heads, d, page, new tokens, lengths, n, first, last
    (1, 1, 8, 32, [1], [1], 1, 0, 0),
    (2, 6, 64, 32, [1, 1, 1, 1], [1, 32, 1000, 64], 4, 1, 1),
    (8, 32, 128, 64, [1] * 5, [5000, 64, 65, 1, 2049], 16, 1, 1),
    (4, 28, 96, 32, [3, 3, 1], [900, 33, 128], 5, 2, 3),
    (1, 16, 256, 128, [2, 1], [6000, 513], 8, 0, 1),
    (1, 17, 192, 32, [1, 4], [900, 640], 7, 1, 0),
    (2, 80, 128, 32, [2, 1], [2000, 770], 9, 0, 0),
    (3, 3, 80, 64, [21, 0, 40], [3000, 500, 41], 12, 1, 2),
    (1, 2, 136, 256, [5], [9000], 3, 0, 3),
    (2, 2, 64, 32, [1], [2000], 62, 1, 1),
    (2, 2, 64, 32, [1], [2000], 200, 1, 1),
]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape", LISTS)
def test_lists(lc, dtype, shape):
    heads, Hq, d, page, news, lens, n, first, last = shape
    say(f"[case] lists {dtype} {shape}")
    pg = Paged(lc, "bf16", heads, d, page, len(lens), -(-max(lens) // page), seed=d)
    b = random_bounds(lc, pg.cache, seed=d + n)
    q = normals((sum(news), Hq, d), seed=n, dtype=dtype)
    for max_new in (max(news), 0, 1):
        check_lists(lc, b, q, news, lens, pg.table, n, first, last, max_new)


@pytest.mark.parametrize("pages,n", [(300, 20), (9000, 100), (9000, 8500)])
def test_lists_of_equal_pages(lc, pages, n):
    """Tables that hold the same pages again and again: most scores are equal, and the first ones are taken.  Also of more
    pages than LDS holds keys."""
    pg = Paged(lc, "bf16", 2, 64, 32, 1, 1, n_pages=7)
    b = random_bounds(lc, pg.cache, seed=3)
    g = torch.Generator().manual_seed(pages)
    table = torch.randint(-1, 8, (2, pages), generator=g).to(torch.int32)     # -1 and 7 are not there
    q = normals((3, 4, 64), seed=1)
    check_lists(lc, b, q, [2, 1], [pages * 32, pages * 32 - 1700], table, n)
    b.code.zero_()                                                            # all the same
    check_lists(lc, b, q, [2, 1], [pages * 32, pages * 32 - 1700], table, n)


def test_lists_of_what_is_no_number(lc):
    pg = Paged(lc, "bf16", 2, 64, 32, 1, 100)
    b = random_bounds(lc, pg.cache, seed=5)
    q = normals((4, 4, 64), seed=2)
    b.scale[pg.table[0, 40].item(), 0] = math.nan
    b.scale[pg.table[0, 41].item()] = math.nan
    b.scale[pg.table[0, 50].item()] = 3e38
    b.scale[pg.table[0, 51].item()] = 0
    q[1, 1, 3] = math.nan
    q[2, 0, 3] = math.inf
    q[3] = 0
    q[0, 3] *= 1e30
    check_lists(lc, b, q, [4], [3200], pg.table, 6)
    check_lists(lc, b, q.bfloat16(), [4], [3200], pg.table, 6)


def test_lists_beyond_tables_and_before_positions(lc):
    """Rows before position 0, lengths beyond the table, no tables, rows of no sequence."""
    pg = Paged(lc, "bf16", 2, 64, 32, 3, 10)
    b = random_bounds(lc, pg.cache, seed=5)
    q = normals((9, 4, 64), seed=2)
    check_lists(lc, b, q[:6], [3, 2, 1], [1, 700, 0], pg.table, 3, 1, 2)
    seqs = lc.Sequences(torch.tensor([2, 5, 6], dtype=torch.int32, device=DEV), torch.tensor([300, 9], dtype=torch.int32, device=DEV),
                        pg.table[:2].contiguous().to(DEV))
    out = torch.full((9, 2, 3), 7, dtype=torch.int32, device=DEV)
    got = b.select(q, seqs, 3, out=out)
    assert got is out and bool((out[[0, 1, 6, 7, 8]] == 7).all()) and not bool((out[2:6] == 7).all(2).any())
    none = b.select(q[:1], pg.seqs([1], [5], torch.zeros((1, 0), dtype=torch.int32)), 3)
    assert bool((none == -1).all())
    assert b.select(q[:0], pg.seqs([0], [5], pg.table[:1]), 3).shape == (0, 2, 3)


# ---- attention ---------------------------------------------------------------------------------------------


def check_blocks(lc, pg, held, q, news, lens, blocks, scale=None, table=None, out=None, gone=None):
    """One call against float64, within the bounds derived in decode_exact."""
    c, d = pg.cache, q.shape[2]
    scale_ = d ** -0.5 if scale is None else scale
    o, lse = c.attend_blocks(q, pg.seqs(news, lens, table), blocks, scale=scale) if out is None else out
    assert o.dtype == q.dtype and lse.dtype == torch.float32
    t, G, lists = 0, q.shape[1] // c.heads, blocks.tolist()
    for s, (n, length) in enumerate(zip(news, lens)):
        keys, vals = held[s]
        for i in range(n):
            p = length - n + i
            for h in range(c.heads):
                j = torch.arange(keys.shape[0], device=DEV)
                seen = torch.zeros(keys.shape[0], dtype=torch.bool, device=DEV)
                for x in lists[t][h]:
                    if x >= 0:
                        seen[x * c.page:(x + 1) * c.page] = True
                seen &= (j <= p) & (j < length)
                if gone is not None:
                    seen &= ~gone[s][:len(seen)]
                want = ref.attention(q[t:t + 1, h * G:(h + 1) * G].double(), keys[:, h:h + 1], vals[:, h:h + 1], seen[None], scale_)
                eo, el = ex.bounds(want, d, q.dtype == torch.float32)
                go, gl = o[t:t + 1, h * G:(h + 1) * G].double(), lse[t:t + 1, h * G:(h + 1) * G].double()
                empty = torch.isinf(want[1])
                assert torch.equal(torch.isinf(gl) & (gl < 0), empty) and bool((go[empty] == 0).all()), (s, i, h)
                assert bool(((go - want[0]).abs() <= eo).all()), (s, i, h, float(((go - want[0]).abs() / eo).max()))
                assert bool(((gl - want[1]).abs()[~empty] <= el[~empty]).all()), (s, i, h)
            t += 1


def random_lists(news, lens, heads, page, n, seed, most=None):
    g = torch.Generator().manual_seed(seed)
    out = torch.full((sum(news), heads, n), -1, dtype=torch.int32)
    t = 0
    for m, length in zip(news, lens):
        for i in range(m):
            count = max(0, (length - m + i) // page + 1)
            for h in range(heads):
                k = min(n, count, most or n)
                out[t, h, :k] = torch.randperm(max(count, 1), generator=g)[:k].to(torch.int32)
            t += 1
    return out.to(DEV)


BLOCKS = [  # heads, q_heads, d, page, new tokens, lengths, n
    (1, 1, 8, 32, [1], [1], 1),
    (2, 6, 64, 32, [1, 1, 1, 1, 1], [1, 31, 32, 33, 0], 2),
    (8, 32, 128, 64, [1, 1, 1], [700, 64, 65], 4),
    (2, 14, 80, 32, [1, 1], [257, 1000], 9),
    (1, 16, 256, 128, [1, 1], [127, 1500], 5),
    (1, 17, 96, 64, [1, 2], [300, 64], 3),
    (2, 80, 128, 64, [1, 1], [200, 770], 6),
    (3, 3, 192, 32, [5, 0, 3], [333, 9, 41], 4),
    (2, 8, 136, 256, [3], [2000], 7),
    (4, 4, 64, 32, [300], [900], 3),
    (1, 4, 128, 64, [1], [30_000], 300),
]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape", BLOCKS)
def test_attend_blocks(lc, kind, dtype, shape):
    heads, Hq, d, page, news, lens, n = shape
    say(f"[case] blocks {kind} {dtype} {shape}")
    pg, held = filled(lc, kind, heads, d, page, lens, seed=d + n)
    q = normals((sum(news), Hq, d), seed=n, dtype=dtype, size=2)
    check_blocks(lc, pg, held, q, news, lens, random_lists(news, lens, heads, page, n, seed=n))
    if sum(news) < 50:
        check_blocks(lc, pg, held, q, news, lens, random_lists(news, lens, heads, page, n, seed=n + 1, most=max(1, n // 3)),
                     scale=-0.3)


@pytest.mark.parametrize("kind", KINDS)
def test_attend_blocks_of_odd_lists(lc, kind):
    """Lists of nothing, of pages that are not there, that lie ahead, beyond the table; what a page listed twice does."""
    pg, held = filled(lc, kind, 2, 64, 32, [400, 100], seed=9)
    q = normals((3, 8, 64), seed=4, dtype=torch.bfloat16)
    blocks = torch.tensor([[[-1] * 4, [5, 4, -1, 0]], [[12, 13, 2 ** 30, -2 ** 31], [1, 13, 7, 2 ** 31 - 1]], [[3, 0, 2, 9], [9, -7, 1, 50]]],
                          dtype=torch.int32, device=DEV)
    table = pg.table.clone()
    table[0, 4], table[0, 7] = -1, pg.cache.n_pages
    gone = [torch.zeros(400, dtype=torch.bool, device=DEV), torch.zeros(100, dtype=torch.bool, device=DEV)]
    gone[0][128:160] = gone[0][224:256] = True
    keep = torch.where((blocks < 0) | (blocks > 12), -1, blocks)
    out = pg.cache.attend_blocks(q, pg.seqs([2, 1], [400, 100], table), blocks)
    check_blocks(lc, pg, held, q, [2, 1], [400, 100], keep, table=table, gone=gone, out=out)
    twice = torch.tensor([[[1, 1, 0, -1]] * 2], dtype=torch.int32, device=DEV)
    o, lse = pg.cache.attend_blocks(q[:1].float(), pg.seqs([1], [400], pg.table[:1]), twice)
    k2 = [torch.cat((x[:64], x[32:64])) for x in held[0]]
    want = ref.attention(q[:1].double(), *k2, torch.ones((1, 96), dtype=torch.bool, device=DEV), 0.125)
    eo, el = ex.bounds(want, 64, True)
    assert bool(((o.double() - want[0]).abs() <= eo).all()) and bool(((lse.double() - want[1]).abs() <= el).all())


@pytest.mark.parametrize("count", [127, 128, 300, 17_000])
def test_many_sequences(lc, count):
    """More sequences than are looked at together, slots without rows among them: each row finds its own."""
    lens, news = [20 + i % 41 for i in range(count)], [(i % 5 != 3) + (i % 97 == 5) for i in range(count)]
    news[-1] = 0
    pg = Paged(lc, "bf16", 1, 64, 32, count, 2, seed=count)
    whole = pg.seqs(lens, lens)
    k, v = (normals((sum(lens), 1, 64), i) for i in range(2))
    pg.cache.append(k, v, whole)
    held = list(zip(*(x.double().split(lens) for x in pg.cache.read(whole, sum(lens), dtype=torch.float32))))
    b = lc.KVBounds(pg.cache)
    b.update(whole, sum(lens))
    q = normals((sum(news), 2, 64), seed=6)
    seqs = pg.seqs(news, lens)
    lists = b.select(q, seqs, 2)
    last = torch.tensor([(n - m + i) // 32 for n, m in zip(lens, news) for i in range(m)])
    assert lists[:, 0, 0].cpu().eq(0).all() and lists[:, 0, 1].cpu().equal(torch.where(last > 0, last, -1).to(torch.int32))
    out = pg.cache.attend_blocks(q, seqs, lists)
    first = torch.tensor([0, *news]).cumsum(0)
    for a in {0, count // 2, max(0, count - 100)}:
        e = min(count, a + 100)
        at = slice(int(first[a]), int(first[e]))
        check_blocks(lc, pg, held[a:e], q[at], news[a:e], lens[a:e], lists[at], out=(out[0][at], out[1][at]))


@pytest.mark.parametrize("kind", ["bf16", "fp8"])
@pytest.mark.parametrize("dtype", DTYPES)
def test_attend_blocks_leaves_out_what_is_not_listed(lc, kind, dtype):
    """NaN and infinities in pages that are not listed, and behind a row in its own page, reach nothing; in a listed page
    they reach the rows that see them."""
    pg, held = filled(lc, kind, 1, 64, 32, [200], seed=2)
    bad = normals((1, 1, 64), 1)
    bad[0, 0, 7] = math.nan
    for at in (40, 198):                                   # page 1, and the newest page behind the first row
        pg.cache.append(bad, bad, pg.seqs([1], [at + 1]))
    q = normals((3, 4, 64), seed=3, dtype=dtype)           # positions 197, 198, 199
    lists = torch.tensor([[[0, 2, 6]], [[0, 2, -1]], [[0, 1, 2]]], dtype=torch.int32, device=DEV)
    o, lse = pg.cache.attend_blocks(q, pg.seqs([3], [200]), lists)
    check_blocks(lc, pg, held, q[:2], [2], [199], lists[:2], out=(o[:2], lse[:2]))
    assert bool(o[2].isnan().any())


def test_attend_blocks_of_strided_rows_and_rows_of_no_sequence(lc):
    pg, held = filled(lc, "bf16", 2, 64, 32, [300, 9], seed=2)
    wide = normals((9, 12, 64), seed=3, dtype=torch.bfloat16)
    lists = random_lists([3, 1], [300, 9], 2, 32, 4, seed=1)
    blocks = torch.full((9, 2, 4), 10 ** 6, dtype=torch.int32, device=DEV)
    blocks[2:6] = lists
    q = wide[:, 2:10]
    seqs = lc.Sequences(torch.tensor([2, 5, 6], dtype=torch.int32, device=DEV), torch.tensor([300, 9], dtype=torch.int32, device=DEV),
                        pg.table.to(DEV))
    out = (torch.full((9, 8, 64), 7.0, dtype=torch.bfloat16, device=DEV), torch.full((9, 8), 7.0, device=DEV))
    pg.cache.attend_blocks(q, seqs, blocks, out=out)
    outside = [0, 1, 6, 7, 8]
    assert bool((out[0][outside] == 7).all()) and bool((out[1][outside] == 7).all())
    check_blocks(lc, pg, held, q[2:6], [3, 1], [300, 9], lists, out=(out[0][2:6], out[1][2:6]))
    empty = pg.cache.attend_blocks(q[:0], pg.seqs([0, 0], [300, 9]), lists[:0])
    assert empty[0].shape == (0, 8, 64)


@pytest.mark.parametrize("kind", ["bf16", "int8"])
def test_chosen_pages_beyond_32_bits(lc, kind):
    n_pages, heads, d, page = 36_000, 8, 128, 128
    last = lambda t, each: (n_pages - 1 - torch.arange(each))[None].to(torch.int32)  # noqa: E731
    pg, held = filled(lc, kind, heads, d, page, [1000], seed=8, n_pages=n_pages, table=last)
    b = lc.KVBounds(pg.cache)
    b.update(pg.seqs([1000], [1000]), 1000)
    q = normals((2, 16, d), seed=1, dtype=torch.bfloat16)
    check_lists(lc, b, q, [2], [1000], pg.table, 3)
    blocks = b.select(q, pg.seqs([2], [1000]), 3)
    check_blocks(lc, pg, held, q, [2], [1000], blocks)


# ---- together ----------------------------------------------------------------------------------------------


@pytest.mark.parametrize("kind", KINDS)
def test_decoding_over_chosen_pages(lc, kind):
    """Steps of append, bounds, choice and attention: lists as defined, attention over them; with room for all pages it is
    that over everything."""
    heads, Hq, d, page, lens = 2, 8, 64, 32, [500, 40, 1]
    pg = Paged(lc, kind, heads, d, page, 3, 20, seed=6)
    k, v = (normals((sum(lens), heads, d), s) for s in (1, 2))
    pg.cache.append(k, v, pg.seqs(lens, lens))
    b = lc.KVBounds(pg.cache)
    b.update(pg.seqs(lens, lens), sum(lens), max_new=max(lens))
    for step in range(40):
        lens = [n + 1 for n in lens]
        seqs = pg.seqs([1, 1, 1], lens)
        k, v, q = (normals((3, h, d), 10 * step + i + 3) for i, h in enumerate((heads, heads, Hq)))
        pg.cache.append(k, v, seqs, max_new=1)
        b.update(seqs, 3, max_new=1)
        if step % 13 == 0 or step > 37:
            whole = pg.seqs(lens, lens)
            kb, vb = pg.cache.read(whole, sum(lens), dtype=torch.float32)
            held = list(zip(kb.double().split(lens), vb.double().split(lens)))
            check_lists(lc, b, q, [1, 1, 1], lens, pg.table, 4, max_new=1)
            check_blocks(lc, pg, held, q, [1, 1, 1], lens, b.select(q, seqs, 4, max_new=1))
            all_of = b.select(q, seqs, 20)
            check_blocks(lc, pg, held, q, [1, 1, 1], lens, all_of)
            assert all_of[0, 0, :lens[0] // page].tolist() == list(range(lens[0] // page))


def test_chosen_pages_on_another_stream_and_in_graphs(lc):
    """A step on a stream of its own; captured steps replayed with inputs and lengths that change, eager steps between; scratch
    shared with lacache_kv_attend; the same bits every time."""
    pg, held = filled(lc, "fp8", 2, 64, 32, [3000, 64, 1999], seed=30)
    b = lc.KVBounds(pg.cache)
    whole = pg.seqs([3000, 64, 1999], [3000, 64, 1999])
    b.update(whole, 5063)
    seqs = pg.seqs([1, 1, 1], [2900, 64, 1500])
    q = normals((3, 8, 64), 1, dtype=torch.bfloat16)
    outs = (torch.empty((3, 8, 64), device=DEV, dtype=torch.bfloat16), torch.empty((3, 8), device=DEV))

    def step(stream=None, outs=None):
        b.update(seqs, 3, max_new=1, stream=stream)
        blocks = b.select(q, seqs, 30, max_new=1, stream=stream)
        return *pg.cache.attend_blocks(q, seqs, blocks, out=outs, stream=stream), blocks

    want = step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = step(stream=side)
    side.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(want, got))
    full = pg.cache.attend(q, seqs, max_new=1)
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step(outs=outs)
        graphs.append(graph)
    for r in range(4):
        q.copy_(normals((3, 8, 64), 5 + r, dtype=torch.bfloat16))
        seqs.lens.copy_(torch.tensor([2901 + r, 64 - 31 * (r % 2), 700 * (r % 3) + 1], dtype=torch.int32))
        want, again = step(), step()
        full = [x.clone() for x in pg.cache.attend(q, seqs, max_new=1)]
        for graph in graphs:
            outs[0].fill_(5)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(outs[0], want[0]) and torch.equal(outs[1], want[1]), r
        assert all(torch.equal(x, y) for x, y in zip(want, again))
        assert all(torch.equal(x, y) for x, y in zip(full, pg.cache.attend(q, seqs, max_new=1)))


def test_calls_that_are_refused(lc):
    pg = Paged(lc, "bf16", 2, 64, 32, 2, 2)
    b = lc.KVBounds(pg.cache)
    q, seqs = torch.zeros((2, 4, 64), device=DEV), pg.seqs([1, 1], [5, 6])
    blocks = torch.zeros((2, 2, 3), dtype=torch.int32, device=DEV)
    for f in (lambda: lc.KVBounds(pg.cache, code=b.code[:1]), lambda: lc.KVBounds(pg.cache, scale=b.scale.double()),
              lambda: lc.KVBounds(pg.cache, code=b.code.cpu()), lambda: b.update(seqs, -1), lambda: b.update(seqs, 2, max_new=-1),
              lambda: b.read(torch.zeros(3, device=DEV)), lambda: b.read(torch.zeros((1, 3), dtype=torch.int32, device=DEV)),
              lambda: b.read(torch.zeros(3, dtype=torch.int32)), lambda: b.select(q.half(), seqs, 3),
              lambda: b.select(q[:, :3], seqs, 3), lambda: b.select(q, seqs, 0), lambda: b.select(q, seqs, 3, first=2, last=2),
              lambda: b.select(q, seqs, 3, first=-1), lambda: b.select(q[..., :32], seqs, 3), lambda: b.select(q.cpu(), seqs, 3),
              lambda: b.select(q, seqs, 3, out=blocks[:1]), lambda: pg.cache.attend_blocks(q, seqs, blocks.long()),
              lambda: pg.cache.attend_blocks(q, seqs, blocks[:1]), lambda: pg.cache.attend_blocks(q, seqs, blocks[..., :0]),
              lambda: pg.cache.attend_blocks(q, seqs, blocks[..., :2]), lambda: pg.cache.attend_blocks(q[:, :3], seqs, blocks),
              lambda: pg.cache.attend_blocks(q, seqs, blocks, scale=math.nan), lambda: pg.cache.attend_blocks(q.half(), seqs, blocks),
              lambda: pg.cache.attend_blocks(q.clone().requires_grad_(), seqs, blocks)):
        with pytest.raises((ValueError, lc.LaCacheError)):
            f()
    with torch.no_grad():
        pg.cache.attend_blocks(q.clone().requires_grad_(), seqs, blocks)
