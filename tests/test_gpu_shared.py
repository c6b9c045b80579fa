"""GPU tests of attention over shared prefixes: against float64, and against the attention that reads each table whole."""
from __future__ import annotations

import math

import pytest
import torch

from tests import decode_exact as ex
from tests import decode_ref as ref
from tests.test_gpu_decode import DEV, DTYPES, KINDS, Paged, check_attend, lc, say  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def tight(monkeypatch):
    monkeypatch.setattr(ref, "bounds", ex.bounds)


def normals(shape, seed, dtype=torch.float32, size=1.0):
    return torch.randn(shape, generator=torch.Generator(DEV).manual_seed(seed), device=DEV).mul_(size).to(dtype)


def shared(lc, kind, heads, d, page, lens, groups, seed, n_pages=None):
    """A cache whose sequences share pages by `groups` (first sequence, end, shared tokens), and what each sequence holds."""
    each = max(1, -(-max([1, *lens, *(n for *_, n in groups)]) // page))
    pg = Paged(lc, kind, heads, d, page, len(lens), each, seed=seed, n_pages=n_pages)
    for a, b, n in groups:
        pg.table[a:b, :n // page] = pg.table[a, :n // page].clone()
    # the longest of a group writes the prefix, the others their own tokens behind it
    whole = [max(0, x) for x in lens]
    k, v = (normals((sum(whole), heads, d), seed + i) for i in range(2))
    k, v = list(k.split(whole)), list(v.split(whole))
    for a, b, n in groups:
        front = n // page * page
        long = max(range(a, b), key=lambda i: whole[i]) if b > a else a
        for i in range(a, b):
            k[i][:front] = k[long][:min(front, whole[i])]
            v[i][:front] = v[long][:min(front, whole[i])]
    seqs = pg.seqs(whole, whole)
    pg.cache.append(torch.cat(k), torch.cat(v), seqs)
    kb, vb = pg.cache.read(seqs, sum(whole), dtype=torch.float32)
    return pg, list(zip(kb.double().split(whole), vb.double().split(whole)))


def prefixes(lc, groups, last=None):
    """The groups as the call takes them; sequences between two groups are groups that share nothing."""
    bounds, lens, at = [groups[0][0] if groups else 0], [], groups[0][0] if groups else 0
    for a, b, n in groups:
        if a > at:
            bounds.append(a)
            lens.append(0)
        bounds.append(b)
        lens.append(n)
        at = b
    return lc.Prefixes(torch.tensor(bounds, dtype=torch.int32, device=DEV), torch.tensor(lens, dtype=torch.int32, device=DEV))


def check(lc, pg, held, q, news, lens, groups, window=0, scale=None, max_new=0, gone=None, table=None):
    p = prefixes(lc, groups)
    out = pg.cache.attend_shared(q, pg.seqs(news, lens, table), p, scale=scale, window=window, max_new=max_new)
    return check_attend(lc, pg, held, q, news, lens, window=window, scale=scale, out=out, gone=gone)


SHARED = [  # heads, q_heads, d, page, new tokens, lengths, groups
    (1, 1, 8, 32, [1, 1], [33, 40], [(0, 2, 32)]),
    (2, 6, 64, 32, [1, 1, 1], [70, 65, 100], [(0, 3, 64)]),
    (8, 32, 128, 64, [1] * 6, [700, 650, 641, 900, 64, 0], [(0, 4, 640)]),
    (2, 14, 80, 32, [1, 1, 1, 1], [257, 1000, 300, 260], [(0, 2, 250), (2, 4, 256)]),
    (1, 16, 256, 128, [1, 1, 2], [527, 513, 600], [(0, 3, 512)]),
    (1, 17, 96, 64, [1, 1, 1], [300, 264, 20], [(0, 2, 260)]),
    (2, 64, 128, 64, [1, 1, 1], [200, 177, 500], [(1, 3, 130)]),
    (4, 12, 96, 64, [21, 3, 0, 21], [221, 400, 250, 231], [(0, 4, 192)]),
    (4, 32, 128, 64, [21, 21, 5], [500, 464, 470], [(0, 3, 448)]),
    (2, 16, 256, 32, [40, 9], [333, 341], [(0, 2, 300)]),
    (1, 2, 192, 32, [151, 3], [600, 500], [(0, 2, 320)]),
    (3, 3, 40, 64, [33, 1, 2], [133, 101, 90], [(0, 2, 64)]),
    (2, 8, 64, 32, [1] * 40, [200 + 7 * i for i in range(40)], [(0, 17, 160), (17, 18, 320), (20, 40, 192)]),
    (1, 4, 64, 32, [1] * 3, [5000, 4900, 4870], [(0, 3, 4864)]),
    (2, 2, 64, 32, [1] * 300, [100 + i % 50 for i in range(300)], [(0, 300, 96)]),
]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape", SHARED)
def test_shared(lc, kind, dtype, shape):
    heads, Hq, d, page, news, lens, groups = shape
    say(f"[case] shared {kind} {dtype} {shape[:6]}")
    pg, held = shared(lc, kind, heads, d, page, lens, groups, seed=d + len(lens))
    q = normals((sum(news), Hq, d), seed=d, dtype=dtype, size=2)
    for max_new in (max(news), 0):
        check(lc, pg, held, q, news, lens, groups, max_new=max_new)
    check(lc, pg, held, q, news, lens, groups, window=100, max_new=max(news))
    check(lc, pg, held, q, news, lens, groups, window=33, scale=-0.2)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", DTYPES)
def test_shared_rows_within_the_prefix(lc, kind, dtype):
    """Sequences that are shorter than what they share, rows in it, before position 0, and of empty slots."""
    lens, news = [200, 150, 40, 0, 3, 97], [1, 40, 9, 2, 7, 2]
    groups = [(0, 6, 96)]
    pg, held = shared(lc, kind, 2, 64, 32, lens, groups, seed=3)
    q = normals((sum(news), 8, 64), seed=5, dtype=dtype)
    for window in (0, 50, 1):
        check(lc, pg, held, q, news, lens, groups, window=window, max_new=40)
        check(lc, pg, held, q, news, lens, groups, window=window)


@pytest.mark.parametrize("new,Hq", [(1, 4), (3, 32), (30, 4)])
def test_groups_of_every_kind(lc, new, Hq):
    """No groups, empty ones, groups of one, of nothing, overlapping ends, counts beyond the table and out of range."""
    lens = [300, 290, 310, 400, 333]
    pg, held = shared(lc, "bf16", 2, 64, 32, lens, [(0, 3, 256), (3, 5, 320)], seed=4)
    q = normals((5 * new, Hq, 64), seed=6, dtype=torch.bfloat16)
    news = [new] * 5
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    for group, n in ((i32(0), i32()), (i32(0, 0, 3, 3, 5, 5), i32(64, 256, 99, 320, 1)), (i32(0, 1, 3, 4, 5), i32(9, 256, 64, 320)),
                     (i32(3, 5), i32(320)), (i32(0, 3, 5), i32(0, 0)), (i32(0, 3, 5), i32(-5, 31)), (i32(0, 3, 9), i32(255, 320)),
                     (i32(-4, 3, 2 ** 31 - 1), i32(256, 320)), (i32(5, 5), i32(64)), (i32(2, 3, 5), i32(2 ** 31 - 1, 63))):
        out = pg.cache.attend_shared(q, pg.seqs(news, lens), lc.Prefixes(group, n), max_new=new)
        check_attend(lc, pg, held, q, news, lens, out=out)
    # a group that shares its whole table
    for i in (0, 1):
        pg.table[1] = pg.table[0]
    same = [held[0], held[0]]
    p = lc.Prefixes(i32(0, 2), i32(2 ** 31 - 1))
    out = pg.cache.attend_shared(q[:2 * new], pg.seqs([new] * 2, [300, 299], pg.table[:2]), p)
    check_attend(lc, pg, same, q[:2 * new], [new] * 2, [300, 299], out=out)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("count,prefix,own", [(64, 16_384, (3, 40)), (64, 1024, (1100, 1500)), (4, 65_536, (1, 30)), (4, 64, (9000, 9500)),
                                              (40, 6400, (1, 3))])
def test_parts_of_unequal_work(lc, dtype, count, prefix, own):
    """Much more over the prefix than over the sequences' own tokens, or much less."""
    lens = [prefix + own[0] + i * (own[1] - own[0]) // (count - 1) for i in range(count)]
    pg, held = shared(lc, "fp8", 8, 64, 64, lens, [(0, count, prefix)], seed=count)
    q = normals((count, 32, 64), seed=6, dtype=dtype)
    check(lc, pg, held, q, [1] * count, lens, [(0, count, prefix)], max_new=1)
    check(lc, pg, held, q, [1] * count, lens, [(0, count, prefix)], max_new=1, window=700)


@pytest.mark.parametrize("count,each", [(390, 3), (260, 2), (900, 1), (17_000, 100)])
def test_many_groups(lc, count, each):
    """More groups and sequences than are looked at together, empty groups and slots without rows among them."""
    lens = [70 + i % 40 for i in range(count)]
    news = [i % 5 != 3 for i in range(count)]
    groups = [(i, min(i + each, count), 64) for i in range(0, count, each) if i % 7]
    pg, held = shared(lc, "bf16", 1, 64, 32, lens, groups, seed=each)
    q = normals((sum(news), 2, 64), seed=6, dtype=torch.bfloat16)
    p = prefixes(lc, groups)
    seqs = pg.seqs(news, lens)
    out = pg.cache.attend_shared(q, seqs, p, max_new=1)
    first = torch.tensor([0, *news]).cumsum(0)
    for a in {0, count // 2, max(0, count - 200)}:          # 200 sequences at a time
        b = min(count, a + 200)
        at = slice(int(first[a]), int(first[b]))
        check_attend(lc, pg, held[a:b], q[at], news[a:b], lens[a:b], out=(out[0][at], out[1][at]))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("new,Hq", [(1, 4), (1, 32), (21, 16)])
def test_shared_pages_that_are_not_there(lc, kind, new, Hq):
    lens = [400, 380, 500]
    pg, held = shared(lc, kind, 2, 64, 32, lens, [(0, 3, 320)], seed=14)
    table = pg.table.clone()
    table[:, 2], table[:, 5] = -1, pg.cache.n_pages
    table[1, 11] = -3
    gone = [torch.zeros(n, dtype=torch.bool, device=DEV) for n in lens]
    for g in gone:
        g[64:96] = g[160:192] = True
    gone[1][352:384] = True
    q = normals((3 * new, Hq, 64), seed=6, dtype=torch.bfloat16)
    out = pg.cache.attend_shared(q, pg.seqs([new] * 3, lens, table), prefixes(lc, [(0, 3, 320)]), max_new=new)
    check_attend(lc, pg, held, q, [new] * 3, lens, out=out, gone=gone)
    table[:, :10] = -1                                     # all of the prefix
    for g in gone:
        g[:320] = True
    out = pg.cache.attend_shared(q, pg.seqs([new] * 3, lens, table), prefixes(lc, [(0, 3, 320)]), max_new=new)
    check_attend(lc, pg, held, q, [new] * 3, lens, out=out, gone=gone)


@pytest.mark.parametrize("kind", ["bf16", "fp8"])
@pytest.mark.parametrize("new,Hq", [(1, 4), (9, 8), (40, 8)])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_values_that_are_no_numbers(lc, kind, new, Hq, bad):
    """In the prefix they reach the rows that see them (a window hides them from some), as without sharing."""
    lens = [170, 130 + new, 300]
    pg, _ = shared(lc, kind, 2, 64, 32, lens, [(0, 3, 128)], seed=14)
    v = normals((1, 2, 64), 3)
    v[0, 1, 5] = bad
    pg.cache.append(torch.zeros_like(v), v, pg.seqs([1], [101], pg.table[:1]))       # position 100
    q = normals((3 * new, Hq, 64), seed=6, dtype=torch.bfloat16)
    for window in (0, 60, 31):
        seqs = pg.seqs([new] * 3, lens)
        want, want_lse = pg.cache.attend(q, seqs, window=window, max_new=new)
        out, lse = pg.cache.attend_shared(q, seqs, prefixes(lc, [(0, 3, 128)]), window=window, max_new=new)
        assert torch.equal(out.isfinite(), want.isfinite()), window
        assert torch.equal(lse.isfinite(), want_lse.isfinite())
        fine = want.isfinite()
        assert bool(((out.float() - want.float()).abs()[fine] <= 2.0 ** -6 * (1 + want.float().abs()[fine])).all())
    if new == 1:
        assert bool(pg.cache.attend_shared(q, seqs, prefixes(lc, [(0, 3, 128)]))[0].isfinite().logical_not().any())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("new,heads,Hq,d", [(1, 2, 8, 128), (21, 2, 8, 64), (4, 1, 4, 256)])
def test_long_prefixes(lc, dtype, new, heads, Hq, d):
    lens = [20_000, 20_100, 19_990, 20_003]
    groups = [(0, 4, 19_968)]
    pg, held = shared(lc, "bf16", heads, d, 64, lens, groups, seed=8)
    q = normals((4 * new, Hq, d), seed=6, dtype=dtype, size=2)
    check(lc, pg, held, q, [new] * 4, lens, groups, max_new=new)
    check(lc, pg, held, q, [new] * 4, lens, groups, max_new=new, window=700)


def test_rows_of_no_sequence_and_strided_rows(lc):
    pg, held = shared(lc, "bf16", 2, 64, 32, [300, 290], [(0, 2, 256)], seed=2)
    wide = normals((9, 12, 64), seed=3, dtype=torch.bfloat16)
    q = wide[:, 2:10]
    seqs = lc.Sequences(torch.tensor([2, 5, 6], dtype=torch.int32, device=DEV), torch.tensor([300, 290], dtype=torch.int32, device=DEV),
                        pg.table.to(DEV))
    out = (torch.full((9, 8, 64), 7.0, dtype=torch.bfloat16, device=DEV), torch.full((9, 8), 7.0, device=DEV))
    version = out[0]._version
    got = pg.cache.attend_shared(q, seqs, prefixes(lc, [(0, 2, 256)]), out=out)
    assert got[0] is out[0] and out[0]._version > version
    outside = [0, 1, 6, 7, 8]
    assert bool((out[0][outside] == 7).all()) and bool((out[1][outside] == 7).all())
    check_attend(lc, pg, held, q[2:6], [3, 1], [300, 290], out=(out[0][2:6], out[1][2:6]))
    none = pg.cache.attend_shared(q[:0], pg.seqs([0, 0], [300, 290]), prefixes(lc, [(0, 2, 256)]))
    assert none[0].shape == (0, 8, 64)


@pytest.mark.parametrize("kind", ["bf16", "int8"])
def test_shared_pages_beyond_32_bits(lc, kind):
    n_pages, heads, d, page = 36_000, 8, 128, 128
    pg = Paged(lc, kind, heads, d, page, 2, 8, n_pages=n_pages)
    pg.table = torch.stack([n_pages - 1 - torch.arange(8)] * 2).to(torch.int32)
    pg.table[1, 7] = n_pages - 30
    k, v = normals((1000, heads, d), 1), normals((1000, heads, d), 2)
    pg.cache.append(k, v, pg.seqs([1000, 0], [1000, 0]))
    pg.cache.append(k[896:], v[896:], pg.seqs([0, 104], [0, 1000]))
    whole = pg.seqs([1000, 1000], [1000, 1000])
    kb, vb = pg.cache.read(whole, 2000, dtype=torch.float32)
    held = list(zip(kb.double().split(1000), vb.double().split(1000)))
    q = normals((4, 16, d), 3, dtype=torch.bfloat16)
    check(lc, pg, held, q, [2, 2], [1000, 1000], [(0, 2, 896)])


def test_streams_graphs_and_scratch(lc):
    """Another stream; captured calls replayed with lengths and groups that change, eager calls of this and of the whole attention
    between, which share the scratch; the same bits every time."""
    lens = [300, 290, 270, 1500]
    pg, held = shared(lc, "fp8", 2, 64, 32, lens, [(0, 3, 256)], seed=30)
    q = normals((4, 8, 64), 1, dtype=torch.bfloat16)
    seqs, p = pg.seqs([1] * 4, lens), prefixes(lc, [(0, 3, 256)])
    outs = (torch.empty((4, 8, 64), device=DEV, dtype=torch.bfloat16), torch.empty((4, 8), device=DEV))

    def call(stream=None, out=None):
        return pg.cache.attend_shared(q, seqs, p, max_new=1, out=out, stream=stream)

    want = call()
    check_attend(lc, pg, held, q, [1] * 4, lens, out=want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = call(stream=side)
    side.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(want, got))
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call(out=outs)
        graphs.append(graph)
    for r in range(4):
        q.copy_(normals((4, 8, 64), 5 + r, dtype=torch.bfloat16))
        now = [300 - r, 290, 270 - 31 * (r % 2), 1500 - 700 * (r % 3)]
        seqs.lens.copy_(torch.tensor(now, dtype=torch.int32))
        p.len.copy_(torch.tensor([256 - 64 * (r % 3)], dtype=torch.int32))
        want, again = call(), call()
        check_attend(lc, pg, held, q, [1] * 4, now, out=want)
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
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    q, seqs, p = torch.zeros((2, 4, 64), device=DEV), pg.seqs([1, 1], [5, 6]), lc.Prefixes(i32(0, 2), i32(32))
    for f in (lambda: lc.Prefixes(i32(0), i32(32)), lambda: lc.Prefixes(i32(0, 2).cpu(), i32(32).cpu()),
              lambda: lc.Prefixes(i32(0, 2).long(), i32(32)), lambda: lc.Prefixes(i32(0, 2), i32(32).float()),
              lambda: pg.cache.attend_shared(q.half(), seqs, p), lambda: pg.cache.attend_shared(q[:, :3], seqs, p),
              lambda: pg.cache.attend_shared(q, seqs, p, window=-1), lambda: pg.cache.attend_shared(q, seqs, p, scale=math.inf),
              lambda: pg.cache.attend_shared(q, seqs, p, max_new=-1), lambda: pg.cache.attend_shared(q.cpu(), seqs, p),
              lambda: pg.cache.attend_shared(q, seqs, p, out=(q[:1], q[:1, :, 0])),
              lambda: pg.cache.attend_shared(q.clone().requires_grad_(), seqs, p)):
        with pytest.raises((ValueError, lc.LaCacheError)):
            f()
    with torch.no_grad():
        pg.cache.attend_shared(q.clone().requires_grad_(), seqs, p)


IDLE = [  # new tokens, lengths, groups: slots without tokens or rows, and sequences shorter than the prefix, come first
    ([1, 1, 1], [0, 290, 310], [(0, 3, 256)]),
    ([1, 1, 1], [40, 290, 310], [(0, 3, 256)]),
    ([1, 1, 1, 1], [0, 0, 70, 333], [(0, 4, 320)]),
    ([0, 1, 1], [300, 290, 270], [(0, 3, 256)]),
    ([1, 1], [40, 70], [(0, 2, 256)]),
    ([1] * 8, [0, 260, 300, 33, 0, 257, 0, 129], [(0, 3, 256), (3, 6, 250), (6, 8, 128)]),
    ([1, 1, 1], [300, 0, 290], [(0, 3, 256)]),
]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("new,Hq,d", [(1, 4, 64), (1, 32, 64), (5, 16, 96), (30, 4, 64), (1, 4, 256), (9, 4, 256)])
@pytest.mark.parametrize("news,lens,groups", IDLE)
def test_any_sequence_of_a_group_may_be_idle(lc, dtype, new, Hq, d, news, lens, groups):
    """Page tables have nothing behind their sequences' own tokens, and nothing at all where a slot has no rows: the others'
    prefix is read all the same, through the table of one that holds it."""
    say(f"[case] idle {dtype} {new} {Hq} {d} {news} {lens} {groups}")
    pg, held = shared(lc, "bf16", 2, d, 32, lens, groups, seed=d + new)
    table = pg.table.clone()
    for i, (n, length) in enumerate(zip(news, lens)):
        table[i, -(-length // 32) if n else 0:] = -1
    news = [n * new for n in news]
    q = normals((sum(news), Hq, d), seed=new, dtype=dtype, size=2)
    for window in (0, 100):
        check(lc, pg, held, q, news, lens, groups, window=window, max_new=new, table=table)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("kind,heads,Hq,d,news,fronts,groups", [
    ("bf16", 2, 8, 64, [600, 417, 33, 1030], [256, 256, 256, 256], [(0, 4, 256)]),
    ("fp8", 1, 4, 128, [700, 1, 350], [640, 640, 0], [(0, 2, 640)]),
    ("int8", 2, 4, 96, [301, 300, 290, 400], [96, 96, 320, 320], [(0, 2, 96), (2, 4, 320)]),
    ("bf16", 1, 2, 256, [500, 450], [512, 512], [(0, 2, 512)])])
def test_prompts_behind_a_prefix(lc, dtype, kind, heads, Hq, d, news, fronts, groups):
    """All of the sequences' own tokens are new, as when instructions that prompts share have been cached before."""
    say(f"[case] prompts {kind} {dtype} {heads} {Hq} {d} {news} {fronts}")
    lens = [n + f for n, f in zip(news, fronts)]
    pg, held = shared(lc, kind, heads, d, 32, lens, groups, seed=d)
    q = normals((sum(news), Hq, d), seed=d, dtype=dtype, size=2)
    check(lc, pg, held, q, news, lens, groups, max_new=max(news))
    check(lc, pg, held, q, news, lens, groups, window=150)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("new,Hq,d", [(1, 8, 64), (21, 8, 64), (1, 4, 256)])
def test_few_of_many_share(lc, dtype, new, Hq, d):
    """Two small groups among sequences that share nothing, of other lengths."""
    lens = [120 + (37 * i) % 500 for i in range(60)]
    for i in (11, 12, 13, 40, 41):
        lens[i] += 256
    groups = [(11, 14, 256), (40, 42, 320)]
    pg, held = shared(lc, "bf16", 2, d, 32, lens, groups, seed=3)
    q = normals((60 * new, Hq, d), seed=5, dtype=dtype)
    check(lc, pg, held, q, [new] * 60, lens, groups, max_new=new)
    check(lc, pg, held, q, [new] * 60, lens, groups, window=90)
