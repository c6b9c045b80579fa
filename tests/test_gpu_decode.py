"""GPU tests of the decode operators through the public calls: rotary positions, writing the paged key-value cache and
reading it back (bit for bit), and the attention over it (against float64)."""
from __future__ import annotations

import math
import sys

import pytest
import torch

from tests import decode_ref as ref

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
KINDS = ("bf16", "fp8", "int8")
DTYPES = (torch.bfloat16, torch.float32)


@pytest.fixture(scope="module")
def lc():
    assert torch.cuda.is_available()
    import paper_2608_01718_amd as m
    return m


def say(*a):
    print(*a, flush=True)
    sys.stdout.flush()


def kind_of(lc, kind):
    return {"bf16": lc.KV_BF16, "fp8": lc.KV_FP8, "int8": lc.KV_INT8}[kind]


# ---- rotary positions --------------------------------------------------------------------------------------


@pytest.mark.parametrize("kw", [dict(n=1, rot=2), dict(n=777, rot=64), dict(n=300, rot=96, base=500000.0, first=131_000),
                                dict(n=513, rot=128, factor=8.0, original=4096.0, magnitude=1.2),
                                dict(n=100, rot=40, factor=4.0, first=5), dict(n=64, rot=256, factor=2.0,
                                                                               original=100.0, low=0.0, high=4.0)])
def test_rope_table(lc, kw):
    """One rounding of the double value: half a unit in the last place, and the double angle's own error (1e-15 of up to
    2e5 turns, with a margin)."""
    got = lc.lacache_rope_table(**kw).cpu().double()
    want = ref.table64(**kw)
    assert got.shape == want.shape
    assert torch.all((got - want).abs() <= want.abs() * 2.0 ** -24 * 1.001 + 2e-9)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("T,H,d,rot", [(1, 1, 2, 2), (1, 32, 128, 128), (7, 5, 80, 40), (33, 3, 96, 96), (130, 8, 64, 20),
                                       (65, 2, 200, 64), (19, 40, 128, 64), (257, 4, 256, 256), (11, 3, 24, 10),
                                       (6, 2, 1024, 128), (3, 1, 13, 8), (1000, 4, 64, 64)])
def test_rope(lc, dtype, pairs, T, H, d, rot):
    """Forward and gradient, for contiguous rows, rows inside a wider tensor, and in place: the float32 formula bit for
    bit, rounded once."""
    say(f"[case] rope T={T} H={H} d={d} rot={rot} pairs={pairs} {dtype}")
    g = torch.Generator().manual_seed(T * 1000 + d)
    table = ref.table64(97, rot, magnitude=1.1).float()
    rope = lc.Rope(table.to(DEV), lc.ROPE_PAIRS if pairs else lc.ROPE_HALF)
    pos = torch.randint(97, (T,), generator=g, dtype=torch.int32)
    wide = torch.randn((T, H + 2, d + 8), generator=g).to(dtype)
    for x in (wide[:, :H, :d].contiguous(), wide[:, 1:H + 1, :d], wide[:, :H, 3:3 + d]):
        for backward in (False, True):
            want = ref.turned(x, table[pos.long()], pairs, backward).to(dtype)
            full = wide.to(DEV)
            dx = x.to(DEV) if x.is_contiguous() else full.as_strided(x.shape, x.stride(), x.storage_offset())
            y = lc.lacache_rope(dx, pos.to(DEV), rope, backward=backward)
            assert torch.equal(y.cpu(), want)
            assert lc.lacache_rope(dx, pos.to(DEV), rope, backward=backward, out=dx) is dx  # in place
            assert torch.equal(dx.cpu(), want)
            if not x.is_contiguous():  # nothing else was written
                back = full.cpu()
                back.as_strided(x.shape, x.stride(), x.storage_offset()).copy_(x)
                assert torch.equal(back, wide)


def test_rope_positions_outside_the_table_take_its_nearest_row(lc):
    x = torch.randn((4, 2, 16))
    table = ref.table64(5, 16).float()
    y = lc.lacache_rope(x.to(DEV), torch.tensor([-3, 0, 4, 2 ** 31 - 1], dtype=torch.int32).to(DEV), lc.Rope(table.to(DEV)))
    assert torch.equal(y.cpu(), ref.turned(x, table[[0, 0, 4, 4]], False))


@pytest.mark.parametrize("pairs", [False, True])
def test_rope_gradient_against_differences(lc, pairs):
    """dx . u is the difference quotient of sum(dy y) along u: the map is linear, so a step of 1 has no truncation error,
    and both sides are sums of T H d float32 products (in double), each within a few roundings."""
    g = torch.Generator().manual_seed(5)
    T, H, d, rot = 9, 3, 48, 32
    rope = lc.Rope(lc.lacache_rope_table(50, rot, factor=4.0, original=20.0, magnitude=1.3),
                   lc.ROPE_PAIRS if pairs else lc.ROPE_HALF)
    pos = torch.randint(50, (T,), generator=g, dtype=torch.int32).to(DEV)
    x, u, dy = (torch.randn((T, H, d), generator=g).to(DEV) for _ in range(3))
    dx = lc.lacache_rope(dy, pos, rope, backward=True).double()
    diff = (lc.lacache_rope(x + u, pos, rope).double() - lc.lacache_rope(x - u, pos, rope).double()) / 2
    left, right = (dx * u.double()).sum(), (dy.double() * diff).sum()
    size = (dy.abs().double() * (x.abs() + u.abs()).double()).sum()
    assert abs(float(left - right)) <= 8 * 2.0 ** -24 * 1.3 * 2 * float(size) / math.sqrt(T * H * d) * 4


def test_rope_of_no_rows(lc):
    rope = lc.Rope(lc.lacache_rope_table(4, 8))
    assert lc.lacache_rope(torch.zeros((0, 2, 8), device=DEV), torch.zeros(0, dtype=torch.int32, device=DEV),
                           rope).shape == (0, 2, 8)
    assert lc.lacache_rope_table(0, 8).shape == (0, 4, 2)


# ---- the paged cache ---------------------------------------------------------------------------------------


class Paged:
    """A cache whose memory holds NaN wherever nothing has been written, and the sequences' page tables."""

    def __init__(self, lc, kind, heads, d, page, n_seq, max_pages, seed=0, spare=3, n_pages=None):
        g = torch.Generator().manual_seed(seed)
        n = n_pages or n_seq * max_pages + spare
        self.lc, self.kind, self.heads, self.d, self.page = lc, kind, heads, d, page
        D = lc._padded(d)
        shape = (n, heads, page // 32, 32 * D)
        if kind == "bf16":
            pools = [torch.full(shape, float("nan"), dtype=torch.bfloat16, device=DEV) for _ in range(2)] + [None, None]
        else:
            raw = [torch.full(shape, 127, dtype=torch.int8, device=DEV) for _ in range(2)]  # 0x7f: NaN in fp8
            sc = [torch.full((n, heads, page), float("nan"), device=DEV) for _ in range(2)]
            pools = [x.view(torch.float8_e4m3fn) if kind == "fp8" else x for x in raw] + sc
        self.cache = lc.KVCache(pools=tuple(pools), d=d)
        self.table = torch.randperm(n, generator=g)[:n_seq * max_pages].view(n_seq, max_pages).to(torch.int32)

    def seqs(self, news, lens, table=None):
        start = torch.tensor([0, *news]).cumsum(0).to(torch.int32)
        return self.lc.Sequences(start.to(DEV), torch.tensor(lens, dtype=torch.int32).to(DEV),
                                 (self.table if table is None else table).contiguous().to(DEV))


def positions(news, lens):
    return torch.cat([torch.arange(n - a, n) for a, n in zip(news, lens)] or [torch.zeros(0, dtype=torch.long)])


def same(got, want):
    """Bit for bit (of a tensor without NaN)."""
    got, want = got.cpu(), want.cpu()
    return got.shape == want.shape and got.dtype == want.dtype and bool((got == want).all())


SHAPES = [  # heads, q_heads, d, rot, page, new tokens, lengths with them
    (1, 1, 8, 8, 32, [1], [1]),
    (2, 6, 64, 64, 32, [1, 1, 1, 1], [1, 32, 33, 64]),
    (3, 3, 80, 40, 64, [5, 0, 31, 70], [5, 17, 90, 133]),
    (8, 32, 128, 128, 64, [1] * 9, [1, 2, 31, 32, 63, 64, 65, 127, 128]),
    (4, 12, 96, 48, 128, [21, 21, 1], [21, 150, 128]),
    (2, 4, 256, 64, 256, [300, 2], [300, 257]),
    (1, 5, 192, 192, 32, [64, 32, 33], [96, 64, 65]),
    (5, 10, 136, 12, 64, [7, 9], [64, 73]),
]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("shape", SHAPES)
def test_append_and_read(lc, kind, dtype, pairs, shape):
    """Codes, scales, turned queries and what is read back, bit for bit; nothing else of the pools changes."""
    heads, Hq, d, rot, page, news, lens = shape
    say(f"[case] append {kind} {dtype} pairs={pairs} {shape}")
    g = torch.Generator().manual_seed(d + page)
    T = sum(news)
    pg = Paged(lc, kind, heads, d, page, len(news), 3 if page > 64 else 5, seed=d)
    seqs = pg.seqs(news, lens)
    table = ref.table64(max(lens), rot).float()
    rope = lc.Rope(table.to(DEV), lc.ROPE_PAIRS if pairs else lc.ROPE_HALF)
    qkv = torch.randn((T, (Hq + 2 * heads) * d), generator=g).mul_(3).to(dtype)
    qkv[T // 2, Hq * d:] = 0                     # a token of zeros
    q, k, v = (x.unflatten(1, (-1, d)) for x in qkv.to(DEV).split([Hq * d, heads * d, heads * d], 1))
    before = [None if t is None else t.clone() for t in (pg.cache.k, pg.cache.v, pg.cache.k_scale, pg.cache.v_scale)]
    q_out = pg.cache.append(k, v, seqs, q=q, rope=rope, max_new=max(news))
    rows = table[positions(news, lens)]
    assert same(q_out, ref.turned(q.cpu(), rows, pairs).to(dtype))
    want_k, want_v = ref.coded(ref.turned(k.cpu(), rows, pairs), kind), ref.coded(v.cpu().float(), kind)
    for out_dtype in DTYPES:
        k_back, v_back = pg.cache.read(seqs, T, dtype=out_dtype, max_new=max(news))
        assert same(k_back, ref.values(*want_k).to(out_dtype))
        assert same(v_back, ref.values(*want_v).to(out_dtype))
    # the layout, element by element, and everything that was not written
    pos = positions(news, lens)
    b = torch.repeat_interleave(torch.arange(len(news)), torch.tensor(news))
    pages, at = pg.table[b, pos // page].long(), pos % page
    D = lc._padded(d)
    t, c = (at % 32)[:, None, None], torch.arange(D)[None, None]
    x, u, e, y, m = c // 32, c // 8 % 4, c % 8, c // 16 % 2, c % 16
    bb, r, gg, i = t // 16, t % 16, t // 4 % 4, t % 4
    base = ((pages[:, None] * heads + torch.arange(heads)) * (page // 32) + at[:, None] // 32)[..., None] * (32 * D)
    if kind == "bf16":
        ik, iv = (((x * 2 + bb) * 4 + u) * 16 + r) * 8 + e, ((((x * 2 + y) * 4 + gg) * 16 + m) * 2 + bb) * 4 + i
    else:
        ik, iv = (((x * 4 + u) * 16 + r) * 2 + bb) * 8 + e, ((((x * 4 + gg) * 16 + m) * 2 + y) * 2 + bb) * 4 + i
    for pool, old, idx, (code, scale), new_scale, old_scale in (
            (pg.cache.k, before[0], base + ik, want_k, pg.cache.k_scale, before[2]),
            (pg.cache.v, before[1], base + iv, want_v, pg.cache.v_scale, before[3])):
        raw = torch.int16 if kind == "bf16" else torch.int8
        want = old.cpu().view(raw).view(-1).clone()
        padded = torch.zeros((T, heads, D), dtype=code.dtype if kind != "fp8" else torch.int8)
        padded[..., :d] = code if kind != "fp8" else code.view(torch.int8)
        want[idx.reshape(-1)] = padded.view(raw).reshape(-1)
        got = pool.cpu().view(raw).view(-1)
        if kind != "int8":  # zeros of either sign
            got, want = (torch.where(z == torch.iinfo(raw).min, torch.zeros_like(z), z) for z in (got, want))
        assert torch.equal(got, want)
        if scale is not None:
            ws = old_scale.cpu().clone()
            ws[pages[:, None], torch.arange(heads), at[:, None]] = scale
            assert torch.equal(new_scale.cpu().view(torch.int32), ws.view(torch.int32))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("spread", [1e-30, 2.0 ** -101, 3e-39, 1e30])
def test_codes_of_tiny_and_huge_heads(lc, kind, spread):
    """Heads below 2^-100 are stored as zeros, others keep their relative precision whatever their size."""
    g = torch.Generator().manual_seed(3)
    k, v = (torch.randn((40, 2, 64), generator=g).clamp_(-3, 3).mul_(spread) for _ in range(2))
    k[3] = 0.9 * 2.0 ** -100
    k[4] = 2.0 ** -100
    pg = Paged(lc, kind, 2, 64, 32, 1, 2)
    seqs = pg.seqs([40], [40])
    pg.cache.append(k.to(DEV), v.to(DEV), seqs)
    kb, vb = pg.cache.read(seqs, 40, dtype=torch.float32)
    for got, x in ((kb, k), (vb, v)):
        assert same(got, ref.values(*ref.coded(x, kind)))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_values_that_are_no_numbers_are_not_lost(lc, kind, dtype, bad):
    """bfloat16 keeps them where they are; 8 bits have none, the whole head of the token reads as NaN.  Other heads and
    tokens are as ever."""
    g = torch.Generator().manual_seed(4)
    k, v = (torch.randn((40, 3, 80), generator=g).to(dtype) for _ in range(2))
    pg = Paged(lc, kind, 3, 80, 32, 1, 2)
    seqs = pg.seqs([40], [40])
    want = [ref.values(*ref.coded(x.float(), kind)) for x in (k, v)]
    for x, w in zip((k, v), want):
        for t, h, c in ((0, 1, 0), (31, 0, 79), (39, 2, 41)):
            x[t, h, c] = bad
            w[t, h, slice(None) if kind != "bf16" else c] = bad if kind == "bf16" else math.nan
    pg.cache.append(k.to(DEV), v.to(DEV), seqs)
    for got, w in zip(pg.cache.read(seqs, 40, dtype=torch.float32), want):
        got = got.cpu()
        assert torch.equal(got.isnan(), w.isnan()) and torch.equal(got[~w.isnan()], w[~w.isnan()])


@pytest.mark.parametrize("kind", KINDS)
def test_positions_that_do_not_exist(lc, kind):
    """Pages outside the pool, positions beyond the page table and negative positions: not stored, read as zeros, their
    queries turned all the same; no other page changes."""
    g = torch.Generator().manual_seed(9)
    news, lens = [40, 70, 6, 0, 4], [33, 70, 6, 0, 100]      # the first has 7 negative positions, the last lies beyond
    pg = Paged(lc, kind, 2, 64, 32, 5, 3, seed=4)
    table = pg.table.clone()
    table[1, 1] = -1
    table[2, 0] = pg.cache.n_pages                           # one past the pool
    table[0, 2], table[3, 0] = 2 ** 31 - 1, -2 ** 31
    seqs = pg.seqs(news, lens, table)
    T = sum(news)
    k, v, q = (torch.randn((T, 2, 64), generator=g) for _ in range(3))
    rot = ref.table64(80, 64).float()
    before = pg.cache.v.cpu().view(torch.int8).clone()
    q_out = pg.cache.append(k.to(DEV), v.to(DEV), seqs, q=q.to(DEV), rope=lc.Rope(rot.to(DEV)))
    pos = positions(news, lens)
    rows = rot[pos.clamp(0, 79)]
    assert same(q_out, ref.turned(q, rows, False))
    b = torch.repeat_interleave(torch.arange(5), torch.tensor(news))
    there = (pos >= 0) & (pos < 96) & ~((b == 1) & (pos // 32 == 1)) & (b != 2) & (b != 3)
    kb, vb = pg.cache.read(seqs, T, dtype=torch.float32)
    assert same(kb, torch.where(there[:, None, None], ref.values(*ref.coded(ref.turned(k, rows, False), kind)), 0.0))
    assert same(vb, torch.where(there[:, None, None], ref.values(*ref.coded(v, kind)), 0.0))
    touched = set(table[b[there], pos[there] // 32].tolist())
    changed = (pg.cache.v.cpu().view(torch.int8) != before).flatten(1).any(1).nonzero()[:, 0].tolist()
    assert set(changed) <= touched


def test_rows_of_no_sequence_are_left_alone(lc):
    """start need not begin at 0 or end at the last row."""
    pg = Paged(lc, "bf16", 1, 64, 32, 2, 2)
    start = torch.tensor([2, 5, 6], dtype=torch.int32).to(DEV)
    seqs = lc.Sequences(start, torch.tensor([3, 9], dtype=torch.int32).to(DEV), pg.table.to(DEV))
    k = torch.randn((9, 1, 64))
    q_out = torch.full((9, 1, 64), 7.0, device=DEV)
    rope = lc.Rope(lc.lacache_rope_table(16, 64))
    pg.cache.append(k.to(DEV), k.to(DEV), seqs, q=k.to(DEV), rope=rope, q_out=q_out)
    o = pg.cache.attend(q_out, seqs, out=(torch.full((9, 1, 64), 7.0, device=DEV), torch.full((9, 1), 7.0, device=DEV)))
    outside = [0, 1, 6, 7, 8]
    assert bool((q_out[outside] == 7).all()) and bool((o[0][outside] == 7).all()) and bool((o[1][outside] == 7).all())
    assert not bool((o[1][2:6] == 7).any())


# ---- attention ---------------------------------------------------------------------------------------------


def filled(lc, kind, heads, d, page, lens, seed, spread=1.0, n_pages=None, table=None):
    """A cache holding random tokens of every sequence, and what it holds as float64 [L, heads, d] each."""
    each = max(1, -(-max([1, *lens]) // page))
    pg = Paged(lc, kind, heads, d, page, len(lens), each, seed=seed, n_pages=n_pages)
    if table is not None:
        pg.table = table(pg.table, each)
    g = torch.Generator(DEV).manual_seed(seed)
    T = sum(lens)
    k, v = (torch.randn((T, heads, d), generator=g, device=DEV).mul_(spread) for _ in range(2))
    whole = pg.seqs(lens, lens)
    pg.cache.append(k, v, whole)
    kb, vb = pg.cache.read(whole, T, dtype=torch.float32)
    return pg, list(zip(kb.double().split(lens), vb.double().split(lens)))


def check_attend(lc, pg, held, q, news, lens, window=0, scale=None, table=None, gone=None, max_new=0, out=None):
    """One call against float64, within the bounds derived in decode_ref."""
    scale_ = q.shape[2] ** -0.5 if scale is None else scale
    o, lse = pg.cache.attend(q, pg.seqs(news, lens, table), scale=scale, window=window, max_new=max_new) \
        if out is None else out
    assert o.dtype == q.dtype and lse.dtype == torch.float32
    r0, worst = 0, 0.0
    for b, (n, length) in enumerate(zip(news, lens)):
        keys, vals = held[b][0][:max(0, length)], held[b][1][:max(0, length)]
        j = torch.arange(keys.shape[0], device=DEV)
        p = torch.arange(length - n, length, device=DEV)[:, None]
        seen = (j <= p) & ((p - j < window) if window else (j >= 0))
        if gone is not None:
            seen &= ~gone[b][:keys.shape[0]]
        for i in range(0, n, 64):  # a part of the rows at a time
            at = slice(r0 + i, r0 + min(n, i + 64))
            want = ref.attention(q[at].double(), keys, vals, seen[i:i + 64], scale_)
            eo, el = ref.bounds(want, q.shape[2], q.dtype == torch.float32)
            go, gl = o[at].double(), lse[at].double()
            empty = torch.isinf(want[1])
            assert torch.equal(torch.isinf(gl) & (gl < 0), empty), (b, i)
            assert bool((go[empty] == 0).all())
            off = (go - want[0]).abs()
            assert bool((off <= eo).all()), (b, i, float((off / eo).max()))
            assert bool(((gl - want[1]).abs()[~empty] <= el[~empty]).all()), (b, i)
            worst = max(worst, float((off / eo).max()) if off.numel() else 0.0)
        r0 += n
    return worst


ATTEND = [  # heads, q_heads, d, page, new tokens, lengths
    (1, 1, 8, 32, [1], [1]),
    (1, 1, 64, 32, [1, 1, 1, 1, 1], [1, 31, 32, 33, 0]),
    (8, 32, 128, 64, [1] * 7, [1, 63, 64, 65, 129, 700, 0]),
    (2, 14, 80, 32, [1, 1], [257, 1000]),
    (16, 16, 64, 256, [1, 1, 1], [255, 256, 257]),
    (1, 16, 256, 128, [1, 1], [127, 513]),
    (1, 17, 96, 64, [1, 1], [300, 64]),
    (2, 64, 128, 64, [1, 1], [200, 77]),
    (1, 128, 64, 64, [1], [150]),
    (4, 12, 96, 64, [21, 3, 0, 21], [21, 400, 50, 131]),
    (4, 32, 128, 64, [21, 21], [500, 64]),
    (2, 16, 256, 32, [40, 9], [333, 41]),
    (1, 2, 192, 32, [151], [600]),
    (3, 3, 40, 64, [33, 1, 2], [33, 1, 90]),
    (2, 8, 128, 64, [300], [300]),
]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape", ATTEND)
def test_attend(lc, kind, dtype, shape):
    heads, Hq, d, page, news, lens = shape
    say(f"[case] attend {kind} {dtype} {shape}")
    pg, held = filled(lc, kind, heads, d, page, lens, seed=d + len(lens))
    q = torch.randn((sum(news), Hq, d), generator=torch.Generator(DEV).manual_seed(1), device=DEV).mul_(2).to(dtype)
    worst = check_attend(lc, pg, held, q, news, lens, max_new=max(news))
    for window in (1, 33, 100):
        worst = max(worst, check_attend(lc, pg, held, q, news, lens, window=window))
    say(f"[ok] {worst:.3f} of the bound")


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", DTYPES)
def test_attend_many_ragged_sequences(lc, kind, dtype):
    """More sequences than a wave has lanes, every length from 0 up, many of them the same, among long ones; one to four
    new tokens."""
    lens = [i if i % 37 else 40 * i for i in range(150)]
    news = [min(n, 1 + i % 4) if n else 1 for i, n in enumerate(lens)]
    pg, held = filled(lc, kind, 2, 64, 32, lens, seed=5)
    q = torch.randn((sum(news), 6, 64), generator=torch.Generator(DEV).manual_seed(2), device=DEV).to(dtype)
    say(f"[case] many sequences {kind} {dtype}")
    check_attend(lc, pg, held, q, news, lens, max_new=4)
    check_attend(lc, pg, held, q, news, lens, window=50)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("new,heads,Hq,d", [(1, 8, 32, 128), (1, 1, 4, 256), (21, 2, 8, 96)])
def test_attend_long_contexts(lc, kind, dtype, new, heads, Hq, d):
    """Contexts that are split over the whole chip, alone and beside short ones."""
    for lens in ([40_001], [3, 20_000, 511, 9000]):
        news = [min(new, n) for n in lens]
        say(f"[case] long {kind} {dtype} new={new} {lens}")
        pg, held = filled(lc, kind, heads, d, 64, lens, seed=7)
        q = torch.randn((sum(news), Hq, d), generator=torch.Generator(DEV).manual_seed(3), device=DEV).mul_(2).to(dtype)
        check_attend(lc, pg, held, q, news, lens, max_new=new)
        check_attend(lc, pg, held, q, news, lens, window=4097)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", DTYPES)
def test_attend_sharp_and_flat_scores(lc, kind, dtype):
    """Scores of hundreds (one position has all the weight, the maximum moves from block to block), of zero and of either
    sign of the scale."""
    lens, news = [700, 65], [3, 2]
    pg, held = filled(lc, kind, 2, 64, 32, lens, seed=11, spread=4.0)
    q = torch.randn((5, 4, 64), generator=torch.Generator(DEV).manual_seed(4), device=DEV).mul_(30).to(dtype)
    for scale in (1.0, 1e-3, 0.0, -0.125):
        say(f"[case] scale {scale} {kind} {dtype}")
        check_attend(lc, pg, held, q, news, lens, scale=scale)


@pytest.mark.parametrize("kind", KINDS)
def test_attend_pages_that_are_not_there(lc, kind):
    """Pages given back (numbers outside the pool) are not seen, wherever they lie; a sequence without any page and one
    whose length passes its page table are rows that see nothing, or what there is."""
    lens, news = [1000, 130, 64, 96], [2, 1, 1, 1]
    pg, held = filled(lc, kind, 2, 128, 32, lens, seed=13)
    table = pg.table.clone()
    table[0, :20] = -1
    table[0, 25] = pg.cache.n_pages
    table[1, 4] = -7
    table[2, :] = -1
    gone = [torch.zeros(n, dtype=torch.bool, device=DEV) for n in lens]
    gone[0][:640] = gone[0][800:832] = True
    gone[1][128:] = True
    gone[2][:] = True
    q = torch.randn((5, 4, 128), generator=torch.Generator(DEV).manual_seed(4), device=DEV).to(torch.bfloat16)
    check_attend(lc, pg, held, q, news, lens, table=table, gone=gone)
    check_attend(lc, pg, held, q, news, lens, table=table, gone=gone, window=70)
    # a length beyond the page table: positions up to 32 * max_pages exist
    cut = table[:, :3]
    gone = [torch.arange(n, device=DEV) >= 96 for n in lens]
    gone[0][:] = True
    gone[2][:] = True
    check_attend(lc, pg, held, q, news, lens, table=cut, gone=gone)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("window", [0, 45])
@pytest.mark.parametrize("length,new,heads,Hq,d", [(75, 3, 2, 4, 64), (130, 9, 2, 6, 96), (300, 21, 2, 8, 128),
                                                   (96, 40, 2, 4, 256), (3000, 150, 2, 2, 64), (64, 64, 2, 2, 192)])
def test_attend_hidden_values_that_are_no_numbers(lc, kind, dtype, bad, window, length, new, heads, Hq, d):
    """An infinity or NaN among the keys or values of a token that some rows see and others do not (later new tokens, and
    tokens that the window has passed): the rows that see it get it (8 bits: in all columns of its head, as a NaN), the
    others are as if it were not there."""
    say(f"[case] no numbers {kind} {dtype} {bad} window={window} {length, new, heads, Hq, d}")
    g = torch.Generator(DEV).manual_seed(d + new)
    k, v = (torch.randn((length, heads, d), generator=g, device=DEV) for _ in range(2))
    pg, clean = (Paged(lc, kind, heads, d, 32, 1, -(-length // 32), seed=d) for _ in range(2))
    seqs = pg.seqs([length], [length])
    clean.cache.append(k, v, seqs)
    keys, vals = (x.double() for x in clean.cache.read(seqs, length, dtype=torch.float32))
    spoiled = torch.zeros((length, heads, d), dtype=torch.bool, device=DEV)   # values that are no numbers
    for t, h, c in ((length - 1, 0, 5), (length - new // 2 - 1, 0, 5), (length - new // 2 - 1, 1, d - 1),
                    (max(0, length - new - 40), 1, 0)):
        v[t, h, c] = bad
        spoiled[t, h, slice(None) if kind != "bf16" else c] = True
    key_at = length - 1 - new // 3
    k[key_at, 1, 3] = math.nan
    pg.cache.append(k, v, seqs)
    q = torch.randn((new, Hq, d), generator=g, device=DEV).to(dtype)
    o, lse = pg.cache.attend(q, pg.seqs([new], [length]), window=window, max_new=new)
    j, p = torch.arange(length, device=DEV), torch.arange(length - new, length, device=DEV)[:, None]
    seen = (j <= p) & ((p - j < window) if window else (j >= 0))
    want = ref.attention(q.double(), keys, vals, seen, d ** -0.5)
    eo, el = ref.bounds(want, d, dtype == torch.float32)
    of = Hq // heads
    no_number = ((seen.double() @ spoiled.double().flatten(1)).view(new, heads, d) > 0).repeat_interleave(of, 1)
    lost = torch.zeros((new, heads), dtype=torch.bool, device=DEV)            # rows without a sum
    lost[:, 1] = seen[:, key_at]
    lost = lost.repeat_interleave(of, 1)
    no_number |= lost[..., None]
    assert torch.equal(~o.isfinite(), no_number)
    assert torch.equal(lse.isnan(), lost)
    assert bool(((o.double() - want[0]).abs() <= eo)[~no_number].all())
    assert bool(((lse.double() - want[1]).abs() <= el)[~lost].all())


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("lens,new", [([70], 1), ([20_001, 40], 1), ([9000], 25)])
def test_attend_of_queries_that_are_no_numbers(lc, kind, dtype, lens, new):
    """A query with a NaN has NaN for a result, also where its context is joined of parts; other rows are as ever."""
    pg, held = filled(lc, kind, 1, 64, 32, lens, seed=9)
    news = [new] * len(lens)
    q = torch.randn((sum(news), 4, 64), generator=torch.Generator(DEV).manual_seed(2), device=DEV).to(dtype)
    seqs = pg.seqs(news, lens)
    want = pg.cache.attend(q, seqs, max_new=new)
    odd = q.clone()
    odd[0, 2, 7] = math.nan
    got = pg.cache.attend(odd, seqs, max_new=new)
    for x, w in zip(got, want):
        assert bool(x[0, 2].isnan().all()) and int(x.isnan().sum()) == x[0, 2].numel()
        x[0, 2] = w[0, 2]
    check_attend(lc, pg, held, q, news, lens, out=got)


def test_attend_rows_before_the_first_position(lc):
    """More rows than the sequence has tokens: the first rows see nothing."""
    pg, held = filled(lc, "bf16", 1, 64, 32, [5, 40], seed=2)
    q = torch.randn((50, 2, 64), device=DEV)
    check_attend(lc, pg, held, q, [9, 41], [5, 40])
    check_attend(lc, pg, [held[0], (held[1][0][:0], held[1][1][:0])], q, [9, 41], [5, -3])


def test_attend_of_strided_rows_and_no_rows(lc):
    pg, held = filled(lc, "fp8", 2, 80, 64, [90, 10], seed=6)
    wide = torch.randn((7, 6 * 80 + 24), device=DEV)
    for shift in (0, 8, 3):  # 3: rows that start off a 16-byte boundary
        q = wide[:, shift:shift + 480].unflatten(1, (6, 80))
        check_attend(lc, pg, held, q, [5, 2], [90, 10])
    empty = pg.cache.attend(torch.zeros((0, 4, 80), device=DEV), pg.seqs([0, 0], [90, 10]))
    assert empty[0].shape == (0, 4, 80) and empty[1].shape == (0, 4)
    none = lc.Sequences(torch.zeros(1, dtype=torch.int32, device=DEV), torch.zeros(0, dtype=torch.int32, device=DEV),
                        torch.zeros((0, 4), dtype=torch.int32, device=DEV))
    assert pg.cache.attend(torch.zeros((0, 4, 80), device=DEV), none)[0].shape == (0, 4, 80)


@pytest.mark.parametrize("kind", ["bf16", "int8"])
def test_offsets_beyond_32_bits(lc, kind):
    """Pools of more than 2^32 elements, the sequence's pages at their end."""
    n_pages, heads, d, page = 36_000, 8, 128, 128                                    # 4.7e9 elements
    last = lambda t, each: (n_pages - 1 - torch.arange(each))[None].to(torch.int32)  # noqa: E731
    pg, held = filled(lc, kind, heads, d, page, [1000], seed=8, n_pages=n_pages, table=last)
    q = torch.randn((2, 16, d), device=DEV).to(torch.bfloat16)
    check_attend(lc, pg, held, q, [2], [1000])


def test_attend_repeats_bit_for_bit(lc):
    pg, _ = filled(lc, "bf16", 4, 128, 64, [5000, 17, 900], seed=21)
    q = torch.randn((3, 32, 128), device=DEV).to(torch.bfloat16)
    seqs = pg.seqs([1, 1, 1], [5000, 17, 900])
    first = pg.cache.attend(q, seqs)
    for _ in range(10):
        again = pg.cache.attend(q, seqs)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


def test_decode_on_another_stream_and_in_a_graph(lc):
    """A step (append, read, attend) on a stream of its own, and captured: replays follow lengths and inputs that change
    between them, with eager work in between."""
    news, lens = [1, 1, 1], [300, 64, 1999]
    pg, _ = filled(lc, "int8", 2, 64, 32, [400, 400, 2100], seed=30)
    g = torch.Generator(DEV).manual_seed(1)
    qkv = torch.empty((3, 8 * 64 + 4 * 64), device=DEV, dtype=torch.bfloat16)
    rope = lc.Rope(lc.lacache_rope_table(3000, 64))
    seqs = pg.seqs(news, lens)
    outs = (torch.empty((3, 8, 64), device=DEV, dtype=torch.bfloat16), torch.empty((3, 8), device=DEV))

    def step(stream=None, outs=None):
        q, k, v = (x.unflatten(1, (-1, 64)) for x in qkv.split([512, 128, 128], 1))
        qr = pg.cache.append(k, v, seqs, q=q, rope=rope, max_new=1, stream=stream)
        return pg.cache.attend(qr, seqs, max_new=1, out=outs, stream=stream), pg.cache.read(seqs, 3, stream=stream)

    qkv.normal_(generator=g)
    (want, want_lse), (wk, wv) = step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    (o, lse), (k, v) = step(stream=side)
    side.synchronize()
    assert torch.equal(o, want) and torch.equal(lse, want_lse) and torch.equal(k, wk) and torch.equal(v, wv)
    step(outs=outs)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(outs=outs)
    for r in range(4):
        qkv.normal_(generator=g)
        seqs.lens.copy_(torch.tensor([301 + r, 64 + 31 * r, 1000 * (r % 3) + 1], dtype=torch.int32))
        (want, want_lse), _ = step()
        outs[0].fill_(5)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[0], want) and torch.equal(outs[1], want_lse), r


def test_graphs_keep_their_scratch(lc):
    """A graph captured before any eager call, eager calls before its first replay, and eager calls that need more scratch
    than the graph was captured with: each gives what a cache of its own gives."""
    lens = [3000, 40, 64]
    pg, _ = filled(lc, "bf16", 2, 64, 32, lens, seed=40)
    other, _ = filled(lc, "bf16", 2, 64, 32, lens, seed=40)
    g = torch.Generator(DEV).manual_seed(1)
    q = torch.randn((3, 8, 64), generator=g, device=DEV).to(torch.bfloat16)
    many = torch.randn((90, 8, 64), generator=g, device=DEV).to(torch.bfloat16)
    one, thirty = (lambda p: p.seqs([1, 1, 1], lens)), (lambda p: p.seqs([30, 30, 30], lens))
    want = [x.clone() for x in other.cache.attend(q, one(other), max_new=1)]
    want_many = [x.clone() for x in other.cache.attend(many, thirty(other), max_new=30)]

    def captured(pg):
        outs, seqs, graph = (torch.zeros_like(want[0]), torch.zeros_like(want[1])), one(pg), torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            pg.cache.attend(q, seqs, max_new=1, out=outs)
        return graph, outs, seqs

    first = captured(pg)
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(pg.cache.attend(q, one(pg), max_new=1), want))
    second = captured(pg)                    # with the scratch of the eager calls
    assert pg.cache._space is not None
    for r in range(3):
        assert all(torch.equal(a, b) for a, b in zip(pg.cache.attend(many, thirty(pg), max_new=30), want_many))
        fill = [torch.full((1 << n,), 255, dtype=torch.uint8, device=DEV) for n in range(12, 27)]  # takes what was freed
        for graph, outs, _ in (first, second):
            for x in outs:
                x.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(outs, want)), r
        assert all(bool((x == 255).all()) for x in fill)
        del fill


# ---- refusals of the binding ---------------------------------------------------------------------------------


def test_binding_refuses(lc):
    bf = torch.bfloat16
    pg = Paged(lc, "bf16", 2, 64, 32, 2, 2)
    seqs = pg.seqs([1, 1], [3, 4])
    x = torch.zeros((2, 2, 64), device=DEV, dtype=bf)
    rope = lc.Rope(lc.lacache_rope_table(8, 64))
    bad = [lambda: pg.cache.append(x, x.float(), seqs), lambda: pg.cache.append(x[:, :1], x, seqs),
           lambda: pg.cache.append(x, x[:1], seqs), lambda: pg.cache.append(x.half(), x.half(), seqs),
           lambda: pg.cache.append(x.cpu(), x.cpu(), seqs), lambda: pg.cache.append(x, x, seqs, q=x[:1], rope=rope),
           lambda: pg.cache.append(x.transpose(0, 1), x, seqs), lambda: pg.cache.append(x, x, seqs, q=x, rope=rope, q_out=x[:1]),
           lambda: pg.cache.attend(x.cpu(), seqs), lambda: pg.cache.attend(x[..., :32], seqs),
           lambda: pg.cache.attend(x, seqs, out=(x[:1], torch.zeros((2, 2), device=DEV))),
           lambda: pg.cache.read(seqs, 2, dtype=torch.float16), lambda: lc.Rope(torch.zeros((4, 8, 2))),
           lambda: lc.Rope(torch.zeros((4, 8), device=DEV)), lambda: lc.KVCache(4, 2, 64, page=48),
           lambda: lc.KVCache(4, 2, 300), lambda: lc.KVCache(pools=(x, x, None, None), d=64),
           lambda: lc.KVCache(pools=(pg.cache.k, pg.cache.v, None, None), d=96),
           lambda: lc.Sequences(seqs.start, seqs.lens.long(), seqs.pages),
           lambda: lc.Sequences(seqs.start[:2], seqs.lens, seqs.pages),
           lambda: lc.lacache_rope(x, torch.zeros(3, dtype=torch.int32, device=DEV), rope),
           lambda: lc.lacache_rope(x.half(), torch.zeros(2, dtype=torch.int32, device=DEV), rope)]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            pytest.fail(f"call {i} was not refused")
    for call in (lambda: pg.cache.attend(torch.zeros((2, 3, 64), device=DEV, dtype=bf), seqs),   # 3 heads over 2
                 lambda: pg.cache.append(x, x, seqs, q=x),                                       # queries without a table
                 lambda: pg.cache.attend(x, seqs, scale=float("nan")), lambda: pg.cache.attend(x, seqs, window=-1),
                 lambda: lc.lacache_rope(x[..., :32], torch.zeros(2, dtype=torch.int32, device=DEV), rope),
                 lambda: lc.lacache_rope_table(4, 7), lambda: lc.lacache_rope_table(4, 8, factor=0.5),
                 lambda: lc.KVCache(pools=(pg.cache.k, pg.cache.v, None, None), d=60).attend(
                     torch.zeros((2, 2, 60), device=DEV, dtype=bf), seqs)):
        with pytest.raises(lc.LaCacheError) as e:
            call()
        assert e.value.code == lc.EINVAL


def test_a_cache_of_its_own_memory(lc):
    """KVCache allocates its pools itself, for every type."""
    for type in (lc.KV_BF16, lc.KV_FP8, lc.KV_INT8):
        c = lc.KVCache(4, 2, 64, page=32, type=type)
        seqs = lc.Sequences(*(torch.tensor(x, dtype=torch.int32, device=DEV) for x in ([0, 40], [40], [[2, 0]])))
        k, v = torch.randn((40, 2, 64), device=DEV), torch.randn((40, 2, 64), device=DEV)
        assert c.append(k, v, seqs) is None
        kb, vb = c.read(seqs, 40, dtype=torch.float32)
        for got, x in ((kb, k), (vb, v)):
            assert float((got - x).norm() / x.norm()) < 0.04     # 2^-4 of each value at most, uniformly spread: 0.036
