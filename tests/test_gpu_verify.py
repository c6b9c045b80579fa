"""GPU tests of sampled verification against 64 bits: whole numbers are equal, probabilities within their roundings."""
from __future__ import annotations

import math

import numpy as np
import pytest
import torch

from tests import draft_ref as ref

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.fixture(scope="module")
def lc():
    import paper_2608_01718_amd as m
    return m


def inputs(B, k, V, dtype, seed=0, size=2.0, noise=0.5):
    g = torch.Generator(DEV).manual_seed(seed * 7919 + B + 31 * k + V)
    logits = torch.randn((B, k + 1, V), generator=g, device=DEV) * size
    draft = (logits[:, :k] + noise * torch.randn((B, k, V), generator=g, device=DEV)).to(dtype)
    logits = logits.to(dtype)
    if k:
        tokens = torch.multinomial(draft.float().softmax(2).flatten(0, 1), 1, generator=g).view(B, k).int()
    else:
        tokens = torch.zeros((B, 0), dtype=torch.int32, device=DEV)
    u, u_next = torch.rand((B, k), generator=g, device=DEV), torch.rand(B, generator=g, device=DEV)
    return logits, draft, tokens, u, u_next


def check(lc, logits, draft, tokens, u, u_next, temperature=None, n_draft=None, got=None):
    B, k, V = logits.shape[0], logits.shape[1] - 1, logits.shape[2]
    got = got or lc.lacache_verify(logits, draft, tokens, u, u_next, temperature, n_draft)
    acc, nxt, p, q = (x.cpu().numpy() for x in got)
    t = [1.0] * B if temperature is None else temperature.tolist()
    n = [k] * B if n_draft is None else n_draft.tolist()
    lg, dr = logits.float().cpu().numpy(), draft.float().cpu().numpy()
    tk, uu, un = tokens.cpu().numpy(), u.cpu().numpy(), u_next.cpu().numpy()
    for b in range(B):
        a, x, pp, qq, near = ref.verify(lg[b], dr[b], tk[b], uu[b], un[b], t[b], n[b])
        # (the reference's own sums are 64 bits: a comparison nearer to its border than this would say nothing)
        assert near > 1e-13, (b, near)
        assert (acc[b], nxt[b]) == (a, x), (b, acc[b], a, nxt[b], x)
        for have, want in ((p[b], pp), (q[b], qq)):
            assert np.all(np.abs(have - want) <= ref.bound(V) * want + 2.0 ** -126), (b, have, want)
    return got


SIZES = [(1, 1, 1), (1, 0, 5), (3, 5, 7), (17, 20, 1000), (5, 70, 3001), (4, 20, 32000), (2, 3, 128256), (70, 2, 2049),
         (300, 1, 257), (1, 4, 8192), (2, 130, 9)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("size", SIZES)
def test_against_64_bits(lc, size, dtype):
    print(f"[case] {size} {dtype}", flush=True)
    check(lc, *inputs(*size, dtype))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_temperatures_drafts_and_greedy(lc, dtype):
    """A batch of everything: temperatures from hot to cold, greedy ones, fewer drafts, counts out of range."""
    B, k, V = 24, 9, 5003
    logits, draft, tokens, u, u_next = inputs(B, k, V, dtype, seed=3)
    t = torch.tensor([0.0, -1.0, math.nan, math.inf, 2.0 ** -61, 2.0 ** 61, 2.0 ** -60, 1e-3, 0.1, 0.5, 1.0, 1.5, 10.0, 2.0 ** 60,
                      *([0.7] * 10)], device=DEV)
    n = torch.tensor([9, 9, 3, 9, 1, 0, 9, 9, 9, 9, 9, 9, 9, 9, 0, 1, 2, 3, 8, 9, 10, -1, 1000, 5], dtype=torch.int32, device=DEV)
    for b in range(6):
        tokens[b] = logits[b, :k].argmax(1).int()
        if b % 2:
            tokens[b, 4] = 17
    # ties of the largest
    logits[0, :, 100] = logits[0, :, 4000] = 40.0
    tokens[0, ::2], tokens[0, 1::2] = 100, 4000
    got = check(lc, logits, draft, tokens, u, u_next, t, n)
    assert got[0][0] == 9 and got[1][0] == 100
    # rows that are not there are not read
    for b in range(B):
        logits[b, min(max(int(n[b]), 0), k) + 1:] = math.nan
        draft[b, min(max(int(n[b]), 0), k):] = math.nan
        if b < 6:
            draft[b] = math.nan
    again = lc.lacache_verify(logits, draft, tokens, u, u_next, t, n)
    assert all(torch.equal(x, y) for x, y in zip(got, again))


@pytest.mark.parametrize("V", [3, 1000, 20011])
def test_comparisons_at_their_borders(lc, V):
    """Random numbers that are the float32 next to p / q on either side: closer than sums in float32 can tell apart."""
    B, k = 12, 6
    logits, draft, tokens, u, u_next = inputs(B, k, V, torch.float32, seed=5, noise=1.0)
    p = logits[:, :k].double().softmax(2).gather(2, tokens.long()[..., None])[..., 0]
    q = draft.double().softmax(2).gather(2, tokens.long()[..., None])[..., 0]
    at = (p / q).clamp(max=1 - 2.0 ** -24).float()
    up, down = torch.nextafter(at, torch.tensor(1.0, device=DEV)), torch.nextafter(at, torch.tensor(0.0, device=DEV))
    some = torch.arange(B * k, device=DEV).view(B, k)
    check(lc, logits, draft, tokens, torch.where(some % 5 == 4, up, down), u_next)
    check(lc, logits, draft, tokens, down, u_next)
    got = check(lc, logits, draft, tokens, torch.where(p < q, up, down), u_next)
    assert int(got[0].min()) < k


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rows_without_probabilities(lc, dtype):
    """Masked logits, rows of them, infinities and NaN in either model, drafts that are no tokens."""
    B, k, V = 14, 3, 700
    logits, draft, tokens, u, u_next = inputs(B, k, V, dtype, seed=8)
    u[:] = 0.3
    lost, inf = -math.inf, math.inf
    logits[0, 0], logits[1, 1], logits[2, 0, 5], logits[3, 0, 699] = lost, lost, inf, math.nan
    draft[4, 0], draft[5, 1], draft[6, 0, 0], draft[7, 0, 650] = lost, lost, inf, math.nan
    tokens[8, 0], tokens[8, 1], tokens[9, 0] = -1, V, 2 ** 31 - 1
    logits[10, :, 50:], draft[10, :, 50:] = lost, lost     # most of the vocabulary filtered out
    tokens[10] = 7
    logits[11, 0, :600] = lost                             # the target has filtered out the draft's token
    tokens[11, 0] = 3
    draft[12, 0, 3], tokens[12, 0] = lost, 3               # a token that the draft model does not give
    logits[13] = torch.finfo(dtype).min                    # the lowest value is a logit like any other
    draft[13] = torch.finfo(dtype).min
    acc, nxt, p, q = check(lc, logits, draft, tokens, u, u_next)
    assert acc[0] == 0 and nxt[0] == -1 and acc[2] == 0 and nxt[2] == -1 and nxt[3] == -1
    assert acc[4] == 0 and nxt[4] >= 0 and acc[12] >= 1 and int(nxt[10]) < 50
    check(lc, logits, draft, tokens, u, u_next, torch.zeros(B, device=DEV))   # greedy


def test_random_numbers_at_their_ends(lc):
    """0 takes the first token with a weight, the largest number below 1 one near the end, 1 and NaN the last."""
    B, k, V = 6, 2, 3000
    logits, draft, tokens, u, u_next = inputs(B, k, V, torch.float32, seed=9)
    logits[:, :, :10] = -math.inf
    logits[:, :, -7:] = -math.inf
    u[:] = 2.0                                             # (no draft is taken)
    draft[:] = -60.0
    draft[:, :, 40] = 0.0
    tokens[:] = 40
    u_next[:] = torch.tensor([0.0, 1 - 2.0 ** -24, 1.0, 2.0, 0.0, 0.5], device=DEV)
    got = check(lc, logits, draft, tokens, u, u_next)
    assert got[0].tolist() == [0] * 6 and got[1][0] == 10 and got[1][2] == got[1][3] == V - 8
    u_next[0] = u[0, 0] = math.nan
    a, x, _, _ = lc.lacache_verify(logits, draft, tokens, u, u_next)
    assert int(a[0]) == 0 and int(x[0]) == V - 8


def test_the_same_distribution(lc):
    """Nothing is left of p - q: the token is drawn from p.  Also where the logits differ by a constant."""
    B, k, V = 4, 1, 4099
    logits, _, tokens, u, u_next = inputs(B, k, V, torch.float32, seed=2)
    logits = (logits * 64).round() / 64                    # (so that the constant changes no difference)
    draft = logits[:, :k].clone()
    draft[2:] += 3.0
    u[:] = 1.5
    got = check(lc, logits, draft, tokens, u, u_next)
    assert got[0].tolist() == [0] * 4


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_strides(lc, dtype):
    """Rows that begin anywhere, of a wider buffer, in another order, and one row for all."""
    B, k, V = 5, 3, 1001
    logits, draft, tokens, u, u_next = inputs(B, k, V, dtype)
    want = check(lc, logits, draft, tokens, u, u_next)
    wide = torch.full((k + 1, B, V + 37), math.nan, dtype=dtype, device=DEV)
    wide[:, :, 5:5 + V] = logits.transpose(0, 1)
    narrow = torch.full((B, k + 2, V + 2), math.nan, dtype=dtype, device=DEV)
    narrow[:, 1:k + 1, 1:V + 1] = draft
    got = lc.lacache_verify(wide[:, :, 5:5 + V].transpose(0, 1), narrow[:, 1:k + 1, 1:V + 1], tokens, u, u_next)
    assert all(torch.equal(x, y) for x, y in zip(want, got))
    check(lc, logits[:1].expand(B, -1, -1), draft[:1].expand(B, -1, -1), tokens, u, u_next)


def test_calls_that_are_refused(lc):
    B, k, V = 2, 3, 50
    logits, draft, tokens, u, u_next = inputs(B, k, V, torch.float32)
    a = dict(logits=logits, draft_logits=draft, draft_tokens=tokens, u_accept=u, u_next=u_next)
    for bad in (dict(logits=logits[0]), dict(logits=logits.half()), dict(logits=logits.cpu()), dict(logits=logits[:, :0]),
                dict(draft_logits=draft[:, :2]), dict(draft_logits=draft.bfloat16()),
                dict(logits=logits.transpose(1, 2).contiguous().transpose(1, 2)),
                dict(draft_logits=draft[:, :, :-1]), dict(draft_tokens=tokens.long()), dict(draft_tokens=tokens[:, :2]),
                dict(u_accept=u.double()), dict(u_accept=u[:1]), dict(u_next=u_next[:1]), dict(temperature=u_next.double()),
                dict(temperature=u_next[:1]), dict(n_draft=u_next), dict(u_next=u_next.cpu()),
                dict(logits=logits.clone().requires_grad_())):
        with pytest.raises((ValueError, lc.LaCacheError)):
            lc.lacache_verify(**{**a, **bad})
    out = lc.lacache_verify(**a)
    with pytest.raises(ValueError):
        lc.lacache_verify(**a, out=out[:3])
    with torch.no_grad():
        lc.lacache_verify(**{**a, "logits": logits.clone().requires_grad_()})
    empty = lc.lacache_verify(logits[:0], draft[:0], tokens[:0], u[:0], u_next[:0])
    assert [tuple(x.shape) for x in empty] == [(0,), (0,), (0, 3), (0, 3)]


def test_streams_outputs_and_graphs(lc):
    """Another stream, results in given tensors, and two captured calls replayed in turn on changing inputs."""
    B, k, V = 9, 5, 6007
    sets = [inputs(B, k, V, torch.bfloat16, seed=s) for s in range(3)]
    want = [check(lc, *x) for x in sets]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    out = tuple(torch.empty_like(x) for x in want[0])
    version = out[0]._version
    got = lc.lacache_verify(*sets[0], out=out, stream=s)
    s.synchronize()
    assert got[0] is out[0] and out[0]._version > version and all(torch.equal(x, y) for x, y in zip(got, want[0]))
    graphs = []
    for x in sets[:2]:
        held = [t.clone() for t in x]
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            res = lc.lacache_verify(*held)
        graphs.append((g, held, res))
    for turn in range(4):
        for i, (g, held, res) in enumerate(graphs):
            which = (turn + i) % 3
            for t, x in zip(held, sets[which]):
                t.copy_(x)
            g.replay()
            eager = lc.lacache_verify(*sets[which])
            torch.cuda.synchronize()
            assert all(torch.equal(x, y) for x, y in zip(res, want[which]))
            assert all(torch.equal(x, y) for x, y in zip(eager, want[which]))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("B,V", [(2, 700), (2, 3000), (2, 150_001), (2, 262_144), (32, 262_147)])
def test_smallest_weights(lc, B, V, dtype):
    """A random number of 0 takes the first token with a weight, however small: weights between 2^-1000 and 2^-1050 (sums of
    them on either side of 2^-1000), in front of all others or behind tokens without any, in pieces and threads of any number of
    them.  What is below 2^-1074 has none."""
    print(f"[case] {B} {V} {dtype}", flush=True)
    u, tokens, drafts = torch.zeros((B, 0), device=DEV), torch.zeros((B, 0), dtype=torch.int32, device=DEV), (B, 0, V)
    for size in (-693.0, -696.0, -700.0, -704.0, -728.0):
        for first in (0, 5, V // 2 + 1):
            logits = torch.full((B, 1, V), size, device=DEV)
            logits[:, :, :first] = -math.inf
            logits[1, :, :first] = -760.0                  # 2^-1096
            logits[:, :, -1] = 0.0
            got = lc.lacache_verify(logits.to(dtype), logits[:, :0].to(dtype), tokens, u, torch.zeros(B, device=DEV))
            assert got[1].tolist() == [first] * B, (size, first)
            assert got[0].tolist() == [0] * B and tuple(got[2].shape) == drafts[:2]


@pytest.mark.parametrize("B,V", [(3, 900), (3, 140_003), (40, 262_145)])
def test_smallest_weights_of_the_same_distribution(lc, B, V):
    """Nothing is left of p - q, and the first token of p, for a random number of 0, is one of 2^-1004."""
    logits = torch.full((B, 2, V), -math.inf, device=DEV)
    logits[:, :, 7:7 + V // 2] = -696.0
    logits[:, :, -2:] = 0.0
    draft = logits[:, :1].clone()
    u = torch.full((B, 1), 2.0, device=DEV)
    got = lc.lacache_verify(logits, draft, torch.full((B, 1), V - 1, dtype=torch.int32, device=DEV), u, torch.zeros(B, device=DEV))
    assert got[0].tolist() == [0] * B and got[1].tolist() == [7] * B


@pytest.mark.parametrize("B,V", [(4, 5003), (3, 140_003), (70, 140_003)])
def test_what_is_left_of_nearly_equal_models(lc, B, V):
    """Rows that differ by two tokens that have changed places: r lies in one of them (at least 10 / (100 V) of 1), and in what
    the roundings of 64 bits leave of the others' p - q (up to 2^-52 of p each, 2^-20 of r together at the most).  A token
    is drawn, and for any random number but the smallest it is that one."""
    g = torch.Generator(DEV).manual_seed(V)
    draft = torch.randn((B, 1, V), generator=g, device=DEV) * 3
    a, b = V // 3, 2 * V // 3
    draft[:, :, a], draft[:, :, b] = 1.0, 3.0
    logits = draft.expand(B, 2, V).clone()
    logits[:, 0, a], logits[:, 0, b] = 3.0, 1.0
    u = torch.full((B, 1), 100.0, device=DEV)
    tokens = torch.full((B, 1), b, dtype=torch.int32, device=DEV)
    for u_next in (0.5, 2.0 ** -18, 1 - 2.0 ** -18):
        got = lc.lacache_verify(logits, draft, tokens, u, torch.full((B,), u_next, device=DEV))
        assert got[0].tolist() == [0] * B and got[1].tolist() == [a] * B, u_next
    got = lc.lacache_verify(logits, draft, tokens, u, torch.zeros(B, device=DEV))
    assert bool((got[1] >= 0).all()) and bool((got[1] <= a).all())


def test_outputs_between_the_rows(lc):
    """Results in the gaps of the logits' own buffer, next to rows."""
    B, k, V = 3, 4, 1001
    logits, draft, tokens, u, u_next = inputs(B, k, V, torch.float32)
    want = check(lc, logits, draft, tokens, u, u_next)
    wide = torch.full((B, k + 1, V + 40), 7.0, device=DEV)
    wide[:, :, 20:20 + V] = logits
    flat, stride = wide.view(-1), V + 40
    gap = [flat[20 + V + i * stride:20 + V + i * stride + 12] for i in range(4)]       # (40 numbers each)
    out = (gap[0][:B].view(torch.int32), gap[1][:B].view(torch.int32), gap[2].view(B, k), gap[3].view(B, k))
    got = lc.lacache_verify(wide[:, :, 20:20 + V], draft, tokens, u, u_next, out=out)
    assert all(torch.equal(x, y) for x, y in zip(want, got))
    assert torch.equal(wide[:, :, 20:20 + V], logits) and bool((flat[:20] == 7).all())
    with pytest.raises(lc.LaCacheError):
        lc.lacache_verify(wide[:, :, 20:20 + V], draft, tokens, u, u_next, out=(*out[:3], flat[20 + V - 1:20 + V + 11].view(B, k)))
