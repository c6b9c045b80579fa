"""GPU tests of sampled verification in every form that its launches take: chunks of 512, 2048 and 8192 logits, pieces of 512 and
1024, three launches and five, one piece a thread and several, more positions than are looked at together."""
from __future__ import annotations

import math

import pytest
import torch

from tests import draft_ref as ref
from tests.test_gpu_verify import DEV, check, inputs, lc  # noqa: F401

DTYPES = [torch.bfloat16, torch.float32]


def form(B, k, V):
    """(logits of a chunk, logits of a piece, whether all is in three launches, pieces of a thread), and the scratch of it."""
    rows, up = B * (2 * k + 1), lambda n, of: -(-n // of)  # noqa: E731
    chunk = 8192 if rows * up(V, 8192) >= 8192 else 2048 if rows * up(V, 2048) >= 2048 else 512
    piece = 1024 if B * up(V, 8192) >= 1024 else 512
    pieces = up(V, piece)
    space = sum(up(n, 16) * 16 for n in (16 * B * pieces, 8 * B * pieces, 8 * rows * up(V, chunk), 20 * B, 4 * B))
    return (chunk, piece, piece == 512 and B * up(pieces, 4) <= 1024, up(pieces, 256)), space


SIZES = [  # B, k, V
    (300, 3, 7001), (100, 20, 16_411), (30, 8, 150_001), (1030, 66, 41), (1030, 2, 2049), (33, 1, 300_007), (3, 1, 140_003),
    (520, 3, 12_289), (4, 2, 262_145), (60, 130, 701), (9000, 0, 77), (130, 12, 8192)]


def test_sizes_take_every_form(lc):
    """(No GPU needed.)  The forms as the scratch of a call shows them."""
    forms = set()
    for size in SIZES:
        f, space = form(*size)
        assert lc.lacache_verify_workspace(size[2], size[0], size[1]) == space, size
        forms.add(f)
    assert {f[:3] for f in forms} >= {(8192, 1024, False), (8192, 512, False), (2048, 512, False), (2048, 512, True),
                                      (8192, 512, True), (2048, 1024, False)}
    assert {(f[1], f[2], f[3] > 1) for f in forms} >= {(512, True, True), (512, False, True), (1024, False, True)}


def bound(V):
    """Relative error of p and q: the exponents' four roundings under the weights (the mean of these exponents is below log2 V +
    2), six exponentials within 2^-22, 3 + 4 x 4 + 4 + 6 roundings of sums over four steps and a wave, one of the result."""
    return (math.log2(V) + 2) * 4 * 2.0 ** -24 * math.log(2) + 6 * 2.0 ** -22 + 30 * 2.0 ** -24


@pytest.fixture(autouse=True)
def all_roundings(monkeypatch):
    monkeypatch.setattr(ref, "bound", bound)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", SIZES)
def test_against_64_bits(lc, size, dtype):
    print(f"[case] {size} {dtype}", flush=True)
    check(lc, *inputs(*size, dtype, seed=1))


MIXED = [(300, 5, 7001), (100, 20, 16_411), (30, 8, 150_001), (1030, 4, 2049), (33, 3, 270_007), (1030, 66, 41)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", MIXED)
def test_temperatures_counts_and_rows_without_probabilities(lc, size, dtype):
    """Every sequence another temperature (greedy ones among them) and another number of drafts; masked logits, whole steps and
    chunks of them, infinities and NaN in the first, a middle and the last step of either model's rows."""
    B, k, V = size
    print(f"[case] {size} {dtype}", flush=True)
    logits, draft, tokens, u, u_next = inputs(B, k, V, dtype, seed=2)
    t = torch.tensor([1.0, 0.0, 0.7, 1e-2, 10.0, math.nan, 2.0 ** -60, 0.3, -1.0, 1.5, 40.0], device=DEV).repeat(-(-B // 11))[:B].contiguous()
    n = torch.tensor([k, k, k - 1, 1000, 0, k, 1, -1], dtype=torch.int32, device=DEV).repeat(-(-B // 8))[:B].contiguous()
    lost, inf = -math.inf, math.inf
    step, first, last = min(2048, V // 4), min(8192, V // 2), V - 1

    def at(i):                                             # sequences 17 apart: every temperature and count in turn
        return slice(i, None, 17)

    logits[at(0), :, :step] = lost
    draft[at(0), :, :step] = lost
    logits[at(1), :, :first] = lost
    logits[at(2), :, step:] = lost
    draft[at(2), :, step:2 * step] = lost
    logits[at(3), 0, last] = math.nan
    logits[at(4), 1, step] = inf
    draft[at(5), 0, last] = math.nan
    draft[at(6), 0, 0] = inf
    logits[at(7), 0] = lost
    draft[at(8), 1 % k] = lost
    logits[at(9), :, last], draft[at(9), :, last] = 30.0, 29.0   # the largest comes last
    tokens[at(9)] = last
    logits[at(10), :, 0], draft[at(10), :, 0] = 30.0, 29.0
    tokens[at(10)] = 0
    tokens[at(11), 0] = V
    tokens[at(12), 0] = -1
    logits[at(13), :, V // 2:V // 2 + 2] = 25.0                  # ties
    got = check(lc, logits, draft, tokens, u, u_next, t, n)
    again = lc.lacache_verify(logits, draft, tokens, u, u_next, t, n)
    assert all(torch.equal(x, y) for x, y in zip(got, again))
    # rows behind the drafts are not read, nor a greedy sequence's draft model
    for b in range(B):
        m = min(max(int(n[b]), 0), k) if b < 40 else k
        logits[b, m + 1:] = math.nan
        draft[b, 0 if b % 11 in (1, 5, 8) else m:] = math.nan
    again = lc.lacache_verify(logits, draft, tokens, u, u_next, t, n)
    assert all(torch.equal(x, y) for x, y in zip(got, again))


@pytest.mark.gpu
@pytest.mark.parametrize("size", [(300, 6, 7001), (100, 20, 16_411), (1030, 66, 41), (1030, 3, 2049), (33, 3, 270_007)])
def test_comparisons_at_their_borders(lc, size):
    """Random numbers that are the float32 next to p / q on either side."""
    B, k, V = size
    print(f"[case] {size}", flush=True)
    logits, draft, tokens, u, u_next = inputs(B, k, V, torch.float32, seed=5, noise=1.0)
    p, q = (torch.stack([x[i, :k].double().softmax(1).gather(1, tokens[i].long()[:, None])[:, 0] for i in range(B)])
            for x in (logits, draft))
    at = (p / q).clamp(max=1 - 2.0 ** -24).float()
    up, down = torch.nextafter(at, torch.tensor(1.0, device=DEV)), torch.nextafter(at, torch.tensor(0.0, device=DEV))
    some = torch.arange(B * k, device=DEV).view(B, k)
    for border in (torch.where(some % (k + 1) == k, up, down), down, torch.where(p < q, up, down)):
        got = check(lc, logits, draft, tokens, border, u_next)
    assert int(got[0].min()) < k


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", [(300, 2, 7001), (1030, 1, 2049), (33, 1, 270_007)])
def test_random_numbers_at_their_ends_and_equal_models(lc, size, dtype):
    """0, numbers of 1 and more and NaN where few tokens have a weight, and models of which nothing is left of p - q."""
    B, k, V = size
    logits, draft, tokens, u, u_next = inputs(B, k, V, dtype, seed=9)
    logits[:, :, :10] = -math.inf
    logits[:, :, -7:] = -math.inf
    u[:] = 2.0 ** 100                                      # no draft is taken
    draft[:] = -60.0
    draft[:, :, 40] = 0.0
    tokens[:] = 40
    u_next[:] = torch.tensor([0.0, 1 - 2.0 ** -24, 1.0, 2.0, 0.5], device=DEV).repeat(-(-B // 5))[:B]
    got = check(lc, logits, draft, tokens, u, u_next)
    assert bool((got[1][::5] == 10).all()) and bool((got[1][2::5] == V - 8).all()) and int(got[0].max()) == 0
    u_next[3::5] = math.nan
    again = lc.lacache_verify(logits, draft, tokens, u, u_next)
    assert all(torch.equal(x, y) for x, y in zip(got, again))
    logits, _, tokens, u, u_next = inputs(B, k, V, torch.float32, seed=12)
    logits = (logits * 64).round() / 64                    # (so that the constant changes no difference)
    draft = logits[:, :k].clone()
    draft[B // 2:] += 3.0
    u[:] = 2.0 ** 100
    got = check(lc, logits, draft, tokens, u, u_next)
    assert int(got[0].max()) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("size", [(300, 3, 7001), (1030, 2, 2049)])
def test_streams_and_graphs(lc, size):
    """Five launches on another stream, and captured and replayed on changing inputs with eager calls between."""
    sets = [inputs(*size, torch.bfloat16, seed=s) for s in range(3)]
    want = [check(lc, *x) for x in sets]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = lc.lacache_verify(*sets[0], stream=s)
    s.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, want[0]))
    held = [t.clone() for t in sets[0]]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        res = lc.lacache_verify(*held)
    for turn in range(4):
        for t, x in zip(held, sets[turn % 3]):
            t.copy_(x)
        graph.replay()
        eager = lc.lacache_verify(*sets[turn % 3])
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(res, want[turn % 3]))
        assert all(torch.equal(x, y) for x, y in zip(eager, want[turn % 3]))
