"""Bounds for attention that charge every rounding what it is, and inputs that show the precision of its weights."""
from __future__ import annotations

import math

import torch


def bounds(want, d, f32):
    """How far out and lse may be from decode_ref.attention()'s.

    A float32 dot product of d terms is within 8 sqrt(d) 2^-24 of sum |q k| (far out in the tail of the random walk); its
    scaling, the exponential, the rescalings, the code scales and the sums are charged 16 roundings more.  A relative error
    t of every weight moves the normalised sum by 2 t sum w |v|.  bfloat16 has 8 significant bits, half a unit of its last
    place is up to 2^-8 of a number.  With bfloat16 rows a weight is two such terms: the first leaves up to 2^-8 of it, the
    second half a unit of that, 2^-17.  The result is rounded once, 2^-8."""
    out, lse, size, largest = want
    t = 2.0 ** -24 * (8 * math.sqrt(d) * largest + 16)
    b = 2 * t[..., None] * size + 2.0 ** -24 * out.abs()
    if not f32:
        b = b + 2.0 ** -17 * 1.01 * size + 2.0 ** -8 * 1.01 * out.abs()
    return b + 1e-37, t + 2.0 ** -22 * torch.where(torch.isinf(lse), 0.0, lse.abs())


def sparse_bounds(want, f32):
    """The same for queries with a single column that is not 0 and a scale of 1: a score is one product, in up to three
    exact terms (3 roundings of it), times log2 e (2, rounded itself) and less the maximum (2): 6.5 of the score; the
    exponential 2, and 8 for rescaling, joining, code scales and sums."""
    out, _, size, largest = want
    t = 2.0 ** -24 * (6.5 * largest + 10)
    b = 2 * t[..., None] * size + 2.0 ** -24 * out.abs()
    if not f32:
        b = b + 2.0 ** -17 * 1.01 * size + 2.0 ** -8 * 1.01 * out.abs()
    return b + 1e-37


def sparse_queries(n, H, d, seed):
    """[n, H, d] with one column of +-0.25 each, another for every row and head."""
    g = torch.Generator().manual_seed(seed)
    q = torch.zeros((n * H, d))
    q[torch.arange(n * H), torch.randperm(n * H, generator=g) % d] = 0.25
    return (q * (torch.randint(2, (n * H, 1), generator=g) * 2 - 1)).view(n, H, d)


def cancelling_values(q, keys, first):
    """Values [L, heads, d] for the queries q [n, H, d] over the keys [L, heads, d] (float64; a scale of 1): column c has two
    tokens, neighbours among the first `first` >= 2 d, whose weights for one of the rows of the head cancel.  What is left
    of the sum is the rounding of the value and the errors of the weights.  A token has one column that is not 0, so that 8
    bits hold it too."""
    (n, H, d), heads = q.shape, keys.shape[1]
    assert first >= 2 * d and n * (H // heads) <= d
    v = torch.zeros_like(keys)
    group, c = H // heads, torch.arange(d)
    for h in range(heads):
        rows = q[:, h * group:(h + 1) * group].reshape(-1, d)
        j = 2 * ((c * 37) % (first // 2) if math.gcd(37, first // 2) == 1 else c)  # not in order of the columns
        s = rows[c % len(rows)] @ keys[:, h].T
        v[j, h, c] = 1.0
        v[j + 1, h, c] = -torch.exp(s[c, j] - s[c, j + 1])
    return v
