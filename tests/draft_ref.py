"""Sampled verification of drafted tokens in 64 bits, a sequence at a time, from its definition (NumPy)."""
from __future__ import annotations

import math

import numpy as np


def softmax(x, t):
    """Probabilities of a row, None where it has none."""
    x = np.asarray(x, np.float64)
    m = x.max() if len(x) else -math.inf
    if not np.isfinite(m) or np.isnan(x).any():
        return None
    e = np.exp((x - m) / t)
    return e / e.sum()


def verify(logits, draft, tokens, u, u_next, t, n):
    """logits [k + 1, V], draft [k, V], tokens and u [k], u_next and t numbers, n drafts.  Returns (accepted, next, p [k],
    q [k], distance): distance is how near the nearest comparison that decided something was to its border (relative)."""
    k, V = len(tokens), len(logits[0])
    n = min(max(n, 0), k)
    greedy = not 2.0 ** -60 <= t <= 2.0 ** 60
    p, q, taken, near = np.zeros(k), np.zeros(k), 0, math.inf
    for j in range(n):
        x, there = int(tokens[j]), 0 <= int(tokens[j]) < V
        if greedy:
            f = np.asarray(logits[j], np.float64)
            fine = np.isfinite(f.max()) and not np.isnan(f).any()
            p[j], q[j] = float(there and fine and f[x] == f.max()), 1.0
            yes = p[j] == 1
        else:
            f, g = softmax(logits[j], t), softmax(draft[j], t)
            p[j] = f[x] if f is not None and there else 0.0
            q[j] = g[x] if f is not None and g is not None and there else 0.0
            yes = f is not None and g is not None and float(u[j]) * q[j] < p[j]
            if taken == j and p[j] > 0 and g is not None:
                near = min(near, abs(float(u[j]) * q[j] - p[j]) / p[j])
        if yes and taken == j:
            taken = j + 1
    if greedy:
        f = np.asarray(logits[taken], np.float64)
        fine = np.isfinite(f.max()) and not np.isnan(f).any()
        return taken, int(f.argmax()) if fine else -1, p, q, near
    f = softmax(logits[taken], t)
    if f is None:
        return taken, -1, p, q, near
    r = f
    g = softmax(draft[taken], t) if taken < n else None
    if g is not None:
        r = np.maximum(0.0, f - g)
        if r.sum() <= 2.0 ** -30:
            r = f
    c = np.cumsum(r.astype(np.longdouble))
    goal = np.longdouble(float(u_next)) * c[-1]
    past = np.nonzero((c > goal) & (r > 0))[0]
    token = int(past[0]) if len(past) else int(np.nonzero(r > 0)[0][-1])
    borders = np.abs(c[r > 0] - goal) / c[-1]
    if 0 < float(u_next) < 1:
        near = min(near, float(borders.min()))
    return taken, token, p, q, near


def bound(V):
    """Relative error of p and q: the exponents' three roundings under the weights (their mean is below log2 V + 2), the
    exponential's 2^-22, 13 roundings of the float32 sums, one of the result."""
    return (math.log2(V) + 2) * 3 * 2.0 ** -24 * math.log(2) + 2.0 ** -22 + 14 * 2.0 ** -24
