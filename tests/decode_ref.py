"""Plain references of the decode operators: rotary positions and the codes of the cache in float32 step by step (what
the operators define bit for bit), attention in float64."""
from __future__ import annotations

import math

import torch

TOP = {"fp8": 448.0, "int8": 127.0}


def turned(x, rows, pairs, backward=False):
    """[T, H, d] (CPU) as float32, its pairs turned by the table rows [T, rot / 2, 2]; every operation rounds."""
    x = x.float().clone()
    half = rows.shape[1]
    c, s = rows[:, None, :, 0], rows[:, None, :, 1]
    s = -s if backward else s
    ia = torch.arange(half) * 2 if pairs else torch.arange(half)
    ib = ia + 1 if pairs else ia + half
    a, b = x[..., ia], x[..., ib]
    x[..., ia], x[..., ib] = a * c - b * s, b * c + a * s
    return x


def table64(n, rot, base=10000.0, factor=1.0, original=0.0, low=1.0, high=32.0, magnitude=1.0, first=0):
    f = base ** (-2.0 * torch.arange(rot // 2, dtype=torch.float64) / rot)
    g = ((original * f / (2 * math.pi) - low) / (high - low)).clamp(0, 1)
    f = (1 - g) * f / factor + g * f
    angle = torch.arange(first, first + n, dtype=torch.float64)[:, None] * f
    return magnitude * torch.stack((angle.cos(), angle.sin()), 2)


def coded(x, kind):
    """float32 [T, H, d] -> (codes, scale [T, H] or None) as they are stored."""
    if kind == "bf16":
        return x.to(torch.bfloat16), None
    top = torch.tensor(TOP[kind])
    m = x.abs().amax(2)
    some = m >= 2.0 ** -100
    inv = torch.where(some, top / torch.where(some, m, 1.0), 0.0)
    y = (x * inv[..., None]).clamp(-top, top)
    code = y.round().to(torch.int8) if kind == "int8" else y.to(torch.float8_e4m3fn)
    return code, torch.where(some, m / top, 0.0)


def values(code, scale):
    return code.float() if scale is None else code.float() * scale[..., None]


def attention(q, keys, vals, seen, scale):
    """q [n, H, d], keys / vals [L, Hkv, d], seen [n, L], all float64.  Returns (out, lse, sum of w |v|, largest
    sum |q k| * scale of a visible position), empty rows as (0, -inf, 0, 0)."""
    n, H, d = q.shape
    hkv = keys.shape[1]
    rep = H // hkv
    kk, vv = keys.repeat_interleave(rep, 1).transpose(0, 1), vals.repeat_interleave(rep, 1).transpose(0, 1)
    qq = q.transpose(0, 1)
    kk = torch.where(seen.any(0)[None, :, None], kk, 0.0)
    vv = torch.where(seen.any(0)[None, :, None], vv, 0.0)
    s = (qq @ kk.transpose(1, 2)) * scale
    s = s.masked_fill(~seen[None], -math.inf)
    size = ((qq.abs() @ kk.abs().transpose(1, 2)) * abs(scale)).masked_fill(~seen[None], 0.0)
    top = s.amax(2, keepdim=True) if s.shape[2] else s.new_full((H, n, 1), -math.inf)
    empty = torch.isinf(top) & (top < 0)
    e = torch.exp(s - torch.where(empty, 0.0, top))
    total = e.sum(2, keepdim=True)
    w = e / torch.where(total > 0, total, 1.0)
    lse = torch.where(empty, -math.inf, top + torch.log(torch.where(total > 0, total, 1.0)))[..., 0]
    largest = size.amax(2) if s.shape[2] else size.new_zeros((H, n))
    return (w @ vv).transpose(0, 1), lse.T, (w @ vv.abs()).transpose(0, 1), largest.T


def bounds(ref, d, f32):
    """How far out and lse may be from attention()'s.

    A float32 dot product of d terms is within a few sqrt(d) roundings of sum |q k| (8 sqrt(d) 2^-24 is far out in the
    tail of the random walk); its scaling, the exponential, the running rescalings, the code scales and the sums are
    charged 16 roundings more.  A relative error t of every weight moves the normalised sum by 2 t sum w |v|.  With
    bfloat16 rows each weight is rounded to 8 bits (2^-9 of it) before the product, and the result (2^-9 of it)."""
    out, lse, size, largest = ref
    t = 2.0 ** -24 * (8 * math.sqrt(d) * largest + 16)
    b = 2 * t[..., None] * size + 2.0 ** -24 * out.abs()
    if not f32:
        b = b + 2.0 ** -9 * 1.01 * size + 2.0 ** -9 * 1.01 * out.abs()
    return b + 1e-37, t + 2.0 ** -22 * torch.where(torch.isinf(lse), 0.0, lse.abs())
