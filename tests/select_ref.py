"""Plain references of the choice of pages: bounds in float64, scores step by step as they are defined."""
from __future__ import annotations

import torch


def bounds(keys):
    """keys [n, d] float64, exact: (code [2, d] int, scale float32)."""
    top = keys.abs().amax()
    if not bool(torch.isfinite(keys).all()):
        return torch.zeros((2, keys.shape[1]), dtype=torch.int8), torch.tensor(float("nan"))
    if top < 2.0 ** -100:
        return torch.zeros((2, keys.shape[1]), dtype=torch.int8), torch.tensor(0.0)
    hi, lo = keys.amax(0), keys.amin(0)
    code = torch.stack(((127 * hi / top).ceil(), (127 * lo / top).floor()))
    return code.to(torch.int8), (top / 127).float()


def scores(q, code, scale):
    """q [H, G, d], code [P, H, 2, d], scale [P, H] (CPU): [H, P] float32."""
    q = q.float()
    top = q.abs().amax(2)
    fine = torch.isfinite(q).all(2)
    unit = torch.where(fine, top * torch.tensor(1 / 127), float("nan"))
    c = torch.where((unit > 0)[..., None], (q / torch.where(unit > 0, unit, 1.0)[..., None]).round().clamp(-127, 127), 0.0).long()
    hi, lo = code[:, :, 0].long(), code[:, :, 1].long()                   # [P, H, d]
    dot = torch.einsum("hgd,phd->hgp", c.clamp(min=0), hi) + torch.einsum("hgd,phd->hgp", c.clamp(max=0), lo)
    s = (dot.float() * scale.T[:, None]) * unit[..., None]
    top = torch.finfo(torch.float32).max
    s = s.clamp(min=-top)
    return torch.where(s.isnan().any(1), float("nan"), s.nan_to_num(nan=-top, posinf=float("inf")).amax(1))


def chosen(score, there, newest, n, first, last):
    """score [P], there [P] bool, the row's pages 0 .. newest: the list."""
    count = min(newest + 1, len(score))
    cand = [i for i in range(count) if there[i]]
    key = {}
    for i in cand:
        x = float(score[i])
        key[i] = (0,) if i < first or i > newest - last else (1,) if x != x else (2, -x)
    best = sorted(sorted(cand, key=lambda i: (*key[i], 0) if len(key[i]) == 1 else key[i] + (0,))[:n]) if len(cand) > n else cand
    return best + [-1] * (n - len(best))
