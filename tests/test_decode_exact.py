"""The bounds of the precision tests tell the documented weights from coarser ones (float64 on the CPU, no GPU needed)."""
import pytest
import torch

from tests import decode_exact as ex
from tests import decode_ref as ref


def rounded(x, terms):
    """x as a sum of bfloat16 terms."""
    out = torch.zeros_like(x)
    for _ in range(terms):
        out = out + (x - out).float().to(torch.bfloat16).double()
    return out


@pytest.mark.parametrize("f32,enough", [(False, 2), (True, 3)])
@pytest.mark.parametrize("n,H,heads,d,L", [(1, 4, 2, 64, 200), (21, 8, 4, 128, 333), (1, 2, 1, 256, 600)])
def test_bounds_see_a_missing_term(f32, enough, n, H, heads, d, L):
    """Attention in float64 but for the weights, which are `terms` bfloat16 terms (and, for bfloat16 rows, the result's
    rounding): within the bound with as many terms as are documented, outside with one less."""
    g = torch.Generator().manual_seed(d)
    keys = torch.randn((L, heads, d), generator=g).to(torch.bfloat16).double()
    q = ex.sparse_queries(n, H, d, seed=n).double()
    vals = ex.cancelling_values(q, keys, L - n).to(torch.bfloat16).double()
    seen = torch.arange(L)[None] <= torch.arange(L - n, L)[:, None]
    want = ref.attention(q, keys, vals, seen, 1.0)
    b = ex.sparse_bounds(want, f32)
    kk, vv = (x.repeat_interleave(H // heads, 1).transpose(0, 1) for x in (keys, vals))
    s = (q.transpose(0, 1) @ kk.transpose(1, 2)).masked_fill(~seen[None], float("-inf"))
    e = torch.exp(s - s.amax(2, keepdim=True))
    for terms in (enough - 1, enough):
        got = ((rounded(e, terms) @ vv) / e.sum(2, keepdim=True)).transpose(0, 1)
        if not f32:
            got = got.float().to(torch.bfloat16).double()
        worst = float(((got - want[0]).abs() / b).max())
        assert worst <= 1 if terms == enough else worst > 2, (terms, worst)
