"""GPU tests of the decode operators under autograd: rotary positions have a gradient, the cache has none and says so, and
tensors that a call writes into are known to have changed."""
import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.fixture(scope="module")
def lc():
    import paper_2608_01718_amd as m
    return m


@pytest.fixture(scope="module")
def rope(lc):
    return lc.Rope(lc.lacache_rope_table(50, 32, magnitude=1.3), lc.ROPE_PAIRS)


def made(lc, dtype=torch.float32, new=3):
    g = torch.Generator(DEV).manual_seed(2)
    cache = lc.KVCache(4, 2, 48, page=32)
    seqs = lc.Sequences(*(torch.tensor(x, dtype=torch.int32, device=DEV) for x in ([0, new], [20], [[2, 1]])))
    q, k, v = (torch.randn((new, h, 48), generator=g, device=DEV).to(dtype) for h in (4, 2, 2))
    return cache, seqs, q, k, v


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("pairs", [False, True])
def test_rope_has_a_gradient(lc, dtype, pairs):
    """The gradient that backward() leaves is that of the call with backward=True, bit for bit, also where the gradient of
    the result is a broadcast one; and the second derivative is the rotation itself."""
    r = lc.Rope(lc.lacache_rope_table(50, 32, magnitude=1.3), lc.ROPE_PAIRS if pairs else lc.ROPE_HALF)
    g = torch.Generator(DEV).manual_seed(1)
    pos = torch.randint(50, (7,), generator=g, device=DEV, dtype=torch.int32)
    x, dy, u = (torch.randn((7, 3, 48), generator=g, device=DEV).to(dtype) for _ in range(3))
    plain = lc.lacache_rope(x, pos, r)
    w = x.clone().requires_grad_()
    y = lc.lacache_rope(w, pos, r)
    assert y.requires_grad and torch.equal(y.detach(), plain)
    y.backward(dy)
    assert torch.equal(w.grad, lc.lacache_rope(dy, pos, r, backward=True))
    w.grad = None
    lc.lacache_rope(w, pos, r).sum().backward()
    assert torch.equal(w.grad, lc.lacache_rope(torch.ones_like(x), pos, r, backward=True))
    # part of a wider projection, as a model has it
    wide = torch.randn((7, 5, 48), generator=g, device=DEV).to(dtype).requires_grad_()
    lc.lacache_rope(wide[:, 1:4], pos, r).backward(dy)
    assert torch.equal(wide.grad[:, 1:4], lc.lacache_rope(dy, pos, r, backward=True))
    assert not bool(wide.grad[:, [0, 4]].any())
    # the transposed call has the rotation for a gradient
    z = dy.clone().requires_grad_()
    lc.lacache_rope(z, pos, r, backward=True).backward(u)
    assert torch.equal(z.grad, lc.lacache_rope(u, pos, r))
    a, b = x.clone().requires_grad_(), dy.clone().requires_grad_()
    (da,) = torch.autograd.grad(lc.lacache_rope(a, pos, r), a, b, create_graph=True)
    (db,) = torch.autograd.grad(da, b, u)
    assert torch.equal(db, lc.lacache_rope(u, pos, r))


def test_rope_gradient_against_differences(lc, rope):
    """The map is linear, so the difference quotient has no truncation error: both sides are float32 sums of 9 x 3 x 48
    products of a few units, and their 2 x 1296 roundings of 2^-24 add up to less than 1e-3 together."""
    g = torch.Generator(DEV).manual_seed(3)
    pos = torch.randint(50, (9,), generator=g, device=DEV, dtype=torch.int32)
    x, u, dy = (torch.randn((9, 3, 48), generator=g, device=DEV) for _ in range(3))
    w = x.clone().requires_grad_()
    (lc.lacache_rope(w, pos, rope) * dy).sum().backward()
    diff = (lc.lacache_rope(x + u, pos, rope).double() - lc.lacache_rope(x - u, pos, rope).double()) / 2
    assert abs(float((w.grad.double() * u).sum() - (diff * dy).sum())) < 1e-3


def test_rope_refuses_where_a_gradient_would_be_lost(lc, rope):
    pos = torch.zeros(3, dtype=torch.int32, device=DEV)
    x = torch.randn((3, 2, 48), device=DEV)
    w = x.clone().requires_grad_()
    table = lc.Rope(rope.table.clone().requires_grad_())
    for call in (lambda: lc.lacache_rope(w, pos, rope, out=torch.empty_like(x)), lambda: lc.lacache_rope(w, pos, rope, out=w),
                 lambda: lc.lacache_rope(x, pos, rope, out=w), lambda: lc.lacache_rope(x, pos, table)):
        with pytest.raises(ValueError):
            call()
        with torch.no_grad():
            call()


def test_the_cache_refuses_where_a_gradient_would_be_lost(lc):
    cache, seqs, q, k, v = made(lc)
    rope = lc.Rope(lc.lacache_rope_table(50, 48))
    table = lc.Rope(rope.table.clone().requires_grad_())
    grad = lambda t: t.clone().requires_grad_()  # noqa: E731
    for call in (lambda: cache.append(grad(k), v, seqs), lambda: cache.append(k, grad(v), seqs),
                 lambda: cache.append(k, v, seqs, q=grad(q), rope=rope), lambda: cache.append(k, v, seqs, rope=table),
                 lambda: cache.append(k, v, seqs, q=q, rope=rope, q_out=grad(q)), lambda: cache.attend(grad(q), seqs),
                 lambda: cache.attend(q, seqs, out=(grad(q), torch.zeros((3, 4), device=DEV))),
                 lambda: cache.read(seqs, 3, dtype=torch.float32, out=(grad(k), v.clone()))):
        with pytest.raises(ValueError, match="gradient"):
            call()
        with torch.no_grad():
            call()


def test_written_tensors_are_known_to_have_changed(lc, rope):
    """autograd keeps a tensor for its backward pass and checks then that nothing has been written into it."""
    cache, seqs, q, k, v = made(lc)
    full = lc.Rope(lc.lacache_rope_table(50, 48))
    pos = torch.zeros(3, dtype=torch.int32, device=DEV)

    def changes(t, call):
        w = torch.ones_like(t).requires_grad_()
        y = (w * t).sum()      # keeps t
        call()
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            y.backward()

    x = torch.randn((3, 2, 48), device=DEV)
    changes(x, lambda: lc.lacache_rope(x, pos, rope, out=x))
    changes(q, lambda: cache.append(k, v, seqs, q=q, rope=full, q_out=q))
    out = torch.zeros_like(q), torch.zeros((3, 4), device=DEV)
    for t in out:
        changes(t, lambda: cache.attend(q, seqs, out=out))
    back = torch.zeros_like(k), torch.zeros_like(v)
    for t in back:
        changes(t, lambda: cache.read(seqs, 3, dtype=torch.float32, out=back))
    table = torch.zeros((4, 16, 2), device=DEV)
    changes(table, lambda: lc.lacache_rope_table(4, 32, out=table))
    coded = lc.KVCache(4, 2, 48, page=32, type=lc.KV_INT8)
    for t in (cache.k, cache.v, coded.k_scale, coded.v_scale):
        changes(t, lambda: (cache if t.dtype == torch.bfloat16 else coded).append(k, v, seqs))
    with torch.inference_mode():  # tensors without versions
        x = torch.randn((3, 2, 48), device=DEV)
        assert lc.lacache_rope(x, pos, rope, out=x) is x
        cache.append(x.new_zeros((3, 2, 48)), x, seqs)
