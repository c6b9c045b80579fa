"""The decode operators together, as examples/speculative_decode.py uses them."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ex():
    from examples import speculative_decode as m
    return m


def plain_logits(model, tokens):
    """The model over whole sequences [B, n] in float64, without a cache."""
    B, n = tokens.shape
    d, (q_dim, kv_dim, _) = model.d, model.sizes
    hq, hkv = q_dim // d, kv_dim // d
    table = torch.view_as_complex(model.rope.table[:n].double())

    def norm(x):
        return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6)

    def turned(x):  # pairs (i, i + d / 2)
        z = torch.complex(x[..., :d // 2].contiguous(), x[..., d // 2:].contiguous()) * table[:, None]
        return torch.cat((z.real, z.imag), -1)

    x = model.embedding[tokens].double()
    hidden = torch.ones((n, n), dtype=torch.bool, device=x.device).triu(1)
    for w_in, w_out in model.layers:
        q, k, v = (norm(x) @ w_in.double()).split(model.sizes, 2)
        q, k = turned(q.unflatten(2, (hq, d))), turned(k.unflatten(2, (hkv, d)))
        v = v.unflatten(2, (hkv, d))
        out = torch.empty_like(q)
        for h in range(hq):
            s = (q[:, :, h] @ k[:, :, h * hkv // hq].transpose(1, 2).contiguous()) * d ** -0.5
            out[:, :, h] = s.masked_fill(hidden, float("-inf")).softmax(2) @ v[:, :, h * hkv // hq]
        x = x + out.flatten(2) @ w_out.double()
    return norm(x) @ model.head.double()


def test_decoded_tokens_are_the_models(ex):
    """After several verifications the cached sequences are what the model says of the whole sequences: its logits for their
    next tokens agree.  float32 activations over a bfloat16 cache: keys and values are each 2^-9 off, scores of a few units
    thus by about 2^-7 and a layer's attention by 2^-6 of itself; two layers 2^-5."""
    lc = ex.lc
    B, n, k, vocab = 5, 37, 6, 500
    pages = torch.arange(B * 4, dtype=torch.int32, device="cuda").flip(0).view(B, 4).contiguous()
    target = ex.Model(vocab, 2, 4, 2, 64, B * 4, 32, 128, seed=1, dtype=torch.float32)
    draft = ex.Model(vocab, 1, 4, 2, 64, B * 4, 32, 128, dtype=torch.float32, first=target)
    g = torch.Generator("cuda").manual_seed(3)
    r = ex.Requests.prompts(target, draft, torch.randint(vocab, (B, n), generator=g, device="cuda"), 128, pages)
    lengths = [r.cached.tolist()]
    for _ in range(6):
        r.step(k)
        lengths.append(r.cached.tolist())
    gained = [b - a for x, y in zip(lengths, lengths[1:]) for a, b in zip(x, y)]
    assert all(1 <= n <= k + 1 for n in gained) and len(set(gained)) > 1      # some drafts stood, some were taken back
    lens = r.cached.tolist()
    # the next token of every sequence, through the caches
    got = target.logits(r.tokens[torch.arange(B, device="cuda"), r.cached.long()],
                        lc.Sequences(torch.arange(B + 1, dtype=torch.int32, device="cuda"), r.cached + 1, pages), 1).double()
    for b in range(B):
        want = plain_logits(target, r.tokens[b:b + 1, :lens[b] + 1])[0, -1]
        assert float((got[b] - want).norm() / want.norm()) < 2.0 ** -5, b


@pytest.mark.parametrize("kv", ["bf16", "fp8", "int8"])
def test_example_runs(ex, kv):
    """The same requests again are served from the cache: their first tokens are decoded alike."""
    assert ex.main(["--requests", "6", "--prompt", "70", "--tokens", "30", "--k", "8", "--vocab", "1000", "--kv", kv]) == 3
