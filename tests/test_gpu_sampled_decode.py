"""Sampled verification, shared prefixes and chosen pages together, as examples/speculative_decode.py uses them."""
import pytest
import torch

from tests.test_gpu_speculative import plain_logits

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ex():
    from examples import speculative_decode as m
    return m


@pytest.mark.parametrize("temperature,shared,chosen", [(0.0, 32, 0), (0.9, 0, 0), (0.9, 32, 0), (0.9, 0, 4), (0.7, 32, 4), (0.0, 0, 4)])
def test_decoded_tokens_are_the_models(ex, temperature, shared, chosen):
    """After several verifications the caches hold the sequences: the model's logits for their next tokens agree with those of the
    whole sequences in float64 (bfloat16 keys and values are 2^-9 off, two layers 2^-5: as without sharing or choice).  With
    lists of four pages, which is what a table has, choosing changes nothing."""
    lc = ex.lc
    B, n, k, vocab = 5, 37, 6, 500
    pages = torch.arange(B * 4, dtype=torch.int32, device="cuda").flip(0).view(B, 4).contiguous()
    if shared:
        pages[:, 0] = pages[0, 0]
    target = ex.Model(vocab, 2, 4, 2, 64, B * 4, 32, 128, seed=1, dtype=torch.float32, chosen=chosen)
    draft = ex.Model(vocab, 1, 4, 2, 64, B * 4, 32, 128, dtype=torch.float32, first=target, chosen=chosen)
    g = torch.Generator("cuda").manual_seed(3)
    prompts = torch.randint(vocab, (B, n), generator=g, device="cuda")
    prompts[:, :shared] = prompts[:1, :shared].clone()
    r = ex.Requests.prompts(target, draft, prompts, 128, pages, shared, temperature, g)
    lengths = [r.cached.tolist()]
    for _ in range(5):
        r.step(k)
        lengths.append(r.cached.tolist())
    gained = [b - a for x, y in zip(lengths, lengths[1:]) for a, b in zip(x, y)]
    assert all(1 <= n <= k + 1 for n in gained) and len(set(gained)) > 1      # some drafts stood, some were taken back
    lens = r.cached.tolist()
    got = target.logits(r.tokens[torch.arange(B, device="cuda"), r.cached.long()],
                        lc.Sequences(torch.arange(B + 1, dtype=torch.int32, device="cuda"), r.cached + 1, pages), 1, r.prefixes,
                        decode=True).double()
    for b in range(B):
        want = plain_logits(target, r.tokens[b:b + 1, :lens[b] + 1])[0, -1]
        assert float((got[b] - want).norm() / want.norm()) < 2.0 ** -5, b


@pytest.mark.parametrize("options", [["--temperature", "0.8"], ["--instructions", "150"], ["--pages", "2"],
                                     ["--temperature", "0.8", "--instructions", "150", "--pages", "3", "--kv", "fp8"]])
def test_example_runs(ex, options):
    served = ex.main(["--requests", "6", "--prompt", "70", "--tokens", "30", "--k", "8", "--vocab", "1000", *options])
    assert 0 <= served <= 3
