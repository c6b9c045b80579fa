"""A semantic cache in front of speculative decoding, on random weights: what a serving loop does with the decode operators.

    python examples/speculative_decode.py [--requests 16] [--prompt 500] [--tokens 120] [--k 20] [--kv fp8]

Every request's first k tokens are decoded speculatively: a draft model proposes k tokens one at a time, the target model
verifies them in one pass, and lacache_accept_length says how many of them stand.  With these tokens as its lookahead a
request is looked up in the semantic cache; a hit is served, the others are decoded to the end and inserted.  Both models
keep their keys and values in pages.  A rejected token's entry stays in its page until the next token of that position is
written over it, so taking tokens back is a matter of the sequences' lengths, which live on the GPU.
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2608_01718_amd as lc  # noqa: E402

KV = {"bf16": lc.KV_BF16, "fp8": lc.KV_FP8, "int8": lc.KV_INT8}


class Model:
    """Attention layers with residuals, an embedding before and a head after them.  first: a model whose first layers,
    embedding and head are this one's too (a draft model that resembles its target)."""

    def __init__(self, vocab, layers, q_heads, kv_heads, d, n_pages, page, positions, kv="bf16", dtype=torch.bfloat16, seed=0,
                 first=None):
        g = torch.Generator("cuda").manual_seed(seed)
        dim, self.sizes, self.d = q_heads * d, [q_heads * d, kv_heads * d, kv_heads * d], d

        def weight(n, m, size):
            return torch.randn((n, m), generator=g, device="cuda").mul_(size).to(dtype)

        if first is None:
            self.embedding, self.head = weight(vocab, dim, 1.0), weight(dim, vocab, 3 * dim ** -0.5)
            self.layers = [(weight(dim, sum(self.sizes), dim ** -0.5), weight(dim, dim, dim ** -0.5)) for _ in range(layers)]
        else:
            self.embedding, self.head, self.layers = first.embedding, first.head, first.layers[:layers]
        self.caches = [lc.KVCache(n_pages, kv_heads, d, page=page, type=KV[kv]) for _ in range(layers)]
        self.rope = lc.Rope(lc.lacache_rope_table(positions, d))

    def logits(self, tokens, seqs, max_new):
        """tokens [rows]: the newest tokens of the sequences, packed.  Caches them and returns [rows, vocab]."""
        x = self.embedding[tokens]
        for cache, (w_in, w_out) in zip(self.caches, self.layers):
            q, k, v = (y.unflatten(1, (-1, self.d)) for y in (_norm(x) @ w_in).split(self.sizes, 1))
            q = cache.append(k, v, seqs, q=q, rope=self.rope, max_new=max_new)
            o, _ = cache.attend(q, seqs, max_new=max_new)
            x = x + o.flatten(1) @ w_out
        return _norm(x) @ self.head


def _norm(x):
    return x * torch.rsqrt(x.float().square().mean(1, keepdim=True) + 1e-6).to(x.dtype)


class Requests:
    """The sequences that are decoded together: tokens [B, room], `cached` [B] how many of each are in the caches (the next
    token is known, and not cached yet), pages [B, max_pages]."""

    def __init__(self, target, draft, tokens, cached, pages):
        self.target, self.draft, self.tokens, self.cached, self.pages = target, draft, tokens, cached, pages

    @classmethod
    def prompts(cls, target, draft, prompts, room, pages):
        B, n = prompts.shape
        tokens = torch.zeros((B, room), dtype=torch.long, device="cuda")
        tokens[:, :n] = prompts
        r = cls(target, draft, tokens, torch.full((B,), n, dtype=torch.int32, device="cuda"), pages)
        seqs = r._newest(n, r.cached)
        draft.logits(prompts.flatten(), seqs, n)
        r.tokens[:, n] = target.logits(prompts.flatten(), seqs, n).view(B, n, -1)[:, -1].argmax(1)
        return r

    def some(self, which):
        return Requests(self.target, self.draft, self.tokens[which], self.cached[which], self.pages[which].contiguous())

    def _newest(self, new, lens):
        """The newest `new` tokens of every sequence."""
        start = torch.arange(len(lens) + 1, dtype=torch.int32, device="cuda") * new
        return lc.Sequences(start, lens, self.pages)

    def step(self, k):
        """k tokens proposed and verified; the accepted ones, and the target's own next one, are in `tokens` then."""
        B = len(self.cached)
        rows = torch.arange(B, device="cuda")
        at = self.cached.long()
        lens = self.cached.clone()
        one = self._newest(1, lens)
        feed = torch.empty((B, k + 1), dtype=torch.long, device="cuda")
        p_draft = torch.empty((B, k), device="cuda")
        feed[:, 0] = self.tokens[rows, at]
        for i in range(k + 1):  # (the last pass only caches the last draft)
            lens += 1
            out = self.draft.logits(feed[:, i], one, 1)
            if i < k:
                p, feed[:, i + 1] = out.float().softmax(1).max(1)
                p_draft[:, i] = p
        verify = self._newest(k + 1, self.cached + (k + 1))
        out = self.target.logits(feed.flatten(), verify, k + 1).view(B, k + 1, -1)
        accepted, _ = lc.lacache_accept_length(out[:, :k].contiguous(), feed[:, 1:].int().contiguous(), p_draft)
        self.tokens[rows[:, None], at[:, None] + 1 + torch.arange(k, device="cuda")] = feed[:, 1:]
        self.tokens[rows, at + 1 + accepted] = out[rows, accepted.long()].argmax(1)
        self.cached += accepted + 1
        return accepted

    def until(self, length, k):
        """Steps until every sequence has `length` tokens."""
        steps, accepted = 0, 0
        while int(self.cached.min()) + 1 < length:
            accepted += int(self.step(k).sum())
            steps += 1
        return steps, accepted


def main(argv=None):
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    p.add_argument("--requests", type=int, default=16)
    p.add_argument("--prompt", type=int, default=500)
    p.add_argument("--tokens", type=int, default=120)
    p.add_argument("--k", type=int, default=20)
    p.add_argument("--kv", choices=KV, default="bf16")
    p.add_argument("--vocab", type=int, default=32_000)
    a = p.parse_args(argv)
    B, page = a.requests, 64
    # a sequence that is far ahead goes on until the slowest is through: room for k + 1 tokens in each of its steps
    room = a.prompt + (a.k + 1) * (a.tokens + 2)
    each = -(-room // page)
    g = torch.Generator("cuda").manual_seed(7)
    pages = torch.randperm(B * each, generator=g, device="cuda").to(torch.int32).view(B, each)
    target = Model(a.vocab, 4, 16, 4, 128, B * each, page, room, a.kv, seed=1)
    draft = Model(a.vocab, 2, 16, 4, 128, B * each, page, room, a.kv, first=target)
    prompts = torch.randint(a.vocab, (B, a.prompt), generator=g, device="cuda")
    prompts[B // 2:] = prompts[:B - B // 2]                # the second half asks the same again
    # random stand-ins for the query and response embeddings of an embedding model
    table = torch.randn((a.vocab, 384), generator=g, device="cuda")
    embed = lambda t: torch.nn.functional.normalize(table[t].mean(1), dim=1)  # noqa: E731
    cache = lc.LaCache(capacity=1024, d=384, k_cap=a.k, in_dtype=lc.F32, max_batch=max(B, 1))
    served = 0
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    for part in (slice(0, B // 2), slice(B // 2, B)):
        ask = prompts[part]
        if not len(ask):
            continue
        r = Requests.prompts(target, draft, ask, room, pages[part].contiguous())
        steps, accepted = r.until(a.prompt + a.k, a.k)
        first = r.tokens[:, a.prompt:a.prompt + a.k]
        lookahead = first.int().contiguous()
        decision = cache.lookup(embed(ask), embed(first), lookahead, 0.9, 0.85, a.k)[3]
        miss = (decision < lc.HIT).nonzero()[:, 0]
        served += len(ask) - len(miss)
        if len(miss):
            rest = r.some(miss)
            more = rest.until(a.prompt + a.tokens, a.k)
            cache.insert(embed(ask[miss]), embed(first[miss]), lookahead[miss].contiguous())
            steps, accepted = steps + more[0], accepted + more[1]
        print(f"{len(ask)} requests, {len(ask) - len(miss)} served from the cache; {steps} verifications, {accepted} drafts "
              f"accepted", flush=True)
    torch.cuda.synchronize()
    print(f"{time.perf_counter() - t0:.2f} s")
    cache.close()
    return served


if __name__ == "__main__":
    main()
