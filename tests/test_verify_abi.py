"""Argument checks of sampled verification: refused before any device work (no GPU needed)."""
import ctypes

import pytest
import torch

EINVAL, FAKE = -1, 1 << 20


@pytest.fixture(scope="module")
def lc():
    import paper_2608_01718_amd as m
    return m


def call(lc, **kw):
    a = dict(logits=FAKE, draft=FAKE, dtype=1, V=100, t_seq=500, t_row=100, d_seq=400, d_row=100, tokens=FAKE, u=FAKE,
             u_next=FAKE, temperature=FAKE, n_draft=FAKE, B=2, k=4, accept_len=FAKE, next_token=FAKE, p=FAKE, q=FAKE,
             workspace=FAKE, bytes=1 << 40, stream=None)
    a.update(kw)
    return lc.raw_library().lacache_verify(*a.values())


@pytest.mark.parametrize("bad", [
    dict(dtype=2), dict(V=0), dict(B=-1), dict(B=65536), dict(k=-1), dict(k=4097), dict(t_seq=-1), dict(t_row=-1),
    dict(d_seq=-1), dict(d_row=-1), dict(bytes=-1), dict(logits=0), dict(draft=0), dict(tokens=0), dict(u=0), dict(u_next=0),
    dict(accept_len=0), dict(next_token=0), dict(p=0), dict(q=0), dict(workspace=0), dict(workspace=FAKE + 8),
    dict(logits=FAKE + 1), dict(draft=FAKE + 1), dict(dtype=0, logits=FAKE + 2), dict(tokens=FAKE + 2), dict(u=FAKE + 1),
    dict(u_next=FAKE + 2), dict(temperature=FAKE + 2), dict(n_draft=FAKE + 1), dict(p=FAKE + 2), dict(q=FAKE + 2),
    dict(accept_len=FAKE + 2), dict(next_token=FAKE + 2), dict(bytes=16), dict(B=65535, V=2 ** 20)])
def test_refused(lc, bad):
    assert call(lc, **bad) == EINVAL


def test_nothing_to_do(lc):
    assert call(lc, B=0, logits=0, draft=0, workspace=0, bytes=0) == 0


def test_workspace(lc):
    for bad in ((0, 1, 1), (10, -1, 1), (10, 65536, 1), (10, 1, -1), (10, 1, 4097)):
        with pytest.raises(lc.LaCacheError):
            lc.lacache_verify_workspace(*bad)
    assert lc.lacache_verify_workspace(1000, 0, 5) == 0
    need = lc.lacache_verify_workspace(128_256, 64, 20)
    assert 0 < need < 2 ** 22
    assert call(lc, V=128_256, B=64, k=20, bytes=need - 1) == EINVAL


def test_binding_wants_gpu_tensors(lc):
    x = torch.zeros((2, 5, 7))
    with pytest.raises(ValueError):
        lc.lacache_verify(x, x[:, :4], torch.zeros((2, 4), dtype=torch.int32), torch.zeros((2, 4)), torch.zeros(2))
    assert ctypes.sizeof(ctypes.c_void_p) == 8


@pytest.mark.parametrize("out", ["accept_len", "next_token", "p", "q"])
def test_outputs_that_overlap(lc, out):
    at = {name: FAKE + 4096 * i for i, name in enumerate(
        ("tokens", "u", "u_next", "temperature", "n_draft", "accept_len", "next_token", "p", "q"))}
    for name in at:
        if name != out:
            for shift in (0, -4, 4):  # (two numbers or eight each)
                assert call(lc, **{**at, out: at[name] + shift}) == EINVAL


WRITTEN = ["accept_len", "next_token", "p", "q", "workspace"]


@pytest.mark.parametrize("out", WRITTEN)
@pytest.mark.parametrize("rows", ["logits", "draft"])
def test_outputs_in_the_logits(lc, out, rows):
    """Any byte of any row, first or last, of either model; rows and sequences apart, together, and in any order."""
    far = {name: (1 << 40) + (1 << 24) * i for i, name in enumerate(("tokens", "u", "u_next", "temperature", "n_draft",
                                                                      "logits", "draft", *WRITTEN))}
    k = 4 if rows == "draft" else 5                        # rows of a sequence
    at = 1 << 30
    for t_seq, t_row in ((k * 100, 100), (100_000, 1000), (100, 5000), (0, 0), (0, 128), (1 << 12, 0), (1 << 40, 1 << 20)):
        strides = dict(d_seq=t_seq, d_row=t_row) if rows == "draft" else dict(t_seq=t_seq, t_row=t_row)
        for b in range(3):
            for j in range(k):
                row = at + 2 * (b * t_seq + j * t_row)
                for x in (row, row + 96, row + 192):       # (200 bytes a row)
                    assert call(lc, **{**far, rows: at, out: x, "B": 3, **strides}) == EINVAL


@pytest.mark.parametrize("out", WRITTEN[:4])
def test_outputs_in_the_workspace(lc, out):
    far = {name: (1 << 40) + (1 << 24) * i for i, name in enumerate(("tokens", "u", "u_next", "temperature", "n_draft",
                                                                      "logits", "draft", *WRITTEN))}
    need = lc.lacache_verify_workspace(100, 2, 4)
    for name in (out, "tokens", "u", "u_next", "temperature", "n_draft"):
        for shift in (0, 16, need - 4):
            assert call(lc, **{**far, name: far["workspace"] + shift}) == EINVAL


def test_strides_beyond_64_bits(lc):
    far = {name: (1 << 40) + (1 << 24) * i for i, name in enumerate(("tokens", "u", "u_next", "temperature", "n_draft",
                                                                      "logits", "draft", *WRITTEN))}
    for bad in ("t_seq", "t_row", "d_seq", "d_row"):
        assert call(lc, **{**far, bad: 1 << 62}) == EINVAL
