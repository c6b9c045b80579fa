"""Python binding of liblacache (the gfx950 LaCache two-stage lookup): argument marshalling only.

Every function mirrors one entry point of ``include/lacache.h`` under the
same name and passes torch device tensors' data pointers and the current HIP
stream straight through; all work runs in the library's kernels.  There is no
fallback: importing this module fails if ``liblacache.so`` has not been built
(``python paper_2608_01718_amd/build.py``).
"""
from __future__ import annotations

import ctypes
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "liblacache.so")

MISS, REJECT, HIT, HIT_EXACT = 0, 1, 2, 3
OK, EINVAL, EFULL, ENOMEM, EHIP = 0, -1, -2, -3, -4
F32, BF16 = 0, 1
MAX_MODELS = 8
KV_BF16, KV_FP8, KV_INT8 = 1, 2, 3
ROPE_HALF, ROPE_PAIRS = 0, 1

if not os.path.exists(LIB_PATH):
    raise ImportError(f"{LIB_PATH} is missing: build it with `python paper_2608_01718_amd/build.py` "
                      "(there is no non-HIP implementation of the lookup)")

_lib = ctypes.CDLL(LIB_PATH)
_P, _i32, _i64, _f32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float
_lib.lacache_create.argtypes = [ctypes.POINTER(_P), _i64, _i32, _i32, ctypes.c_int, _i32, _i32]
_lib.lacache_create_ensemble.argtypes = [ctypes.POINTER(_P), _i64, _i32, _i32, ctypes.c_int, _i32, _i32, _i32,
                                         ctypes.POINTER(_i32)]
_lib.lacache_models.argtypes = [_P]
_lib.lacache_models.restype = _i32
_lib.lacache_insert_ensemble.argtypes = [_P, _P, ctypes.POINTER(_P), _P, _i32, ctypes.POINTER(_i64), _P]
_lib.lacache_lookup_ensemble.argtypes = [_P, _P, ctypes.POINTER(_P), _P, _i32, _f32, ctypes.POINTER(_f32), _i32,
                                         _P, _P, _P, _P, _P]
_lib.lacache_export_prefix.argtypes = [_P, _i32, _i64, _i32, _P, _P]
_lib.lacache_calibrate.argtypes = [_P, _i32, _P, _P, _i64, _f32, _f32, _P, _P, _P]
_lib.lacache_calibrate_noalloc.argtypes = [_P, _P, ctypes.c_int, _i32, _i64, _f32, _f32, _P, _P, _P]
_lib.lacache_accept_length.argtypes = [_P, ctypes.c_int, _i32, _P, _P, _i32, _i32, _P, _P, _P]
_lib.lacache_enable_lsh.argtypes = [_P, _i32, _P, _i32, _P]
_lib.lacache_lookup_lsh.argtypes = [_P, _P, _P, _P, _i32, _f32, _f32, _i32, _i32, _P, _P, _P, _P, _P, _P]
_lib.lacache_export_signatures.argtypes = [_P, _i64, _i32, _P, _P]
_lib.lacache_destroy.argtypes = [_P]
_lib.lacache_insert.argtypes = [_P, _P, _P, _P, _i32, ctypes.POINTER(_i64), _P]
_lib.lacache_lookup.argtypes = [_P, _P, _P, _P, _i32, _f32, _f32, _i32, _P, _P, _P, _P, _P]
_lib.lacache_size.argtypes = [_P]
_lib.lacache_size.restype = _i64
_lib.lacache_export.argtypes = [_P, _i64, _i32, _P, _P, _P, _P]
_lib.lacache_set_small_batch.argtypes = [_P, _i32]
_lib.lacache_profile.argtypes = [_P, _i32]
_lib.lacache_profile_read.argtypes = [_P, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(_i64)]
_lib.lacache_replay_fallbacks.argtypes = [_P, ctypes.POINTER(_i64)]


class _KV(ctypes.Structure):
    _fields_ = [("k", _P), ("v", _P), ("k_scale", _P), ("v_scale", _P), ("n_pages", _i64), ("page", _i32),
                ("heads", _i32), ("d", _i32), ("type", ctypes.c_int)]


class _Seqs(ctypes.Structure):
    _fields_ = [("start", _P), ("lens", _P), ("pages", _P), ("n_seq", _i32), ("max_pages", _i32)]


class _Bounds(ctypes.Structure):
    _fields_ = [("code", _P), ("scale", _P)]


class _Prefixes(ctypes.Structure):
    _fields_ = [("group", _P), ("len", _P), ("n_groups", _i32)]


class _Rotary(ctypes.Structure):
    _fields_ = [("table", _P), ("n_pos", _i64), ("rot", _i32), ("style", ctypes.c_int)]


_f64 = ctypes.c_double
_lib.lacache_rope_table.argtypes = [_P, _i64, _i64, _i32, _f64, _f64, _f64, _f64, _f64, _f64, _P]
_lib.lacache_rope.argtypes = [_P, _P, ctypes.c_int, _i64, _i32, _i32, _i64, _i64, _i64, _i64, _P, _P, _i32, _P]
_lib.lacache_kv_append.argtypes = [_P, _P, _P, _P, ctypes.c_int, _i64, _i64, _i64, _P, _P, _i32, _i64, _P, _i32, _P]
_lib.lacache_kv_read.argtypes = [_P, _P, _P, _P, ctypes.c_int, _i64, _i32, _P]
_lib.lacache_kv_attend_workspace.argtypes = [_P, ctypes.c_int, _i32, _i32, _i32]
_lib.lacache_kv_attend_workspace.restype = _i64
_lib.lacache_kv_attend.argtypes = [_P, _P, _P, ctypes.c_int, _i64, _i32, _i64, _i32, _f32, _i32, _P, _P, _P, _i64, _P]
_lib.lacache_kv_attend_shared_workspace.argtypes = [_P, ctypes.c_int, _i64, _i32, _i32, _i32, _i32]
_lib.lacache_kv_attend_shared_workspace.restype = _i64
_lib.lacache_kv_attend_shared.argtypes = [_P, _P, _P, _P, ctypes.c_int, _i64, _i32, _i64, _i32, _f32, _i32, _P, _P, _P, _i64,
                                          _P]
_lib.lacache_kv_bound.argtypes = [_P, _P, _P, _i64, _i32, _P]
_lib.lacache_kv_bounds_read.argtypes = [_P, _P, _P, _i64, _P, _P, _P]
_lib.lacache_kv_select_workspace.argtypes = [_P, _i64, _i32]
_lib.lacache_kv_select_workspace.restype = _i64
_lib.lacache_kv_select.argtypes = [_P, _P, _P, _P, ctypes.c_int, _i64, _i32, _i64, _i32, _i32, _i32, _i32, _P, _P, _i64, _P]
_lib.lacache_kv_attend_blocks_workspace.argtypes = [_P, _i64, _i32, _i32]
_lib.lacache_kv_attend_blocks_workspace.restype = _i64
_lib.lacache_kv_attend_blocks.argtypes = [_P, _P, _P, ctypes.c_int, _i64, _i32, _i64, _P, _i32, _f32, _P, _P, _P, _i64, _P]
_lib.lacache_verify_workspace.argtypes = [_i32, _i32, _i32]
_lib.lacache_verify_workspace.restype = _i64
_lib.lacache_verify.argtypes = [_P, _P, ctypes.c_int, _i32, _i64, _i64, _i64, _i64, _P, _P, _P, _P, _P, _i32, _i32, _P, _P,
                                _P, _P, _P, _i64, _P]
_lib.lacache_strerror.argtypes = [ctypes.c_int]
_lib.lacache_strerror.restype = ctypes.c_char_p

EXPORTED = ("lacache_create", "lacache_create_ensemble", "lacache_models", "lacache_destroy", "lacache_insert",
            "lacache_insert_ensemble", "lacache_lookup", "lacache_lookup_ensemble", "lacache_size",
            "lacache_export", "lacache_export_prefix", "lacache_calibrate", "lacache_calibrate_noalloc",
            "lacache_accept_length",
            "lacache_enable_lsh", "lacache_lookup_lsh", "lacache_export_signatures",
            "lacache_set_small_batch",
            "lacache_profile", "lacache_profile_read", "lacache_replay_fallbacks", "lacache_strerror",
            "lacache_rope_table", "lacache_rope", "lacache_kv_append", "lacache_kv_read",
            "lacache_kv_attend_workspace", "lacache_kv_attend", "lacache_verify_workspace", "lacache_verify",
            "lacache_kv_attend_shared_workspace", "lacache_kv_attend_shared", "lacache_kv_bound", "lacache_kv_bounds_read",
            "lacache_kv_select_workspace", "lacache_kv_select",
            "lacache_kv_attend_blocks_workspace", "lacache_kv_attend_blocks")


class LaCacheError(RuntimeError):
    def __init__(self, code: int, what: str):
        super().__init__(f"{what}: {lacache_strerror(code)} ({code})")
        self.code = code


def lacache_strerror(code: int) -> str:
    return _lib.lacache_strerror(code).decode()


def _check(code: int, what: str) -> None:
    if code != OK:
        raise LaCacheError(code, what)


def _stream(device: int, stream) -> int:
    if stream is None:
        stream = torch.cuda.current_stream(device)
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _vec(t: torch.Tensor, dtype: int, rows: int, d: int, device: int, name: str) -> int:
    want = (torch.float32,) if dtype == F32 else (torch.bfloat16, torch.int16, torch.uint16)
    if t.dtype not in want or t.device.type != "cuda" or t.device.index != device:
        raise ValueError(f"{name}: expected a {want} tensor on cuda:{device}, got {t.dtype} on {t.device}")
    if tuple(t.shape) != (rows, d) or not t.is_contiguous():
        raise ValueError(f"{name}: expected a contiguous [{rows}, {d}] tensor, got {tuple(t.shape)}")
    return t.data_ptr()


def _ints(t: torch.Tensor, shape, device: int, name: str) -> int:
    if t.dtype != torch.int32 or t.device.type != "cuda" or t.device.index != device:
        raise ValueError(f"{name}: expected an int32 tensor on cuda:{device}")
    if tuple(t.shape) != tuple(shape) or not t.is_contiguous():
        raise ValueError(f"{name}: expected a contiguous {list(shape)} tensor, got {tuple(t.shape)}")
    return t.data_ptr()


class LaCache:
    """A handle of the C library plus the sizes it was created with.  ``d_resp`` (one dimension per prefix
    model) makes an ensemble cache through lacache_create_ensemble; without it the cache has one prefix
    model of dimension d."""

    def __init__(self, capacity: int, d: int, k_cap: int, in_dtype: int = BF16, max_batch: int = 4096,
                 device: int = 0, d_resp=None):
        self.capacity, self.d, self.k_cap, self.in_dtype = capacity, d, k_cap, in_dtype
        self.max_batch, self.device = max_batch, device
        h = _P()
        if d_resp is None:
            self.d_resp = (d,)
            _check(_lib.lacache_create(ctypes.byref(h), capacity, d, k_cap, in_dtype, max_batch, device),
                   "lacache_create")
        else:
            self.d_resp = tuple(int(x) for x in d_resp)
            arr = (_i32 * max(1, len(self.d_resp)))(*self.d_resp)
            _check(_lib.lacache_create_ensemble(ctypes.byref(h), capacity, d, k_cap, in_dtype, max_batch, device,
                                                len(self.d_resp), arr), "lacache_create_ensemble")
        self._h = h

    @property
    def m(self) -> int:
        return len(self.d_resp)

    @property
    def handle(self):
        if self._h is None:
            raise ValueError("the cache has been destroyed")
        return self._h

    def insert(self, keys, resp_emb, resp_tokens, stream=None) -> int:
        return lacache_insert(self, keys, resp_emb, resp_tokens, stream)

    def lookup(self, queries, lookahead_emb, lookahead_tokens, tau_q, tau_r, k, out=None, stream=None):
        return lacache_lookup(self, queries, lookahead_emb, lookahead_tokens, tau_q, tau_r, k, out, stream)

    def export(self, first: int, n: int, stream=None):
        return lacache_export(self, first, n, stream)

    def insert_ensemble(self, keys, resp_embs, resp_tokens, stream=None) -> int:
        return lacache_insert_ensemble(self, keys, resp_embs, resp_tokens, stream)

    def lookup_ensemble(self, queries, lookahead_embs, lookahead_tokens, tau_q, tau_r, k, out=None, stream=None):
        return lacache_lookup_ensemble(self, queries, lookahead_embs, lookahead_tokens, tau_q, tau_r, k, out,
                                       stream)

    def export_prefix(self, model: int, first: int, n: int, stream=None):
        return lacache_export_prefix(self, model, first, n, stream)

    def enable_lsh(self, bits: int, hyperplanes, max_candidates: int = 256, stream=None) -> None:
        lacache_enable_lsh(self, bits, hyperplanes, max_candidates, stream)

    def lookup_lsh(self, queries, lookahead_emb, lookahead_tokens, tau_q, tau_r, k, radius, out=None, stream=None):
        return lacache_lookup_lsh(self, queries, lookahead_emb, lookahead_tokens, tau_q, tau_r, k, radius, out,
                                  stream)

    def export_signatures(self, first: int, n: int, stream=None):
        return lacache_export_signatures(self, first, n, stream)

    def calibrate(self, a, b, percentile: float, cap: float, which: int = -1, out=None, stream=None):
        return lacache_calibrate(self, which, a, b, percentile, cap, out, stream)

    def size(self) -> int:
        return lacache_size(self)

    def set_small_batch(self, b_small: int) -> None:
        lacache_set_small_batch(self, b_small)

    def profile(self, every) -> None:
        lacache_profile(self, every)

    def profile_read(self):
        return lacache_profile_read(self)

    def replay_fallbacks(self) -> int:
        return lacache_replay_fallbacks(self)

    def close(self) -> None:
        if getattr(self, "_h", None) is not None:
            lacache_destroy(self)

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def lacache_create(capacity: int, d: int, k_cap: int, in_dtype: int = BF16, max_batch: int = 4096,
                   device: int = 0) -> LaCache:
    return LaCache(capacity, d, k_cap, in_dtype, max_batch, device)


def lacache_create_ensemble(capacity: int, d: int, k_cap: int, in_dtype: int, max_batch: int, device: int,
                            d_resp) -> LaCache:
    return LaCache(capacity, d, k_cap, in_dtype, max_batch, device, d_resp=d_resp)


def lacache_models(c: LaCache) -> int:
    return int(_lib.lacache_models(c.handle))


def lacache_destroy(c: LaCache) -> None:
    h, c._h = c._h, None
    _check(_lib.lacache_destroy(h), "lacache_destroy")


def lacache_insert(c: LaCache, keys, resp_emb, resp_tokens, stream=None) -> int:
    n = keys.shape[0]
    first = _i64(-1)
    _check(_lib.lacache_insert(c.handle, _vec(keys, c.in_dtype, n, c.d, c.device, "keys"),
                               _vec(resp_emb, c.in_dtype, n, c.d, c.device, "resp_emb"),
                               _ints(resp_tokens, (n, c.k_cap), c.device, "resp_tokens"), n, ctypes.byref(first),
                               _stream(c.device, stream)), "lacache_insert")
    return first.value


def lacache_insert_ensemble(c: LaCache, keys, resp_embs, resp_tokens, stream=None) -> int:
    """resp_embs: one [n][d_resp[i]] tensor per prefix model."""
    n = keys.shape[0]
    if len(resp_embs) != c.m:
        raise ValueError(f"resp_embs: expected {c.m} tensors, got {len(resp_embs)}")
    ptrs = (_P * c.m)(*[_vec(e, c.in_dtype, n, c.d_resp[i], c.device, f"resp_embs[{i}]")
                         for i, e in enumerate(resp_embs)])
    first = _i64(-1)
    _check(_lib.lacache_insert_ensemble(c.handle, _vec(keys, c.in_dtype, n, c.d, c.device, "keys"), ptrs,
                                        _ints(resp_tokens, (n, c.k_cap), c.device, "resp_tokens"), n,
                                        ctypes.byref(first), _stream(c.device, stream)), "lacache_insert_ensemble")
    return first.value


def lacache_lookup_ensemble(c: LaCache, queries, lookahead_embs, lookahead_tokens, tau_q: float, tau_r, k: int,
                            out=None, stream=None):
    """lookahead_embs: one [B][d_resp[i]] tensor per prefix model; tau_r: one threshold per model.
    Returns (idx int32 [B], score f32 [B], resp_score f32 [B][m], decision int32 [B])."""
    B = queries.shape[0]
    m = c.m
    dev = torch.device("cuda", c.device)
    if len(lookahead_embs) != m or len(tau_r) != m:
        raise ValueError(f"expected {m} lookahead embeddings and {m} thresholds")
    if out is None:
        out = (torch.empty(B, dtype=torch.int32, device=dev), torch.empty(B, dtype=torch.float32, device=dev),
               torch.empty((B, m), dtype=torch.float32, device=dev), torch.empty(B, dtype=torch.int32, device=dev))
    idx, score, resp, dec = out
    for t, dt, n, nm in ((idx, torch.int32, B, "idx"), (score, torch.float32, B, "score"),
                         (resp, torch.float32, B * m, "resp"), (dec, torch.int32, B, "decision")):
        if t.dtype != dt or t.device != dev or t.numel() != n or not t.is_contiguous():
            raise ValueError(f"{nm}: expected a contiguous {dt} tensor of {n} elements on {dev}")
    ptrs = (_P * m)(*[_vec(e, c.in_dtype, B, c.d_resp[i], c.device, f"lookahead_embs[{i}]")
                      for i, e in enumerate(lookahead_embs)])
    taus = (_f32 * m)(*[float(t) for t in tau_r])
    _check(_lib.lacache_lookup_ensemble(c.handle, _vec(queries, c.in_dtype, B, c.d, c.device, "queries"), ptrs,
                                        _ints(lookahead_tokens, (B, k), c.device, "lookahead_tokens"), B,
                                        float(tau_q), taus, int(k), idx.data_ptr(), score.data_ptr(),
                                        resp.data_ptr(), dec.data_ptr(), _stream(c.device, stream)),
           "lacache_lookup_ensemble")
    return out


def lacache_lookup(c: LaCache, queries, lookahead_emb, lookahead_tokens, tau_q: float, tau_r: float, k: int,
                   out=None, stream=None):
    """Returns (idx int32, score f32, resp_score f32, decision int32), each [B], on the cache's device."""
    B = queries.shape[0]
    dev = torch.device("cuda", c.device)
    if out is None:
        out = (torch.empty(B, dtype=torch.int32, device=dev), torch.empty(B, dtype=torch.float32, device=dev),
               torch.empty(B, dtype=torch.float32, device=dev), torch.empty(B, dtype=torch.int32, device=dev))
    idx, score, resp, dec = out
    for t, dt, nm in ((idx, torch.int32, "idx"), (score, torch.float32, "score"), (resp, torch.float32, "resp"),
                      (dec, torch.int32, "decision")):
        if t.dtype != dt or t.device != dev or t.numel() != B or not t.is_contiguous():
            raise ValueError(f"{nm}: expected a contiguous [{B}] {dt} tensor on {dev}")
    _check(_lib.lacache_lookup(c.handle, _vec(queries, c.in_dtype, B, c.d, c.device, "queries"),
                               _vec(lookahead_emb, c.in_dtype, B, c.d, c.device, "lookahead_emb"),
                               _ints(lookahead_tokens, (B, k), c.device, "lookahead_tokens"), B, float(tau_q),
                               float(tau_r), int(k), idx.data_ptr(), score.data_ptr(), resp.data_ptr(),
                               dec.data_ptr(), _stream(c.device, stream)), "lacache_lookup")
    return out


def lacache_size(c: LaCache) -> int:
    return int(_lib.lacache_size(c.handle))


def lacache_export(c: LaCache, first: int, n: int, stream=None):
    """Returns (keys bf16-bits int16 [n][d], emb int16 [n][d], tokens int32 [n][k_cap]) as stored."""
    dev = torch.device("cuda", c.device)
    keys = torch.empty((n, c.d), dtype=torch.int16, device=dev)
    emb = torch.empty((n, c.d_resp[0]), dtype=torch.int16, device=dev)
    tok = torch.empty((n, c.k_cap), dtype=torch.int32, device=dev)
    _check(_lib.lacache_export(c.handle, first, n, keys.data_ptr(), emb.data_ptr(), tok.data_ptr(),
                               _stream(c.device, stream)), "lacache_export")
    return keys, emb, tok


def lacache_export_prefix(c: LaCache, model: int, first: int, n: int, stream=None):
    """The stored prefix embeddings of one model, bf16 bits as int16 [n][d_resp[model]]."""
    if not 0 <= model < c.m:
        raise ValueError(f"model must be in [0, {c.m})")
    emb = torch.empty((n, c.d_resp[model]), dtype=torch.int16, device=torch.device("cuda", c.device))
    _check(_lib.lacache_export_prefix(c.handle, model, first, n, emb.data_ptr(), _stream(c.device, stream)),
           "lacache_export_prefix")
    return emb


def lacache_calibrate(c: LaCache, which: int, a, b, percentile: float, cap: float, out=None, stream=None):
    """Pair cosines and the capped percentile threshold (Appendix A.2).  which = -1: key-model vectors of
    dimension d; else prefix model `which`.  Returns (sims f32 [n], tau f32 [2] = (percentile, min(cap, .)))
    on the cache's device."""
    # an out-of-range `which` is passed through for the library to reject
    dim = c.d_resp[which] if 0 <= which < c.m else (c.d if which == -1 else a.shape[1])
    n = a.shape[0]
    dev = torch.device("cuda", c.device)
    if out is None:
        out = (torch.empty(n, dtype=torch.float32, device=dev), torch.empty(2, dtype=torch.float32, device=dev))
    sims, tau = out
    for t, k, nm in ((sims, n, "sims"), (tau, 2, "tau")):
        if t.dtype != torch.float32 or t.device != dev or t.numel() != k or not t.is_contiguous():
            raise ValueError(f"{nm}: expected a contiguous float32 tensor of {k} elements on {dev}")
    _check(_lib.lacache_calibrate(c.handle, int(which), _vec(a, c.in_dtype, n, dim, c.device, "a"),
                                  _vec(b, c.in_dtype, n, dim, c.device, "b"), n, float(percentile), float(cap),
                                  sims.data_ptr(), tau.data_ptr(), _stream(c.device, stream)), "lacache_calibrate")
    return out


def lacache_calibrate_noalloc(a, b, percentile: float, cap: float, out=None, stream=None):
    """lacache_calibrate without a handle, with the library's static scratch: a, b [n][d] float32 or bfloat16
    (int16/uint16 bits) on the current device.  Returns (sims f32 [n], tau f32 [2]); with `out` given no device
    memory is allocated here either."""
    if a.dim() != 2 or a.shape != b.shape or a.dtype != b.dtype:
        raise ValueError("a, b: expected two [n, d] tensors of one dtype")
    dtype = F32 if a.dtype == torch.float32 else BF16
    n, d = a.shape
    dev = a.device
    if out is None:
        out = (torch.empty(n, dtype=torch.float32, device=dev), torch.empty(2, dtype=torch.float32, device=dev))
    sims, tau = out
    for t, k, nm in ((sims, n, "sims"), (tau, 2, "tau")):
        if t.dtype != torch.float32 or t.device != dev or t.numel() != k or not t.is_contiguous():
            raise ValueError(f"{nm}: expected a contiguous float32 tensor of {k} elements on {dev}")
    _check(_lib.lacache_calibrate_noalloc(_vec(a, dtype, n, d, dev.index, "a"), _vec(b, dtype, n, d, dev.index, "b"),
                                          dtype, d, n, float(percentile), float(cap), sims.data_ptr(),
                                          tau.data_ptr(), _stream(dev.index, stream)),
           "lacache_calibrate_noalloc")
    return out


def lacache_accept_length(logits, draft_tokens, p_draft, out=None, stream=None):
    """Speculative-decoding acceptance (Section 4.3).  logits: [B][k][V] float32 or bfloat16 (int16/uint16
    bits) on a GPU; draft_tokens [B][k] int32; p_draft [B][k] float32.  Returns (accept_len int32 [B],
    p_target float32 [B][k]) on the same device."""
    if logits.dim() != 3 or logits.device.type != "cuda" or not logits.is_contiguous():
        raise ValueError("logits: expected a contiguous [B, k, V] tensor on a GPU")
    B, k, V = logits.shape
    dtype = F32 if logits.dtype == torch.float32 else BF16
    if dtype == BF16 and logits.dtype not in (torch.bfloat16, torch.int16, torch.uint16):
        raise ValueError(f"logits: unsupported dtype {logits.dtype}")
    dev = logits.device
    for t, dt, nm in ((draft_tokens, torch.int32, "draft_tokens"), (p_draft, torch.float32, "p_draft")):
        if t.dtype != dt or t.device != dev or tuple(t.shape) != (B, k) or not t.is_contiguous():
            raise ValueError(f"{nm}: expected a contiguous [{B}, {k}] {dt} tensor on {dev}")
    if out is None:
        out = (torch.empty(B, dtype=torch.int32, device=dev), torch.empty((B, k), dtype=torch.float32, device=dev))
    acc, pt = out
    if acc.dtype != torch.int32 or acc.numel() != B or pt.dtype != torch.float32 or pt.numel() != B * k:
        raise ValueError("out: expected (int32 [B], float32 [B, k])")
    if acc.device != dev or pt.device != dev:
        raise ValueError(f"out: expected tensors on {dev}")
    with torch.cuda.device(dev):  # the entry point runs on the calling thread's current device
        _check(_lib.lacache_accept_length(logits.data_ptr(), dtype, V, draft_tokens.data_ptr(), p_draft.data_ptr(),
                                          B, k, acc.data_ptr(), pt.data_ptr(), _stream(dev.index, stream)),
               "lacache_accept_length")
    return out


def lacache_enable_lsh(c: LaCache, bits: int, hyperplanes, max_candidates: int = 256, stream=None) -> None:
    """hyperplanes: [bits][d] bfloat16 (or int16/uint16 bits) on the cache's device."""
    hp = _vec(hyperplanes, BF16, bits, c.d, c.device, "hyperplanes")
    _check(_lib.lacache_enable_lsh(c.handle, int(bits), hp, int(max_candidates), _stream(c.device, stream)),
           "lacache_enable_lsh")
    c.lsh_bits = int(bits)


def lacache_lookup_lsh(c: LaCache, queries, lookahead_emb, lookahead_tokens, tau_q: float, tau_r: float, k: int,
                       radius: int, out=None, stream=None):
    """Returns (idx int32, score f32, resp_score f32, decision int32, n_cand int32), each [B]."""
    B = queries.shape[0]
    dev = torch.device("cuda", c.device)
    if out is None:
        out = (torch.empty(B, dtype=torch.int32, device=dev), torch.empty(B, dtype=torch.float32, device=dev),
               torch.empty(B, dtype=torch.float32, device=dev), torch.empty(B, dtype=torch.int32, device=dev),
               torch.empty(B, dtype=torch.int32, device=dev))
    for t, dt, nm in zip(out, (torch.int32, torch.float32, torch.float32, torch.int32, torch.int32),
                         ("idx", "score", "resp", "decision", "n_cand")):
        if t.dtype != dt or t.device != dev or t.numel() != B or not t.is_contiguous():
            raise ValueError(f"{nm}: expected a contiguous [{B}] {dt} tensor on {dev}")
    _check(_lib.lacache_lookup_lsh(c.handle, _vec(queries, c.in_dtype, B, c.d, c.device, "queries"),
                                   _vec(lookahead_emb, c.in_dtype, B, c.d, c.device, "lookahead_emb"),
                                   _ints(lookahead_tokens, (B, k), c.device, "lookahead_tokens"), B, float(tau_q),
                                   float(tau_r), int(k), int(radius), *(t.data_ptr() for t in out),
                                   _stream(c.device, stream)), "lacache_lookup_lsh")
    return out


def lacache_export_signatures(c: LaCache, first: int, n: int, stream=None):
    """The stored LSH signatures as int32 bit patterns [n][bits / 32] (view as uint32 on the host)."""
    bits = getattr(c, "lsh_bits", 0)
    if not bits:
        raise ValueError("the LSH index is not enabled")
    sig = torch.empty((n, bits // 32), dtype=torch.int32, device=torch.device("cuda", c.device))
    _check(_lib.lacache_export_signatures(c.handle, first, n, sig.data_ptr(), _stream(c.device, stream)),
           "lacache_export_signatures")
    return sig


def lacache_set_small_batch(c: LaCache, b_small: int) -> None:
    _check(_lib.lacache_set_small_batch(c.handle, b_small), "lacache_set_small_batch")


def lacache_profile(c: LaCache, every) -> None:
    """Time every `every`-th stage-1 launch from now on (True: every launch; False or 0: stop)."""
    n = int(every)  # True -> 1, False -> 0
    _check(_lib.lacache_profile(c.handle, n), "lacache_profile")


def lacache_profile_read(c: LaCache):
    """(total stage-1 milliseconds, number of launches timed) since profiling was enabled or last read."""
    ms, n = ctypes.c_double(0), _i64(0)
    _check(_lib.lacache_profile_read(c.handle, ctypes.byref(ms), ctypes.byref(n)), "lacache_profile_read")
    return ms.value, n.value


def lacache_replay_fallbacks(c: LaCache) -> int:
    """Queries since create whose large-batch group replay did not reproduce their stage-1 score (0 in correct
    operation); synchronises the device."""
    n = _i64(0)
    _check(_lib.lacache_replay_fallbacks(c.handle, ctypes.byref(n)), "lacache_replay_fallbacks")
    return n.value


_KV_DTYPES = {KV_BF16: torch.bfloat16, KV_FP8: torch.float8_e4m3fn, KV_INT8: torch.int8}
_KV_TYPES = {t: k for k, t in _KV_DTYPES.items()}
_ROW_DTYPES = {torch.float32: F32, torch.bfloat16: BF16}


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)  # (torch.cuda.current_stream takes a microsecond more)


def _on(index: int, stream, f, *args) -> int:
    """f(*args, stream) with GPU `index` as the calling thread's current device."""
    raw = _raw_stream(index) if stream is None and _raw_stream is not None else _stream(index, stream)
    if torch.cuda.current_device() == index:
        return f(*args, raw)
    with torch.cuda.device(index):
        return f(*args, raw)


def _rows(t: torch.Tensor, heads: int, d: int, index: int, dtype, name: str) -> int:
    """The row stride of [rows, heads, d] activations whose rows are each contiguous."""
    if t.dtype != dtype or t.get_device() != index:
        raise ValueError(f"{name}: expected a {dtype} tensor on cuda:{index}, got {t.dtype} on {t.device}")
    shape, stride = t.shape, t.stride()
    if len(shape) != 3 or shape[1] != heads or shape[2] != d or (
            shape[0] and ((d > 1 and stride[2] != 1) or (heads > 1 and stride[1] != d))):
        raise ValueError(f"{name}: expected [rows, {heads}, {d}] with contiguous rows, got {tuple(shape)} with strides "
                         f"{stride}")
    return stride[0]


def _made(like: torch.Tensor, shape, dtype, stream, zeros=False):
    """An empty (or zero) tensor on the GPU of `like` that belongs to the stream the call runs on."""
    make = like.new_zeros if zeros else like.new_empty
    if stream is None:
        return make(shape, dtype=dtype)
    if not isinstance(stream, torch.cuda.Stream):
        handle = stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)
        stream = torch.cuda.ExternalStream(handle, device=like.device) if handle else \
            torch.cuda.default_stream(like.device)
    with torch.cuda.stream(stream):
        return make(shape, dtype=dtype)


def _capturing(index: int, stream) -> bool:
    """Whether the stream of the call is recording a graph."""
    handle = _stream(index, stream)
    with torch.cuda.stream(torch.cuda.ExternalStream(handle, device=index) if handle else torch.cuda.default_stream(index)):
        return torch.cuda.is_current_stream_capturing()


def _given(t: torch.Tensor, shape, dtype, index: int, name: str) -> torch.Tensor:
    if t.dtype != dtype or t.get_device() != index or t.shape != (shape if type(shape) is torch.Size else torch.Size(shape)) or \
            not t.is_contiguous():
        raise ValueError(f"{name}: expected a contiguous {list(shape)} {dtype} tensor on cuda:{index}")
    return t


_written = torch.autograd.graph.increment_version  # what autograd goes by to see that a tensor it keeps was written into


class Rope:
    """A rotary table [positions, rot / 2, 2] (cos, sin; float32, for example from lacache_rope_table) and the layout of
    the pairs."""

    def __init__(self, table: torch.Tensor, style: int = ROPE_HALF):
        if table.dtype != torch.float32 or table.device.type != "cuda" or table.dim() != 3 or table.shape[2] != 2 or \
                not table.is_contiguous():
            raise ValueError("table: expected a contiguous float32 [positions, rot / 2, 2] tensor on a GPU")
        self.table, self.style, self.rot, self.index = table, style, 2 * table.shape[1], table.get_device()
        self._c = _Rotary(table.data_ptr(), table.shape[0], self.rot, style)
        self._ref = ctypes.addressof(self._c)


class Sequences:
    """The sequences of a call: start [n + 1] (their rows in the packed row tensors), lens [n] (their tokens, the new
    ones included), pages [n, max_pages]; int32 on one GPU."""

    def __init__(self, start: torch.Tensor, lens: torch.Tensor, pages: torch.Tensor):
        n, dev = lens.shape[0], lens.device
        if dev.type != "cuda" or pages.dim() != 2:
            raise ValueError("sequences: expected tensors on a GPU, pages as [sequences, max_pages]")
        _ints(start, (n + 1,), dev.index, "start")
        _ints(lens, (n,), dev.index, "lens")
        _ints(pages, (n, pages.shape[1]), dev.index, "pages")
        self.start, self.lens, self.pages, self.index = start, lens, pages, dev.index
        self._c = _Seqs(start.data_ptr(), lens.data_ptr(), pages.data_ptr(), n, pages.shape[1])
        self._ref = ctypes.addressof(self._c)

    def __len__(self) -> int:
        return self._c.n_seq


class Prefixes:
    """Tokens that sequences share: sequences group[g] .. group[g + 1] - 1 begin with the same len[g] tokens (whole pages of
    them), and their page tables with the same pages, as far as their own tokens reach (slots without tokens or new rows may
    have any table).  group [n + 1] and len [n], int32 on one GPU."""

    def __init__(self, group: torch.Tensor, len: torch.Tensor):
        n, dev = len.shape[0], len.device
        if dev.type != "cuda":
            raise ValueError("prefixes: expected tensors on a GPU")
        _ints(group, (n + 1,), dev.index, "group")
        _ints(len, (n,), dev.index, "len")
        self.group, self.len, self.index = group, len, dev.index
        self._c = _Prefixes(group.data_ptr(), len.data_ptr(), n)
        self._ref = ctypes.addressof(self._c)


def _no_gradient(name: str) -> ValueError:
    """What autograd would want to follow: the cache keeps numbers, and no graph."""
    return ValueError(f"{name}: has no gradient, and a tensor requires one (torch.no_grad() or detach() say that none is "
                      "wanted)")


class KVCache:
    """A paged key-value cache: the pools of lacache_kv in torch tensors, and the scratch of its attention.  Without
    `pools` they are allocated here (zeros): k and v [n_pages, heads, page / 32, 32 D] (D: d padded to 64, 96, 128, 192 or
    256) bfloat16, float8_e4m3fn or int8, and for the last two k_scale and v_scale [n_pages, heads, page] float32.  With
    pools = (k, v, k_scale, v_scale) these tensors are used.  Calls on one cache are ordered on one stream (or by events):
    they share the pools and the scratch.  No gradient passes through a cache: with autograd on, its calls refuse tensors that
    require one."""

    def __init__(self, n_pages: int = 0, heads: int = 0, d: int = 0, page: int = 64, type: int = KV_BF16, device: int = 0,
                 pools=None):
        if pools is None:
            if type not in _KV_DTYPES or not _kv_fits(n_pages, heads, d, page):
                raise ValueError("KVCache: expected a KV_ type, at least one head, a page of 32, 64, 128 or 256 tokens and d as a "
                                 "multiple of 8 up to 256")
            dev = torch.device("cuda", device)
            shape = (n_pages, heads, page // 32, 32 * _padded(d))
            # (zeros of a one-byte type: fp8 has no fill everywhere, its zero is the byte 0)
            k, v = (torch.zeros(shape, dtype=torch.bfloat16 if type == KV_BF16 else torch.int8, device=dev)
                    .view(_KV_DTYPES[type]) for _ in range(2))
            ks, vs = (None if type == KV_BF16 else torch.zeros((n_pages, heads, page), device=dev) for _ in range(2))
        else:
            k, v, ks, vs = pools
            if k.dim() != 4 or k.dtype not in _KV_TYPES or k.device.type != "cuda":
                raise ValueError("pools: expected [n_pages, heads, page / 32, 32 D] tensors on a GPU")
            dev, type = k.device, _KV_TYPES[k.dtype]
            n_pages, heads, page = k.shape[0], k.shape[1], 32 * k.shape[2]
            if not 1 <= d <= 256 or k.shape[3] != 32 * _padded(d):
                raise ValueError(f"pools: tiles of {k.shape[3]} elements do not fit d = {d}")
            if not _kv_fits(n_pages, heads, d, page):
                raise LaCacheError(EINVAL, f"pools of {n_pages} pages, {heads} heads, d = {d}, {page} tokens a page")
            _given(k, k.shape, k.dtype, dev.index, "k")
            _given(v, k.shape, k.dtype, dev.index, "v")
            for t, name in ((ks, "k_scale"), (vs, "v_scale")):
                if type != KV_BF16:
                    _given(t, (n_pages, heads, page), torch.float32, dev.index, name)
                elif t is not None:
                    raise ValueError(f"{name}: a bfloat16 cache has no scales")
        self.k, self.v, self.k_scale, self.v_scale = k, v, ks, vs
        self.n_pages, self.heads, self.d, self.page, self.type, self.index = n_pages, heads, d, page, type, k.get_device()
        self._c = _KV(k.data_ptr(), v.data_ptr(), *(0 if t is None else t.data_ptr() for t in (ks, vs)), n_pages, page,
                      heads, d, type)
        self._ref = ctypes.addressof(self._c)
        self._pools = tuple(t for t in (k, v, ks, vs) if t is not None)
        self._need, self._space, self._outgrown = {}, None, []

    def _scratch(self, like, need: int, stream):
        """Larger scratch.  What it replaces stays: a captured graph may have it among its arguments.  Scratch made while a
        graph is captured is that graph's alone, since its zeros are written when the graph runs, not before."""
        space = _made(like, (need,), torch.uint8, stream, zeros=True)
        if _capturing(self.index, stream):
            return space
        if self._space is not None:
            self._outgrown.append(self._space)
        self._space = space
        return space

    def append(self, k, v, seqs, q=None, rope=None, q_out=None, max_new=0, stream=None):
        return lacache_kv_append(self, k, v, seqs, q, rope, q_out, max_new, stream)

    def read(self, seqs, rows, dtype=torch.bfloat16, out=None, max_new=0, stream=None):
        return lacache_kv_read(self, seqs, rows, dtype, out, max_new, stream)

    def attend(self, q, seqs, scale=None, window=0, max_new=0, out=None, stream=None):
        return lacache_kv_attend(self, q, seqs, scale, window, max_new, out, stream)

    def attend_shared(self, q, seqs, prefixes, scale=None, window=0, max_new=0, out=None, stream=None):
        return lacache_kv_attend_shared(self, q, seqs, prefixes, scale, window, max_new, out, stream)

    def attend_blocks(self, q, seqs, blocks, scale=None, out=None, stream=None):
        return lacache_kv_attend_blocks(self, q, seqs, blocks, scale, out, stream)


class KVBounds:
    """Bounds of the keys of a cache's pages, in 8 bits: code [n_pages, heads, 2, D] int8 (the largest value of each column,
    then the smallest) and scale [n_pages, heads] float32.  Allocated here (zeros) if they are not given."""

    def __init__(self, cache: KVCache, code=None, scale=None):
        shape = (cache.n_pages, cache.heads, 2, _padded(cache.d))
        self.code = cache.k.new_zeros(shape, dtype=torch.int8) if code is None else \
            _given(code, shape, torch.int8, cache.index, "code")
        self.scale = cache.k.new_zeros(shape[:2], dtype=torch.float32) if scale is None else \
            _given(scale, shape[:2], torch.float32, cache.index, "scale")
        self.cache = cache
        self._c = _Bounds(self.code.data_ptr(), self.scale.data_ptr())
        self._ref = ctypes.addressof(self._c)

    def update(self, seqs, rows, max_new=0, stream=None):
        return lacache_kv_bound(self, seqs, rows, max_new, stream)

    def read(self, pages, out=None, stream=None):
        return lacache_kv_bounds_read(self, pages, out, stream)

    def select(self, q, seqs, n_blocks, first=1, last=1, max_new=0, out=None, stream=None):
        return lacache_kv_select(self, q, seqs, n_blocks, first, last, max_new, out, stream)


def _kv_fits(n_pages: int, heads: int, d: int, page: int) -> bool:
    """What the calls take (lacache_kv)."""
    return 0 <= n_pages < 1 << 31 and 1 <= heads <= 65535 and 8 <= d <= 256 and d % 8 == 0 and page in (32, 64, 128, 256)


def _padded(d: int) -> int:
    return next(D for D in (64, 96, 128, 192, 256) if d <= D)


def lacache_rope_table(n: int, rot: int, base: float = 10000.0, factor: float = 1.0, original: float = 0.0,
                       low: float = 1.0, high: float = 32.0, magnitude: float = 1.0, first: int = 0, device: int = 0,
                       out=None, stream=None):
    """(cos, sin) of positions first .. first+n-1 for rot / 2 pairs, [n, rot / 2, 2] float32, scaled by parts for long
    contexts if factor > 1."""
    shape = (n, rot // 2, 2)
    if out is None:
        out = _made(torch.empty(0, device=torch.device("cuda", device)), shape, torch.float32, stream)
    _given(out, shape, torch.float32, device, "out")
    _check(_on(device, stream, _lib.lacache_rope_table, out.data_ptr(), first, n, rot, base, factor, original, low, high,
               magnitude), "lacache_rope_table")
    _written(out)
    return out


class _RopeGrad(torch.autograd.Function):
    """lacache_rope under autograd: the gradient is the other rotation of the two."""

    @staticmethod
    def forward(ctx, x, pos, rope, backward, stream):
        ctx.rope, ctx.turns_back = rope, backward
        ctx.save_for_backward(pos, rope.table)
        return lacache_rope(x, pos, rope, backward, None, stream)

    @staticmethod
    def backward(ctx, dy):
        pos, _ = ctx.saved_tensors
        dy = dy if dy.stride(2) == 1 else dy.contiguous()
        return lacache_rope(dy, pos, ctx.rope, not ctx.turns_back), None, None, None, None


def lacache_rope(x, pos, rope: Rope, backward: bool = False, out=None, stream=None):
    """x [rows, H, d] float32 or bfloat16 (any strides, the last one 1), pos [rows] int32.  Returns the turned rows
    (`out`, which may be x; otherwise a new contiguous tensor); with backward=True the gradient of the input from that of
    the output.  autograd differentiates it with respect to x (not through `out`, and not with respect to the table)."""
    if torch.is_grad_enabled():
        if rope.table.requires_grad or (out is not None and (x.requires_grad or out.requires_grad)):
            raise ValueError("a table that needs a gradient has none, nor does a result written into `out`")
        if x.requires_grad:
            return _RopeGrad.apply(x, pos, rope, bool(backward), stream)
    index, dtype, shape, xs = x.get_device(), _ROW_DTYPES.get(x.dtype), x.shape, x.stride()
    if len(shape) != 3 or dtype is None or index < 0 or (shape[2] > 1 and xs[2] != 1):
        raise ValueError("x: expected a float32 or bfloat16 [rows, H, d] tensor on a GPU, its last stride 1")
    rows, H, d = shape
    given = out is not None
    if not given:
        out = _made(x, shape, x.dtype, stream)
    elif out.shape != shape or out.dtype != x.dtype or out.get_device() != index or (d > 1 and out.stride(2) != 1):
        raise ValueError(f"out: expected {tuple(shape)} {x.dtype} on cuda:{index}, its last stride 1")
    if rope.index != index or pos.dtype != torch.int32 or pos.get_device() != index or pos.shape != shape[:1] or \
            not pos.is_contiguous():
        raise ValueError(f"expected a table and {rows} contiguous int32 positions on cuda:{index}")
    ys = out.stride()
    _check(_on(index, stream, _lib.lacache_rope, x.data_ptr(), out.data_ptr(), dtype, rows, H, d, xs[0], xs[1], ys[0],
               ys[1], pos.data_ptr(), rope._ref, int(backward)), "lacache_rope")
    if given:
        _written(out)
    return out


def lacache_kv_append(c: KVCache, k, v, seqs: Sequences, q=None, rope=None, q_out=None, max_new: int = 0, stream=None):
    """Store the new tokens k, v [rows, heads, d] (float32 or bfloat16, for example parts of one projection's output) of
    every sequence; k and q [rows, q_heads, d] are turned by `rope`.  Returns the turned q (None without q)."""
    index, kind = c.index, k.dtype
    dtype = _ROW_DTYPES.get(kind)
    if dtype is None:
        raise ValueError(f"k: unsupported dtype {kind}")
    if torch.is_grad_enabled() and (k.requires_grad or v.requires_grad or (q is not None and q.requires_grad) or
                                    (q_out is not None and q_out.requires_grad) or
                                    (rope is not None and rope.table.requires_grad)):
        raise _no_gradient("lacache_kv_append")
    k_row, v_row = _rows(k, c.heads, c.d, index, kind, "k"), _rows(v, c.heads, c.d, index, kind, "v")
    rows = k.shape[0]
    if v.shape[0] != rows or seqs.index != index or (rope is not None and rope.index != index):
        raise ValueError(f"expected {rows} rows of v, and sequences and table on cuda:{index}")
    q_ptr = o_ptr = None
    q_row = q_heads = 0
    given = False
    if q is not None:
        q_heads = q.shape[1]
        q_row = _rows(q, q_heads, c.d, index, kind, "q")
        if q.shape[0] != rows:
            raise ValueError(f"q: expected {rows} rows")
        given = q_out is not None
        q_out = _given(q_out, q.shape, kind, index, "q_out") if given else _made(q, q.shape, kind, stream)
        q_ptr, o_ptr = q.data_ptr(), q_out.data_ptr()
    _check(_on(index, stream, _lib.lacache_kv_append, c._ref, seqs._ref, k.data_ptr(), v.data_ptr(), dtype, rows, k_row,
               v_row, q_ptr, o_ptr, q_heads, q_row, None if rope is None else rope._ref, max_new), "lacache_kv_append")
    _written(c._pools)
    if given:
        _written(q_out)
    return q_out if q is not None else None


def lacache_kv_read(c: KVCache, seqs: Sequences, rows: int, dtype=torch.bfloat16, out=None, max_new: int = 0,
                    stream=None):
    """The newest tokens of every sequence as (k, v), each [rows, heads, d] of dtype; rows is start[-1]."""
    index, kind = c.index, _ROW_DTYPES.get(dtype)
    if kind is None or seqs.index != index:
        raise ValueError(f"expected float32 or bfloat16, and sequences on cuda:{index}")
    shape = (rows, c.heads, c.d)
    if out is None:
        k, v = _made(c.k, shape, dtype, stream), _made(c.k, shape, dtype, stream)
    else:
        k, v = _given(out[0], shape, dtype, index, "k"), _given(out[1], shape, dtype, index, "v")
        if torch.is_grad_enabled() and (k.requires_grad or v.requires_grad):
            raise _no_gradient("lacache_kv_read")
    _check(_on(index, stream, _lib.lacache_kv_read, c._ref, seqs._ref, k.data_ptr(), v.data_ptr(), kind, rows, max_new),
           "lacache_kv_read")
    if out is not None:
        _written((k, v))
    return k, v


def lacache_kv_attend_workspace(c: KVCache, dtype: int, n_seq: int, q_heads: int, max_new: int = 0) -> int:
    """Bytes of scratch that lacache_kv_attend needs (dtype: F32 or BF16)."""
    with torch.cuda.device(c.index):
        n = int(_lib.lacache_kv_attend_workspace(c._ref, dtype, n_seq, q_heads, max_new))
    if n < 0:
        raise LaCacheError(n, "lacache_kv_attend_workspace")
    return n


def lacache_kv_attend(c: KVCache, q, seqs: Sequences, scale=None, window: int = 0, max_new: int = 0, out=None,
                      stream=None):
    """Attention of the new rows q [rows, q_heads, d] (already turned) over the cached tokens.  scale defaults to
    1 / sqrt(d).  Returns (out [rows, q_heads, d] of q's dtype, lse [rows, q_heads] float32)."""
    index, kind, shape = c.index, q.dtype, q.shape
    dtype = _ROW_DTYPES.get(kind)
    if dtype is None or len(shape) != 3 or seqs.index != index:
        raise ValueError(f"q: expected float32 or bfloat16 [rows, q_heads, d], and sequences on cuda:{index}")
    rows, q_heads = shape[0], shape[1]
    q_row = _rows(q, q_heads, c.d, index, kind, "q")
    given = out is not None
    if torch.is_grad_enabled() and (q.requires_grad or (given and (out[0].requires_grad or out[1].requires_grad))):
        raise _no_gradient("lacache_kv_attend")
    if not given:
        out = (_made(q, shape, kind, stream), _made(q, shape[:2], torch.float32, stream))
    else:
        _given(out[0], shape, kind, index, "out")
        _given(out[1], shape[:2], torch.float32, index, "lse")
    key = (dtype, seqs._c.n_seq, q_heads, max_new)
    need = c._need.get(key)
    if need is None:
        need = c._need[key] = lacache_kv_attend_workspace(c, *key)
    space = c._space
    if space is None or space.numel() < need:
        space = c._scratch(q, need, stream)
    _check(_on(index, stream, _lib.lacache_kv_attend, c._ref, seqs._ref, q.data_ptr(), dtype, rows, q_heads, q_row,
               max_new, c.d ** -0.5 if scale is None else scale, window, out[0].data_ptr(), out[1].data_ptr(),
               space.data_ptr(), space.numel()), "lacache_kv_attend")
    if given:
        _written(out)
    return out


def _keep(sizes: dict, key, need: int) -> int:
    if len(sizes) >= 4096:  # (calls of ever other sizes)
        sizes.clear()
    sizes[key] = need
    return need


def lacache_kv_attend_shared_workspace(c: KVCache, dtype: int, rows: int, n_seq: int, n_groups: int, q_heads: int,
                                       max_new: int = 0) -> int:
    """Bytes of scratch that lacache_kv_attend_shared needs (dtype: F32 or BF16)."""
    with torch.cuda.device(c.index):
        n = int(_lib.lacache_kv_attend_shared_workspace(c._ref, dtype, rows, n_seq, n_groups, q_heads, max_new))
    if n < 0:
        raise LaCacheError(n, "lacache_kv_attend_shared_workspace")
    return n


def lacache_kv_attend_shared(c: KVCache, q, seqs: Sequences, prefixes: Prefixes, scale=None, window: int = 0, max_new: int = 0,
                             out=None, stream=None):
    """lacache_kv_attend of sequences of which groups begin with the same pages, which are read once for all of a group's
    rows: for a few new tokens of each behind some thousands that they share (prompts are faster, and take less scratch, in
    lacache_kv_attend).  Returns (out, lse) as that call."""
    index, kind, shape = c.index, q.dtype, q.shape
    dtype = _ROW_DTYPES.get(kind)
    if dtype is None or len(shape) != 3 or seqs.index != index or prefixes.index != index:
        raise ValueError(f"q: expected float32 or bfloat16 [rows, q_heads, d], and sequences and prefixes on cuda:{index}")
    rows, q_heads = shape[0], shape[1]
    q_row = _rows(q, q_heads, c.d, index, kind, "q")
    given = out is not None
    if torch.is_grad_enabled() and (q.requires_grad or (given and (out[0].requires_grad or out[1].requires_grad))):
        raise _no_gradient("lacache_kv_attend_shared")
    if not given:
        out = (_made(q, shape, kind, stream), _made(q, shape[:2], torch.float32, stream))
    else:
        _given(out[0], shape, kind, index, "out")
        _given(out[1], shape[:2], torch.float32, index, "lse")
    key = ("shared", dtype, rows, seqs._c.n_seq, prefixes._c.n_groups, q_heads, max_new)
    need = c._need.get(key)
    if need is None:
        need = _keep(c._need, key, lacache_kv_attend_shared_workspace(c, *key[1:]))
    space = _made(q, (need,), torch.uint8, stream)  # (all rows' sums: too much to keep for the largest call)
    _check(_on(index, stream, _lib.lacache_kv_attend_shared, c._ref, seqs._ref, prefixes._ref, q.data_ptr(), dtype, rows, q_heads,
               q_row, max_new, c.d ** -0.5 if scale is None else scale, window, out[0].data_ptr(), out[1].data_ptr(),
               space.data_ptr(), need), "lacache_kv_attend_shared")
    if given:
        _written(out)
    return out


def lacache_kv_bound(b: KVBounds, seqs: Sequences, rows: int, max_new: int = 0, stream=None) -> None:
    """Bounds of the pages that the newest tokens of every sequence lie in (rows is start[-1]), after each append."""
    c = b.cache
    if seqs.index != c.index:
        raise ValueError(f"expected sequences on cuda:{c.index}")
    _check(_on(c.index, stream, _lib.lacache_kv_bound, c._ref, b._ref, seqs._ref, rows, max_new), "lacache_kv_bound")
    _written((b.code, b.scale))


def lacache_kv_bounds_read(b: KVBounds, pages, out=None, stream=None):
    """The bounds of pages [n] (int32) as (most, least), each [n, heads, d] float32."""
    c = b.cache
    n = pages.shape[0] if pages.dim() == 1 else -1
    _given(pages, (n,) if n >= 0 else (0,), torch.int32, c.index, "pages")
    shape = (n, c.heads, c.d)
    given = out is not None
    if not given:
        out = _made(c.k, (2, *shape), torch.float32, stream).unbind(0)
    else:
        _given(out[0], shape, torch.float32, c.index, "most")
        _given(out[1], shape, torch.float32, c.index, "least")
        if torch.is_grad_enabled() and (out[0].requires_grad or out[1].requires_grad):
            raise _no_gradient("lacache_kv_bounds_read")
    _check(_on(c.index, stream, _lib.lacache_kv_bounds_read, c._ref, b._ref, pages.data_ptr(), n, out[0].data_ptr(),
               out[1].data_ptr()), "lacache_kv_bounds_read")
    if given:
        _written(out)
    return out


def lacache_kv_select_workspace(c: KVCache, rows: int, max_pages: int) -> int:
    """Bytes of scratch that lacache_kv_select needs."""
    n = int(_lib.lacache_kv_select_workspace(c._ref, rows, max_pages))
    if n < 0:
        raise LaCacheError(n, "lacache_kv_select_workspace")
    return n


def lacache_kv_select(b: KVBounds, q, seqs: Sequences, n_blocks: int, first: int = 1, last: int = 1, max_new: int = 0,
                      out=None, stream=None):
    """The pages whose keys may give the new rows q [rows, q_heads, d] their largest scores: [rows, heads, n_blocks] int32
    indices into the page tables, rising, -1 behind them.  The first `first` pages and the `last` newest are always there."""
    c = b.cache
    index, kind, shape = c.index, q.dtype, q.shape
    dtype = _ROW_DTYPES.get(kind)
    if dtype is None or len(shape) != 3 or seqs.index != index:
        raise ValueError(f"q: expected float32 or bfloat16 [rows, q_heads, d], and sequences on cuda:{index}")
    q_row = _rows(q, shape[1], c.d, index, kind, "q")
    given = out is not None
    if n_blocks < 1 or first < 0 or last < 0 or first + last > n_blocks:
        raise ValueError("expected n_blocks >= 1, first >= 0, last >= 0 and first + last <= n_blocks")
    out = _given(out, (shape[0], c.heads, n_blocks), torch.int32, index, "out") if given else \
        _made(q, (shape[0], c.heads, n_blocks), torch.int32, stream)
    key = ("select", shape[0], seqs._c.max_pages)
    need = c._need.get(key)
    if need is None:
        need = _keep(c._need, key, lacache_kv_select_workspace(c, shape[0], seqs._c.max_pages))
    space = _made(q, (need,), torch.uint8, stream)
    _check(_on(index, stream, _lib.lacache_kv_select, c._ref, b._ref, seqs._ref, q.data_ptr(), dtype, shape[0], shape[1], q_row,
               n_blocks, first, last, max_new, out.data_ptr(), space.data_ptr(), need), "lacache_kv_select")
    if given:
        _written(out)
    return out


def lacache_kv_attend_blocks_workspace(c: KVCache, rows: int, q_heads: int, n_blocks: int) -> int:
    """Bytes of scratch that lacache_kv_attend_blocks needs."""
    with torch.cuda.device(c.index):
        n = int(_lib.lacache_kv_attend_blocks_workspace(c._ref, rows, q_heads, n_blocks))
    if n < 0:
        raise LaCacheError(n, "lacache_kv_attend_blocks_workspace")
    return n


def lacache_kv_attend_blocks(c: KVCache, q, seqs: Sequences, blocks, scale=None, out=None, stream=None):
    """Attention of the new rows q [rows, q_heads, d] (already turned) over the pages of their lists, blocks [rows, heads, n]
    int32 indices into the page tables (for example of KVBounds.select).  Returns (out, lse) as lacache_kv_attend."""
    index, kind, shape = c.index, q.dtype, q.shape
    dtype = _ROW_DTYPES.get(kind)
    if dtype is None or len(shape) != 3 or seqs.index != index:
        raise ValueError(f"q: expected float32 or bfloat16 [rows, q_heads, d], and sequences on cuda:{index}")
    rows, q_heads = shape[0], shape[1]
    q_row = _rows(q, q_heads, c.d, index, kind, "q")
    if blocks.dim() != 3 or blocks.shape[2] < 1:
        raise ValueError(f"blocks: expected [{rows}, {c.heads}, n] with n >= 1, got {tuple(blocks.shape)}")
    n = blocks.shape[2]
    _given(blocks, (rows, c.heads, n), torch.int32, index, "blocks")
    given = out is not None
    if torch.is_grad_enabled() and (q.requires_grad or (given and (out[0].requires_grad or out[1].requires_grad))):
        raise _no_gradient("lacache_kv_attend_blocks")
    if not given:
        out = (_made(q, shape, kind, stream), _made(q, shape[:2], torch.float32, stream))
    else:
        _given(out[0], shape, kind, index, "out")
        _given(out[1], shape[:2], torch.float32, index, "lse")
    key = ("blocks", rows, q_heads, n)
    need = c._need.get(key)
    if need is None:
        need = _keep(c._need, key, lacache_kv_attend_blocks_workspace(c, rows, q_heads, n))
    space = c._space
    if need and (space is None or space.numel() < need):
        space = c._scratch(q, need, stream)
    _check(_on(index, stream, _lib.lacache_kv_attend_blocks, c._ref, seqs._ref, q.data_ptr(), dtype, rows, q_heads, q_row,
               blocks.data_ptr(), n, c.d ** -0.5 if scale is None else scale, out[0].data_ptr(), out[1].data_ptr(),
               space.data_ptr() if need else None, space.numel() if need else 0), "lacache_kv_attend_blocks")
    if given:
        _written(out)
    return out


def lacache_verify_workspace(V: int, B: int, k: int) -> int:
    """Bytes of scratch that lacache_verify needs."""
    n = int(_lib.lacache_verify_workspace(V, B, k))
    if n < 0:
        raise LaCacheError(n, "lacache_verify_workspace")
    return n


def _logits(t, shape, dtype, index: int, name: str):
    """The strides of [B, rows, V] logits whose rows are each contiguous."""
    stride = t.stride()
    if t.dtype != dtype or t.get_device() != index or t.shape != shape or (shape[2] > 1 and t.numel() and stride[2] != 1):
        raise ValueError(f"{name}: expected {list(shape)} {dtype} on cuda:{index} with contiguous rows, got {tuple(t.shape)} "
                         f"{t.dtype} on {t.device} with strides {stride}")
    return stride[0], stride[1]


_verify_need = {}  # bytes of scratch by (V, B, k); a thread that empties it costs others a question again, no more


def lacache_verify(logits, draft_logits, draft_tokens, u_accept, u_next, temperature=None, n_draft=None, out=None,
                   stream=None):
    """Verification of drafted tokens by rejection: logits [B, k + 1, V] of the target model and draft_logits [B, k, V] of
    the draft model (float32 or bfloat16, rows contiguous), draft_tokens [B, k] int32, u_accept [B, k] and u_next [B]
    float32 random numbers from [0, 1), temperature [B] float32 (1 where it is not given; 0 is greedy), n_draft [B] int32
    (k where it is not given).  Returns (accept_len [B] int32, next_token [B] int32, p_target [B, k], p_draft [B, k])."""
    dtype, shape, index = logits.dtype, logits.shape, logits.get_device()
    kind = _ROW_DTYPES.get(dtype)
    if len(shape) != 3 or index < 0 or kind is None or shape[1] < 1:
        raise ValueError("logits: expected a float32 or bfloat16 [B, k + 1, V] tensor on a GPU")
    B, k, V = shape[0], shape[1] - 1, shape[2]
    per_draft, per_seq = torch.Size((B, k)), torch.Size((B,))
    t_seq, t_row = _logits(logits, shape, dtype, index, "logits")
    d_seq, d_row = _logits(draft_logits, torch.Size((B, k, V)), dtype, index, "draft_logits")
    _given(draft_tokens, per_draft, torch.int32, index, "draft_tokens")
    _given(u_accept, per_draft, torch.float32, index, "u_accept")
    _given(u_next, per_seq, torch.float32, index, "u_next")
    if temperature is not None:
        _given(temperature, per_seq, torch.float32, index, "temperature")
    if n_draft is not None:
        _given(n_draft, per_seq, torch.int32, index, "n_draft")
    given = out is not None
    if torch.is_grad_enabled() and (logits.requires_grad or draft_logits.requires_grad or u_accept.requires_grad or
                                    u_next.requires_grad or (temperature is not None and temperature.requires_grad) or
                                    (given and any(t.requires_grad for t in out))):
        raise _no_gradient("lacache_verify")
    if given:
        for t, s, kind_of, name in zip(out, (per_seq, per_seq, per_draft, per_draft),
                                       (torch.int32, torch.int32, torch.float32, torch.float32),
                                       ("accept_len", "next_token", "p_target", "p_draft"), strict=True):
            _given(t, s, kind_of, index, name)
        out = tuple(out)
    else:  # (two allocations, not four)
        out = _made(logits, (2, B), torch.int32, stream).unbind(0) + _made(logits, (2, B, k), torch.float32, stream).unbind(0)
    need = _verify_need.get((V, B, k))
    if need is None:
        need = _keep(_verify_need, (V, B, k), lacache_verify_workspace(V, B, k))
    space = _made(logits, (need,), torch.uint8, stream)
    _check(_on(index, stream, _lib.lacache_verify, logits.data_ptr(), draft_logits.data_ptr(), kind, V, t_seq, t_row, d_seq,
               d_row, draft_tokens.data_ptr(), u_accept.data_ptr(), u_next.data_ptr(),
               None if temperature is None else temperature.data_ptr(), None if n_draft is None else n_draft.data_ptr(), B, k,
               out[0].data_ptr(), out[1].data_ptr(), out[2].data_ptr(), out[3].data_ptr(), space.data_ptr(), need),
           "lacache_verify")
    if given:
        _written(out)
    return out


def raw_library() -> ctypes.CDLL:
    """The loaded C library, for callers that pass raw pointers themselves."""
    return _lib
