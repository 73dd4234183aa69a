"""The cache of a serving loop: storing rows, attention over 8-bit rows, the weight that rows gather, and eviction by it.  Argument marshalling
only, like binding.py, natively for the calls of every token; the calls are described in include/llla.h."""
from __future__ import annotations

import contextlib
import ctypes
from typing import NamedTuple, Optional

import torch

from . import binding
from .binding import LlaError, _DTYPES, _Strides, _stream_ptr, _strides4

BLOCK = 64                                  # slots of a head that share an exponent (LLLA_CACHE_BLOCK)
CACHE_DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.int8: 2, torch.float8_e4m3fn: 3}
_CODES = (torch.int8, torch.float8_e4m3fn)


class Cache(NamedTuple):
    """Keys and values of B sequences and H cache heads.

    K, V           [B, H, L_max, d], float32, bfloat16, or codes: int8 or float8_e4m3fn
    k_exp, v_exp   with codes: int8 [B, H, ceil(L_max / 64)]; a row is code * 2^exp of its block of 64 slots
    scores         float32 [B, H, L_max], the weight that a row has gathered, or None
    pos            int32 [B, H, L_max], the position in its sequence that a row stands for, or None (its slot)
    """
    K: torch.Tensor
    V: torch.Tensor
    k_exp: Optional[torch.Tensor] = None
    v_exp: Optional[torch.Tensor] = None
    scores: Optional[torch.Tensor] = None
    pos: Optional[torch.Tensor] = None

    def values(self, dtype=torch.float32):
        """(K, V) as numbers, for inspection: codes times their powers of two."""
        def rows(c, e):
            if e is None:
                return c.to(dtype)
            power = torch.where(e == -128, torch.nan, torch.exp2(e.to(torch.float64)))
            return (c.to(torch.float64) * power.repeat_interleave(BLOCK, 2)[:, :, :c.shape[2], None]).to(dtype)
        return rows(self.K, self.k_exp), rows(self.V, self.v_exp)


def cache_alloc(B: int, H: int, L_max: int, d: int, dtype=torch.int8, device="cuda", scores: bool = False, pos: bool = False) -> Cache:
    """An empty cache for L_max rows of B sequences and H cache heads."""
    if dtype not in CACHE_DTYPES:
        raise ValueError("a cache holds float32, bfloat16, int8 or float8_e4m3fn rows")
    K, V = (torch.zeros((B, H, L_max, d), dtype=dtype, device=device) for _ in range(2))
    blocks = (L_max + BLOCK - 1) // BLOCK
    ke, ve = (torch.zeros((B, H, blocks), dtype=torch.int8, device=device) if dtype in _CODES else None for _ in range(2))
    return Cache(K, V, ke, ve, torch.zeros((B, H, L_max), device=device) if scores else None,
                 torch.zeros((B, H, L_max), dtype=torch.int32, device=device) if pos else None)


class _CacheStruct(ctypes.Structure):
    _fields_ = [("K", ctypes.c_void_p), ("V", ctypes.c_void_p), ("sk", _Strides), ("sv", _Strides), ("k_exp", ctypes.c_void_p),
                ("v_exp", ctypes.c_void_p), ("scores", ctypes.c_void_p), ("pos", ctypes.c_void_p), ("B", ctypes.c_int), ("H", ctypes.c_int),
                ("L_max", ctypes.c_int), ("d", ctypes.c_int), ("type", ctypes.c_int)]


def declare(L) -> None:
    """The C ABI's signatures, on a loaded library."""
    vp, sz, i32, f32, cp = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int, ctypes.c_float, ctypes.POINTER(_CacheStruct)
    L.llla_cache_append.argtypes = [cp, vp, vp, _Strides, _Strides, i32, i32, vp, vp, vp, vp]
    L.llla_cache_append.restype = i32
    L.llla_decode_q8_workspace_bytes.argtypes = [cp, i32]
    L.llla_decode_q8_workspace_bytes.restype = sz
    L.llla_decode_q8.argtypes = [vp, cp, vp, vp, i32, i32, i32, f32, f32, vp, sz, vp]
    L.llla_decode_q8.restype = i32
    L.llla_cache_scores_workspace_bytes.argtypes = [cp, i32, i32, i32]
    L.llla_cache_scores_workspace_bytes.restype = sz
    L.llla_cache_scores.argtypes = [vp, cp, _Strides, vp, i32, i32, i32, f32, vp, sz, vp]
    L.llla_cache_scores.restype = i32
    L.llla_cache_evict_workspace_bytes.argtypes = [cp, i32]
    L.llla_cache_evict_workspace_bytes.restype = sz
    L.llla_cache_evict.argtypes = [cp, cp, vp, i32, i32, i32, vp, vp, vp, sz, vp]
    L.llla_cache_evict.restype = i32


def _words(t, what, shape, dtype, device):
    """Address of an optional contiguous array of the cache or a call."""
    if t is None:
        return None
    if t.dtype != dtype or tuple(t.shape) != shape or not t.is_contiguous() or t.device != device:
        raise ValueError("%s must be a contiguous %s tensor %s on the cache's device" % (what, str(dtype).replace("torch.", ""), list(shape)))
    return t.data_ptr()


def _struct(cache) -> _CacheStruct:
    """The C ABI's cache, checked."""
    K, V = cache.K, cache.V
    if not (K.is_cuda and V.is_cuda):
        raise ValueError("a cache lies in device memory; this library has no CPU path")
    if K.dtype != V.dtype or K.dtype not in CACHE_DTYPES:
        raise ValueError("K and V must share dtype float32, bfloat16, int8 or float8_e4m3fn")
    if K.dim() != 4 or K.shape != V.shape or K.device != V.device:
        raise ValueError("K and V must have the same [B, H, L_max, d] shape, on one device")
    B, H, L, d = K.shape
    sk, sv = _strides4(K, V)
    ke = ve = None
    if K.dtype in _CODES:
        if cache.k_exp is None or cache.v_exp is None:
            raise ValueError("a cache of codes needs the exponents k_exp and v_exp")
        shape = (B, H, (L + BLOCK - 1) // BLOCK)
        ke = _words(cache.k_exp, "k_exp", shape, torch.int8, K.device)
        ve = _words(cache.v_exp, "v_exp", shape, torch.int8, K.device)
    return _CacheStruct(K.data_ptr(), V.data_ptr(), sk, sv, ke, ve, _words(cache.scores, "scores", (B, H, L), torch.float32, K.device),
                        _words(cache.pos, "pos", (B, H, L), torch.int32, K.device), B, H, L, d, CACHE_DTYPES[K.dtype])


def _on(device, stream):
    """Makes the call's device, and stream if one is given, torch's current ones: what the call allocates then belongs to that stream."""
    if stream is not None:
        if stream.device != device:
            raise ValueError("the stream must be one of the cache's device")
        return torch.cuda.stream(stream)
    if device.index != torch._C._cuda_getDevice():
        return torch.cuda.device(device)
    return contextlib.nullcontext()


def _scratch(need: int, device, workspace):
    """Address and size of the caller's scratch, or of scratch of this call's own."""
    if workspace is None:
        workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=device)
    elif workspace.device != device or not workspace.is_contiguous():
        raise ValueError("the workspace must be a contiguous tensor on the cache's device")
    return workspace, workspace.data_ptr(), workspace.numel() * workspace.element_size()


def _lengths(t, what, B, device):
    return None if t is None else _words(t, what, (B,), torch.int32, device)


def _native(stream, *tensors):
    """Addresses for the native extension, which takes the ordinary forms of a call on the current stream; None: marshalled here.  (One token's rows
    for 512 heads, 4.5 us on the GPU: 12.4 -> 5.0 us a call.)"""
    if stream is not None:
        return None
    return binding._entries.get(binding._use_measure) or binding._entry_points(*tensors)


def llla_cache_append(cache: Cache, k, v, seqlens=None, new_lens=None, first_pos=None, stream=None) -> None:
    """Stores k, v ([B, H, n, d], float32 or bfloat16): row i of sequence b goes to slot seqlens[b] + i (seqlens None: 0).  ``new_lens``: int32 [B],
    how many of the n rows a sequence brings; ``first_pos``: int32 [B], position of its first new row, for cache.pos (None: its slot).
    cache.scores becomes 0 there.  The lengths are the caller's to add to."""
    fn = _native(stream, cache.K, k, v)
    st = NotImplemented if fn is None else binding._host.cache_append(fn[4], cache, k, v, seqlens, new_lens, first_pos, binding._current_stream)
    if st is not NotImplemented:
        if st != 0:
            raise LlaError(st, "llla_cache_append")
        return
    c = _struct(cache)
    device = cache.K.device
    if k.dtype != v.dtype or k.dtype not in _DTYPES or k.device != device or v.device != device:
        raise ValueError("k and v must share dtype float32 or bfloat16, on the cache's device")
    if k.dim() != 4 or k.shape != v.shape or (k.shape[0], k.shape[1], k.shape[3]) != (c.B, c.H, c.d):
        raise ValueError("k and v must be [B, H, n, d] of the cache's B, H and d")
    sk, sv = _strides4(k, v)
    lens = [_lengths(t, w, c.B, device) for t, w in ((seqlens, "seqlens"), (new_lens, "new_lens"), (first_pos, "first_pos"))]
    with _on(device, stream):
        st = binding.lib().llla_cache_append(c, k.data_ptr(), v.data_ptr(), sk, sv, k.shape[2], _DTYPES[k.dtype], *lens, _stream_ptr(stream))
    if st != 0:
        raise LlaError(st, "llla_cache_append")


def decode_q8_workspace_bytes(cache: Cache, H: int) -> int:
    return int(binding.lib().llla_decode_q8_workspace_bytes(_struct(cache), H))


def llla_decode_q8(q, cache: Cache, lam: float, scale: float, seqlens=None, out_dtype=None, workspace=None, out=None, stream=None):
    """One query per (sequence, query head), q [B, H, d], against a cache of codes; query head h reads cache head h // (H // cache heads).
    Returns [B, H, d] (zero for empty sequences)."""
    fn = _native(stream, cache.K, q)
    r = NotImplemented if fn is None else binding._host.decode_q8(fn[5], fn[6], q, cache, lam, scale, seqlens, out_dtype, workspace, out, binding._current_stream)
    if r is not NotImplemented:
        if type(r) is int:
            raise LlaError(r, "llla_decode_q8")
        return r
    c = _struct(cache)
    device = cache.K.device
    if cache.K.dtype not in _CODES:
        raise ValueError("llla_decode_q8 reads caches of codes (int8, float8_e4m3fn); llla_decode those of numbers")
    if q.dtype not in _DTYPES or q.device != device or q.dim() != 3 or not q.is_contiguous() or (q.shape[0], q.shape[2]) != (c.B, c.d):
        raise ValueError("q must be a contiguous float32 or bfloat16 tensor [B, H, d] of the cache's B and d, on its device")
    H = q.shape[1]
    out_dtype = torch.float32 if out_dtype is None else out_dtype
    lens = _lengths(seqlens, "seqlens", c.B, device)
    L = binding.lib()
    with _on(device, stream):
        if out is None:
            if out_dtype not in _DTYPES:
                raise ValueError("the result is float32 or bfloat16")
            out = torch.empty(q.shape, dtype=out_dtype, device=device)
        elif out.dtype not in _DTYPES or out.shape != q.shape or not out.is_contiguous() or out.device != device:
            raise ValueError("out must be a contiguous float32 or bfloat16 tensor of q's shape")
        keep, ws, size = _scratch(int(L.llla_decode_q8_workspace_bytes(c, H)), device, workspace)
        st = L.llla_decode_q8(q.data_ptr(), c, out.data_ptr(), lens, H, _DTYPES[q.dtype], _DTYPES[out.dtype], float(lam), float(scale), ws, size,
                              _stream_ptr(stream))
    if st != 0:
        raise LlaError(st, "llla_decode_q8")
    return out


def cache_scores_workspace_bytes(cache: Cache, H: int, nq: int, dtype) -> int:
    return int(binding.lib().llla_cache_scores_workspace_bytes(_struct(cache), H, nq, _DTYPES[dtype]))


def llla_cache_scores(Q, cache: Cache, scale: float, seqlens=None, workspace=None, stream=None):
    """Adds to cache.scores what share of every query's kernel weight each row has.  Q: [B, H, nq, d], the queries of the last nq rows of each
    sequence, or [B, H, d], those of the last one.  Returns cache.scores."""
    fn = _native(stream, cache.K, Q)
    st = NotImplemented if fn is None else binding._host.cache_scores(fn[7], fn[8], Q, cache, scale, seqlens, workspace, binding._current_stream)
    if st is not NotImplemented:
        if st != 0:
            raise LlaError(st, "llla_cache_scores")
        return cache.scores
    c = _struct(cache)
    device = cache.K.device
    if cache.scores is None:
        raise ValueError("the cache has no scores")
    if Q.dim() == 3:
        Q = Q[:, :, None]
    if Q.dtype not in _DTYPES or Q.device != device or Q.dim() != 4 or (Q.shape[0], Q.shape[3]) != (c.B, c.d):
        raise ValueError("Q must be a float32 or bfloat16 tensor [B, H, nq, d] or [B, H, d] of the cache's B and d, on its device")
    if cache.K.dtype not in _CODES and cache.K.dtype != Q.dtype:
        raise ValueError("a cache of numbers and its queries must share their dtype")
    H, nq = Q.shape[1], Q.shape[2]
    sq = _strides4(Q)[0]
    lens = _lengths(seqlens, "seqlens", c.B, device)
    L = binding.lib()
    with _on(device, stream):
        keep, ws, size = _scratch(int(L.llla_cache_scores_workspace_bytes(c, H, nq, _DTYPES[Q.dtype])), device, workspace)
        st = L.llla_cache_scores(Q.data_ptr(), c, sq, lens, H, nq, _DTYPES[Q.dtype], float(scale), ws, size, _stream_ptr(stream))
    if st != 0:
        raise LlaError(st, "llla_cache_scores")
    return cache.scores


def cache_evict_workspace_bytes(cache: Cache, keep: int) -> int:
    return int(binding.lib().llla_cache_evict_workspace_bytes(_struct(cache), keep))


def llla_cache_evict(cache: Cache, keep: int, seqlens=None, sinks: int = 0, recent: int = 0, into: Optional[Cache] = None, index=None, lens_out=None,
                     workspace=None, stream=None):
    """Keeps ``keep`` rows of every (sequence, head): the first ``sinks`` and last ``recent`` positions, then those of largest cache.scores (equal
    ones by lower slot).  In place, rows move into the slots of rows given up; with ``into`` they are copied there in the order of their
    slots.  ``index``: int32 [B, H, keep], receives the slot that each row was in.  Returns the lengths afterwards, int32 [B]."""
    c = _struct(cache)
    device = cache.K.device
    if cache.scores is None:
        raise ValueError("the cache has no scores")
    to = None
    if into is not None:
        to = _struct(into)
        if into.K.device != device or into.K.dtype != cache.K.dtype:
            raise ValueError("the other cache must be of the same dtype and on the same device")
    at = _words(index, "index", (c.B, c.H, keep), torch.int32, device)
    lens = _lengths(seqlens, "seqlens", c.B, device)
    L = binding.lib()
    with _on(device, stream):
        if lens_out is None:
            lens_out = torch.empty(c.B, dtype=torch.int32, device=device)
        got = _lengths(lens_out, "lens_out", c.B, device)
        held, ws, size = _scratch(int(L.llla_cache_evict_workspace_bytes(c, keep)), device, workspace)
        st = L.llla_cache_evict(c, to, lens, keep, sinks, recent, got, at, ws, size, _stream_ptr(stream))
    if st != 0:
        raise LlaError(st, "llla_cache_evict")
    return lens_out
