"""Host-side checks of the cache calls (no GPU needed): bad arguments are refused before anything is launched, with the status that names them."""
import ctypes

import pytest
import torch

import paper_2510_01450_amd as llla
from paper_2510_01450_amd.binding import _Strides
from paper_2510_01450_amd.cache import _CacheStruct

FAKE = 0x10000                              # never dereferenced: every call below fails a check first
F32, BF16, I8, E4M3 = 0, 1, 2, 3


def _cache(B=2, H=2, L=128, d=64, type=I8, **kw):
    s = _Strides(H * L * d, L * d, d)
    f = dict(K=FAKE, V=2 * FAKE, sk=s, sv=s, k_exp=3 * FAKE, v_exp=4 * FAKE, scores=5 * FAKE, pos=6 * FAKE, B=B, H=H, L_max=L, d=d, type=type)
    f.update(kw)
    return _CacheStruct(*[f[n] for n, _ in _CacheStruct._fields_])


def _append(c, k=FAKE, v=FAKE, sk=None, n=3, din=BF16, seqlens=None, new=None, first=None):
    s = sk or _Strides(2 * n * 64, n * 64, 64)
    return llla.lib().llla_cache_append(c, k, v, s, s, n, din, seqlens, new, first, None)


def _decode(c, q=FAKE, o=FAKE, seqlens=None, H=4, din=BF16, dout=BF16, lam=1e-2, scale=0.1):
    return llla.lib().llla_decode_q8(q, c, o, seqlens, H, din, dout, lam, scale, None, 0, None)


def _scores(c, Q=FAKE, sq=None, seqlens=None, H=4, nq=3, din=BF16, scale=0.1, ws=0, size=0):
    return llla.lib().llla_cache_scores(Q, c, sq or _Strides(H * nq * 64, nq * 64, 64), seqlens, H, nq, din, scale, ws, size, None)


def _evict(c, into=None, seqlens=None, keep=100, sinks=0, recent=0, lens=FAKE, index=None, ws=0, size=0):
    return llla.lib().llla_cache_evict(c, into, seqlens, keep, sinks, recent, lens, index, ws, size, None)


# what is wrong with a cache itself
BAD_CACHES = [
    (dict(K=0), 1), (dict(V=0), 1), (dict(k_exp=0), 1), (dict(v_exp=0), 1),
    (dict(B=0), 2), (dict(L=0), 2), (dict(d=-1), 2), (dict(B=70000), 2), (dict(sk=_Strides(0, 64 * 128, 64)), 2), (dict(sv=_Strides(16384, 0, 64)), 2),
    (dict(sk=_Strides(16384, 8192, 48)), 2), (dict(sk=_Strides(1 << 40, 1 << 34, 1 << 27)), 2), (dict(sv=_Strides(16384, 8192, -64)), 2),
    (dict(sk=_Strides(1 << 40, 1 << 34, 1 << 25)), 2), (dict(L=(1 << 30) + 64), 2),
    (dict(type=4), 3), (dict(type=-1), 3),
    (dict(K=FAKE + 8), 5), (dict(V=FAKE + 1), 5), (dict(sk=_Strides(16384, 8192, 72)), 5), (dict(scores=FAKE + 2), 5), (dict(pos=FAKE + 1), 5),
    (dict(d=48), 7), (dict(d=256), 7),
]


@pytest.mark.parametrize("kw,code", BAD_CACHES)
def test_bad_caches(kw, code):
    c = _cache(**kw)
    assert _append(c) == code and _decode(c) == code
    assert _evict(c, keep=1 if kw.get("L") == 0 else 100) == code
    if not set(kw) & {"V", "sv", "v_exp"}:
        assert _scores(c) == code               # (reads no values)
    good = _cache(K=7 * FAKE, V=8 * FAKE, k_exp=9 * FAKE, v_exp=10 * FAKE, scores=11 * FAKE, pos=12 * FAKE)
    assert _evict(good, into=c) == code


def test_missing_cache():
    assert _append(None) == 1 and _decode(None) == 1 and _scores(None) == 1 and _evict(None) == 1


@pytest.mark.parametrize("kw,code", [
    (dict(k=0), 1), (dict(v=0), 1), (dict(n=0), 2), (dict(n=-2), 2), (dict(sk=_Strides(0, 192, 64)), 2), (dict(sk=_Strides(384, 192, 32)), 2),
    (dict(din=I8), 3), (dict(din=7), 3), (dict(k=FAKE + 8), 5), (dict(sk=_Strides(384, 196, 64)), 5), (dict(seqlens=FAKE + 2), 5), (dict(new=FAKE + 1), 5),
    (dict(first=FAKE + 3), 5),
])
def test_append_refuses(kw, code):
    assert _append(_cache(), **kw) == code


def test_keys_and_values_in_one_array():
    """Read, they may be one; written, they would be written twice."""
    for kw in (dict(V=FAKE), dict(v_exp=3 * FAKE)):
        assert _append(_cache(**kw)) == 4 and _evict(_cache(**kw)) == 4
        assert _evict(_cache(), into=_cache(**dict(dict(K=7 * FAKE, V=8 * FAKE, k_exp=9 * FAKE, v_exp=10 * FAKE, scores=0, pos=0), **{k: 7 * FAKE if k == "V" else 9 * FAKE for k in kw}))) == 4
        assert _scores(_cache(**kw)) == 6


@pytest.mark.parametrize("kw,code", [
    (dict(q=0), 1), (dict(o=0), 1), (dict(H=3), 2), (dict(H=0), 2), (dict(H=-2), 2), (dict(H=65536), 2), (dict(din=I8), 3), (dict(dout=E4M3), 3),
    (dict(lam=0.0), 4), (dict(lam=float("nan")), 4), (dict(lam=float("inf")), 4), (dict(scale=float("inf")), 4), (dict(q=FAKE + 4), 5), (dict(o=FAKE + 8), 5),
    (dict(seqlens=FAKE + 2), 5),
])
def test_decode_refuses(kw, code):
    assert _decode(_cache(), **kw) == code


def test_decode_takes_codes_only():
    for t in (F32, BF16):
        assert _decode(_cache(type=t)) == 3
        assert llla.lib().llla_decode_q8_workspace_bytes(_cache(type=t), 4) == 0
    assert llla.lib().llla_decode_q8_workspace_bytes(_cache(), 3) == 0


@pytest.mark.parametrize("kw,code", [
    (dict(Q=0), 1), (dict(H=3), 2), (dict(nq=0), 2), (dict(sq=_Strides(768, 192, 16)), 2), (dict(din=I8), 3), (dict(scale=float("nan")), 4),
    (dict(Q=FAKE + 2), 5), (dict(sq=_Strides(768, 193, 64)), 5), (dict(seqlens=FAKE + 2), 5),
    (dict(), 6), (dict(ws=FAKE + 16, size=1 << 30), 6), (dict(ws=FAKE, size=16), 6),
])
def test_scores_refuse(kw, code):
    assert _scores(_cache(), **kw) == code


def test_scores_need_an_array_and_the_queries_type():
    assert _scores(_cache(scores=0)) == 1
    assert _scores(_cache(type=F32)) == 3 and _scores(_cache(type=BF16), din=F32) == 3
    assert _scores(_cache(type=F32), din=F32) == 6
    assert _scores(_cache(V=0, v_exp=0)) == 6               # values are not read


@pytest.mark.parametrize("kw,code", [
    (dict(lens=0), 1), (dict(keep=0), 2), (dict(keep=129), 2), (dict(sinks=-1), 4), (dict(recent=-1), 4), (dict(sinks=60, recent=41), 4),
    (dict(sinks=2147483647, recent=2147483647), 4), (dict(seqlens=FAKE), 4), (dict(lens=FAKE + 2), 5), (dict(seqlens=FAKE + 1), 5), (dict(index=FAKE + 1), 5),
    (dict(), 6), (dict(ws=FAKE + 16, size=1 << 30), 6), (dict(ws=FAKE, size=64), 6),
])
def test_evict_refuses(kw, code):
    assert _evict(_cache(), **kw) == code


def test_evict_refuses_another_cache_that_does_not_fit():
    c = _cache()
    other = dict(K=7 * FAKE, V=8 * FAKE, k_exp=9 * FAKE, v_exp=10 * FAKE, scores=11 * FAKE, pos=12 * FAKE)
    assert _evict(c, into=_cache(**other)) == 6             # all is well but for the workspace
    assert _evict(c, into=_cache(**dict(other, scores=0, pos=0))) == 6
    for kw, code in ((dict(B=1), 2), (dict(H=1), 2), (dict(L=99), 2), (dict(d=32), 2), (dict(type=E4M3), 3), (dict(K=FAKE), 4), (dict(V=2 * FAKE), 4),
                     (dict(V=7 * FAKE), 4), (dict(k_exp=3 * FAKE), 4), (dict(v_exp=4 * FAKE), 4), (dict(scores=5 * FAKE), 4), (dict(pos=6 * FAKE), 4)):
        assert _evict(c, into=_cache(**dict(other, **kw))) == code, kw
    assert _evict(_cache(scores=0)) == 1


def test_workspace_sizes():
    L = llla.lib()
    c = _cache(B=1, H=16, L=32768)
    assert L.llla_decode_q8_workspace_bytes(c, 16) > 0 and L.llla_decode_q8_workspace_bytes(_cache(L=64), 4) == 0
    # decode steps keep their logits; prompts one number per query, and two per query and part of the keys, never more than 4096 parts of 256 queries (8 MiB): nothing
    # of the size of queries times keys
    assert 16 * 32768 * 4 <= L.llla_cache_scores_workspace_bytes(c, 16, 1, BF16) < 16 * 32768 * 4 + (1 << 20)
    assert L.llla_cache_scores_workspace_bytes(c, 16, 32768, BF16) <= 16 * 32768 * 4 + (8 << 20) + 512
    # slots of the rows that move; long rows also three histograms of 2048 bins
    assert L.llla_cache_evict_workspace_bytes(_cache(B=1, H=16, L=16384), 4096) <= 16 * 4 * (2 * 4096 + 256)
    assert L.llla_cache_evict_workspace_bytes(c, 4096) <= 16 * 4 * (2 * 4096 + 3 * 2048 + 256)
    assert L.llla_cache_evict_workspace_bytes(c, 0) == 0 and L.llla_cache_evict_workspace_bytes(c, 40000) == 0


def test_bindings_have_no_cpu_path_and_word_mistakes():
    cache = llla.cache_alloc(1, 1, 64, 16, torch.int8, "cpu", scores=True)
    x = torch.zeros(1, 1, 4, 16)
    for call in (lambda: llla.llla_cache_append(cache, x, x), lambda: llla.llla_decode_q8(x[:, :, 0], cache, 1e-2, 0.1),
                 lambda: llla.llla_cache_scores(x, cache, 0.1), lambda: llla.llla_cache_evict(cache, 5)):
        with pytest.raises(ValueError, match="device memory"):
            call()
    with pytest.raises(ValueError):
        llla.cache_alloc(1, 1, 64, 16, torch.float16, "cpu")


def test_values_of_a_cache():
    cache = llla.cache_alloc(1, 1, 70, 16, torch.int8, "cpu")
    cache.K[0, 0, 3] = 5
    cache.K[0, 0, 65] = -127
    cache.V[0, 0, 66] = 1
    cache.k_exp[0, 0] = torch.tensor([-2, 3], dtype=torch.int8)
    cache.v_exp[0, 0, 1] = -128
    K, V = cache.values()
    assert K[0, 0, 3, 0] == 1.25 and K[0, 0, 65, 1] == -1016 and not K[0, 0, 4].any()
    assert not V[0, 0, :64].any() and torch.isnan(V[0, 0, 64:]).all()
