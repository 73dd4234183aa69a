"""Decode over 8-bit caches against the fp64 oracle on the rows that the codes stand for (exact numbers), through the same gate as the other decode calls:
1e-4 for an fp32 result; a bf16 result adds half a step, 2^-8 of the value."""
import math

import numpy as np
import pytest
import torch

import cache_reference as ref
import oracle
import paper_2510_01450_amd as llla
from parity import check

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
I8, E4M3, BF16, F32 = torch.int8, torch.float8_e4m3fn, torch.bfloat16, torch.float32
LAM = 1e-2


def _case(B, H, HC, L, d, dtype, q_dtype, seed, unit=False, spread=0.3):
    g = torch.Generator(device="cpu").manual_seed(seed)
    K, V, q = (torch.randn(s, generator=g) for s in ((B, HC, L, d), (B, HC, L, d), (B, H, d)))
    if unit:
        K, q = K / K.norm(dim=-1, keepdim=True), q / q.norm(dim=-1, keepdim=True)
    else:
        K = K * torch.exp(spread * torch.randn((B, HC, L, 1), generator=g))
    V = V * torch.exp(spread * torch.randn((B, HC, L, 1), generator=g))
    cache = llla.cache_alloc(B, HC, L, d, dtype, DEV)
    llla.llla_cache_append(cache, K.to(DEV), V.to(DEV))
    return q.to(q_dtype).to(DEV), cache


def _oracle(q, cache, scale, lens, lam=LAM):
    K, V = (x.cpu() for x in cache.values())               # (fp32: exact)
    group = q.shape[1] // K.shape[1]
    K, V = (x.repeat_interleave(group, 1).contiguous() for x in (K, V))
    return np.asarray(oracle.decode(q.float().cpu(), K, V, lam, scale, seqlens=[max(n, 1) for n in lens]))


def _check(got, q, cache, scale, lens, what, lam=LAM, far=0.0):
    want = _oracle(q, cache, scale, lens, lam)
    got = got.float().cpu().numpy()
    d = q.shape[-1]
    tol = 1e-4 + (2.0 ** -8 if what.endswith("bf16") else 0.0) + far
    for b, n in enumerate(lens):
        if n == 0:
            assert not got[b].any()
            continue
        # the gate's factor of ten below 4 d keys stands for |z|^2 / lambda = 10^4 (unit variance, d = 64): the part of 1 - z . rho that is left of moments in
        # 24 bits; larger keys lose as much more
        t = tol
        if n < 4 * d:
            K = cache.values()[0][b, :, :n].double().repeat_interleave(q.shape[1] // cache.K.shape[1], 0)
            t = tol * max(1.0, float((K - q[b, :, None].double()).square().sum(-1).max()) / (1e4 * lam))
        print(check(got[b:b + 1, :, None, :], want[b:b + 1, :, None, :], np.array([n - 1]), d, t, what + " L=%d" % n))


@pytest.mark.parametrize("dtype", [I8, E4M3])
@pytest.mark.parametrize("d", [16, 32, 64, 128])
@pytest.mark.parametrize("L", [1, 2, 31, 63, 64, 65, 100, 127, 257, 1000])
def test_lengths(dtype, d, L):
    for q_dtype, out in ((F32, F32), (BF16, BF16)):
        q, cache = _case(2, 2, 2, L, d, dtype, q_dtype, 100 * d + L, unit=out == F32)
        got = llla.llla_decode_q8(q, cache, LAM, 1 / math.sqrt(d), out_dtype=out)
        assert got.dtype == out
        _check(got, q, cache, 1 / math.sqrt(d), [L, L], "d=%d %s %s" % (d, dtype, "bf16" if out == BF16 else "f32"))


@pytest.mark.parametrize("dtype", [I8, E4M3])
@pytest.mark.parametrize("d,group", [(64, 1), (64, 4), (128, 2), (128, 8), (32, 3), (16, 5)])
def test_lengths_of_their_own(dtype, d, group):
    """Empty, short (key space), long sequences in one batch; several query heads to a cache head; bf16 queries with an fp32 result."""
    lens = [0, 1, 50, 64, 65, 700, 1999, 2500]
    q, cache = _case(8, 2 * group, 2, 2500, d, dtype, BF16, d + group)
    seq = torch.tensor(lens, dtype=torch.int32, device=DEV)
    got = llla.llla_decode_q8(q, cache, LAM, 1 / math.sqrt(d), seqlens=seq)
    _check(got, q, cache, 1 / math.sqrt(d), lens, "d=%d group=%d" % (d, group))
    # A bf16 result of more than 4 d keys has one term: x = w k is off by 2^-11 of itself, a moment by at most 2^-11 of the sum of w |k| |k|'.  The solve passes
    # that on by one over the smallest eigenvalue of Sigma / omega, (1 - sqrt(d / n))^2 of the keys' variance, 1/3 at d = 128 and 700 keys: 3 x 2^-11, up to
    # 2^-9.  It comes in from mu, Sigma and the value moments, and weights that differ leave fewer keys than n: 2^-7 in all.
    got = llla.llla_decode_q8(q, cache, LAM, 1 / math.sqrt(d), seqlens=seq, out_dtype=BF16)
    assert got.dtype == BF16
    _check(got, q, cache, 1 / math.sqrt(d), lens, "d=%d group=%d bf16" % (d, group), far=2.0 ** -7)


@pytest.mark.parametrize("B,H,L,d", [(1, 1, 20000, 64), (1, 4, 9000, 128), (3, 7, 3333, 64), (40, 16, 300, 64), (64, 16, 130, 32), (2, 300, 200, 16), (17, 9, 1111, 128)])
@pytest.mark.parametrize("dtype,out", [(I8, F32), (I8, BF16), (E4M3, BF16)])
def test_shapes_of_the_cut(B, H, L, d, dtype, out):
    """Few heads and long caches (many records), more heads than workgroups fit, numbers that divide nothing; with and without lengths, and without scratch.
    bf16 results: half a step, 2^-8, and the rounding of weights and weighted keys to 11 bits, which is random: 2^-11 is four times that of each."""
    q, cache = _case(B, H, H, L, d, dtype, F32, B + L, unit=True)
    scale = 1 / math.sqrt(d)
    tol = 1e-4 if out == F32 else 2.0 ** -8 + 2.0 ** -11
    got = llla.llla_decode_q8(q, cache, LAM, scale, out_dtype=out).float()
    lens = [L - (i * 7) % (L // 2) for i in range(B)]
    ragged = llla.llla_decode_q8(q, cache, LAM, scale, seqlens=torch.tensor(lens, dtype=torch.int32, device=DEV), out_dtype=out).float()
    none = llla.llla_decode_q8(q, cache, LAM, scale, workspace=torch.empty(256, dtype=torch.uint8, device=DEV), out_dtype=out).float()
    heads = [(b, h) for b in range(B) for h in range(H)][:: max(1, B * H // 24)]
    K, V = (x.cpu() for x in cache.values())
    for what, out, ns in (("even", got, [L] * B), ("ragged", ragged, lens), ("no scratch", none, [L] * B)):
        for b, h in heads:
            want = np.asarray(oracle.decode(q[b:b + 1, h:h + 1].cpu(), K[b:b + 1, h:h + 1].contiguous(), V[b:b + 1, h:h + 1].contiguous(), LAM, scale, seqlens=[ns[b]]))
            check(out[b:b + 1, h:h + 1].cpu().numpy()[:, :, None], want[:, :, None], np.array([ns[b] - 1]), d, tol, "%s %d %d" % (what, b, h))


def test_same_as_the_decode_of_the_numbers():
    """llla_decode of the fp32 rows that the codes stand for: the same result but for rounding (both within 1e-4 of the oracle)."""
    q, cache = _case(2, 8, 8, 4000, 64, E4M3, F32, 5, unit=True)
    K, V = cache.values()
    a, b = llla.llla_decode_q8(q, cache, LAM, 0.125), llla.llla_decode(q, K, V, LAM, 0.125)
    assert float((a - b).norm() / b.norm()) < 2e-4


@pytest.mark.parametrize("dtype", [I8, E4M3])
@pytest.mark.parametrize("d,L", [(16, 700), (32, 700), (64, 700), (128, 1500)])
def test_results_carry_24_bits(dtype, d, L):
    """Unit keys, many for the features: the moments are well conditioned, so an fp32 result is off by the roundings of their sums, a few dozen of 2^-24 at most
    (3.8e-6 is 64; 7e-7 seen).  Every head of several seeds: one weighted key in a hundred thousand with a term that does not belong to the other
    showed as 2e-5 in one head of twenty."""
    for seed in range(4):
        q, cache = _case(2, 16, 16, L, d, dtype, F32, 50 + seed, unit=True)
        got = llla.llla_decode_q8(q, cache, LAM, 1 / math.sqrt(d)).cpu().double()
        want = torch.from_numpy(_oracle(q, cache, 1 / math.sqrt(d), [L, L])).double()
        err = (got - want).norm(dim=-1) / want.norm(dim=-1)
        assert float(err.max()) < 64 * 2.0 ** -24, (seed, float(err.max()))


@pytest.mark.parametrize("dtype", [I8, E4M3])
@pytest.mark.parametrize("d", [64, 128, 32])
def test_peaked_and_flat_weights(dtype, d):
    """One key that holds nearly all weight, at the front, inside and at the end (the reference exponent moves late or not at all); weights all equal;
    logits of +-80.

    A key at distance |z| from the query that holds nearly all weight w = 1: 1 - z . rho and delta are lambda / (lambda + |z|^2) of the moments they are differences
    of.  Each of omega, mu, Sigma and sum w k v^T is rounded at least twice at the size of that key's own terms, when a head's parts are merged and when the
    mean is taken out, by 2^-24 of them at most, so the result, whatever the moments were summed with, may be off by 8 x 2^-24 |z|^2 / lambda of the
    values: 2.7e-2 at |z| = 24 (llla_decode on the same rows in fp32: 2.5e-3 at d = 32 and 64, up to 1.2e-2 at d = 128)."""
    L = 3000
    for kind in ("front", "middle", "end", "flat", "steep"):
        q, cache = _case(1, 2, 2, L, d, dtype, F32, 77, unit=True)
        K, V = (x.cpu() for x in cache.values())
        scale = 1.0
        if kind == "flat":
            q = torch.zeros_like(q)
        elif kind == "steep":
            scale = 80.0
        else:
            at = {"front": 3, "middle": L // 2 + 5, "end": L - 1}[kind]
            K[0, :, at] = 25.0 * q[0].cpu()
        cache = llla.cache_alloc(1, 2, L, d, dtype, DEV)
        llla.llla_cache_append(cache, K.to(DEV), V.to(DEV))
        got = llla.llla_decode_q8(q, cache, LAM, scale)
        _check(got, q, cache, scale, [L], "%s d=%d" % (kind, d), far=8 * 2.0 ** -24 * 24 ** 2 / LAM if kind in ("front", "middle", "end") else 0.0)


@pytest.mark.parametrize("dtype", [I8, E4M3])
def test_blocks_of_very_different_size(dtype):
    """Keys of one block 2^-12 of the others', values between 2^-30 and 2^30; all weight on the small ones."""
    L, d = 1500, 64
    g = torch.Generator(device="cpu").manual_seed(4)
    K, V, q = torch.randn((1, 2, L, d), generator=g), torch.randn((1, 2, L, d), generator=g), torch.randn((1, 2, d), generator=g)
    K = K / K.norm(dim=-1, keepdim=True)
    K[:, :, 640:704] *= 2.0 ** -12
    for power in (-30, 0, 30):
        cache = llla.cache_alloc(1, 2, L, d, dtype, DEV)
        llla.llla_cache_append(cache, K.to(DEV), (V * 2.0 ** power).to(DEV))
        qd = (q / q.norm(dim=-1, keepdim=True)).to(DEV)
        got = llla.llla_decode_q8(qd, cache, LAM, 0.125)
        _check(got, qd, cache, 0.125, [L], "2^%d" % power)


@pytest.mark.parametrize("d", [16, 32, 64, 128])
def test_every_code(d):
    """All codes of both formats, keys of e4m3 down to its subnormal numbers, against the oracle."""
    for dtype, codes in ((I8, torch.arange(-127, 128).to(torch.int8)), (E4M3, torch.cat([torch.arange(0, 127), torch.arange(128, 255)]).to(torch.uint8).view(E4M3))):
        L = 256 * 3
        cache = llla.cache_alloc(1, 1, L, d, dtype, DEV)
        n = codes.numel()
        i = (torch.arange(L)[:, None] * 7 + torch.arange(d)[None] * 31) % n
        ref.bits(cache.K)[0, 0] = ref.bits(codes)[i].to(DEV)
        ref.bits(cache.V)[0, 0] = ref.bits(codes)[(i * 5 + 3) % n].to(DEV)
        cache.k_exp.fill_(-7 if dtype == I8 else -8)
        cache.v_exp.fill_(-7 if dtype == I8 else -8)
        q = torch.randn((1, 1, d), generator=torch.Generator().manual_seed(d)).to(DEV)
        for L1 in (40, L):
            lens = torch.tensor([L1], dtype=torch.int32, device=DEV)
            got = llla.llla_decode_q8(q, cache, 0.1, 1 / math.sqrt(d), seqlens=lens)
            _check(got, q, cache, 1 / math.sqrt(d), [L1], "codes d=%d" % d, lam=0.1)


@pytest.mark.parametrize("dtype", [I8, E4M3])
@pytest.mark.parametrize("d", [64, 128])
def test_marked_blocks_and_what_lies_behind_the_length(dtype, d):
    """A block marked as not finite makes its heads' results NaN, and no other's; rows and exponents behind the length do not matter."""
    L = 1000
    q, cache = _case(2, 4, 2, L, d, dtype, F32, 9, unit=True)
    lens = torch.tensor([700, 40], dtype=torch.int32, device=DEV)
    want = llla.llla_decode_q8(q, cache, LAM, 0.1, seqlens=lens)
    assert torch.isfinite(want).all()
    cache.k_exp[:, :, 11:] = -128                             # from slot 704 on
    cache.k_exp[1, :, 1:] = -128
    ref.bits(cache.K)[0, :, 700:] = 0x7f
    ref.bits(cache.V)[0, :, 700:] = 0x7f
    assert torch.equal(llla.llla_decode_q8(q, cache, LAM, 0.1, seqlens=lens), want)
    for t, block in ((cache.k_exp, 3), (cache.v_exp, 5)):
        was = int(t[0, 1, block])
        t[0, 1, block] = -128
        got = llla.llla_decode_q8(q, cache, LAM, 0.1, seqlens=lens)
        assert torch.isnan(got[0, 2:]).all() and torch.equal(got[0, :2], want[0, :2]) and torch.equal(got[1], want[1])
        t[0, 1, block] = was
    cache.v_exp[1, 0, 0] = -128
    got = llla.llla_decode_q8(q, cache, LAM, 0.1, seqlens=lens)
    assert torch.isnan(got[1, :2]).all() and torch.equal(got[1, 2:], want[1, 2:]) and torch.equal(got[0], want[0])


def test_strides_output_and_stream():
    """Caches that are parts of larger tensors; the caller's result and scratch; another stream."""
    q, cache = _case(2, 4, 4, 900, 64, I8, BF16, 12)
    want = llla.llla_decode_q8(q, cache, LAM, 0.125, out_dtype=BF16)
    big = torch.zeros((2, 950, 4, 80), dtype=I8, device=DEV)
    K = big[:, :900, :, :64].transpose(1, 2)
    K.copy_(cache.K)
    V = torch.zeros((2, 5, 901, 96), dtype=I8, device=DEV)[:, 1:, 1:, 32:]
    V.copy_(cache.V)
    c = cache._replace(K=K, V=V)
    out = torch.empty((2, 4, 64), dtype=BF16, device=DEV)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = llla.llla_decode_q8(q, c, LAM, 0.125, out=out, stream=s, workspace=torch.empty(llla.decode_q8_workspace_bytes(c, 4) + 256, dtype=torch.uint8, device=DEV))
    torch.cuda.current_stream().wait_stream(s)
    assert got is out and torch.equal(got, want)


def test_offsets_beyond_32_bits():
    """A head that begins 4.5 GB into its cache, and rows 2.3 GB apart inside one."""
    d, L, HC = 64, 600, 2
    q, cache = _case(1, 2, 2, L, d, I8, F32, 15, unit=True)
    want = llla.llla_decode_q8(q, cache, LAM, 0.125)
    flat = torch.zeros(9 * (1 << 30) // 2 + L * d + 64, dtype=I8, device=DEV)
    K = flat.as_strided((1, HC, L, d), (0, 9 * (1 << 30) // 2, d, 1))
    K.copy_(cache.K)
    assert torch.equal(llla.llla_decode_q8(q, cache._replace(K=K), LAM, 0.125), want)
    del K, flat
    pitch = 4 * (1 << 20)
    flat = torch.zeros(L * pitch + 2 * d, dtype=I8, device=DEV)
    V = flat.as_strided((1, HC, L, d), (0, d, pitch, 1))
    V.copy_(cache.V)
    assert torch.equal(llla.llla_decode_q8(q, cache._replace(V=V), LAM, 0.125), want)


@pytest.mark.parametrize("d", [16, 32])
@pytest.mark.parametrize("L", [90, 140])
def test_rows_as_far_apart_as_they_may_be(d, L):
    """The largest row stride; lengths that end inside a block (rows of a transfer are read from 32-bit offsets)."""
    pitch = (1 << 25) - 16
    q, cache = _case(1, 2, 2, L, d, E4M3, BF16, L + d, unit=True)
    want = llla.llla_decode_q8(q, cache, LAM, 0.25)
    flat = torch.zeros((L - 1) * pitch + 2 * d, dtype=torch.uint8, device=DEV).view(E4M3)
    K = flat.as_strided((1, 2, L, d), (0, d, pitch, 1))
    K.copy_(cache.K)
    assert torch.equal(llla.llla_decode_q8(q, cache._replace(K=K), LAM, 0.25), want)
    one = llla.llla_decode_q8(q, cache, LAM, 0.25, out_dtype=BF16)
    assert torch.equal(llla.llla_decode_q8(q, cache._replace(K=K), LAM, 0.25, out_dtype=BF16), one)


@pytest.mark.parametrize("d", [16, 64, 128])
@pytest.mark.parametrize("out", [F32, BF16])
def test_without_a_workspace(d, out):
    """A workspace that is too small is none: one workgroup per head, every kind of length; and the others behind the result stay as they were."""
    lens = [0, 1, 64, 65, 4 * d, 4 * d + 1, 1500]
    q, cache = _case(7, 4, 2, 1500, d, E4M3, BF16, d, spread=0.1)
    seq = torch.tensor(lens, dtype=torch.int32, device=DEV)
    room = torch.full((9, 4, d), 7.0, dtype=out, device=DEV)
    got = llla.llla_decode_q8(q, cache, LAM, 1 / math.sqrt(d), seqlens=seq, out=room[1:8], workspace=torch.empty(256, dtype=torch.uint8, device=DEV))
    _check(got, q, cache, 1 / math.sqrt(d), lens, "no workspace d=%d %s" % (d, "bf16" if out == BF16 else "f32"), far=2.0 ** -7 if out == BF16 else 0.0)
    assert bool((room[0] == 7).all()) and bool((room[8] == 7).all())
