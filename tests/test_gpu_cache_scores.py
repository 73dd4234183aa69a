"""Shares of the kernel weight against 64 bits.  Tolerance: a logit is a sum of d products of exact operands, d + 4 roundings of at most
2^-24 A, A = |scale| max |q| max |k| log2(e) the size of what is summed (fp32 operands in three bf16 leave out 2^-23 A more); a share has the errors of its own
logit, of its query's largest one and of the logarithm of the sum, ln 2 times, and some 2^-20 for the sums and exponentials.  A sum of shares is off
by that much of itself, and by half a step of the score it is added to."""
import math

import pytest
import torch

import cache_reference as ref
import paper_2510_01450_amd as llla

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
I8, E4M3, BF16, F32 = torch.int8, torch.float8_e4m3fn, torch.bfloat16, torch.float32


def _case(B, H, HC, L, d, dtype, nq, q_dtype, seed):
    g = torch.Generator(device="cpu").manual_seed(seed)
    K, Q = torch.randn((B, HC, L, d), generator=g), torch.randn((B, H, nq, d), generator=g)
    cache = llla.cache_alloc(B, HC, L, d, dtype, DEV, scores=True)
    if dtype in ref.CODES:
        llla.llla_cache_append(cache, K.to(DEV), K.to(DEV))
    else:
        cache.K.copy_(K.to(DEV))
    cache.scores.copy_(torch.rand((B, HC, L), generator=g).to(DEV))
    return cache, Q.to(q_dtype).to(DEV)


def _check(cache, Q, scale, lens, before, what):
    host = ref.Host(cache)
    if Q.dim() == 3:
        Q = Q[:, :, None]
    add = ref.scores(host, Q.cpu(), scale, lens)
    d = Q.shape[-1]
    A = abs(scale) * 1.4427 * max((Q.float().norm(dim=-1).max() * max(host.rows("K", b, h).norm(dim=-1).nan_to_num().max() for b in range(host.B) for h in range(host.H))).item(), 1.0)
    rel = 3 * math.log(2) * (d + 6) * 2.0 ** -24 * A + 2.0 ** -20
    got, was = cache.scores.double().cpu(), before.double().cpu()
    for b, n in enumerate(lens):
        assert torch.equal(got[b, :, n:], was[b, :, n:]), what + ": behind the length"
        err = (got[b, :, :n] - was[b, :, :n] - add[b, :, :n]).abs()
        bound = rel * add[b, :, :n] + 2.0 ** -23 * (was[b, :, :n] + add[b, :, :n]) + 1e-30
        assert bool((err <= bound).all()), "%s: sequence %d: %.3g of its bound" % (what, b, float((err / bound).max()))


TYPES = [(I8, BF16), (I8, F32), (E4M3, BF16), (E4M3, F32), (BF16, BF16), (F32, F32)]


@pytest.mark.parametrize("dtype,q_dtype", TYPES)
@pytest.mark.parametrize("d", [16, 32, 64, 128])
def test_types_and_lengths(dtype, q_dtype, d):
    """One query, few, many; more queries than rows (those in front of slot 0 see nothing); empty sequences."""
    for nq, lens in ((1, [0, 1, 64, 65, 200]), (5, [0, 3, 5, 130, 199]), (70, [0, 20, 70, 128, 200]), (200, [1, 150, 200, 0, 64])):
        cache, Q = _case(5, 4, 2, 200, d, dtype, nq, q_dtype, d + nq)
        before = cache.scores.clone()
        got = llla.llla_cache_scores(Q if nq > 1 else Q[:, :, 0], cache, 1 / math.sqrt(d), seqlens=torch.tensor(lens, dtype=torch.int32, device=DEV))
        assert got is cache.scores
        _check(cache, Q, 1 / math.sqrt(d), lens, before, "%s %s d=%d nq=%d" % (dtype, q_dtype, d, nq))


@pytest.mark.parametrize("dtype,q_dtype,group,nq", [(I8, BF16, 1, 1), (I8, F32, 8, 1), (BF16, BF16, 4, 1), (F32, F32, 16, 1), (F32, F32, 3, 11), (E4M3, BF16, 2, 31), (BF16, BF16, 1, 64), (BF16, BF16, 1, 65)])
def test_long_caches(dtype, q_dtype, group, nq):
    """Parts of the keys, with logits stored and formed again, one cache head with many readers."""
    L = 9001
    cache, Q = _case(1, 2 * group, 2, L, 64, dtype, nq, q_dtype, nq)
    before = cache.scores.clone()
    llla.llla_cache_scores(Q, cache, 0.125)
    _check(cache, Q, 0.125, [L], before, "long")


@pytest.mark.parametrize("dtype", [I8, BF16, F32])
def test_peaked_weights_and_accumulation(dtype):
    """Logits of +-60, called twice: the second adds the same again."""
    q_dtype = F32 if dtype == F32 else BF16
    cache, Q = _case(1, 2, 2, 700, 32, dtype, 3, q_dtype, 2)
    scale = 3.0
    before = cache.scores.clone()
    llla.llla_cache_scores(Q, cache, scale)
    once = cache.scores.clone()
    _check(cache, Q, scale, [700], before, "first")
    llla.llla_cache_scores(Q, cache, scale)
    _check(cache, Q, scale, [700], once, "second")


@pytest.mark.parametrize("scale", [-0.3, 0.0])
@pytest.mark.parametrize("nq", [1, 90])
def test_scales_that_are_not_positive(scale, nq):
    for dtype, q_dtype in ((E4M3, BF16), (BF16, BF16), (F32, F32)):
        cache, Q = _case(2, 4, 2, 333, 32, dtype, nq, q_dtype, 3)
        before = cache.scores.clone()
        llla.llla_cache_scores(Q, cache, scale, seqlens=torch.tensor([333, 100], dtype=torch.int32, device=DEV))
        _check(cache, Q, scale, [333, 100], before, "scale %g nq=%d" % (scale, nq))


@pytest.mark.parametrize("dtype,q_dtype,H,HC,nq,L", [(F32, F32, 16, 4, 40, 2999), (BF16, BF16, 6, 2, 100, 1500), (I8, F32, 8, 8, 300, 700), (E4M3, BF16, 2, 1, 129, 4000)])
def test_many_queries_of_few_heads(dtype, q_dtype, H, HC, nq, L):
    """More queries than a workgroup's waves share, keys cut into parts; groups of query heads, lengths of their own."""
    cache, Q = _case(2, H, HC, L, 64, dtype, nq, q_dtype, nq)
    lens = [L, L // 3]
    before = cache.scores.clone()
    llla.llla_cache_scores(Q, cache, 0.125, seqlens=torch.tensor(lens, dtype=torch.int32, device=DEV))
    _check(cache, Q, 0.125, lens, before, "many")


def test_sums_to_the_number_of_queries():
    cache, Q = _case(2, 4, 4, 3000, 64, BF16, 3000, BF16, 6)
    cache.scores.zero_()
    llla.llla_cache_scores(Q, cache, 0.125)
    # every query's shares sum to one: 3000 of them, each sum within 2^-16
    assert float((cache.scores.double().sum(-1) - 3000).abs().max()) < 3000 * 2.0 ** -16


def test_marked_blocks_and_rows_behind_the_length():
    cache, Q = _case(2, 2, 2, 400, 32, I8, 1, BF16, 8)
    lens = torch.tensor([300, 100], dtype=torch.int32, device=DEV)
    cache.scores.zero_()
    llla.llla_cache_scores(Q, cache, 0.2, seqlens=lens)
    want = cache.scores.clone()
    cache.k_exp[:, :, 5:] = -128
    cache.k_exp[1, 1, 1] = -128
    cache.scores.zero_()
    llla.llla_cache_scores(Q, cache, 0.2, seqlens=lens)
    assert torch.equal(cache.scores[0], want[0]) and torch.equal(cache.scores[1, 0], want[1, 0])
    assert torch.isnan(cache.scores[1, 1, :100]).all() and not cache.scores[1, 1, 100:].any()
    # rows behind the length that are not numbers (fp32), for one query and many
    for nq in (1, 90):
        cache, Q = _case(1, 2, 2, 300, 32, F32, nq, F32, 9)
        lens = torch.tensor([201], dtype=torch.int32, device=DEV)
        cache.scores.zero_()
        llla.llla_cache_scores(Q, cache, 0.2, seqlens=lens)
        want = cache.scores.clone()
        cache.K[:, :, 201:] = float("nan")
        cache.scores.zero_()
        llla.llla_cache_scores(Q, cache, 0.2, seqlens=lens)
        assert torch.equal(cache.scores, want)


def test_strides_and_stream():
    cache, Q = _case(2, 4, 2, 500, 64, BF16, 7, BF16, 10)
    before = cache.scores.clone()
    want = llla.llla_cache_scores(Q, cache, 0.125).clone()
    cache.scores.copy_(before)
    K = torch.zeros((2, 500, 3, 72), dtype=BF16, device=DEV)[:, :, 1:, 8:].transpose(1, 2)
    K.copy_(cache.K)
    Qt = torch.zeros((2, 7, 4, 64), dtype=BF16, device=DEV).transpose(1, 2)
    Qt.copy_(Q)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    llla.llla_cache_scores(Qt, cache._replace(K=K), 0.125, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(cache.scores, want)


@pytest.mark.parametrize("nq", [1, 80])
def test_offsets_beyond_32_bits(nq):
    """Rows 4 MB apart, 2.5 GB in all: the same bits as with rows together."""
    cache, Q = _case(1, 2, 2, 620, 64, I8, nq, BF16, 11)
    before = cache.scores.clone()
    want = llla.llla_cache_scores(Q, cache, 0.125).clone()
    cache.scores.copy_(before)
    flat = torch.zeros(620 * (4 << 20) + 128, dtype=I8, device=DEV)
    K = flat.as_strided((1, 2, 620, 64), (0, 64, 4 << 20, 1))
    K.copy_(cache.K)
    assert torch.equal(llla.llla_cache_scores(Q, cache._replace(K=K), 0.125), want)
