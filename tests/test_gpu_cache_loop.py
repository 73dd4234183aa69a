"""The cache calls together, as a serving loop makes them: rows stored, attended to, scored, and given up when the cache is full; the same loop in a HIP
graph, on two streams, and by graphs that share a workspace.  Every call's tolerance is that of its own tests."""
import math

import pytest
import torch

import cache_reference as ref
import paper_2510_01450_amd as llla
import test_gpu_cache_rows as rows
import test_gpu_cache_scores as shares
import test_gpu_decode_q8 as attention

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
I8, E4M3, BF16, F32 = torch.int8, torch.float8_e4m3fn, torch.bfloat16, torch.float32
LAM = 1e-2


def _tokens(gen, B, H, HC, n, d, dtype):
    k, v = (torch.randn((B, HC, n, d), generator=gen).to(dtype).to(DEV) for _ in range(2))
    return k, v, torch.randn((B, H, n, d), generator=gen).to(dtype).to(DEV)


def _fresh(cache):
    return llla.Cache(*(None if t is None else t.clone() for t in cache))


def _same(a, b, what):
    for name, x, y in zip(a._fields, a, b):
        if x is not None:
            assert torch.equal(ref.bits(x), ref.bits(y)), "%s: %s" % (what, name)


@pytest.mark.parametrize("dtype,q_dtype,d,group", [(I8, BF16, 64, 1), (I8, F32, 128, 2), (E4M3, BF16, 128, 4), (E4M3, F32, 32, 2), (I8, F32, 16, 1)])
def test_serving_loop(dtype, q_dtype, d, group):
    """Prompts of their own lengths (one empty) in a padded batch, cut down to a budget; then single tokens until the caches are full again, and an eviction
    in place.  Each call's effect on the whole cache against the plain form."""
    B, HC, L, prompt, budget = 3, 2, 150, 140, 100
    H, scale = HC * group, 1 / math.sqrt(d)
    gen = torch.Generator().manual_seed(d)
    cache = llla.cache_alloc(B, HC, L, d, dtype, DEV, scores=True, pos=True)
    k, v, q = _tokens(gen, B, H, HC, prompt, d, q_dtype)
    lens = [140, 0, 77]
    host = rows._append(cache, k, v, None, lens, None)
    rows._same(cache, host, "prompt")
    # (a padded batch: the last queries of a shorter sequence stand in front of its length)
    for b, n in enumerate(lens):
        if n:
            q[b] = q[b].roll(prompt - n, 1)
    at = torch.tensor(lens, dtype=torch.int32, device=DEV)
    before = cache.scores.clone()
    llla.llla_cache_scores(q, cache, scale, seqlens=at)
    shares._check(cache, q, scale, lens, before, "prompt")
    rows._evict(cache, lens, budget, sinks=4, recent=16)
    lens = [min(n, budget) for n in lens]
    position = torch.tensor([140, 0, 77], dtype=torch.int32)
    for step in range(L - budget + 3):
        if max(lens) == L:
            rows._evict(cache, lens, budget, sinks=4, recent=16)
            lens = [min(n, budget) for n in lens]
        k, v, q = _tokens(gen, B, H, HC, 1, d, q_dtype)
        host = rows._append(cache, k, v, lens, None, position.tolist())
        rows._same(cache, host, "step %d" % step)
        lens = [n + 1 for n in lens]
        position += 1
        at = torch.tensor(lens, dtype=torch.int32, device=DEV)
        q = q[:, :, 0].contiguous()
        got = llla.llla_decode_q8(q, cache, LAM, scale, seqlens=at)
        if step % 13 == 0:
            attention._check(got, q, cache, scale, lens, "step")
        before = cache.scores.clone()
        llla.llla_cache_scores(q, cache, scale, seqlens=at)
        shares._check(cache, q, scale, lens, before, "step %d" % step)


class _Step:
    """One token: stored, attended to, scored; the cache cut back to its budget when `evict`."""

    def __init__(self, seed, dtype, d, L, budget, workspace=None, B=2, HC=2, group=2):
        gen = torch.Generator().manual_seed(seed)
        self.d, self.budget, self.group = d, budget, group
        self.cache = llla.cache_alloc(B, HC, L, d, dtype, DEV, scores=True, pos=True)
        k, v, _ = _tokens(gen, B, HC * group, HC, L, d, BF16)
        llla.llla_cache_append(self.cache, k, v, new_lens=torch.full((B,), budget, dtype=torch.int32, device=DEV))
        self.lens = torch.full((B,), budget, dtype=torch.int32, device=DEV)
        self.pos = self.lens.clone()
        self.k, self.v, q = _tokens(gen, B, HC * group, HC, 1, d, BF16)
        self.q = q[:, :, 0].contiguous()
        self.out = torch.empty_like(self.q)
        self.after = torch.empty_like(self.lens)
        self.ws = workspace

    def token(self, seed):
        gen = torch.Generator().manual_seed(seed)
        k, v, q = _tokens(gen, *self.q.shape[:2], self.k.shape[1], 1, self.d, BF16)
        self.k.copy_(k), self.v.copy_(v), self.q.copy_(q[:, :, 0])

    def run(self, evict=True):
        scale = 1 / math.sqrt(self.d)
        llla.llla_cache_append(self.cache, self.k, self.v, seqlens=self.lens, first_pos=self.pos)
        self.lens += 1
        self.pos += 1
        llla.llla_decode_q8(self.q, self.cache, LAM, scale, seqlens=self.lens, out=self.out, workspace=self.ws)
        llla.llla_cache_scores(self.q, self.cache, scale, seqlens=self.lens, workspace=self.ws)
        if evict:
            llla.llla_cache_evict(self.cache, self.budget, seqlens=self.lens, sinks=2, recent=8, lens_out=self.after, workspace=self.ws)
            self.lens.copy_(self.after)

    def same(self, other, what):
        _same(self.cache, other.cache, what)
        assert torch.equal(self.out, other.out) and torch.equal(self.lens, other.lens), what


def _capture(step):
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step.run()
    return graph


@pytest.mark.parametrize("dtype,d,L,budget", [(I8, 64, 700, 600), (E4M3, 128, 300, 200), (I8, 32, 20000, 17000), (E4M3, 16, 70, 40)])
def test_captured_step(dtype, d, L, budget):
    """Replays of a captured step, with other calls and synchronizations between them, against the same steps made eagerly: equal bits."""
    graphed, eager, other = (_Step(s, dtype, d, L, budget) for s in (1, 1, 2))
    for s in (graphed, eager):
        s.token(5)
        s.run()
    graph = _capture(graphed)
    graphed.same(eager, "capturing changes nothing")
    for i in range(6):
        for s in (graphed, eager):
            s.token(100 + i)
        graph.replay()
        other.token(i)
        other.run()
        if i % 2:
            torch.cuda.synchronize()
        eager.run()
        graphed.same(eager, "replay %d" % i)
    assert int(graphed.pos[0]) == budget + 7 and int(graphed.lens[0]) == budget


def test_graphs_and_calls_that_share_a_workspace():
    """A workspace holds nothing from one call for the next: two graphs and eager calls take turns in one."""
    probe = [_Step(s, dtype, d, L, b) for s, (dtype, d, L, b) in enumerate([(I8, 64, 900, 800), (E4M3, 128, 20000, 18000)])]
    need = max(max(llla.decode_q8_workspace_bytes(p.cache, 4), llla.cache_scores_workspace_bytes(p.cache, 4, 1, BF16), llla.cache_evict_workspace_bytes(p.cache, p.budget))
               for p in probe)
    ws = torch.full((need,), 0xA5, dtype=torch.uint8, device=DEV)
    shared = [_Step(s, dtype, d, L, b, ws) for s, (dtype, d, L, b) in enumerate([(I8, 64, 900, 800), (E4M3, 128, 20000, 18000)])]
    for a, b in zip(shared, probe):
        a.token(3), b.token(3)
        a.run(), b.run()
    graphs = [_capture(s) for s in shared]
    for i in range(4):
        ws.fill_(255 * (i % 2))
        for n in ((0, 1) if i % 2 else (1, 0)):
            shared[n].token(50 + i), probe[n].token(50 + i)
            if i == 2:
                shared[n].run()
            else:
                graphs[n].replay()
            probe[n].run()
            shared[n].same(probe[n], "turn %d of %d" % (i, n))


def test_two_streams_at_once():
    """Calls of two loops on two streams, with scratch of their own, in flight together."""
    kinds = [(I8, 64, 4000, 3900), (E4M3, 128, 4000, 3900)]
    alone, together = ([_Step(s, *k, B=4, HC=4) for s, k in enumerate(kinds)] for _ in range(2))
    for s in alone:
        for i in range(4):
            s.run(evict=i == 3)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in kinds]
    for i in range(4):
        for s, st in zip(together, streams):
            with torch.cuda.stream(st):
                s.run(evict=i == 3)
    torch.cuda.synchronize()
    for a, b in zip(alone, together):
        a.same(b, "streams")


def test_copies_that_leave_a_snapshot():
    """Evicting into another cache leaves the source as it was; decoding from the copy sees the rows kept."""
    s = _Step(7, I8, 64, 500, 400)
    s.run(evict=False)
    before = _fresh(s.cache)
    to = llla.cache_alloc(2, 2, 300, 64, I8, DEV, scores=True, pos=True)
    lens = llla.llla_cache_evict(s.cache, 256, seqlens=s.lens, sinks=2, recent=8, into=to)
    _same(s.cache, before, "the source")
    assert lens.cpu().tolist() == [256, 256]
    q = s.q.float()
    got = llla.llla_decode_q8(q, to, LAM, 0.125, seqlens=lens)
    attention._check(got, q, to, 0.125, [256, 256], "copy")
