"""Plain implementations of the cache calls in 64 bits, on the CPU, one row or block at a time."""
import math

import torch

BLOCK = 64
LARGEST = {torch.int8: 127.0, torch.float8_e4m3fn: 448.0}
CODES = tuple(LARGEST)


def least_exponent(top, dtype):
    """The smallest e >= -120 with top <= LARGEST 2^e; -128 if top is not finite."""
    if not math.isfinite(top):
        return -128
    e = -120
    while top > LARGEST[dtype] * 2.0 ** e:
        e += 1
    return e


def to_codes(x, dtype):
    """float64 numbers of at most the format's largest, to nearest even."""
    return torch.round(x).to(torch.int8) if dtype == torch.int8 else x.to(torch.float32).to(dtype)


def bits(t):
    """The tensor with a type that every operation has."""
    return t.view(torch.uint8) if t.dtype == torch.float8_e4m3fn else t


def values(c, e):
    """[n, d] rows as float64."""
    if e is None:
        return c.double()
    power = torch.tensor([math.nan if int(x) == -128 else 2.0 ** int(x) for x in e], dtype=torch.float64)
    return c.double() * power.repeat_interleave(BLOCK)[:c.shape[0], None]


class Host:
    """A cache on the host: lists of one head's tensors by (b, h)."""

    def __init__(self, cache):
        self.dtype = cache.K.dtype
        self.B, self.H, self.L, self.d = cache.K.shape
        f = lambda t: None if t is None else t.detach().cpu().clone()
        self.K, self.V, self.ke, self.ve, self.scores, self.pos = (f(t) for t in cache)

    def tensors(self):
        return {k: getattr(self, k) for k in ("K", "V", "ke", "ve", "scores", "pos") if getattr(self, k) is not None}

    def rows(self, which, b, h):
        c, e = (self.K, self.ke) if which == "K" else (self.V, self.ve)
        return values(c[b, h], None if e is None else e[b, h])


def append(host, k, v, lens, counts, first):
    for b in range(host.B):
        n, length = counts[b], lens[b]
        for h in range(host.H):
            for c, e, x in ((host.K, host.ke, k), (host.V, host.ve, v)):
                for i in range(n):
                    if length + i < host.L and e is None:
                        c[b, h, length + i] = x[b, h, i].to(c.dtype)
                if e is None:
                    continue
                end = min(length + n, host.L)
                for blk in range(length // BLOCK, -(-end // BLOCK)):
                    s0, s1 = max(length, blk * BLOCK), min(end, (blk + 1) * BLOCK)
                    if s0 >= s1:
                        continue
                    new = x[b, h, s0 - length:s1 - length].double()
                    top = new.abs().max().item() if torch.isfinite(new).all() else math.inf
                    need = least_exponent(top, host.dtype)
                    old = slice(blk * BLOCK, s0)
                    if s0 > blk * BLOCK:
                        was = int(e[b, h, blk])
                        need = -128 if -128 in (was, need) else max(was, need)
                        if need != -128 and need != was:
                            bits(c)[b, h, old] = bits(to_codes(c[b, h, old].double() * 2.0 ** (was - need), host.dtype))
                    e[b, h, blk] = need
                    put = torch.zeros_like(new) if need == -128 else new * 2.0 ** -need
                    bits(c)[b, h, s0:s1] = bits(to_codes(put, host.dtype))
            for i in range(n):
                if length + i < host.L:
                    if host.scores is not None:
                        host.scores[b, h, length + i] = 0.0
                    if host.pos is not None:
                        host.pos[b, h, length + i] = (length if first is None else first[b]) + i


def scores(host, Q, scale, lens):
    """What is added to host.scores, float64 [B, H, L]."""
    B, HQ, nq, _ = Q.shape
    out = torch.zeros((B, host.H, host.L), dtype=torch.float64)
    for b in range(B):
        L = lens[b]
        for hq in range(HQ):
            h = hq // (HQ // host.H)
            K = host.rows("K", b, h)[:L]
            for i in range(nq):
                seen = L - nq + i + 1
                if seen <= 0:
                    continue
                t = K[:seen] @ Q[b, hq, i].double() * scale
                w = torch.exp(t - t.max())
                out[b, h, :seen] += w / w.sum()
    return out


def ranked(host, b, h, length, sinks, recent):
    """Slots of a head, best first."""
    pos = host.pos[b, h] if host.pos is not None else torch.arange(host.L)
    newest = int(pos[:length].max()) if length else 0

    def key(s):
        p, score = int(pos[s]), float(host.scores[b, h, s])
        safe = p < sinks or (recent > 0 and p > newest - recent)
        return (0 if safe else 1, 0.0 if safe else -(-math.inf if math.isnan(score) else score), 0 if safe or not math.isnan(score) else 1, s)
    return sorted(range(length), key=key)


def evict(host, into, lens, keep, sinks, recent):
    """Changes `host` (into None) or `into`; returns (lengths, index [B][H] of lists)."""
    index = [[None] * host.H for _ in range(host.B)]
    source = {k: v.clone() for k, v in host.tensors().items()}
    for b in range(host.B):
        for h in range(host.H):
            length = lens[b]
            stay = sorted(ranked(host, b, h, length, sinks, recent)[:keep])
            if into is None:
                target = host
                holes = [s for s in range(min(keep, length)) if s not in set(stay)]
                movers = [s for s in stay if s >= keep]
                assert len(holes) == len(movers)
                moves = list(zip(movers, holes))
                place = {d: s for s, d in moves}
                index[b][h] = [place.get(j, j) for j in range(min(keep, length))]
            else:
                target = into
                moves = [(s, j) for j, s in enumerate(stay)]
                index[b][h] = stay
            for name, en in (("K", "ke"), ("V", "ve")):
                c = getattr(target, name)
                if en not in source:
                    for s, d in moves:
                        c[b, h, d] = source[name][b, h, s]
                    continue
                e, se = getattr(target, en), source[en]
                for blk in sorted({d // BLOCK for _, d in moves}):
                    here = [(s, d) for s, d in moves if d // BLOCK == blk]
                    was = int(source[en][b, h, blk]) if into is None else -120
                    now = was
                    for s, _ in here:
                        row = source[name][b, h, s].double().abs()
                        es = int(se[b, h, s // BLOCK])
                        top = row.max().item()
                        need = -128 if es == -128 or not math.isfinite(top) else least_exponent(top * 2.0 ** es, host.dtype)
                        now = -128 if -128 in (now, need) else max(now, need)
                    if into is None and now not in (was, -128):
                        rows = slice(blk * BLOCK, min((blk + 1) * BLOCK, keep))
                        bits(c)[b, h, rows] = bits(to_codes(source[name][b, h, rows].double() * 2.0 ** (was - now), host.dtype))
                    for s, d in here:
                        es = int(se[b, h, s // BLOCK])
                        row = source[name][b, h, s]
                        bits(c)[b, h, d] = bits(row if now == -128 else to_codes(row.double() * 2.0 ** (es - now), host.dtype))
                    e[b, h, blk] = now
            for s, d in moves:
                if target.scores is not None:
                    target.scores[b, h, d] = source["scores"][b, h, s]
                if target.pos is not None:
                    target.pos[b, h, d] = source["pos"][b, h, s] if "pos" in source else s
    return [min(n, keep) for n in lens], index
