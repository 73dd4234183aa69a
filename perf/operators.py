"""The calls of a serving loop's cache that this library is held to: storing rows, attention over 8-bit rows, the accumulated weight
of cached keys, and eviction by it.

A case is a dict of plain values:
  op      "append" | "decode_q8" | "scores" | "evict"
  B       sequences
  H, HC   query heads and cache heads; H // HC query heads read one cache head
  n       capacity of the cache
  d       head dimension, one of 16, 32, 64, 128
  cache   "int8" | "e4m3" (codes with one power of two for every 64 rows of a head) | "bf16" | "f32"
  dtype   "bf16" | "f32": new rows (append), queries
  out     type of the result (decode_q8)
  m       rows stored per sequence (append; evict: stored before each eviction, 0 = none), queries per sequence (scores)
  keep    evict: rows kept per head
  ragged  every sequence has a length of its own, between an eighth of the capacity and all of it
  into    evict: into another cache, in the order of the slots (otherwise in place)
Every attention uses the ridge 1e-2 and the scale 1/sqrt(d).

Codes and exponents of 8-bit caches are whole numbers here and equal bit for bit: the exponent follows from the largest value, products with
a power of two are exact, and codes are rounded to nearest even.
"""
import math

import torch

own = False

LAMBDA = 1e-2
BLOCK = 64                                   # rows that share an exponent
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "int8": torch.int8, "e4m3": torch.float8_e4m3fn}
# a block's values are code * 2^e, e the smallest with max|x| <= LIMIT * 2^e: LIMIT = FRACTION * 2^POWER
FRACTION = {"int8": 127.0 / 128.0, "e4m3": 0.875}
POWER = {"int8": 7, "e4m3": 9}
LEAST = -120                                 # least exponent: smaller values are stored as zero


def _case(op, B, H, HC, n, d, cache, dtype="bf16", out="bf16", m=0, keep=0, ragged=False, into=False, name=None):
    case = {"op": op, "B": B, "H": H, "HC": HC, "n": n, "d": d, "cache": cache, "dtype": dtype, "out": out, "m": m, "keep": keep,
            "ragged": ragged, "into": into}
    if name is not None:
        case["name"] = name
    return case


def listed():
    return [
        # one generated token of a single conversation
        _case("decode_q8", 1, 16, 16, 4096, 64, "int8", name="decode_single"),
        # one generated token of a full serving batch, all caches full
        _case("decode_q8", 32, 16, 16, 32768, 64, "int8", name="decode_batch"),
        # a serving batch of conversations of different lengths, four query heads to a cache head, the larger head dimension
        _case("decode_q8", 16, 16, 4, 16384, 128, "e4m3", ragged=True, name="decode_ragged_d128"),
        # an fp32 model with many small heads
        _case("decode_q8", 8, 32, 32, 4096, 32, "int8", "f32", "f32", name="decode_small_heads_f32"),
        # a chunk of every prompt of a batch goes behind what is there
        _case("append", 8, 16, 16, 8192, 64, "int8", m=2047, ragged=True, name="append_chunk"),
        # the new token of every conversation of a batch
        _case("append", 64, 8, 8, 8192, 128, "e4m3", m=1, ragged=True, name="append_token"),
        # what the new token's query looks at, a full batch
        _case("scores", 32, 16, 16, 32768, 64, "int8", m=1, name="scores_batch"),
        # what a whole prompt looks at
        _case("scores", 2, 16, 16, 4096, 64, "bf16", m=4096, name="scores_prompt"),
        # what the last tokens of every prompt look at, shared cache heads, fp32
        _case("scores", 4, 16, 4, 3001, 128, "f32", "f32", m=32, ragged=True, name="scores_window_f32"),
        # long prompts become caches of an eighth
        _case("evict", 4, 16, 16, 32768, 128, "bf16", keep=4096, into=True, name="evict_prompts"),
        # a loop at its budget: 64 new rows come, 64 old ones go, in place
        _case("evict", 32, 8, 8, 4160, 64, "int8", m=64, keep=4096, name="evict_step"),
        # one very long document
        _case("evict", 1, 8, 8, 131071, 128, "e4m3", keep=16385, into=True, name="evict_long"),
    ]


def _between(rng, low, high):
    """A whole number, uniform in its logarithm."""
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    op = rng.choice(["decode_q8", "decode_q8", "append", "scores", "scores", "evict"])
    d = rng.choice([64, 64, 128, 128, 32, 16])
    HC = rng.choice([1, 2, 4, 8, 16])
    H = HC * rng.choice([1, 1, 2, 4])
    codes = rng.choice(["int8", "e4m3"])
    ragged = rng.random() < 0.5
    if op == "decode_q8":
        out = rng.choice(["bf16", "bf16", "f32"])
        # results in fp32 of some more keys than features mean little: the ridge alone holds the system up
        n = _between(rng, 1, 32768) if out == "bf16" else _between(rng, 1, 64) if rng.random() < 0.25 else _between(rng, 32 * d if ragged else 4 * d, 32768)
        B = _between(rng, 1, max(1, min(64, (1 << 23) * 64 // (max(d, 64) * H * n))))
        return _case(op, B, H, HC, n, d, codes, "f32" if out == "f32" else "bf16", out, ragged=ragged)
    if op == "append":
        n = _between(rng, 2, 16384)
        m = rng.choice([1, _between(rng, 1, max(1, n // 2))])
        B = _between(rng, 1, max(1, min(64, (1 << 25) // (HC * n * d))))
        return _case(op, B, HC, HC, n, d, rng.choice([codes, codes, "bf16"]), rng.choice(["bf16", "f32"]) if codes == "int8" else "bf16", m=m, ragged=ragged)
    cache = rng.choice([codes, "bf16", "f32"])
    dtype = cache if cache in ("bf16", "f32") else rng.choice(["bf16", "f32"])
    if op == "scores":
        n = _between(rng, 1, 32768)
        m = rng.choice([1, _between(rng, 1, min(n, 64)), _between(rng, 1, min(n, 4096))])
        m = min(m, max(1, (1 << 28) // (H * n)))
        B = _between(rng, 1, max(1, min(64, (1 << 28) // (H * n * m + 16 * HC * n))))
        return _case(op, B, H, HC, n, d, cache, dtype, m=m, ragged=ragged)
    n = _between(rng, 2, 65536)
    B = _between(rng, 1, max(1, min(32, (1 << 26) // (HC * n * d))))
    if rng.random() < 0.5:
        return _case(op, B, HC, HC, n, d, cache, dtype, keep=_between(rng, 1, n), ragged=ragged, into=True)
    m = _between(rng, 1, max(1, min(n // 8, 512)))
    return _case(op, B, HC, HC, max(n, 2), d, cache, dtype, m=m, keep=max(n, 2) - m)


def _recent(case):
    """Rows that the loop protects as the newest ones, beside the first four."""
    return max(0, min(case["keep"] - 4, max(case["m"], 64)))


def _sinks(case):
    return min(4, case["keep"] - _recent(case))


# ---- the format ------------------------------------------------------------------------------------------------------------
def _least_exponent(top, cache):
    """The smallest e >= LEAST with top <= LIMIT * 2^e."""
    f, x = torch.frexp(top)
    return torch.where(top > 0, x - POWER[cache] + (f > FRACTION[cache]).to(x.dtype), LEAST).clamp_(min=LEAST)


def _power(e):
    """2^e in fp32 as a tensor; exact for every exponent that a block can have."""
    return torch.ldexp(torch.ones((), dtype=torch.float32, device=e.device), e.to(torch.int32))


def _codes(x, cache):
    """fp32 values in units of a block's power as codes, rounded to nearest even."""
    return torch.round(x).to(torch.int8) if cache == "int8" else x.to(torch.float8_e4m3fn)


def _quantised(x, cache):
    """[B, H, n, d] fp32 as (codes, exponents [B, H, blocks])."""
    B, H, n, d = x.shape
    blocks = -(-n // BLOCK)
    x = torch.nn.functional.pad(x, (0, 0, 0, blocks * BLOCK - n)).view(B, H, blocks, BLOCK, d)
    e = _least_exponent(x.abs().amax((3, 4)), cache)
    c = _codes(x / _power(e)[..., None, None], cache).view(B, H, blocks * BLOCK, d)[:, :, :n].contiguous()
    return c, e.to(torch.int8)


def _bits(c):
    """The tensor as one that can be indexed and assigned whatever its type."""
    return c.view(torch.int8) if c.dtype == torch.float8_e4m3fn else c


def _values(c, e, dtype=torch.float32):
    """Rows of a cache as numbers."""
    if e is None:
        return c.to(dtype)
    return c.to(dtype) * _power(e).to(dtype).repeat_interleave(BLOCK, 2)[:, :, :c.shape[2], None]


# ---- inputs ----------------------------------------------------------------------------------------------------------------
def _normal(gen, shape, dtype=torch.float32):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32).to(dtype)


def _rows(gen, shape, unit):
    """Keys or values: tokens of different size, or (fp32 models) of length one."""
    x = _normal(gen, shape)
    if unit:
        return x / x.norm(dim=-1, keepdim=True)
    return x * torch.exp(0.2 * _normal(gen, shape[:-1] + (1,)))


def prepare(case, seed):
    """What a serving loop holds before the call: the cache with its lengths, the new rows or queries."""
    B, H, HC, n, d, m = (case[k] for k in ("B", "H", "HC", "n", "d", "m"))
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dt, unit = TYPES[case["dtype"]], case["out"] == "f32"
    s = {"case": case, "scale": 1.0 / math.sqrt(d), "ke": None, "ve": None, "lens": None, "pos": None}
    if case["ragged"]:
        s["lens"] = torch.randint(max(1, n // 8), n + 1, (B,), generator=gen, device="cuda", dtype=torch.int32)
    K, V = _rows(gen, (B, HC, n, d), unit), _rows(gen, (B, HC, n, d), unit)
    if case["cache"] in POWER:
        s["K"], s["ke"] = _quantised(K, case["cache"])
        s["V"], s["ve"] = _quantised(V, case["cache"])
    else:
        s["K"], s["V"] = K.to(TYPES[case["cache"]]), V.to(TYPES[case["cache"]])
    del K, V
    if case["op"] == "append":
        # room for the new rows; some sequences of a ragged batch bring fewer
        full = n - m if s["lens"] is None else s["lens"]
        s["lens"] = torch.full((B,), n - m, device="cuda", dtype=torch.int32) if s["lens"] is None else full.clamp(max=n - m)
        if case["ragged"]:
            s["new"] = torch.randint((m + 1) // 2, m + 1, (B,), generator=gen, device="cuda", dtype=torch.int32)
        else:
            s["new"] = None
    if m and case["op"] != "scores":
        s["k"], s["v"] = _rows(gen, (B, HC, m, d), False).to(dt), _rows(gen, (B, HC, m, d), False).to(dt)
    if case["op"] == "decode_q8":
        q = _normal(gen, (B, H, d))
        s["q"] = (q / q.norm(dim=-1, keepdim=True) if unit else q).to(dt)
    if case["op"] == "scores":
        s["q"] = _normal(gen, (B, H, m, d), dt)
    if case["op"] in ("scores", "evict"):
        # weights gathered so far: a few keys hold most of it; in front of a call that adds to them, of the size of what it adds
        s["scores"] = torch.exp(3.0 * _normal(gen, (B, HC, n))) if case["op"] == "evict" else torch.exp(_normal(gen, (B, HC, n))) * (H // HC * m / n)
    if case["op"] == "evict":
        # where the rows of a cache that has evicted before come from
        first = torch.arange(n, device="cuda", dtype=torch.int32)
        s["pos"] = torch.stack([first[torch.randperm(n, generator=gen, device="cuda")] for _ in range(B)])[:, None].expand(B, HC, n).contiguous()
        if m:
            s["full"] = torch.full((B,), n, device="cuda", dtype=torch.int32)
            s["kept"] = torch.full((B,), case["keep"], device="cuda", dtype=torch.int32)
            s["next"] = torch.full((B,), n, device="cuda", dtype=torch.int32)
        if case["into"]:
            k = case["keep"]
            blocks = -(-k // BLOCK)
            s["Ki"], s["Vi"] = (torch.zeros((B, HC, k, d), device="cuda", dtype=s["K"].dtype) for _ in range(2))
            s["kei"], s["vei"] = (torch.zeros((B, HC, blocks), device="cuda", dtype=torch.int8) if s["ke"] is not None else None for _ in range(2))
            s["scoresi"] = torch.zeros((B, HC, k), device="cuda")
            s["posi"] = torch.zeros((B, HC, k), device="cuda", dtype=torch.int32)
    return s


# ---- plain forms -----------------------------------------------------------------------------------------------------------
def _heads(x, group):
    """One cache head for every query head."""
    return x if group == 1 else x.repeat_interleave(group, 1)


def _lengths(s, n):
    return torch.full((s["case"]["B"],), n, device="cuda") if s["lens"] is None else s["lens"].long()


def _plain_decode(s):
    case, q = s["case"], s["q"]
    n, d, group = case["n"], case["d"], case["H"] // case["HC"]
    # 64 bits where 1 - z . rho cancels (few keys for the features) or the result is to hold 24 bits of it
    wide = torch.float64 if case["out"] == "f32" or n <= 32 * d else torch.float32
    K, V = _heads(_values(s["K"], s["ke"], wide), group), _heads(_values(s["V"], s["ve"], wide), group)
    qw = q.to(wide)
    seen = torch.arange(n, device="cuda") < _lengths(s, n)[:, None, None]
    t = torch.where(seen, s["scale"] * torch.matmul(K, qw[..., None])[..., 0], -math.inf)
    w = torch.exp(t - t.amax(-1, keepdim=True))
    z = K - qw[:, :, None]
    wz = w[..., None] * z
    S = torch.matmul(wz.transpose(-1, -2).contiguous(), z).double() + LAMBDA * torch.eye(d, device="cuda", dtype=torch.float64)
    mu = wz.double().sum(2)
    rho = torch.linalg.solve(S, mu)
    delta = w.double().sum(-1) - (mu * rho).sum(-1)
    a = w * (1 - torch.matmul(z, rho.to(wide)[..., None])[..., 0]) / delta.to(wide)[..., None]
    return torch.matmul(a[:, :, None], V)[:, :, 0].to(TYPES[case["out"]])


def _plain_append(s, lens, new):
    """Rows k, v of every sequence behind its lens rows: whole windows of blocks are read, changed and written back."""
    case, n, m = s["case"], s["case"]["n"], s["case"]["m"]
    B = case["B"]
    lens = lens.long()
    count = torch.full((B,), m, device="cuda") if new is None else new.long()
    first = lens // BLOCK * BLOCK
    wide = -(-(m + BLOCK - 1) // BLOCK) * BLOCK
    slot = first[:, None] + torch.arange(wide, device="cuda")                      # [B, wide]
    i = slot - lens[:, None]
    is_new = (i >= 0) & (i < count[:, None]) & (slot < n)
    is_old = (i < 0) & (slot < n)
    b, at = torch.nonzero(is_new | is_old, as_tuple=True)
    blocks = slot[:, ::BLOCK] // BLOCK
    has_new = is_new.view(B, -1, BLOCK).any(-1)
    bb, bat = torch.nonzero(has_new, as_tuple=True)
    for x, c, e in ((s["k"], s["K"], s["ke"]), (s["v"], s["V"], s["ve"])):
        rows = torch.gather(x.float(), 2, i.clamp(0, m - 1)[:, None, :, None].expand(-1, x.shape[1], -1, x.shape[3]))
        if e is None:
            nb, nat = torch.nonzero(is_new, as_tuple=True)
            c[nb, :, slot[nb, nat]] = rows[nb, :, nat].to(c.dtype)
            continue
        shape = rows.shape[:2] + (wide // BLOCK, BLOCK, rows.shape[3])
        top = torch.where(is_new[:, None, :, None], rows.abs(), 0).view(shape).amax((3, 4))
        was = e.long().gather(2, blocks.clamp(max=e.shape[2] - 1)[:, None].expand(-1, e.shape[1], -1)).int()
        open_ = is_old.view(B, -1, BLOCK).any(-1)[:, None]
        now = _least_exponent(top, case["cache"])
        now = torch.where(open_, torch.maximum(now, was), now)
        old = torch.gather(c.view(torch.int8), 2, slot.clamp(max=n - 1)[:, None, :, None].expand(-1, c.shape[1], -1, c.shape[3])).view(c.dtype).float()
        old = old.view(shape) * _power(torch.where(open_, was - now, 0))[..., None, None]
        put = torch.where(is_new[:, None, :, None].view(B, 1, -1, BLOCK, 1), rows.view(shape) / _power(now)[..., None, None], old)
        put = _bits(_codes(put, case["cache"]).view(rows.shape))
        _bits(c)[b, :, slot[b, at]] = put[b, :, at]
        e[bb, :, blocks[bb, bat]] = now.to(torch.int8)[bb, :, bat]
    if s["pos"] is not None:
        nb, nat = torch.nonzero(is_new, as_tuple=True)
        s["pos"][nb, :, slot[nb, nat]] = (s["next"][nb] + i[nb, nat]).int()[:, None]
        s["scores"][nb, :, slot[nb, nat]] = 0.0


def _plain_scores(s):
    case, n, m, group = s["case"], s["case"]["n"], s["case"]["m"], s["case"]["H"] // s["case"]["HC"]
    K = _heads(_values(s["K"], s["ke"]), group)
    t = torch.matmul(s["q"].float(), K.transpose(-1, -2).contiguous()) * s["scale"]
    # query i of m stands at row len - m + i and sees the rows up to its own
    last = _lengths(s, n)[:, None] - m + torch.arange(m, device="cuda")
    t = torch.where(torch.arange(n, device="cuda") <= last[:, None, :, None], t, -math.inf)
    w = torch.exp(t - t.amax(-1, keepdim=True).clamp(min=torch.finfo(torch.float32).min))
    p = w / w.sum(-1, keepdim=True).clamp(min=torch.finfo(torch.float32).tiny)
    s["scores"] += p.sum(2).view(case["B"], case["HC"], group, n).sum(2)
    return s["scores"]


def _plain_evict(s, lens):
    case = s["case"]
    B, HC, n, keep = case["B"], case["HC"], case["n"], case["keep"]
    slots = torch.arange(n, device="cuda")
    live = (slots < lens.long()[:, None])[:, None].expand(B, HC, n)
    pos, scores = s["pos"], s["scores"]
    newest = torch.where(live, pos, -1).amax(-1, keepdim=True)
    safe = live & ((pos < _sinks(case)) | (pos > newest - _recent(case)))
    rank = torch.where(safe, math.inf, torch.where(live, scores, -math.inf))
    order = torch.sort(rank, dim=-1, descending=True, stable=True).indices[..., :keep]
    kept = torch.zeros((B, HC, n), dtype=torch.bool, device="cuda").scatter_(2, order, True) & live
    lens_out = lens.clamp(max=keep)
    count = kept.sum(-1, keepdim=True)
    if case["into"]:
        src = torch.sort((~kept).to(torch.int8), dim=-1, stable=True).indices[..., :keep]       # kept slots in their order
        dst = torch.arange(keep, device="cuda").expand(B, HC, keep)
        move = dst < count
        to = {k: s[k + "i"] for k in ("K", "V", "ke", "ve", "scores", "pos")}
    else:
        most = min(keep, n - keep)
        hole = live & ~kept & (slots < keep)
        src = torch.sort((~(kept & (slots >= keep))).to(torch.int8), dim=-1, stable=True).indices[..., :most]
        dst = torch.sort((~hole).to(torch.int8), dim=-1, stable=True).indices[..., :most]
        move = torch.arange(most, device="cuda") < hole.sum(-1, keepdim=True)
        to = {k: s[k] for k in ("K", "V", "ke", "ve", "scores", "pos")}
    b, h, i = torch.nonzero(move, as_tuple=True)
    at, frm = dst[b, h, i], src[b, h, i]
    for c, e in (("K", "ke"), ("V", "ve")):
        if s[e] is None:
            to[c][b, h, at] = s[c][b, h, frm]
            continue
        was = s[e][b, h, frm // BLOCK].int()
        rows = _bits(s[c])[b, h, frm].view(s[c].dtype).float()
        need = torch.where(rows.abs().amax(-1) > 0, was + _least_exponent(rows.abs().amax(-1), case["cache"]), LEAST).clamp(min=LEAST)
        blocks = to[e].shape[2]
        now = torch.full((B, HC, blocks), LEAST, device="cuda", dtype=torch.int32)
        if not case["into"]:
            now = to[e].int()
        flat = (b * HC + h) * blocks + at // BLOCK
        now = now.view(-1).scatter_reduce(0, flat, need, "amax").view(B, HC, blocks)
        if not case["into"]:
            shift = _power(to[e].int() - now).repeat_interleave(BLOCK, 2)[:, :, :keep, None]
            grown = _codes(to[c][:, :, :keep].float() * shift, case["cache"])
            _bits(to[c])[:, :, :keep] = _bits(grown)
        _bits(to[c])[b, h, at] = _bits(_codes(rows * _power(was - now[b, h, at // BLOCK])[:, None], case["cache"]))
        if case["into"]:
            held = torch.arange(blocks, device="cuda") * BLOCK < count
            now = torch.where(held, now, to[e].int())
        to[e].copy_(now.to(torch.int8))
    to["scores"][b, h, at] = scores[b, h, frm]
    to["pos"][b, h, at] = pos[b, h, frm]
    return lens_out


# ---- one pass --------------------------------------------------------------------------------------------------------------
def _state(s, suffix=""):
    """The cache's own buffers, as far as the call changes them."""
    got = {k: s[k + suffix] for k in ("K", "V", "ke", "ve", "scores", "pos") if s.get(k + suffix) is not None}
    return got


def run(s):
    case = s["case"]
    op = case["op"]
    if own:
        import paper_2510_01450_amd as llla
        cache = llla.Cache(s["K"], s["V"], s["ke"], s["ve"], s.get("scores"), s["pos"])
        if op == "append":
            llla.llla_cache_append(cache, s["k"], s["v"], seqlens=s["lens"], new_lens=s["new"])
            return _state(s)
        if op == "decode_q8":
            return llla.llla_decode_q8(s["q"], cache, LAMBDA, s["scale"], seqlens=s["lens"], out_dtype=TYPES[case["out"]])
        if op == "scores":
            return llla.llla_cache_scores(s["q"], cache, s["scale"], seqlens=s["lens"])
        if case["into"]:
            to = llla.Cache(s["Ki"], s["Vi"], s["kei"], s["vei"], s["scoresi"], s["posi"])
            lens = llla.llla_cache_evict(cache, case["keep"], seqlens=s["lens"], sinks=_sinks(case), recent=_recent(case), into=to)
            return {**_state(s, "i"), "lens": lens}
        llla.llla_cache_append(cache, s["k"], s["v"], seqlens=s["kept"], first_pos=s["next"])
        lens = llla.llla_cache_evict(cache, case["keep"], seqlens=s["full"], sinks=_sinks(case), recent=_recent(case))
    else:
        if op == "append":
            _plain_append(s, s["lens"], s["new"])
            return _state(s)
        if op == "decode_q8":
            return _plain_decode(s)
        if op == "scores":
            return _plain_scores(s)
        if case["into"]:
            lens = _plain_evict(s, _lengths(s, case["n"]).int())
            return {**_state(s, "i"), "lens": lens}
        _plain_append(s, s["kept"], None)
        lens = _plain_evict(s, s["full"])
    s["next"] += case["m"]
    return {**_state(s), "lens": lens}


# ---- what a pass cannot do without -------------------------------------------------------------------------------------------
def work(case):
    """Bytes: rows, exponents, scores and results once each.  Operations: decode as in the library's other decode, the logits and
    exponentials of scores; a few per value of the others."""
    B, H, HC, n, d, m, keep = (case[k] for k in ("B", "H", "HC", "n", "d", "m", "keep"))
    size = {"f32": 4, "bf16": 2, "int8": 1, "e4m3": 1}
    c, e = size[case["cache"]], size[case["dtype"]]
    live = n * (9 / 16 if case["ragged"] else 1.0)                  # mean length of a ragged batch
    row = 2 * (d * c + (1 / BLOCK if c == 1 else 0))                # a key and a value with their share of the exponents
    if case["op"] == "decode_q8":
        return {"bytes": B * (HC * live * row + H * d * (e + size[case["out"]])), "flops": B * H * (live * (d * d + 11 * d) + d ** 3 / 3 + 4 * d * d)}
    if case["op"] == "append":
        rows = B * HC * (m * 3 / 4 if case["ragged"] and m > 1 else m)
        return {"bytes": rows * (2 * d * e + row), "flops": rows * 2 * d * 4}
    if case["op"] == "scores":
        pairs = B * H * (m * (live - (m - 1) / 2) if live > m else live * (live + 1) / 2)
        return {"bytes": B * (HC * live * (row / 2 + 8) + H * m * d * e), "flops": pairs * (2 * d + 4)}
    if case["into"]:
        rows = B * HC * min(keep, live)
        return {"bytes": B * HC * live * 8 + rows * (2 * row + 8), "flops": B * HC * live * 4}
    rows = B * HC * m
    return {"bytes": B * HC * n * 8 + rows * (2 * d * e + 3 * row + 24), "flops": B * HC * n * 4}


# ---- the definitions in 64 bits ------------------------------------------------------------------------------------------------
def _exact_decode(case, s):
    """Per query head the weighted ridge regression of the values on [1, k - q] by its normal equations; the intercept is the result."""
    group, d, n = case["H"] // case["HC"], case["d"], case["n"]
    out = torch.empty((case["B"], case["H"], d), dtype=torch.float64, device="cuda")
    for b in range(case["B"]):
        L = n if s["lens"] is None else int(s["lens"][b])
        for h in range(case["HC"]):
            def rows(c, e):
                power = torch.exp2(s[e][b, h].double())[torch.arange(L, device="cuda") // BLOCK]
                return s[c][b, h, :L].double() * power[:, None]
            K, V = rows("K", "ke"), rows("V", "ve")
            q = s["q"][b, h * group:(h + 1) * group].double()
            logits = torch.matmul(q, K.t().contiguous()) * s["scale"]
            w = torch.exp(logits - logits.max(1, keepdim=True).values)
            X = torch.cat([torch.ones((group, L, 1), dtype=torch.float64, device="cuda"), K[None] - q[:, None]], 2)
            XtW = (X * w[:, :, None]).transpose(1, 2).contiguous()
            ridge = torch.full((d + 1,), LAMBDA, dtype=torch.float64, device="cuda")
            ridge[0] = 0.0
            fit = torch.linalg.solve(torch.matmul(XtW, X) + torch.diag(ridge), torch.matmul(XtW, V[None].expand(group, L, d)))
            out[b, h * group:(h + 1) * group] = fit[:, 0]
    return out


def _exact_scores(case, s):
    group, n, m = case["H"] // case["HC"], case["n"], case["m"]
    out = s["scores"].double()
    for b in range(case["B"]):
        L = n if s["lens"] is None else int(s["lens"][b])
        for h in range(case["H"]):
            K = s["K"][b, h // group, :L].double()
            if s["ke"] is not None:
                K = K * torch.exp2(s["ke"][b, h // group].double())[torch.arange(L, device="cuda") // BLOCK][:, None]
            skip = max(0, m - L)                                  # queries in front of the first row
            logits = torch.matmul(s["q"][b, h, skip:].double(), K.t().contiguous()) * s["scale"]
            hidden = torch.ones((m - skip, L), dtype=torch.bool, device="cuda").triu(L - m + skip + 1)
            logits.masked_fill_(hidden, -math.inf)
            out[b, h // group, :L] += torch.softmax(logits, 1).sum(0)
    return out


def _exact_moved(case, s):
    """Rows of caches that hold numbers: copies of what was there."""
    B, HC, n, keep = case["B"], case["HC"], case["n"], case["keep"]
    suffix, out = "i" if case["into"] else "", {}
    held = {k: s[k].double().clone() for k in ("K", "V", "scores") if s[k].dtype not in (torch.int8, torch.float8_e4m3fn)}
    pos = s["pos"].clone()
    if case["m"]:
        held["scores"][:, :, keep:] = 0.0
        pos[:, :, keep:] = s["next"][:, None, None] + torch.arange(case["m"], device="cuda", dtype=torch.int32)
        for c, x in (("K", "k"), ("V", "v")):
            if c in held:
                held[c][:, :, keep:] = s[x].double()
    got = {k: (s[k + suffix].double().clone() if case["into"] else v.clone()) for k, v in held.items()}
    for b in range(B):
        L = n if s["lens"] is None else int(s["lens"][b])
        for h in range(HC):
            p = pos[b, h, :L]
            safe = ((p < _sinks(case)) | (p > p.max() - _recent(case))).double()
            # by (safe, score, lower slot)
            best = torch.sort(held["scores"][b, h, :L], descending=True, stable=True).indices
            best = best[torch.sort(safe[best], descending=True, stable=True).indices][:keep]
            if case["into"]:
                frm = best.sort().values
                at = torch.arange(frm.numel(), device="cuda")
            else:
                stays = torch.zeros(L, dtype=torch.bool, device="cuda")
                stays[best] = True
                frm, at = torch.nonzero(stays[keep:])[:, 0] + keep, torch.nonzero(~stays[:keep])[:, 0]
            for k in got:
                got[k][b, h, at] = held[k][b, h, frm]
    return got


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "decode_q8":
        return _exact_decode(case, s)
    if case["op"] == "scores":
        return _exact_scores(case, s)
    if case["op"] == "append":
        return None if case["cache"] in POWER else _exact_append(case, s)
    return _exact_moved(case, s)


def _exact_append(case, s):
    got = {"K": s["K"].double(), "V": s["V"].double()}
    for b in range(case["B"]):
        L, count = int(s["lens"][b]), case["m"] if s["new"] is None else int(s["new"][b])
        got["K"][b, :, L:L + count] = s["k"][b, :, :count].double()
        got["V"][b, :, L:L + count] = s["v"][b, :, :count].double()
    return got
