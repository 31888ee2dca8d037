"""Performance cases of a paged cache held in 4 bits, of the attention that reads it, and of rotary positions with several axes.

A generation that continues a clip turns its queries and keys by their places in time, height and width (``rope``), writes the new
keys and values of each candidate into pages of 4-bit codes (``append``), attends to them (``attn``), and takes the tokens of a
sequence out again as bf16 for whatever does not read the codes (``read``; a pass of ``append`` reads back what it has written).

The codes: 32 channels of a token share a scale, the nearest number of five significant bits to their largest magnitude over 7; a code
is the nearest whole number of scales, -7 .. 7, so that every value that the cache stands for is a bf16 number.

``own`` selects between the library's calls and the plain form: elementary tensor operations in 32 bits (angles in 64).
"""
from __future__ import annotations

import math
import random

import torch

own = False

_HEADS = ((24, 24), (32, 32), (32, 8), (24, 8), (16, 2), (2, 2))
_SECTIONS = {(64, 1): (32,), (64, 2): (16, 16), (64, 3): (12, 10, 10), (128, 1): (64,), (128, 2): (32, 32), (128, 3): (22, 21, 21)}


def listed():
    return [
        # ---- rotary positions of queries and keys.  axes: time, height, width; start: how far into the generation the first frame lies
        # the next audio token of one candidate: the smallest call
        dict(name="rope one token", op="rope", B=1, N=1, H=24, Hkv=24, d=128, axes=1, start=5000, halves=False, inverse=False),
        # a whole latent clip (21 x 30 x 52)
        dict(name="rope a clip", op="rope", B=1, N=32760, H=24, Hkv=24, d=128, axes=3, start=0, halves=False, inverse=False),
        # back from positions far into a long generation (the gradient's direction), two halves of a head, grouped heads, odd sizes
        dict(name="rope back, odd sizes", op="rope", B=3, N=1009, H=24, Hkv=8, d=64, axes=2, start=300000, halves=True, inverse=True),
        # ---- new tokens into the cache, and the last ones out of it again
        dict(name="append a token each", op="append", n=16, L=1, Hkv=24, d=128, page=64, own_min=1, own_max=1000, ragged=False),
        dict(name="append a frame each", op="append", n=4, L=1560, Hkv=24, d=128, page=32, own_min=1, own_max=4000, ragged=True),
        # ---- whole sequences out of the cache
        # two short ones of different lengths
        dict(name="read short sequences", op="read", n=2, Hkv=8, d=64, page=16, own_min=77, own_max=333),
        # the finished clip (16 x 48 x 64 latents) of a model with grouped heads
        dict(name="read a clip", op="read", n=1, Hkv=8, d=128, page=128, own_min=49152, own_max=49152),
        # ---- attention.  prefix: tokens that all sequences share; each one's own length is drawn from own_min..own_max
        # the next audio token of one candidate behind a short beginning: the smallest call
        dict(name="attn one token, short clip", op="attn", B=1, L=1, H=24, Hkv=24, d=128, page=64, prefix=256, own_min=40, own_max=40, causal=False, idle=0),
        # sixteen candidates of one clip (31 x 24 x 24 latents), a token each, half a thousand own tokens
        dict(name="attn one token, 16 candidates", op="attn", B=16, L=1, H=24, Hkv=24, d=128, page=64, prefix=17856, own_min=1, own_max=1000, causal=False, idle=0),
        # sixty-four candidates of a long clip, four query heads to a key head, ragged continuations
        dict(name="attn one token, 64 candidates", op="attn", B=64, L=1, H=32, Hkv=8, d=128, page=128, prefix=49152, own_min=100, own_max=2048, causal=False, idle=0),
        # a few tokens at once, three query heads to a key head, small pages, two batch rows whose sequence is empty
        dict(name="attn few tokens, odd sizes", op="attn", B=5, L=7, H=24, Hkv=8, d=64, page=16, prefix=1008, own_min=7, own_max=333, causal=True, idle=2),
        # the next latent frame (30 x 52) of four candidates behind eight shared frames, tokens of a frame see each other: the largest
        dict(name="attn frame of 4 candidates", op="attn", B=4, L=1560, H=24, Hkv=24, d=128, page=32, prefix=12480, own_min=1560, own_max=1560, causal=False, idle=0),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        c = _draw(rng)
        if _cost(c) <= most and _memory(c) <= 24e9:
            return c


def _draw(rng):
    op = rng.choice(("attn", "attn", "attn", "append", "read", "rope"))
    H, Hkv = rng.choice(_HEADS)
    d, page = rng.choice((64, 128)), rng.choice((16, 32, 64, 128))
    if op == "rope":
        return dict(op=op, B=_log(rng, 1, 8), N=_log(rng, 1, 33000), H=H, Hkv=Hkv, d=d, axes=rng.randint(1, 3), start=_log(rng, 1, 1 << 20),
                    halves=rng.random() < 0.5, inverse=rng.random() < 0.5)
    if op == "append":
        return dict(op=op, n=_log(rng, 1, 64), L=_log(rng, 1, 2000), Hkv=Hkv, d=d, page=page, own_min=_log(rng, 1, 300), own_max=_log(rng, 300, 3000),
                    ragged=rng.random() < 0.5)
    if op == "read":
        own_min = _log(rng, 1, 20000)
        return dict(op=op, n=_log(rng, 1, 32), Hkv=Hkv, d=d, page=page, own_min=own_min, own_max=max(own_min, _log(rng, 1, 50000)))
    B = _log(rng, 1, 64)
    L = 1 if rng.random() < 0.5 else _log(rng, 2, 1600)
    prefix = 0 if rng.random() < 0.15 else _log(rng, page, 50000) // page * page
    own_min = 0 if rng.random() < 0.2 else _log(rng, 1, 1600)
    idle = 1 if B > 1 and rng.random() < 0.2 else 0
    return dict(op=op, B=B, L=L, H=H, Hkv=Hkv, d=d, page=page, prefix=prefix, own_min=own_min, own_max=max(own_min, _log(rng, 1, 4000)),
                causal=rng.random() < 0.5, idle=idle)


def _cost(c):
    w = work(c)
    return max(w["bytes"] / 6e12, w["flops"] / 1.2e15)


def _memory(c):
    """Bytes that the plain form holds at once, about."""
    if c["op"] == "rope":
        return 24.0 * c["B"] * c["N"] * (c["H"] + c["Hkv"]) * c["d"]
    if c["op"] == "append":
        return 8.0 * c["n"] * (c["own_max"] + 8 * c["L"] + 128) * c["Hkv"] * c["d"]
    if c["op"] == "read":
        return 40.0 * c["n"] * (c["own_max"] + c["page"]) * c["Hkv"] * c["d"]
    keys = c["prefix"] + c["own_max"]
    return 16.0 * c["B"] * c["L"] * c["H"] * keys + 24.0 * c["d"] * c["Hkv"] * (c["prefix"] + c["B"] * (c["own_max"] + c["page"]))


# ------------------------------------------------------------------------------------------------ sizes that a case's own numbers decide
def _spread(lo, hi, n, salt):
    """n lengths of lo..hi, spread evenly over the range, in a shuffled order that depends on the case alone."""
    v = [lo + (hi - lo) * k // max(1, n - 1) for k in range(n)] if n > 1 else [hi]
    random.Random(1000003 * n + salt).shuffle(v)
    return v


def _attn_lengths(c):
    v = [c["prefix"] + x for x in _spread(c["own_min"], c["own_max"], c["B"], c["own_max"])]
    for k in range(c["idle"]):           # batch rows whose sequence holds nothing (never the first one)
        v[-1 - k] = 0
    return v


def _append_sizes(c):
    """Tokens of each sequence with the new ones, new ones, and how many are read back: the new ones and up to sixteen in front of them."""
    lens = _spread(c["own_min"], c["own_max"], c["n"], c["L"])
    counts = [max(0, c["L"] - (37 * k) % (c["L"] // 2 + 1)) for k in range(c["n"])] if c["ragged"] else [c["L"]] * c["n"]
    return [n + k for n, k in zip(lens, counts)], counts, [min(n, 16) + k for n, k in zip(lens, counts)]


def _up(n, page):
    return -(-n // page)


def work(case):
    c = case
    if c["op"] == "rope":
        values = float(c["B"] * c["N"] * (c["H"] + c["Hkv"]) * c["d"])
        return {"bytes": 4.0 * values + 4.0 * c["B"] * c["N"] * c["axes"] + 4.0 * c["d"], "flops": 3.0 * values}
    token = c["Hkv"] * c["d"]            # values of a token's keys; 4.5 bits each in the cache, 16 outside
    if c["op"] == "append":
        _, counts, back = _append_sizes(c)
        return {"bytes": 2.0 * token * (sum(counts) * (2 + 0.5625) + sum(back) * 0.5625 + c["n"] * (c["L"] + 16) * 2), "flops": 0.0}
    if c["op"] == "read":
        lens = _spread(c["own_min"], c["own_max"], c["n"], c["own_max"])
        return {"bytes": 2.0 * token * (sum(lens) * 0.5625 + c["n"] * c["own_max"] * 2), "flops": 0.0}
    lens = _attn_lengths(c)
    keys = 0
    for n in lens:
        keys += sum(max(0, n - c["L"] + i + 1) for i in range(c["L"])) if c["causal"] else n * c["L"]
    cached = c["prefix"] + sum(max(0, n - c["prefix"]) for n in lens)
    return {"bytes": 2 * 0.5625 * cached * token + c["B"] * c["L"] * c["H"] * (4.0 * c["d"] + 4.0), "flops": 4.0 * keys * c["H"] * c["d"]}


# ------------------------------------------------------------------------------------------------ inputs
def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _normal(gen, *size):
    return torch.empty(size, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)


def _quantise(x):
    """Codes (whole numbers in fp32) [..., d] and scales [..., d/32] of x [..., d]."""
    g = x.float().unflatten(-1, (-1, 32))
    scale = g.abs().amax(-1) / 7
    scale = ((scale.view(torch.int32) + 0x40000) & ~0x7FFFF).view(torch.float32)       # to five significant bits
    return torch.round(g / torch.where(scale > 0, scale, 1.0)[..., None]).flatten(-2), scale


def _pack(x):
    """Bytes of a token [..., d/2] of codes and [..., d/16] of scales: four bytes hold eight channels, the low halves of their two 16-bit
    words the even ones and the high halves the odd ones."""
    code, scale = _quantise(x)
    u = (code + 8).to(torch.uint8).unflatten(-1, (-1, 8))
    return (u[..., (0, 4, 1, 5)] | (u[..., (2, 6, 3, 7)] << 4)).flatten(-2), scale.to(torch.bfloat16).view(torch.uint8)


def _parts(pool, d):
    """Views of a pool [..., page, d/2 + d/16]: codes [..., page/16, 16, d/2] and scales [..., page/16, 16, d/16].  Sixteen tokens keep their codes
    next to each other, and their scales behind these."""
    blocks = pool.flatten(-2).unflatten(-1, (-1, 16 * (d // 2 + d // 16)))
    return blocks[..., :8 * d].unflatten(-1, (16, d // 2)), blocks[..., 8 * d:].unflatten(-1, (16, d // 16))


def _filled_pool(gen, pages, c):
    """A pool of keys and one of values, each [pages, Hkv, page, bytes of a token], that hold what was written to them."""
    pool = torch.empty((2, pages, c["Hkv"], c["page"], c["d"] // 2 + c["d"] // 16), dtype=torch.uint8, device="cuda")
    for kind in pool:
        codes, scales = _parts(kind, c["d"])
        step = max(1, (1 << 27) // (c["Hkv"] * c["page"] * c["d"]))
        for at in range(0, pages, step):
            n = min(step, pages - at)
            a, b = _pack(_normal(gen, n, c["Hkv"], c["page"] // 16, 16, c["d"]))
            codes[at:at + n], scales[at:at + n] = a, b
    return pool


def _tables(lens, page, rng, room=3):
    need = [_up(n, page) for n in lens]
    pages = list(range(sum(need) + room))
    rng.shuffle(pages)
    at, table = 0, []
    for k in need:
        table.append(pages[at:at + k] + [-1] * (max(need) - k))
        at += k
    return _ints(table), len(pages)


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rng = random.Random(seed)
    s = {"case": c}
    page = c.get("page")
    if c["op"] == "rope":
        # tokens of a sequence next to each other in storage, as a projection leaves them
        s["q"] = _normal(gen, c["B"], c["N"], c["H"], c["d"]).transpose(1, 2)
        s["k"] = _normal(gen, c["B"], c["N"], c["Hkv"], c["d"]).transpose(1, 2)
        # frames of 30 x 52 tokens, each batch entry somewhere else in its generation
        at = torch.arange(c["N"], device="cuda")
        place = (at, torch.stack((at // 52, at % 52), 1), torch.stack((at // 1560, at // 52 % 30, at % 52), 1))[c["axes"] - 1].reshape(c["N"], -1)
        first = torch.tensor([c["start"] + rng.randint(0, 99) for _ in range(c["B"])], device="cuda")
        pos = place[None].repeat(c["B"], 1, 1)
        pos[:, :, 0] += first[:, None]
        s["pos"] = pos.int()
        s["sections"] = _SECTIONS[c["d"], c["axes"]]
        # turns of a channel pair for a step along its axis
        s["freq"] = torch.cat([10000.0 ** (-torch.arange(n, dtype=torch.float64) / n) for n in s["sections"]]).cuda() / (2 * math.pi)
        return s
    if c["op"] == "append":
        lens, counts, back = _append_sizes(c)
        s["table"], pages = _tables(lens, page, rng)
        kv = _filled_pool(gen, pages, c)
        new = _normal(gen, 2, c["n"], c["L"], c["Hkv"], c["d"]).transpose(2, 3)
        order = list(range(c["n"]))
        rng.shuffle(order)
        s.update(k=kv[0], v=kv[1], k_new=new[0], v_new=new[1], length=_ints(lens), seq=_ints(order), count=_ints([counts[i] for i in order]),
                 back=_ints([back[i] for i in order]))
        return s
    if c["op"] == "read":
        lens = _spread(c["own_min"], c["own_max"], c["n"], c["own_max"])
        s["table"], pages = _tables(lens, page, rng)
        kv = _filled_pool(gen, pages, c)
        s.update(k=kv[0], v=kv[1], length=_ints(lens))
        return s
    lens = _attn_lengths(c)
    shared = c["prefix"] // page
    need = [max(0, _up(n, page) - shared) for n in lens]
    pages = list(range(shared + sum(need) + 2))
    rng.shuffle(pages)
    width = max(1, shared + max(need))
    first, at, table = pages[:shared], shared, []
    for n, k in zip(lens, need):
        row = (first if n else []) + pages[at:at + k]
        at += k
        table.append(row + [-1] * (width - len(row)))
    kv = _filled_pool(gen, len(pages), c)
    q = torch.empty((c["B"], c["L"], c["H"], c["d"]), dtype=torch.bfloat16, device="cuda").normal_(0.0, 1.5, generator=gen)
    s.update(k=kv[0], v=kv[1], table=_ints(table), length=_ints(lens), shared=shared, q=q.transpose(1, 2))
    return s


# ------------------------------------------------------------------------------------------------ one pass
def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(s):
    from paper_2608_15522_b200 import binding as av
    c = s["case"]
    if c["op"] == "rope":
        q, k = av.avsa_rope(s["q"], s["k"], s["pos"], s["freq"], s["sections"], halves=c["halves"], inverse=c["inverse"])
        return {"q": q, "k": k}
    if c["op"] == "append":
        av.avsa_cache_write_q4(s["k_new"], s["v_new"], s["k"], s["v"], s["table"], s["length"], seq=s["seq"], count=s["count"])
        k, v = av.avsa_cache_read_q4(s["k"], s["v"], s["table"], s["length"], c["L"] + 16, seq=s["seq"], count=s["back"])
        return {"k": k, "v": v}
    if c["op"] == "read":
        k, v = av.avsa_cache_read_q4(s["k"], s["v"], s["table"], s["length"], c["own_max"], count=s["length"])
        return {"k": k, "v": v}
    o, lse, _ = av.avsa_prefix_attn_q4(s["q"], s["k"], s["v"], s["table"], s["length"], prefix_pages=s["shared"], causal=c["causal"], want_lse=True)
    return {"o": o, "lse": lse}


def _run_plain(s):
    return {"rope": _plain_rope, "append": _plain_append, "read": _plain_read, "attn": _plain_attn}[s["case"]["op"]](s)


def _plain_rope(s):
    c = s["case"]
    axis = torch.cat([torch.full((n,), i) for i, n in enumerate(s["sections"])]).cuda()
    turns = s["pos"].double()[:, :, axis] * s["freq"]
    angle = ((turns - torch.round(turns)) * (2 * math.pi))[:, None]
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    if c["inverse"]:
        sin = -sin
    out = {}
    for name in ("q", "k"):
        x = s[name].float()
        a, b = x.chunk(2, 3) if c["halves"] else (x[..., 0::2], x[..., 1::2])
        y = (a * cos - b * sin, a * sin + b * cos)
        out[name] = (torch.cat(y, 3) if c["halves"] else torch.stack(y, 4).flatten(3)).to(torch.bfloat16)
    return out


def _values(codes, scales):
    """fp32 [..., d] of bytes [..., d/2] and [..., d/16]."""
    lo, hi = (codes & 15).unflatten(-1, (-1, 4)), (codes >> 4).unflatten(-1, (-1, 4))
    u = torch.stack((lo[..., 0], lo[..., 2], hi[..., 0], hi[..., 2], lo[..., 1], lo[..., 3], hi[..., 1], hi[..., 3]), -1).flatten(-2)
    scale = scales.contiguous().view(torch.bfloat16).float()
    return ((u.float() - 8).unflatten(-1, (-1, 32)) * scale[..., None]).flatten(-2)


def _last_tokens(s, count, seq, T):
    """bf16 keys and values [n,Hkv,T,d]: the last count tokens of sequences seq, zeros behind them."""
    c, page = s["case"], s["case"]["page"]
    t = torch.arange(T, device=count.device)
    here = t < count[:, None]
    at = (s["length"].long()[seq] - count)[:, None] + t
    at = torch.where(here, at, 0)
    pages = torch.where(here, s["table"].long()[seq].gather(1, at // page), 0)
    out = []
    for pool in (s["k"], s["v"]):
        codes, scales = _parts(pool, c["d"])
        x = _values(codes[pages, :, at % page // 16, at % 16], scales[pages, :, at % page // 16, at % 16])      # [n,T,Hkv,d]
        out.append(x.masked_fill_(~here[:, :, None, None], 0.0).transpose(1, 2).to(torch.bfloat16).contiguous())
    return {"k": out[0], "v": out[1]}


def _plain_append(s):
    c, page, seq, count = s["case"], s["case"]["page"], s["seq"].long(), s["count"].long()
    n, t = torch.nonzero(torch.arange(c["L"], device=seq.device) < count[:, None], as_tuple=True)
    at = s["length"].long()[seq[n]] - count[n] + t
    to = s["table"].long()[seq[n], at // page]
    for new, pool in ((s["k_new"], s["k"]), (s["v_new"], s["v"])):
        codes, scales = _parts(pool, c["d"])
        a, b = _pack(new.transpose(1, 2)[n, t])
        codes[to, :, at % page // 16, at % 16], scales[to, :, at % page // 16, at % 16] = a, b
    return _last_tokens(s, s["back"].long(), seq, c["L"] + 16)


def _plain_read(s):
    length = s["length"].long()
    return _last_tokens(s, length, torch.arange(length.shape[0], device=length.device), s["case"]["own_max"])


def _plain_attn(s):
    c, q, table, length = s["case"], s["q"], s["table"].long(), s["length"].long()
    B, H, L, d = q.shape
    Hkv, page, shared = c["Hkv"], c["page"], s["shared"]
    G, np_ = H // Hkv, s["shared"] * c["page"]
    scale = 1.0 / math.sqrt(d)
    limit = (length[:, None] - L + 1 + torch.arange(L, device=q.device)) if c["causal"] else length[:, None].expand(B, L)
    limit = limit.clamp(min=0)
    qf = q.float().reshape(B, Hkv, G * L, d)
    limit = limit[:, None].expand(B, G, L).reshape(B, 1, G * L, 1)

    def values(pool, pages):      # [*pages,Hkv,page,d]
        codes, scales = _parts(pool[pages], d)
        return _values(codes, scales).flatten(-3, -2)

    # the shared beginning, once: the rows of all sequences against it
    donor = table[length.argmax(), :shared]
    kp, vp = (values(pool, donor).transpose(0, 1).reshape(Hkv, np_, d) for pool in (s["k"], s["v"]))
    rows = qf.transpose(0, 1).reshape(Hkv, B * G * L, d)
    sp = (rows @ kp.transpose(1, 2)).view(Hkv, B, G * L, np_).transpose(0, 1)
    # each sequence's own pages
    mine = table[:, shared:].clamp(min=0)
    n_own = mine.shape[1] * page
    ko, vo = (values(pool, mine).transpose(1, 2).reshape(B, Hkv, n_own, d) for pool in (s["k"], s["v"]))
    position = torch.arange(np_ + n_own, device=q.device)
    scores = torch.cat([sp, qf @ ko.transpose(2, 3)], dim=3)
    scores = scores.mul_(scale).masked_fill_(position >= limit, float("-inf"))
    lse = torch.logsumexp(scores, dim=3)
    p = scores.sub_(torch.where(lse == float("-inf"), 0.0, lse)[..., None]).exp_()
    o = p[..., np_:] @ vo
    o = o + (p[..., :np_].transpose(0, 1).reshape(Hkv, B * G * L, np_) @ vp).view(Hkv, B, G * L, d).transpose(0, 1)
    return {"o": o.reshape(B, H, L, d).to(torch.bfloat16), "lse": lse.reshape(B, H, L)}


# ------------------------------------------------------------------------------------------------ the definition in 64 bits
def _token_values(pool, page, place, head, d):
    """What token `place` of page `page` (tensors of the same shape) stands for in one key head, fp64 [..., d], byte by byte of the pool."""
    memory = pool[:, head].reshape(pool.shape[0], -1).long()
    block = (place // 16) * (16 * (d // 2 + d // 16))
    ch = torch.arange(d, device=pool.device)
    word, i = ch // 8, ch % 8
    byte = memory[page[..., None], (block + place % 16 * (d // 2))[..., None] + 4 * word + 2 * (i % 2) + i // 4]
    code = (byte >> (4 * (i // 2 % 2))) % 16 - 8
    at = (block + 8 * d + place % 16 * (d // 16))[..., None] + 2 * (ch // 32)
    bits = memory[page[..., None], at] + 256 * memory[page[..., None], at + 1]
    exponent, fraction = bits // 128 % 256, bits % 128
    value = torch.where(exponent > 0, 128 + fraction, 2 * fraction).double() * torch.exp2((exponent - 134).double())
    return code.double() * value


def _stands_for(x):
    """What bf16 x [..., d] becomes in the cache, fp64."""
    g = x.double().reshape(*x.shape[:-1], -1, 32)
    part, power = torch.frexp(g.abs().max(dim=-1, keepdim=True).values / 7)
    step = torch.ldexp(torch.floor(part * 32 + 0.5) / 32, power)
    return torch.where(step > 0, torch.round(g / torch.where(step > 0, step, 1.0)) * step, 0.0).reshape(x.shape)


def exact(case, seed):
    s = prepare(case, seed)
    c, device = case, "cuda"
    if c["op"] == "rope":
        out, at = {}, 0
        for name in ("q", "k"):
            x = s[name].double()
            y = torch.empty_like(x)
            pair = 0
            for axis, n in enumerate(s["sections"]):
                for i in range(n):
                    z = torch.exp(1j * (2 * math.pi * torch.remainder(s["pos"][:, :, axis].double() * s["freq"][pair], 1.0)))
                    z = (z.conj() if c["inverse"] else z)[:, None]
                    a, b = (pair, pair + c["d"] // 2) if c["halves"] else (2 * pair, 2 * pair + 1)
                    turned = torch.complex(x[..., a], x[..., b]) * z
                    y[..., a], y[..., b] = turned.real, turned.imag
                    pair += 1
            out[name] = y
        return out
    page = c["page"]
    if c["op"] in ("append", "read"):
        lens = s["length"].tolist()
        if c["op"] == "append":
            order, counts, back, T = s["seq"].tolist(), s["count"].tolist(), s["back"].tolist(), c["L"] + 16
        else:
            order, counts, back, T = range(c["n"]), [0] * c["n"], lens, c["own_max"]
        out = {}
        for name in ("k", "v"):
            y = torch.zeros((c["n"], c["Hkv"], T, c["d"]), dtype=torch.float64, device=device)
            for row, seq in enumerate(order):
                old = back[row] - counts[row]
                at = lens[seq] - back[row] + torch.arange(old, device=device)
                pages = s["table"][seq].long()[at // page]
                for h in range(c["Hkv"]):
                    y[row, h, :old] = _token_values(s[name], pages, at % page, h, c["d"])
                if counts[row]:
                    y[row, :, old:back[row]] = _stands_for(s[name + "_new"][row, :, :counts[row]])
            out[name] = y
        return out
    q, causal = s["q"], c["causal"]
    B, H, L, d = q.shape
    group = H // c["Hkv"]
    o = torch.zeros((B, H, L, d), dtype=torch.float64, device=device)
    lse = torch.full((B, H, L), float("-inf"), dtype=torch.float64, device=device)
    lengths = s["length"].tolist()
    for b in range(B):
        n = lengths[b]
        if n == 0:
            continue
        at = torch.arange(n, device=device)
        pages, places = s["table"][b].long()[at // page], at % page
        hidden = at[None, :] > (torch.arange(L, device=device)[:, None] + n - L) if causal else None
        for g in range(c["Hkv"]):
            k, v = _token_values(s["k"], pages, places, g, d), _token_values(s["v"], pages, places, g, d)
            for h in range(g * group, (g + 1) * group):
                x = q[b, h].double() @ k.T / math.sqrt(d)
                if causal:
                    x[hidden] = float("-inf")
                top = x.amax(1, keepdim=True)
                top = torch.where(torch.isinf(top), 0.0, top)
                e = torch.exp(x - top)
                z = e.sum(1, keepdim=True)
                o[b, h] = torch.where(z > 0, (e @ v) / z, 0.0)
                lse[b, h] = (top + torch.log(z))[:, 0]
    return {"o": o, "lse": lse}
