"""Performance cases of the paged K/V cache and of the attention that reads it.

A generation that continues a clip keeps the keys and values of what it has made in pages of a pool.  Several candidates that begin alike
share the pages of their beginning (``fork``), the new tokens of each are added to its own pages (``append``), attention runs over
the shared beginning, read once for all, and each candidate's own continuation (``attn``), and rejected candidates give their pages back,
after which the pool is compacted (``prune``).

``own`` selects between the library's calls and the plain form: elementary tensor operations in 32 bits.
"""
from __future__ import annotations

import math
import random

import torch

own = False

_HEADS = ((24, 24), (32, 32), (32, 8), (24, 8), (16, 2), (2, 2))


def listed():
    return [
        # ---- attention.  prefix: tokens that all sequences share; each one's own length is drawn from own_min..own_max
        # the next audio token of one candidate behind a short beginning: the smallest call
        dict(name="attn one token, short clip", op="attn", B=1, L=1, H=24, Hkv=24, d=128, page=64, prefix=256, own_min=40, own_max=40, causal=False, idle=0),
        # sixteen candidates of one clip (31 x 24 x 24 latents), a token each, half a thousand own tokens
        dict(name="attn one token, 16 candidates", op="attn", B=16, L=1, H=24, Hkv=24, d=128, page=64, prefix=17856, own_min=1, own_max=1000, causal=False, idle=0),
        # sixty-four candidates of a long clip (16 x 48 x 64 latents), four query heads to a key head, ragged continuations
        dict(name="attn one token, 64 candidates", op="attn", B=64, L=1, H=32, Hkv=8, d=128, page=128, prefix=49152, own_min=100, own_max=2048, causal=False, idle=0),
        # a few tokens at once, three query heads to a key head, small pages, two batch rows whose sequence is empty
        dict(name="attn few tokens, odd sizes", op="attn", B=5, L=7, H=24, Hkv=8, d=64, page=16, prefix=1008, own_min=7, own_max=333, causal=True, idle=2),
        # the next latent frame (30 x 52) of four candidates behind eight shared frames, tokens of a frame see each other: the largest
        dict(name="attn frame of 4 candidates", op="attn", B=4, L=1560, H=24, Hkv=24, d=128, page=32, prefix=12480, own_min=1560, own_max=1560, causal=False, idle=0),
        # sequences that share nothing, a causal block of tokens each
        dict(name="attn causal block, no prefix", op="attn", B=3, L=509, H=32, Hkv=8, d=64, page=64, prefix=0, own_min=509, own_max=3000, causal=True, idle=0),
        # ---- new tokens into the cache: pages are reserved, then one layer's keys and values written
        dict(name="append a token each", op="append", n=16, L=1, Hkv=24, d=128, page=64, own_min=1, own_max=1000, ragged=False),
        dict(name="append a frame each", op="append", n=4, L=1560, Hkv=24, d=128, page=32, own_min=1, own_max=4000, ragged=True),
        # ---- branches: every parent gets `children` of them; planes = 2 x layers
        dict(name="fork one layer's cache", op="fork", parents=1, children=3, planes=2, Hkv=24, d=128, page=64, own_min=1000, own_max=2000),
        dict(name="fork a model's cache", op="fork", parents=8, children=4, planes=40, Hkv=24, d=128, page=128, own_min=500, own_max=700),
        # ---- rejected candidates give their pages back and the pool is compacted
        dict(name="prune one layer's cache", op="prune", seqs=12, drop=6, planes=2, Hkv=8, d=128, page=16, prefix=512, own_min=30, own_max=300),
        dict(name="prune a model's cache", op="prune", seqs=32, drop=16, planes=40, Hkv=24, d=128, page=128, prefix=1024, own_min=300, own_max=1200),
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
    op = rng.choice(("attn", "attn", "attn", "append", "fork", "prune"))
    H, Hkv = rng.choice(_HEADS)
    d, page = rng.choice((64, 128)), rng.choice((16, 32, 64, 128))
    if op == "attn":
        B = _log(rng, 1, 64)
        L = 1 if rng.random() < 0.5 else _log(rng, 2, 1600)
        prefix = 0 if rng.random() < 0.15 else _log(rng, page, 50000) // page * page
        own_min = 0 if rng.random() < 0.2 else _log(rng, 1, 1600)
        idle = 1 if B > 1 and rng.random() < 0.2 else 0
        return dict(op=op, B=B, L=L, H=H, Hkv=Hkv, d=d, page=page, prefix=prefix, own_min=own_min, own_max=max(own_min, _log(rng, 1, 4000)),
                    causal=rng.random() < 0.5, idle=idle)
    if op == "append":
        return dict(op=op, n=_log(rng, 1, 64), L=_log(rng, 1, 2000), Hkv=Hkv, d=d, page=page, own_min=_log(rng, 1, 300), own_max=_log(rng, 300, 3000),
                    ragged=rng.random() < 0.5)
    if op == "fork":
        return dict(op=op, parents=_log(rng, 1, 8), children=_log(rng, 1, 8), planes=2 * _log(rng, 1, 20), Hkv=Hkv, d=d, page=page,
                    own_min=_log(rng, 1, 300), own_max=_log(rng, 300, 1500))
    seqs = _log(rng, 2, 48)
    return dict(op=op, seqs=seqs, drop=rng.randint(1, seqs - 1), planes=2 * _log(rng, 1, 20), Hkv=Hkv, d=d, page=page,
                prefix=_log(rng, page, 2000) // page * page, own_min=_log(rng, 1, 200), own_max=_log(rng, 200, 1200))


def _cost(c):
    w = work(c)
    return max(w["bytes"] / 6e12, w["flops"] / 1.2e15)


def _memory(c):
    """Bytes that the plain form holds at once, about."""
    if c["op"] == "attn":
        keys = c["prefix"] + c["own_max"]
        return 16.0 * c["B"] * c["L"] * c["H"] * keys + 16.0 * c["d"] * c["Hkv"] * (c["prefix"] + c["B"] * (c["own_max"] + c["page"]))
    if c["op"] == "append":
        return 8.0 * c["n"] * (c["own_max"] + 2 * c["L"]) * c["Hkv"] * c["d"]
    tokens = c["parents"] * (1 + c["children"]) * (c["own_max"] + c["page"]) if c["op"] == "fork" else c["prefix"] + c["seqs"] * (c["own_max"] + c["page"])
    return 4.0 * c["planes"] * tokens * c["Hkv"] * c["d"]


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


def _up(n, page):
    return -(-n // page)


def _append_sizes(c):
    lens = _spread(c["own_min"], c["own_max"], c["n"], c["L"])
    counts = [max(0, c["L"] - (37 * k) % (c["L"] // 2 + 1)) for k in range(c["n"])] if c["ragged"] else [c["L"]] * c["n"]
    return lens, counts


def _fork_sizes(c):
    return _spread(c["own_min"], c["own_max"], c["parents"], c["children"])


def _prune_sizes(c):
    return [c["prefix"] + x for x in _spread(c["own_min"], c["own_max"], c["seqs"], c["drop"])]


def work(case):
    c = case
    if c["op"] == "attn":
        lens = _attn_lengths(c)
        rows = c["L"] * c["H"]
        keys = 0
        for n in lens:
            keys += sum(max(0, n - c["L"] + i + 1) for i in range(c["L"])) if c["causal"] else n * c["L"]
        cached = c["prefix"] + sum(max(0, n - c["prefix"]) for n in lens)
        return {"bytes": 4.0 * cached * c["Hkv"] * c["d"] + c["B"] * rows * (4.0 * c["d"] + 4.0), "flops": 4.0 * keys * c["H"] * c["d"]}
    token = 2.0 * c["Hkv"] * c["d"]
    if c["op"] == "append":
        _, counts = _append_sizes(c)
        return {"bytes": 2 * 2 * token * sum(counts), "flops": 0.0}
    if c["op"] == "fork":
        lens = _fork_sizes(c)
        return {"bytes": 2.0 * c["planes"] * c["page"] * token * c["children"] * sum(n % c["page"] > 0 for n in lens)
                + 8.0 * c["children"] * sum(_up(n, c["page"]) for n in lens), "flops": 0.0}
    _, ref, _, freed, _ = _prune_layout(c, 0)
    live = [r > 0 for r in freed]
    moves = sum(live[sum(live):])
    return {"bytes": 2.0 * c["planes"] * c["page"] * token * moves + 8.0 * (len(ref) + c["seqs"] * _prune_width(c)), "flops": 0.0}


def _prune_width(c):
    return _up(c["prefix"] + c["own_max"], c["page"])


def _prune_layout(c, seed):
    """table, ref, dropped sequences, ref after the drop, lengths: pages are numbered as the case alone decides, so that its work is known."""
    lens = _prune_sizes(c)
    shared = c["prefix"] // c["page"]
    need = [_up(n, c["page"]) - shared for n in lens]
    pages = list(range(shared + sum(need) + 3))
    rng = random.Random(77 + len(pages))
    rng.shuffle(pages)
    it = iter(pages)
    first = [next(it) for _ in range(shared)]
    width = _prune_width(c)
    table, ref = [], [0] * len(pages)
    for k in range(c["seqs"]):
        row = first + [next(it) for _ in range(need[k])]
        for p in row:
            ref[p] += 1
        table.append(row + [-1] * (width - len(row)))
    drop = rng.sample(range(c["seqs"]), c["drop"])
    freed = list(ref)
    for k in drop:
        for p in table[k]:
            if p >= 0:
                freed[p] -= 1
    return table, ref, drop, freed, lens


# ------------------------------------------------------------------------------------------------ inputs
def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _pool(gen, planes, pages, c):
    t = torch.empty((planes, pages, c["Hkv"], c["page"], c["d"]), dtype=torch.bfloat16, device="cuda")
    return t.normal_(generator=gen)


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rng = random.Random(seed)
    s = {"case": c}
    page = c["page"]
    if c["op"] == "attn":
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
        kv = _pool(gen, 2, len(pages), c)
        s.update(k=kv[0], v=kv[1], table=_ints(table), length=_ints(lens), shared=shared)
        # tokens of a sequence next to each other in storage, as a projection leaves them
        q = torch.empty((c["B"], c["L"], c["H"], c["d"]), dtype=torch.bfloat16, device="cuda").normal_(0.0, 1.5, generator=gen)
        s["q"] = q.transpose(1, 2)
        return s
    if c["op"] == "append":
        lens, counts = _append_sizes(c)
        need = [_up(n, page) for n in lens]
        total = sum(_up(n + k, page) for n, k in zip(lens, counts))
        pages = list(range(total + 5))
        rng.shuffle(pages)
        width = max(_up(n + k, page) for n, k in zip(lens, counts))
        at, table, ref = 0, [], [0] * len(pages)
        for k in need:
            row = pages[at:at + k]
            at += k
            for p in row:
                ref[p] += 1
            table.append(row + [-1] * (width - k))
        kv = _pool(gen, 2, len(pages), c)
        new = torch.empty((2, c["n"], c["L"], c["Hkv"], c["d"]), dtype=torch.bfloat16, device="cuda").normal_(generator=gen).transpose(2, 3)
        order = list(range(c["n"]))
        rng.shuffle(order)
        s.update(k=kv[0], v=kv[1], k_new=new[0], v_new=new[1], table=_ints(table), length=_ints(lens), ref=_ints(ref), seq=_ints(order),
                 count=_ints([counts[i] for i in order]))
    elif c["op"] == "fork":
        lens = _fork_sizes(c)
        n = c["parents"] * c["children"]
        need = [_up(x, page) for x in lens]
        pages = list(range(sum(need) + n + 4))
        rng.shuffle(pages)
        at, table, ref = 0, [], [0] * len(pages)
        for k in need:
            row = pages[at:at + k]
            at += k
            for p in row:
                ref[p] += 1
            table.append(row + [-1] * (max(need) - k))
        table += [[-1] * max(need)] * n
        s.update(pool=_pool(gen, c["planes"], len(pages), c), table=_ints(table), length=_ints(lens + [0] * n), ref=_ints(ref),
                 parent=_ints([k // c["children"] for k in range(n)]), child=_ints([c["parents"] + k for k in range(n)]))
    else:
        table, ref, drop, _, lens = _prune_layout(c, seed)
        s.update(pool=_pool(gen, c["planes"], len(ref), c), table=_ints(table), length=_ints(lens), ref=_ints(ref), drop=_ints(drop))
    s["out"] = tuple(torch.empty_like(s[k]) for k in ("table", "length", "ref"))
    return s


# ------------------------------------------------------------------------------------------------ one pass
def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(s):
    from paper_2608_15522_b200 import binding as av
    op = s["case"]["op"]
    if op == "attn":
        o, lse, _ = av.avsa_prefix_attn(s["q"], s["k"], s["v"], s["table"], s["length"], prefix_pages=s["shared"], causal=s["case"]["causal"], want_lse=True)
        return {"o": o, "lse": lse}
    if op == "append":
        table, length, ref, _ = av.avsa_cache_extend(s["table"], s["length"], s["ref"], s["seq"], s["count"], s["case"]["page"], out=s["out"])
        av.avsa_cache_write(s["k_new"], s["v_new"], s["k"], s["v"], table, length, seq=s["seq"], count=s["count"])
        return {"table": table, "length": length, "ref": ref, "k": s["k"], "v": s["v"]}
    if op == "fork":
        table, length, ref, _ = av.avsa_cache_fork(s["pool"], s["table"], s["length"], s["ref"], s["parent"], s["child"], out=s["out"])
        return {"table": table, "length": length, "ref": ref, "pool": s["pool"]}
    table, length, ref, _ = av.avsa_cache_free(s["table"], s["length"], s["ref"], s["drop"], out=s["out"])
    n_live, _ = av.avsa_cache_compact(s["pool"], table, length, ref)
    return {"table": table, "length": length, "ref": ref, "n_live": n_live, "pool": s["pool"]}


def _run_plain(s):
    return {"attn": _plain_attn, "append": _plain_append, "fork": _plain_fork, "prune": _plain_prune}[s["case"]["op"]](s)


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
    # the shared beginning, once: the rows of all sequences against it
    donor = table[length.argmax(), :shared]
    kp = s["k"][donor].transpose(0, 1).reshape(Hkv, np_, d).float()
    vp = s["v"][donor].transpose(0, 1).reshape(Hkv, np_, d).float()
    rows = qf.transpose(0, 1).reshape(Hkv, B * G * L, d)
    sp = (rows @ kp.transpose(1, 2)).view(Hkv, B, G * L, np_).transpose(0, 1)
    # each sequence's own pages
    mine = table[:, shared:]
    n_own = mine.shape[1] * page
    ko = s["k"][mine.clamp(min=0)].transpose(1, 2).reshape(B, Hkv, n_own, d).float()
    vo = s["v"][mine.clamp(min=0)].transpose(1, 2).reshape(B, Hkv, n_own, d).float()
    position = torch.arange(np_ + n_own, device=q.device)
    vo = vo.masked_fill((position[np_:] >= length[:, None])[:, None, :, None], 0.0)
    scores = torch.cat([sp, qf @ ko.transpose(2, 3)], dim=3)
    scores = scores.mul_(scale).masked_fill_(position >= limit, float("-inf"))
    lse = torch.logsumexp(scores, dim=3)
    p = scores.sub_(torch.where(lse == float("-inf"), 0.0, lse)[..., None]).exp_()
    o = p[..., np_:] @ vo
    o = o + (p[..., :np_].transpose(0, 1).reshape(Hkv, B * G * L, np_) @ vp).view(Hkv, B, G * L, d).transpose(0, 1)
    return {"o": o.reshape(B, H, L, d).to(torch.bfloat16), "lse": lse.reshape(B, H, L)}


def _plain_append(s):
    page, seq, count = s["case"]["page"], s["seq"].long(), s["count"].long()
    table, length, ref = (t.clone() for t in (s["table"], s["length"], s["ref"]))
    n = length[seq].long()
    have = (n + page - 1) // page
    need = (n + count + page - 1) // page - have
    first = need.cumsum(0) - need
    free = torch.nonzero(ref == 0)[:, 0]
    j = torch.arange(table.shape[1], device=seq.device)
    at = (j >= have[:, None]) & (j < (have + need)[:, None])            # the entries that get a page
    page_of = free[(first[:, None] + j - have[:, None]).clamp(0, free.shape[0] - 1)]
    table[seq] = torch.where(at, page_of.int(), table[seq])
    ref[page_of[at]] = 1
    length[seq] += s["count"]
    t = torch.arange(s["k_new"].shape[2], device=seq.device)
    b, t = torch.nonzero(t < count[:, None], as_tuple=True)
    pos = n[b] + t
    to = table[seq[b], pos // page].long()
    s["k"][to, :, pos % page] = s["k_new"].transpose(1, 2)[b, t]
    s["v"][to, :, pos % page] = s["v_new"].transpose(1, 2)[b, t]
    return {"table": table, "length": length, "ref": ref, "k": s["k"], "v": s["v"]}


def _plain_fork(s):
    page, parent, child = s["case"]["page"], s["parent"].long(), s["child"].long()
    table, length, ref = (t.clone() for t in (s["table"], s["length"], s["ref"]))
    n = length[parent].long()
    whole, begun = n // page, n % page > 0
    rows = s["table"][parent]
    j = torch.arange(table.shape[1], device=parent.device)
    keep = j < whole[:, None]
    ref.index_add_(0, rows[keep].long(), torch.ones_like(rows[keep]))
    free = torch.nonzero(s["ref"] == 0)[:, 0]
    rank = begun.long().cumsum(0) - 1
    dst = free[rank.clamp(min=0)]
    new = torch.where(keep, rows, torch.where((j == whole[:, None]) & begun[:, None], dst[:, None].int(), -1))
    table[child] = new
    length[child] = n.int()
    ref[dst[begun]] = 1
    src = rows.gather(1, whole.clamp(max=table.shape[1] - 1)[:, None])[:, 0].long()
    s["pool"][:, dst[begun]] = s["pool"][:, src[begun]]
    return {"table": table, "length": length, "ref": ref, "pool": s["pool"]}


def _plain_prune(s):
    drop = s["drop"].long()
    table, length, ref = (t.clone() for t in (s["table"], s["length"], s["ref"]))
    rows = table[drop]
    gone = rows[rows >= 0].long()
    ref.index_add_(0, gone, torch.full_like(gone, -1, dtype=torch.int32))
    table[drop] = -1
    length[drop] = 0
    live = ref > 0
    n_live = live.sum()
    index = torch.arange(ref.shape[0], device=ref.device)
    holes = torch.nonzero(~live & (index < n_live))[:, 0]
    moved = torch.nonzero(live & (index >= n_live))[:, 0]
    place = index.clone()
    place[moved] = holes
    table = torch.where(table >= 0, place[table.clamp(min=0).long()].int(), table)
    ref[holes] = ref[moved]
    ref[moved] = 0
    s["pool"][:, holes] = s["pool"][:, moved]
    return {"table": table, "length": length, "ref": ref, "n_live": n_live.int().reshape(1), "pool": s["pool"]}


# ------------------------------------------------------------------------------------------------ the definition in 64 bits
def exact(case, seed):
    """Attention position by position of the table; the other operators move data and compute whole numbers."""
    if case["op"] != "attn":
        return None
    s = prepare(case, seed)
    q, page, causal = s["q"], case["page"], case["causal"]
    B, H, L, d = q.shape
    group = H // case["Hkv"]
    o = torch.zeros((B, H, L, d), dtype=torch.float64, device=q.device)
    lse = torch.full((B, H, L), float("-inf"), dtype=torch.float64, device=q.device)
    lengths = s["length"].tolist()
    for b in range(B):
        n = lengths[b]
        if n == 0:
            continue
        at = torch.arange(n, device=q.device)
        pages, places = s["table"][b].long()[at // page], at % page
        hidden = at[None, :] > (torch.arange(L, device=q.device)[:, None] + n - L) if causal else None
        for g in range(case["Hkv"]):
            k, v = s["k"][pages, g, places].double(), s["v"][pages, g, places].double()
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
