"""Plain statement of the paged K/V cache and of the attention over it, in numpy (whole numbers; attention in 64 bits).

State: table [seqs,width] (pages of a sequence in order, -1 behind the last one), length [seqs], ref [pages] (sequences that
hold the page, 0 = free).  Every function returns the state behind the call and leaves its arguments alone.
"""
from __future__ import annotations

import numpy as np


def _up(n, page):
    return -(-int(n) // page)


def _free(ref):
    return [int(p) for p in np.nonzero(ref <= 0)[0]]


def extend(table, length, ref, seq, count, page):
    """Returns (table, length, ref, refused list entries): free pages are dealt out in list order, lowest first; an entry whose pages cannot all
    be had changes nothing, and those behind it do not get what it left."""
    table, length, ref0 = table.copy(), length.copy(), ref
    ref = ref.copy()
    free, at, refused, seen = _free(ref0), 0, [], set()
    for k, (s, c) in enumerate(zip(seq, count)):
        if s < 0:
            continue
        if s >= len(length) or s in seen or c < 0 or int(length[s]) + c > table.shape[1] * page:
            refused.append(k)
            seen.add(int(s))
            continue
        seen.add(int(s))
        have, need = _up(length[s], page), _up(int(length[s]) + c, page) - _up(length[s], page)
        mine, at = free[at:at + need], at + need
        if len(mine) < need:
            refused.append(k)
            continue
        table[s, have:have + need] = mine
        ref[mine] = 1
        length[s] += c
    return table, length, ref, refused


def write(k_new, v_new, k_pool, v_pool, table, length, seq, count):
    """Pools [pages,Hkv,page,d] changed in place; k_new/v_new [n,Hkv,L,d]."""
    page = k_pool.shape[2]
    for b, (s, c) in enumerate(zip(seq, count)):
        if s < 0:
            continue
        for j in range(int(c)):
            pos = int(length[s]) - int(c) + j
            p = table[s, pos // page]
            k_pool[p, :, pos % page] = k_new[b, :, j]
            v_pool[p, :, pos % page] = v_new[b, :, j]


def fork(table, length, ref, parent, child, page):
    """Returns (table, length, ref, moves, refused); moves: (from, to) pages whose contents are copied."""
    table0, length0 = table, length
    table, length, free, ref = table.copy(), length.copy(), _free(ref), ref.copy()
    moves, refused, at, seen = [], [], 0, set()
    for k, (p, s) in enumerate(zip(parent, child)):
        if p < 0 or s < 0:
            continue
        if s >= len(length) or p >= len(length) or s in seen or length0[s] != 0:
            refused.append(k)
            seen.add(int(s))
            continue
        seen.add(int(s))
        whole, begun = divmod(int(length0[p]), page)
        row = np.full(table.shape[1], -1, table.dtype)
        row[:whole] = table0[p, :whole]
        if begun:
            if at >= len(free):
                refused.append(k)
                at += 1
                continue
            row[whole] = free[at]
            moves.append((int(table0[p, whole]), free[at]))
            ref[free[at]] = 1
            at += 1
        np.add.at(ref, row[:whole], 1)
        table[s], length[s] = row, length0[p]
    return table, length, ref, moves, refused


def free(table, length, ref, seq):
    table, length, ref = table.copy(), length.copy(), ref.copy()
    for s in seq:
        if s < 0 or s >= len(length):
            continue
        np.add.at(ref, table[s][table[s] >= 0], -1)
        table[s], length[s] = -1, 0
    return table, length, ref


def compact(table, ref):
    """Returns (table, ref, n_live, moves)."""
    n = int((ref > 0).sum())
    holes = [p for p in range(n) if ref[p] <= 0]
    used = [p for p in range(n, len(ref)) if ref[p] > 0]
    place = np.arange(len(ref))
    place[used] = holes
    new = np.where(ref > 0, ref, 0)
    new[holes] = ref[used]
    new[n:] = 0
    return np.where(table >= 0, place[np.maximum(table, 0)], -1).astype(table.dtype), new.astype(ref.dtype), n, list(zip(used, holes))


def limits(length, seq, B, L, causal, count=None):
    """[B,L]: how many of its sequence's tokens a row sees.  count [B]: the first count[b] rows are the sequence's last tokens (None: all L)."""
    out = np.zeros((B, L), np.int64)
    for b in range(B):
        s = int(seq[b])
        if s >= 0:
            n, i = L if count is None else int(count[b]), np.arange(L)
            out[b] = np.where(i < n, np.maximum(0, length[s] - n + 1 + i), 0) if causal else length[s]
    return out


def prefix_attention(q, k_pool, v_pool, table, length, seq=None, causal=False, scale=None, count=None):
    """q [B,H,L,d], pools [pages,Hkv,page,d] in fp64 -> (o, lse); an empty row is 0 and -inf."""
    B, H, L, d = q.shape
    Hkv, page = k_pool.shape[1:3]
    seq = np.arange(B) if seq is None else seq
    scale = scale or 1.0 / np.sqrt(d)
    lim = limits(length, seq, B, L, causal, count)
    o, lse = np.zeros((B, H, L, d)), np.full((B, H, L), -np.inf)
    for b in range(B):
        n = int(length[seq[b]]) if seq[b] >= 0 else 0
        if n == 0:
            continue
        at = np.arange(n)
        pages = table[seq[b], at // page]
        for g in range(Hkv):
            k, v = k_pool[pages, g, at % page], v_pool[pages, g, at % page]
            rows = q[b, g * (H // Hkv):(g + 1) * (H // Hkv)].reshape(-1, d)
            x = rows @ k.T * scale
            hidden = at[None, :] >= np.tile(lim[b], H // Hkv)[:, None]
            x[hidden] = -np.inf
            top = x.max(1, keepdims=True)
            top = np.where(np.isneginf(top), 0.0, top)
            e = np.exp(x - top)
            z = e.sum(1, keepdims=True)
            with np.errstate(divide="ignore", invalid="ignore"):
                o[b, g * (H // Hkv):(g + 1) * (H // Hkv)] = np.where(z > 0, (e @ v) / z, 0.0).reshape(-1, L, d)
                lse[b, g * (H // Hkv):(g + 1) * (H // Hkv)] = (top + np.log(z)).reshape(-1, L)
    return o, lse
