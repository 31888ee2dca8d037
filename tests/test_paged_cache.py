"""Paged K/V cache and the attention over it, against the plain statement in oracle/cache_oracle.py.

What decides pages is compared exactly, page contents bit for bit, attention with the bars of the other attention calls
(parity_bars.py: bf16 P and bf16 O give 2^-9 relative each, fp32 sums a few 1e-6; LSE is fp32 throughout).
"""
import math
import os
import random

import numpy as np
import pytest
import torch

from oracle import cache_oracle as orc
from paper_2608_15522_b200 import binding as av
from parity_bars import close_lse, close_o

gpu = pytest.mark.gpu


# ------------------------------------------------------------------------------------------------ states
def random_state(rng, seqs, page, pages, most, shared=0):
    """Sequences of 0..most tokens whose first `shared` pages are the same (of a shorter one: all it has)."""
    order = list(range(pages))
    rng.shuffle(order)
    width = -(-most // page) + 2
    first, order = order[:shared], order[shared:]
    table, length, ref = np.full((seqs, width), -1, np.int32), np.zeros(seqs, np.int32), np.zeros(pages, np.int32)
    for s in range(seqs):
        n = rng.choice((0, 1, page - 1, page, page + 1, rng.randint(0, most))) if shared == 0 else rng.randint(shared * page, most)
        need = -(-n // page)
        row = first[:need] + [order.pop() for _ in range(max(0, need - shared))]
        table[s, :need], length[s] = row, n
        np.add.at(ref, row, 1)
    return table, length, ref


def check_state(table, length, ref, page):
    """Each page is held as often as ref says, rows have exactly the pages of their length."""
    held = np.zeros_like(ref)
    for row, n in zip(table, length):
        used = -(-int(n) // page)
        assert (row[:used] >= 0).all() and (row[used:] == -1).all()
        np.add.at(held, row[:used], 1)
    assert np.array_equal(held, ref)


def cu(x):
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def nump(t):
    return t.cpu().numpy()


def status(ws):
    return av.avsa_read_status(ws)[0]


# ------------------------------------------------------------------------------------------------ the oracle itself
@pytest.mark.parametrize("seed", range(20))
def test_oracle_keeps_its_state(seed):
    """Random changes one after the other leave pages held exactly as often as ref says, and tokens where they were."""
    rng = random.Random(seed)
    page, pages, seqs = rng.choice((16, 32)), 60, 8
    table, length, ref = random_state(rng, seqs, page, pages, 90)
    content = {}            # (page, place) -> token
    tokens = [[] for _ in range(seqs)]

    def put(s, n0):
        for pos in range(n0, int(length[s])):
            tokens[s].append(rng.random())
            content[table[s, pos // page], pos % page] = tokens[s][pos]

    for s in range(seqs):
        put(s, 0)
    for _ in range(12):
        kind = rng.choice(("extend", "fork", "free", "compact"))
        if kind == "extend":
            seq = rng.sample(range(seqs), 3)
            before = length.copy()
            table, length, ref, _ = orc.extend(table, length, ref, seq, [rng.randint(0, 20) for _ in seq], page)
            for s in seq:
                put(s, int(before[s]))
        elif kind == "fork":
            parent, child = rng.choice(range(seqs)), rng.choice(range(seqs))
            table, length, ref, moves, refused = orc.fork(table, length, ref, [parent], [child], page)
            for a, b in moves:
                content.update({(b, i): content[a, i] for i in range(page) if (a, i) in content})
            if not refused:
                tokens[child] = list(tokens[parent])
        elif kind == "free":
            s = rng.choice(range(seqs))
            table, length, ref = orc.free(table, length, ref, [s, s])
            tokens[s] = []
        else:
            table, ref, n, moves = orc.compact(table, ref)
            for a, b in moves:
                content.update({(b, i): content[a, i] for i in range(page) if (a, i) in content})
            assert (ref[:n] > 0).all() and (ref[n:] == 0).all()
        check_state(table, length, ref, page)
        for s in range(seqs):
            assert [content[table[s, i // page], i % page] for i in range(int(length[s]))] == tokens[s]


def test_oracle_attention_closed_forms():
    """Equal keys: the mean of the values; one token: its value; nothing: zero and -inf; causal rows see one token more each."""
    page, d = 16, 64
    k, v = np.ones((3, 1, page, d)), np.random.default_rng(0).normal(size=(3, 1, page, d))
    table, length = np.array([[2, 0], [1, -1], [-1, -1]], np.int32), np.array([20, 1, 0], np.int32)
    o, lse = orc.prefix_attention(np.ones((3, 2, 1, d)), k, v, table, length)
    seen = np.concatenate([v[2, 0], v[0, 0, :4]])
    assert np.allclose(o[0, :, 0], seen.mean(0)) and np.allclose(lse[0], math.log(20) + math.sqrt(d))
    assert np.allclose(o[1, :, 0], v[1, 0, 0]) and np.allclose(lse[1], math.sqrt(d))
    assert (o[2] == 0).all() and np.isneginf(lse[2]).all()
    o, lse = orc.prefix_attention(np.ones((1, 1, 22, d)), k, v, table, length, causal=True)
    assert (o[0, 0, :2] == 0).all() and np.isneginf(lse[0, 0, :2]).all()
    for i in range(2, 22):
        assert np.allclose(o[0, 0, i], seen[:i - 1].mean(0))


# ------------------------------------------------------------------------------------------------ refusals
def _cache(**kw):
    base = dict(table=1 << 20, length=2 << 20, ref=3 << 20, table_out=1 << 20, length_out=2 << 20, ref_out=3 << 20, seqs=4, width=8, pages=100, page=16)
    return av._Cache(**{**base, **kw})


def _pages(**kw):
    return av._Pages(**{**dict(ptr=1 << 24, planes=2, page_bytes=4096, stride_plane=409600, stride_page=4096), **kw})


@pytest.mark.parametrize("change,want", [
    (dict(seqs=0), 1), (dict(width=0), 1), (dict(pages=-1), 1), (dict(table=None), 1), (dict(ref_out=None), 1), (dict(length=(2 << 20) + 2), 1),
    (dict(page=48), 2), (dict(seqs=1 << 16, width=1 << 16), 2),
    (dict(table_out=(1 << 20) + 4), 1),          # overlaps what is read
    (dict(ref_out=2 << 20), 1), (dict(table_out=4 << 20, length_out=4 << 20), 1)])
def test_cache_calls_refuse(change, want):
    """Before anything is enqueued (the addresses are made up)."""
    lib, c = av.load_library(), _cache(**change)
    assert lib.avsa_cache_extend(c, 8192, 8192, 2, 1 << 16, 1 << 30, 0) == want
    assert lib.avsa_cache_fork(c, _pages(), 8192, 8192, 2, 1 << 16, 1 << 30, 0) == want
    assert lib.avsa_cache_compact(c, _pages(), 8192, 1 << 16, 1 << 30, 0) == want
    if "page" not in change:
        assert lib.avsa_cache_free(c, 8192, 2, 1 << 16, 1 << 30, 0) == want


def test_cache_calls_refuse_lists_workspaces_and_pools():
    lib, c = av.load_library(), _cache()
    need = av.avsa_cache_workspace_bytes(4, 100, 2)
    assert lib.avsa_cache_extend(c, None, 8192, 2, 1 << 16, 1 << 30, 0) == av.AVSA_ERR_INVALID_ARG
    assert lib.avsa_cache_extend(c, 8192, 8192, -1, 1 << 16, 1 << 30, 0) == av.AVSA_ERR_INVALID_ARG
    assert lib.avsa_cache_extend(c, 8192, 8192, 2, None, 1 << 30, 0) == av.AVSA_ERR_WORKSPACE
    assert lib.avsa_cache_extend(c, 8192, 8192, 2, 1 << 16, need - 1, 0) == av.AVSA_ERR_WORKSPACE
    assert lib.avsa_cache_extend(c, 8192, 8192, 2, (1 << 16) + 8, 1 << 30, 0) == av.AVSA_ERR_INVALID_ARG
    for bad in (dict(ptr=None), dict(ptr=(1 << 24) + 8), dict(planes=0), dict(page_bytes=4088), dict(stride_page=4080), dict(stride_plane=8)):
        assert lib.avsa_cache_fork(c, _pages(**bad), 8192, 8192, 2, 1 << 16, 1 << 30, 0) == av.AVSA_ERR_INVALID_ARG
        assert lib.avsa_cache_compact(c, _pages(**bad), 8192, 1 << 16, 1 << 30, 0) == av.AVSA_ERR_INVALID_ARG
    assert lib.avsa_cache_compact(c, _pages(), None, 1 << 16, 1 << 30, 0) == av.AVSA_ERR_INVALID_ARG
    assert av.avsa_cache_workspace_bytes(0, 1, 1) == 0 and av.avsa_cache_workspace_bytes(1, 1, -1) == 0


_T = av._Bf16Tensor4(1 << 24, 2 * 64 * 64, 64 * 64, 64)


@pytest.mark.parametrize("change,want", [
    (dict(B=-1), 1), (dict(H=0), 1), (dict(L=-1), 1), (dict(pages=0), 1), (dict(seqs=0), 1), (dict(width=0), 1), (dict(prefix=-1), 1), (dict(prefix=9), 1),
    (dict(H=5), 1), (dict(flags=2), 1), (dict(B=5), 1), (dict(d=96), 2), (dict(page=8), 2), (dict(page=256), 2), (dict(H=65536), 2), (dict(H=258), 2),
    (dict(seqs=1 << 16, width=1 << 16), 2), (dict(B=65536, seqs=1 << 17), 2), (dict(scale=-1.0), 1), (dict(scale=float("nan")), 1), (dict(scale=float("inf")), 1),
    (dict(q=av._Bf16Tensor4(None, 8, 8, 64)), 1), (dict(q=av._Bf16Tensor4((1 << 24) + 8, 8192, 4096, 64)), 1), (dict(k=av._Bf16Tensor4(1 << 24, 8192, 4096, 4)), 1),
    (dict(v=av._Bf16Tensor4(1 << 24, 8192, 0, 64)), 1), (dict(table=None), 1), (dict(length=None), 1), (dict(o=None), 1), (dict(o=(1 << 24) + 2), 1),
    (dict(ws=None), 3), (dict(ws_bytes=255), 3), (dict(ws=(1 << 16) + 16), 1)])
def test_attention_refuses(change, want):
    a = dict(B=4, H=4, Hkv=2, L=3, d=64, page=64, pages=10, seqs=4, width=8, q=_T, k=_T, v=_T, table=8192, length=8192, seq=None, prefix=2, flags=0, scale=0.0,
             o=1 << 25, lse=None, ws=1 << 16, ws_bytes=1 << 40)
    a.update(change)
    assert av.load_library().avsa_prefix_attn(*a.values(), 0) == want


def test_attention_of_nothing_is_no_error():
    lib = av.load_library()
    for B, L in ((0, 3), (4, 0)):
        assert lib.avsa_prefix_attn(B, 4, 2, L, 64, 64, 10, 4, 8, _T, _T, _T, 8192, 8192, None, 0, 0, 0.0, None, None, None, 0, 0) == av.AVSA_OK


def test_write_refuses():
    lib = av.load_library()
    good = dict(n=2, Hkv=2, L=3, d=64, page=64, pages=10, seqs=4, width=8, kn=_T, vn=_T, k=_T, v=_T, table=8192, length=8192, seq=None, count=None)
    for change, want in ((dict(n=-1), 1), (dict(n=5), 1), (dict(Hkv=0), 1), (dict(d=32), 2), (dict(page=24), 2), (dict(table=None), 1), (dict(length=None), 1),
                         (dict(kn=av._Bf16Tensor4(None, 8192, 4096, 64)), 1), (dict(v=av._Bf16Tensor4(1 << 24, 8192, 4096, 60)), 1), (dict(n=0), 0), (dict(L=0), 0)):
        assert lib.avsa_cache_write(*{**good, **change}.values(), 0) == want, change


def test_integers_off_their_grid_are_refused():
    """int32 arrays begin at multiples of four bytes, the optional ones too."""
    lib = av.load_library()
    attn = dict(B=4, H=4, Hkv=2, L=3, d=64, page=64, pages=10, seqs=4, width=8, q=_T, k=_T, v=_T, table=8192, length=8192, seq=None, prefix=2, flags=0, scale=0.0,
                o=1 << 25, lse=None, ws=1 << 16, ws_bytes=1 << 40)
    write = dict(n=2, Hkv=2, L=3, d=64, page=64, pages=10, seqs=4, width=8, kn=_T, vn=_T, k=_T, v=_T, table=8192, length=8192, seq=None, count=None)
    for name in ("table", "length", "seq", "lse"):
        assert lib.avsa_prefix_attn(*{**attn, name: 8194}.values(), 0) == av.AVSA_ERR_INVALID_ARG, name
    for name in ("table", "length", "seq", "count"):
        assert lib.avsa_cache_write(*{**write, name: 8193}.values(), 0) == av.AVSA_ERR_INVALID_ARG, name
    for a, b in ((8194, 8192), (8192, 8193)):
        assert lib.avsa_cache_extend(_cache(), a, b, 2, 1 << 16, 1 << 30, 0) == av.AVSA_ERR_INVALID_ARG
        assert lib.avsa_cache_fork(_cache(), _pages(), a, b, 2, 1 << 16, 1 << 30, 0) == av.AVSA_ERR_INVALID_ARG
    assert lib.avsa_cache_free(_cache(), 8194, 2, 1 << 16, 1 << 30, 0) == av.AVSA_ERR_INVALID_ARG


def test_wrappers_refuse_what_is_no_cuda_tensor():
    i = torch.zeros(4, dtype=torch.int32)
    t = torch.zeros((4, 2), dtype=torch.int32)
    q = torch.zeros((4, 2, 1, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="CUDA"):
        av.avsa_prefix_attn(q, q, q, t, i)
    with pytest.raises(TypeError, match="expected a tensor"):
        av.avsa_cache_free([1], i, i, i)
    with pytest.raises(ValueError, match="CUDA"):
        av.avsa_cache_extend(t, i, i, i, i, 16)
    with pytest.raises(ValueError, match="CUDA"):
        av.avsa_cache_write(q, q, q, q, t, i)


@gpu
def test_wrappers_refuse_shapes_types_and_layouts():
    i, t = ints([0] * 4), ints([[0, 0]] * 4)
    q = torch.zeros((4, 2, 1, 64), dtype=torch.bfloat16, device="cuda")
    pool = torch.zeros((5, 2, 16, 64), dtype=torch.bfloat16, device="cuda")
    ref = ints([0] * 5)
    ok = dict(q=q, k_pool=pool, v_pool=pool, table=t, length=i)
    for change in (dict(q=q.float()), dict(q=q[0]), dict(k_pool=pool[:4]), dict(k_pool=pool.transpose(2, 3)), dict(table=t.long()), dict(table=t[:, :1]),
                   dict(length=i[:3]), dict(seq=i[:2]), dict(lse=torch.zeros(3, device="cuda"), want_lse=True), dict(o=q[:2]), dict(o=q.transpose(1, 2).contiguous().transpose(1, 2)[:, :, :, ::2])):
        with pytest.raises((ValueError, RuntimeError)):
            av.avsa_prefix_attn(**{**ok, **change})
    with pytest.raises(TypeError):
        av.avsa_prefix_attn(**ok, prefix_pages=1.0)
    with pytest.raises(av.AvsaError):
        av.avsa_prefix_attn(**ok, prefix_pages=3)
    planes = torch.zeros((2, 5, 2, 16, 64), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError, match="one piece"):
        av.avsa_cache_fork(planes[:, :, :, :8], t, i, ref, i[:1], i[1:2])
    with pytest.raises(ValueError, match="as many pages"):
        av.avsa_cache_compact(planes[:, :4], t, i, ref)
    with pytest.raises(ValueError, match="different lengths"):
        av.avsa_cache_extend(t, i, ref, i, i[:2], 16)
    with pytest.raises(av.AvsaError):
        av.avsa_cache_extend(t, i, ref, i, i, 24)
    with pytest.raises(ValueError):
        av.avsa_cache_free(t, i, ref, i, out=(t[:2], i, ref))


# ------------------------------------------------------------------------------------------------ changes of the cache
def call(fn, state, *rest, out, **kw):
    """The call on copies of the state, in place or into other arrays full of rubbish; returns the state behind it and the workspace."""
    given = tuple(cu(x) for x in state)
    before = tuple(x.clone() for x in given)
    target = tuple(torch.full_like(x, 77) for x in given) if out else None
    got = fn(*given, *rest, out=target, **kw)
    if out:
        for x, y in zip(given, before):
            assert torch.equal(x, y), "what is read has changed"
    return tuple(nump(x) for x in got[:3]), got[3]


SIZES = [(1, 16, 4, 30), (7, 16, 60, 100), (40, 64, 700, 900), (300, 16, 9000, 400), (64, 32, 70000, 3000)]      # seqs, page, pages, most


@gpu
@pytest.mark.parametrize("out", [False, True])
@pytest.mark.parametrize("seqs,page,pages,most", SIZES)
def test_extend(seqs, page, pages, most, out):
    rng = random.Random(seqs)
    table, length, ref = random_state(rng, seqs, page, pages, most)
    for n in sorted({1, seqs // 2 or 1, seqs}):
        seq = rng.sample(range(seqs), n)
        count = [rng.choice((0, 1, page, rng.randint(0, 2 * page))) for _ in seq]
        if n > 2:
            seq[1] = -1
        *want, refused = orc.extend(table, length, ref, seq, count, page)
        got, ws = call(av.avsa_cache_extend, (table, length, ref), ints(seq), ints(count), page, out=out)
        for g, w in zip(got, want):
            assert np.array_equal(g, w)
        assert status(ws) == (av.AVSA_OK if not refused else av.AVSA_ERR_NO_PAGES)
        if not refused:
            check_state(*got, page)


@gpu
@pytest.mark.parametrize("out", [False, True])
def test_extend_refuses_what_cannot_be_had(out):
    """Too few pages, a full row, a sequence twice, out of range or of a negative count: the others get theirs."""
    page = 16
    table, length, ref = np.full((5, 4), -1, np.int32), np.zeros(5, np.int32), np.array([1, 0, 0, 1, 0, 0], np.int32)
    table[0, 0], length[0], table[1, 0], length[1] = 0, 16, 3, 3
    for seq, count, code in (([2, 1, 3], [17, 40, 14], av.AVSA_ERR_NO_PAGES), ([0], [49], av.AVSA_ERR_NO_PAGES), ([2, 2], [5, 6], av.AVSA_ERR_BAD_TABLE),
                             ([5, 1], [1, 1], av.AVSA_ERR_BAD_TABLE), ([0, 1], [-1, 14], av.AVSA_ERR_BAD_TABLE), ([], [], av.AVSA_OK),
                             ([1], [2 ** 31 - 1], av.AVSA_ERR_NO_PAGES)):
        *want, _ = orc.extend(table, length, ref, seq, count, page)
        got, ws = call(av.avsa_cache_extend, (table, length, ref), ints(seq), ints(count), page, out=out)
        for g, w in zip(got, want):
            assert np.array_equal(g, w), (seq, count)
        assert status(ws) == code


@gpu
@pytest.mark.parametrize("layout", ["heads", "tokens"])
@pytest.mark.parametrize("n,Hkv,L,d,page,ragged", [(1, 1, 1, 64, 16, False), (5, 3, 1, 128, 32, False), (4, 24, 37, 128, 64, True), (9, 8, 200, 64, 16, True), (3, 2, 130, 128, 128, False)])
def test_write(n, Hkv, L, d, page, ragged, layout):
    rng = random.Random(n * L)
    most = L + 3 * page
    table, length, ref = random_state(rng, n + 2, page, (n + 2) * (most // page + 2), most)
    seq = rng.sample(range(n + 2), n)
    count = [min(int(length[s]), rng.randint(0, L) if ragged else L) for s in seq]
    if n > 3:
        seq[2] = -1
    pools = [torch.randn((len(ref), Hkv, page, d), device="cuda").bfloat16() for _ in range(2)]
    if layout == "tokens":
        pools = [p.transpose(1, 2).contiguous().transpose(1, 2) for p in pools]
    new = [torch.randn((n, L, Hkv, d), device="cuda").bfloat16().transpose(1, 2) for _ in range(2)]
    want = [p.float().cpu().numpy() for p in pools]
    orc.write(*(x.float().cpu().numpy() for x in new), *want, table, length, seq, count)
    av.avsa_cache_write(*new, *pools, cu(table), cu(length), seq=ints(seq), count=ints(count))
    for p, w in zip(pools, want):
        assert np.array_equal(p.float().cpu().numpy(), w)


@gpu
def test_write_leaves_out_tokens_without_a_page():
    """Before the sequence's begin, behind the table, of a page out of range: nothing is written there, the others are."""
    page, d = 16, 64
    pool = torch.zeros((4, 1, page, d), dtype=torch.bfloat16, device="cuda")
    v = pool.clone()
    new = torch.ones((4, 1, 20, d), dtype=torch.bfloat16, device="cuda")
    table, length = ints([[0, -1], [1, 9], [2, 3], [-1, -1]]), ints([5, 20, 40, 3])
    av.avsa_cache_write(new, new, pool, v, table, length)
    want = torch.zeros_like(pool)
    want[0, 0, :5] = 1          # tokens 0..4 of 20: the others lie before the sequence
    want[1] = 1                 # 16..19 in a page out of range
    want[3, 0, 4:] = 1          # positions 20..31; 32..39 have no entry
    assert torch.equal(pool, want) and torch.equal(v, want)


@gpu
@pytest.mark.parametrize("out", [False, True])
@pytest.mark.parametrize("seqs,page,pages,most", SIZES)
@pytest.mark.parametrize("layout", ["heads", "tokens"])
def test_fork_then_prune(seqs, page, pages, most, out, layout):
    """Branches of several parents, then some sequences give their pages back and the pool is compacted: state and page contents."""
    rng = random.Random(seqs + page)
    Hkv, d, planes = (3, 64, 3) if pages < 10000 else (1, 64, 1)
    table, length, ref = random_state(rng, seqs, page, pages, most)
    if seqs == 1:
        table, length = np.concatenate([table, table * 0 - 1]), np.concatenate([length * 0, [0]]).astype(np.int32)
        length[0], table[0, :2], ref[:] = page + 3, (0, 1), (1, 1, 0, 0)
    pool = torch.randint(-30000, 30000, (planes, pages, Hkv, page, d), device="cuda", dtype=torch.int16).view(torch.bfloat16)
    if layout == "tokens":
        pool = pool.transpose(2, 3).contiguous().transpose(2, 3)
    bits = lambda: nump(pool.contiguous().view(torch.int16)).copy()
    empty = [s for s in range(len(length)) if length[s] == 0]
    busy = [s for s in range(len(length)) if length[s] > 0]
    child = empty[:20]
    parent = [rng.choice(busy) for _ in child]
    content = bits()
    *want, moves, refused = orc.fork(table, length, ref, parent, child, page)
    (t, n, r), ws = call(lambda *s, **kw: av.avsa_cache_fork(pool, *s, **kw), (table, length, ref), ints(parent), ints(child), out=out)
    for g, w in zip((t, n, r), want):
        assert np.array_equal(g, w)
    for a, b in moves:
        content[:, b] = content[:, a]
    assert np.array_equal(bits(), content)
    assert status(ws) == (av.AVSA_OK if not refused else av.AVSA_ERR_NO_PAGES)
    if not refused:
        check_state(t, n, r, page)
    table, length, ref = want
    drop = rng.sample(range(len(length)), (len(length) + 1) // 2)
    want = orc.free(table, length, ref, drop)
    (t, n, r), ws = call(av.avsa_cache_free, (table, length, ref), ints(drop + [-1, drop[0]]), out=out)
    for g, w in zip((t, n, r), want):
        assert np.array_equal(g, w)
    assert status(ws) == av.AVSA_OK
    table, length, ref = want
    want_table, want_ref, live, moves = orc.compact(table, ref)
    given = [cu(x) for x in (table, length, ref)]
    target = [torch.full_like(x, 77) for x in given] if out else given
    n_live, ws = av.avsa_cache_compact(pool, *given, out=tuple(target) if out else None)
    assert int(n_live) == live and status(ws) == av.AVSA_OK
    for g, w in zip(target, (want_table, length, want_ref)):
        assert np.array_equal(nump(g), w)
    for a, b in moves:
        content[:, b] = content[:, a]
    assert np.array_equal(bits(), content)


@gpu
def test_fork_refuses_what_cannot_be_had():
    page, d = 16, 64
    table, length, ref = np.full((6, 3), -1, np.int32), np.zeros(6, np.int32), np.array([1, 1, 0], np.int32)
    table[0, :2], length[0] = (0, 1), 20
    pool = torch.randn((1, 3, 1, page, d), device="cuda").bfloat16()
    for parent, child, code in (([0, 0, 5], [1, 2, 3], av.AVSA_ERR_NO_PAGES), ([0, 0], [1, 1], av.AVSA_ERR_BAD_TABLE), ([1, 0], [0, 2], av.AVSA_ERR_BAD_TABLE),
                                ([0, 6], [7, 1], av.AVSA_ERR_BAD_TABLE), ([-1, 0, 0], [1, -1, 2], av.AVSA_OK), ([], [], av.AVSA_OK), ([1], [1], av.AVSA_OK)):
        *want, _, _ = orc.fork(table, length, ref, parent, child, page)
        got, ws = call(lambda *s, **kw: av.avsa_cache_fork(pool, *s, **kw), (table, length, ref), ints(parent), ints(child), out=False)
        for g, w in zip(got, want):
            assert np.array_equal(g, w), (parent, child)
        assert status(ws) == code, (parent, child)


@gpu
def test_fork_entries_that_are_left_out_take_no_place():
    """A negative parent leaves its entry out; a later one may name the same child."""
    table, length, ref = np.array([[0, 1], [-1, -1]], np.int32), np.array([20, 0], np.int32), np.array([1, 1, 0], np.int32)
    pool = torch.randn((1, 3, 1, 16, 64), device="cuda").bfloat16()
    want = orc.fork(table, length, ref, [-1, 0], [1, 1], 16)
    assert not want[4] and want[3] == [(1, 2)]
    state = [cu(x) for x in (table, length, ref)]
    ws = av.avsa_cache_fork(pool, *state, ints([-1, 0]), ints([1, 1]))[3]
    assert status(ws) == av.AVSA_OK
    for g, w in zip(state, want):
        assert np.array_equal(nump(g), w)
    assert torch.equal(pool[:, 2], pool[:, 1])


@gpu
def test_malformed_rows_are_reported():
    """Pages out of range and pages that nobody holds: reported, nothing outside the arrays touched."""
    table, length, ref = ints([[0, 9, -3]]), ints([40]), ints([0, 0, 1])
    _, _, _, ws = av.avsa_cache_free(table, length, ref, ints([0, 4]))
    assert status(ws) == av.AVSA_ERR_BAD_TABLE and table.tolist() == [[-1, -1, -1]]
    pool = torch.zeros((1, 3, 1, 16, 64), dtype=torch.bfloat16, device="cuda")
    n_live, ws = av.avsa_cache_compact(pool, ints([[2, 1, 7]]), ints([40]), ints([0, 0, 1]))
    assert status(ws) == av.AVSA_ERR_BAD_TABLE and int(n_live) == 1
    _, _, _, ws = av.avsa_cache_fork(pool, ints([[7, -5, 9], [-1, -1, -1]]), ints([40, 0]), ints([0, 0, 1]), ints([0]), ints([1]))
    assert status(ws) == av.AVSA_ERR_BAD_TABLE


@gpu
def test_compact_of_a_full_and_of_an_empty_pool():
    pool = torch.randn((2, 5, 1, 16, 64), device="cuda").bfloat16()
    before = pool.clone()
    for ref, live in (([1] * 5, 5), ([0] * 5, 0)):
        table = ints([[0, 1, 2, 3, 4]]) if live else ints([[-1] * 5])
        n, ws = av.avsa_cache_compact(pool, table, ints([80 if live else 0]), ints(ref))
        assert int(n) == live and status(ws) == av.AVSA_OK and torch.equal(pool, before)


# ------------------------------------------------------------------------------------------------ attention
def attention_case(B, H, Hkv, L, d, page, lengths, shared=0, seed=0, q_layout="bhld", kv_layout="heads", idle=(), poison=True, spread=1.0, width=None):
    """Sequences of the given lengths, the first `shared` pages the same; what no sequence holds is NaN."""
    gen = torch.Generator().manual_seed(seed)
    rng = random.Random(seed)
    seqs = len(lengths)
    need = [max(0, -(-n // page) - shared) for n in lengths]
    pages = shared + sum(need) + 3
    order = list(range(pages))
    rng.shuffle(order)
    first, order = order[:shared], order[shared:]
    table = np.full((seqs, width or max(1, max(-(-n // page) for n in lengths) + 1)), -1, np.int32)
    held = np.zeros((pages, page), bool)
    for s, n in enumerate(lengths):
        used = -(-n // page)
        row = first[:used] + [order.pop() for _ in range(max(0, used - shared))]
        table[s, :used] = row
        for t in range(n):
            held[row[t // page], t % page] = True
    kv = torch.randn((2, pages, Hkv, page, d), generator=gen)
    kv[0] *= spread
    if poison:
        kv = torch.where(torch.from_numpy(held)[None, :, None, :, None], kv, float("nan"))
    kv = kv.bfloat16().cuda()
    if kv_layout == "tokens":
        kv = kv.transpose(2, 3).contiguous().transpose(2, 3)
    q = torch.randn((B, H, L, d), generator=gen).bfloat16().cuda()
    if q_layout == "blhd":
        q = q.transpose(1, 2).contiguous().transpose(1, 2)
    return q, kv[0], kv[1], table, np.array(lengths, np.int32)


def check_attention(q, k, v, table, length, prefix_pages=0, seq=None, causal=False, scale=0.0, what="", **kw):
    o, lse, ws = av.avsa_prefix_attn(q, k, v, cu(table), cu(length), prefix_pages=prefix_pages, seq=None if seq is None else ints(seq), causal=causal,
                                     softmax_scale=scale, want_lse=True, **kw)
    assert status(ws) == av.AVSA_OK
    f64 = lambda t: t.double().cpu().numpy()
    want, want_lse = orc.prefix_attention(f64(q), f64(k), f64(v), table, length, seq, causal, scale or None)
    got, got_lse = f64(o), f64(lse)
    empty = np.isneginf(want_lse)
    assert np.array_equal(np.isneginf(got_lse), empty), what
    assert (got[empty] == 0).all(), what
    if not empty.all():
        close_o(got[~empty], want[~empty], what)
        close_lse(got_lse[~empty], want_lse[~empty], what)
    return o, lse, ws


@gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("n", [0, 1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 255, 257, 400])
def test_attention_lengths(n, page, d):
    """One token against n of them, alone and beside a longer sequence."""
    check_attention(*attention_case(2, 3, 3, 1, d, page, [n, 300], seed=n), what=f"{n}")
    check_attention(*attention_case(1, 2, 1, 1, d, page, [n], seed=n), what=f"{n} alone")


@gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("H,Hkv", [(1, 1), (2, 2), (6, 2), (8, 1), (14, 2), (128, 1), (16, 16)])
@pytest.mark.parametrize("L", [1, 2, 7, 33, 130])
@pytest.mark.parametrize("causal", [False, True])
def test_attention_heads_and_queries(H, Hkv, L, d, causal):
    if H * L > 5000:
        L = 17
    case = attention_case(3, H, Hkv, L, d, 32, [200, 64, 131], seed=H + L, q_layout="blhd")
    check_attention(*case, causal=causal)


@gpu
@pytest.mark.parametrize("kv_layout", ["heads", "tokens"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page,shared", [(16, 1), (16, 63), (32, 20), (64, 3), (128, 5)])
@pytest.mark.parametrize("B,L,H,Hkv", [(1, 1, 2, 2), (9, 1, 4, 4), (40, 1, 8, 2), (6, 5, 6, 2), (3, 50, 3, 1), (2, 150, 2, 2)])
@pytest.mark.parametrize("causal", [False, True])
def test_attention_behind_a_shared_beginning(B, L, H, Hkv, page, shared, d, causal, kv_layout):
    rng = random.Random(B * page)
    n = shared * page
    lengths = [n + rng.choice((0, 1, page, rng.randint(0, 300))) for _ in range(B)]
    if B > 4:
        lengths[2], lengths[4] = 0, max(1, n - page // 2)      # one holds nothing, one is a part of the beginning
    lengths[-1] = max(lengths[-1], n)
    case = attention_case(B, H, Hkv, L, d, page, lengths, shared=shared, seed=B, kv_layout=kv_layout)
    a = check_attention(*case, prefix_pages=shared, causal=causal, what="shared")
    b = check_attention(*case, prefix_pages=0, causal=causal, what="each by itself")
    for x, y in zip(a[:2], b[:2]):
        assert torch.allclose(x.float(), y.float(), atol=2e-2, rtol=2e-2)


@gpu
def test_attention_of_chosen_sequences():
    """Batch entries in another order than the sequences, one of them without any."""
    q, k, v, table, length = attention_case(5, 4, 2, 3, 64, 16, [40, 77, 0, 130, 16, 99, 64], shared=0, seed=5)
    for causal in (False, True):
        check_attention(q, k, v, table, length, seq=[6, -1, 3, 2, 0], causal=causal)
    q, k, v, table, length = attention_case(4, 4, 4, 1, 128, 16, [400, 333, 390, 350, 401, 320], shared=20, seed=6)
    check_attention(q, k, v, table, length, seq=[5, 4, -1, 1], prefix_pages=20)


@gpu
@pytest.mark.parametrize("scale", [0.02, 0.7])
@pytest.mark.parametrize("L,shared", [(1, 0), (1, 20), (200, 0), (200, 20)])
def test_attention_scales(L, shared, scale):
    check_attention(*attention_case(3, 2, 2, L, 128, 32, [700, 640, 903], shared=shared), prefix_pages=shared, scale=scale)


@gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("L,shared,causal", [(1, 0, False), (1, 40, False), (5, 40, True), (300, 0, True), (300, 40, False)])
@pytest.mark.parametrize("grow", [30.0, 300.0])
def test_attention_maxima_that_grow_along_the_keys(L, shared, causal, d, grow):
    """Logits that rise by `grow` (as powers of e) from the first key to the last: every reference is outgrown."""
    q, k, v, table, length = attention_case(2, 2, 1, L, d, 32, [1400, 1500], shared=shared, seed=3, poison=False)
    one = torch.zeros(d, device="cuda")
    one[0] = 1.0
    q = (q.float() * (1 - one) + one * 4.0).bfloat16()
    k = k.clone()
    for s in range(2):
        for t in range(int(length[s])):
            k[table[s, t // 32], :, t % 32, 0] = grow * math.sqrt(d) / 4.0 * t / 1500
    check_attention(q, k, v, table, length, prefix_pages=shared, causal=causal)


@gpu
def test_attention_reproduces_and_ignores_old_memory():
    """Bit for bit: run after run, whatever workspace and outputs held, on another stream, and as a replayed graph."""
    q, k, v, table, length = attention_case(20, 8, 4, 2, 128, 64, [1500 + 13 * i for i in range(20)], shared=20, seed=9)
    t, n = cu(table), cu(length)
    first = av.avsa_prefix_attn(q, k, v, t, n, prefix_pages=20, want_lse=True)
    for fill in (0, 255):
        ws = torch.full_like(first[2], fill)
        o, lse = torch.full_like(first[0], float("nan")), torch.full_like(first[1], float("nan"))
        av.avsa_prefix_attn(q, k, v, t, n, prefix_pages=20, want_lse=True, o=o, lse=lse, ws=ws)
        assert torch.equal(o, first[0]) and torch.equal(lse, first[1])
    o2 = av.avsa_prefix_attn(q, k, v, t, n, prefix_pages=20)
    assert o2[1] is None and torch.equal(o2[0], first[0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        o3 = av.avsa_prefix_attn(q, k, v, t, n, prefix_pages=20)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(o3[0], first[0])
    graph = torch.cuda.CUDAGraph()
    o, lse, ws = torch.empty_like(first[0]), torch.empty_like(first[1]), torch.empty_like(first[2])
    with torch.cuda.graph(graph):
        av.avsa_prefix_attn(q, k, v, t, n, prefix_pages=20, want_lse=True, o=o, lse=lse, ws=ws)
    for _ in range(3):
        o.zero_()
        graph.replay()
        assert torch.equal(o, first[0]) and torch.equal(lse, first[1])


@gpu
def test_attention_reports_malformed_tables():
    """Pages out of range contribute nothing, lengths beyond the row are cut: reported, and the other sequences are right."""
    q, k, v, table, length = attention_case(3, 2, 2, 1, 64, 16, [100, 100, 100], seed=1)
    f64 = lambda t: t.double().cpu().numpy()
    want, _ = orc.prefix_attention(f64(q), f64(k), f64(v), table, length)
    for change in ("page", "negative", "length", "sequence"):
        t, n, seq = table.copy(), length.copy(), [0, 1, 2]
        if change == "page":
            t[1, 2] = 1000
        elif change == "negative":
            t[1, 2] = -1
        elif change == "length":
            n[1] = 10 ** 6
            t[1, :] = 0
        else:
            seq[1] = 3
        o, _, ws = av.avsa_prefix_attn(q, k, v, cu(t), cu(n), seq=ints(seq))
        assert status(ws) == av.AVSA_ERR_BAD_TABLE, change
        close_o(f64(o)[[0, 2]], want[[0, 2]], change)


@gpu
def test_attention_offsets_beyond_32_bits():
    """Pages whose distance from the pool's beginning passes 2^32 elements, and a table row far into the pool."""
    free = torch.cuda.mem_get_info()[0]
    page, d, pages = 64, 128, 6
    step = (1 << 30) + 64            # elements between pages: page 5 begins beyond 5 * 2^30 (> 2^32)
    if free < 2 * (5 * step + page * d) * 2 + (2 << 30):
        pytest.skip("too little free memory")
    flat = torch.empty(5 * step + page * d, dtype=torch.bfloat16, device="cuda")
    pool = flat.as_strided((pages, 1, page, d), (step, page * d, d, 1))
    k0, v0 = (torch.randn((pages, 1, page, d), device="cuda").bfloat16() for _ in range(2))
    flat2 = torch.empty_like(flat)
    vpool = flat2.as_strided(pool.shape, pool.stride())
    pool.copy_(k0)
    vpool.copy_(v0)
    table, length = np.array([[5, 0, 4], [3, 5, 1]], np.int32), np.array([170, 192], np.int32)
    q = torch.randn((2, 2, 1, d), device="cuda").bfloat16()
    o, _, ws = av.avsa_prefix_attn(q, pool, vpool, cu(table), cu(length))
    want, _ = orc.prefix_attention(*(x.double().cpu().numpy() for x in (q, k0, v0)), table, length)
    close_o(o.double().cpu().numpy(), want, "far pages")
    new = torch.randn((2, 1, 3, d), device="cuda").bfloat16()
    av.avsa_cache_write(new, new, pool, vpool, cu(table), cu(length))
    assert torch.equal(pool[4, 0, 39:42], new[0, 0]) and torch.equal(vpool[1, 0, 61:64], new[1, 0])


# ------------------------------------------------------------------------------------------------ every way the work is cut
def exact_on_gpu(q, k, v, table, length, seq=None, causal=False):
    """orc.prefix_attention for sizes that numpy takes too long for: the same statement in 64 bits on the GPU."""
    B, H, L, d = q.shape
    page, group = k.shape[2], H // k.shape[1]
    o = torch.zeros((B, H, L, d), dtype=torch.float64, device="cuda")
    lse = torch.full((B, H, L), float("-inf"), dtype=torch.float64, device="cuda")
    for b in range(B):
        s = b if seq is None else seq[b]
        n = int(length[s]) if s >= 0 else 0
        if n == 0:
            continue
        at = torch.arange(n, device="cuda")
        pages = cu(table)[s].long()[at // page]
        kk, vv = k[pages, :, at % page].double().transpose(0, 1), v[pages, :, at % page].double().transpose(0, 1)      # [Hkv,n,d]
        x = q[b].double().reshape(-1, group * L, d) @ kk.transpose(1, 2) / math.sqrt(d)
        if causal:
            lim = torch.arange(L, device="cuda").repeat(group) + n - L + 1
            x.masked_fill_(at[None, :] >= lim[:, None], float("-inf"))
        z = torch.logsumexp(x, 2)
        w = torch.exp(x - torch.where(torch.isinf(z), 0.0, z)[..., None])
        o[b], lse[b] = (w @ vv).reshape(H, L, d), z.reshape(H, L)
    return o, lse


def check_on_gpu(q, k, v, table, length, what, **kw):
    seq = kw.pop("seq", None)
    o, lse, ws = av.avsa_prefix_attn(q, k, v, cu(table), cu(length), seq=None if seq is None else ints(seq), want_lse=True, **kw)
    assert status(ws) == av.AVSA_OK
    want, want_lse = exact_on_gpu(q, k, v, table, length, seq, kw.get("causal", False))
    empty = torch.isinf(want_lse)
    assert torch.equal(torch.isinf(lse), empty) and (o[empty] == 0).all(), what
    close_o(o.double()[~empty].cpu().numpy(), want[~empty].cpu().numpy(), what)
    close_lse(lse.double()[~empty].cpu().numpy(), want_lse[~empty].cpu().numpy(), what)
    return o, lse, ws


def lengths_behind(rng, B, shared, page, most):
    """Ragged lengths behind a shared beginning; with a few of them one sequence holds nothing and one a part of the beginning."""
    v = [shared * page + rng.choice((0, 1, page - 1, rng.randint(0, most))) for _ in range(B)]
    if B > 3:
        v[1], v[2] = 0, shared * page // 2 + 3
    v[-1] = shared * page + most
    return v


@gpu
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B,L,H,Hkv,page,tokens,most", [
    (8, 1, 32, 32, 16, 2048, 300),        # 8 stacked rows: parts by warps' products of one column block
    (16, 1, 24, 24, 64, 2048, 700),       # 16: two
    (30, 1, 16, 16, 32, 2048, 100),       # 30: two row tiles
    (4, 7, 24, 24, 64, 4096, 90),         # 28 rows, several tokens
    (40, 1, 32, 8, 128, 2048, 500),       # 160: the tile kernel, own keys by warps
    (64, 1, 32, 4, 64, 2048, 260),        # 512: four row tiles side by side
    (200, 1, 16, 2, 16, 2048, 40),        # 1600: thirteen, in two turns
    (12, 10, 24, 8, 32, 4096, 200),       # 30 rows a sequence, gathered (three query heads to a key head)
    (12, 20, 8, 2, 32, 16384, 400),       # 80 rows: the tile kernel for both
    (9, 50, 24, 8, 64, 16384, 333)])      # 150: two row tiles of own rows, gathered
def test_attention_stacked(B, L, H, Hkv, page, tokens, most, d, causal):
    """The beginning is read for the rows of all sequences at once; the same call without saying that it is shared gives the same."""
    rng = random.Random(B + d)
    shared = tokens // page
    case = attention_case(B, H, Hkv, L, d, page, lengths_behind(rng, B, shared, page, most), shared=shared, seed=B, q_layout="blhd")
    a = check_on_gpu(*case, "stacked", prefix_pages=shared, causal=causal)
    b = check_on_gpu(*case, "each by itself", causal=causal)
    assert torch.allclose(a[0].float(), b[0].float(), atol=2e-2, rtol=2e-2)


@gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B,L,H,Hkv,width,lengths", [
    (1, 1, 8, 8, 400, (6000,)),           # few items, long rows: parts that another kernel joins
    (1, 3, 8, 2, 400, (6400,)),
    (2, 1, 4, 1, 500, (1, 7900)),
    (1, 31, 4, 4, 300, (4700,)),
    (3, 1, 24, 24, 60, (900, 0, 17)),     # a cluster of CTAs an item
    (20, 2, 16, 16, 80, tuple(range(5, 1285, 64))),
    (70, 1, 32, 8, 300, tuple(range(1, 4700, 67))[:70])])
def test_attention_of_few_rows(B, L, H, Hkv, width, lengths, d):
    rng = random.Random(d)
    case = attention_case(B, H, Hkv, L, d, 16, list(lengths), seed=B, width=width)
    for causal in (False, True):
        check_on_gpu(*case, "few rows", causal=causal)


@gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B,L,H,Hkv,page,lengths,causal", [
    (1, 700, 32, 32, 64, (3000,), False),          # whole items off a queue, the last ones cut
    (1, 2500, 8, 8, 128, (2500,), True),
    (3, 509, 32, 8, 64, (509, 3000, 1754), True),
    (5, 200, 24, 8, 32, (1000, 77, 0, 500, 640), True),
    (2, 129, 6, 6, 16, (2000, 129), False),        # fewer items than SMs
    (1, 33, 2, 2, 16, (5000,), False)])
def test_attention_of_many_rows(B, L, H, Hkv, page, lengths, causal, d):
    check_on_gpu(*attention_case(B, H, Hkv, L, d, page, list(lengths), seed=L, q_layout="blhd"), "many rows", causal=causal)


@gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B,L,H,Hkv,tokens", [(16, 1, 24, 24, 2048), (40, 1, 32, 8, 2048), (12, 20, 8, 2, 16384), (1, 300, 4, 4, 0)])
def test_attention_rows_that_outgrow_their_reference(B, L, H, Hkv, tokens, d):
    """Logits that rise by 300 (as powers of e) along the keys: every way of cutting, the tile kernel's second run among them."""
    page, shared = 64, tokens // 64
    q, k, v, table, length = attention_case(B, H, Hkv, L, d, page, [tokens + 700 + b for b in range(B)], shared=shared, seed=4, poison=False)
    one = torch.zeros(d, device="cuda")
    one[0] = 1.0
    q = (q.float() * (1 - one) + one * 4.0).bfloat16()
    k = k.clone()
    for s in range(B):
        at = torch.arange(int(length[s]), device="cuda")
        k[cu(table)[s].long()[at // page], :, at % page, 0] = (300.0 * math.sqrt(d) / 4.0 * at / (tokens + 800)).bfloat16()[:, None].expand(-1, Hkv)
    _, _, ws = check_on_gpu(q, k, v, table, length, "growing", prefix_pages=shared)
    if L >= 300:
        assert av.avsa_redo_count(ws) > 0


@gpu
@pytest.mark.parametrize("B,L,H,Hkv", [(8, 1, 32, 32), (40, 1, 32, 8), (12, 20, 8, 2)])
def test_attention_stacked_reports_and_reproduces(B, L, H, Hkv):
    """A page out of range in the beginning and behind it, a length that is cut; the same bits twice, on memory full of ones."""
    page, shared = 64, 256 if L > 1 else 32
    q, k, v, table, length = attention_case(B, H, Hkv, L, 64, page, [shared * page + 100] * B, shared=shared, seed=2)
    first = av.avsa_prefix_attn(q, k, v, cu(table), cu(length), prefix_pages=shared, want_lse=True)
    again = av.avsa_prefix_attn(q, k, v, cu(table), cu(length), prefix_pages=shared, want_lse=True, ws=torch.full_like(first[2], 255))
    assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1]) and status(again[2]) == av.AVSA_OK
    for where in ((0, 5), (3, shared), (B - 1, shared + 1)):
        bad = table.copy()
        bad[where] = 10 ** 6
        assert status(av.avsa_prefix_attn(q, k, v, cu(bad), cu(length), prefix_pages=shared)[2]) == av.AVSA_ERR_BAD_TABLE, where
    bad = length.copy()
    bad[3] = -5
    assert status(av.avsa_prefix_attn(q, k, v, cu(table), cu(bad), prefix_pages=shared)[2]) == av.AVSA_ERR_BAD_TABLE


@gpu
def test_attention_workspaces_depend_on_the_shape_alone():
    """What the query says is enough for every call of the shape, whatever the lengths."""
    for B, L, H, Hkv, page, width, prefix in ((1, 1, 8, 8, 16, 400, 0), (16, 1, 24, 24, 64, 60, 32), (40, 1, 32, 8, 128, 40, 16), (3, 509, 32, 8, 64, 50, 0)):
        need = av.avsa_prefix_attn_workspace_bytes(B, H, Hkv, L, 64, page, width, prefix)
        assert need > 256
        q = torch.randn((B, H, L, 64), device="cuda").bfloat16()
        pool = torch.randn((width, Hkv, page, 64), device="cuda").bfloat16()
        table = torch.arange(width, dtype=torch.int32, device="cuda").repeat(B, 1)
        guard = torch.full((need + 4096,), 77, dtype=torch.uint8, device="cuda")
        for n in (width * page, prefix * page, 1, 0):
            av.avsa_prefix_attn(q, pool, pool, table, ints([n] * B), prefix_pages=prefix, ws=guard[:need])
            assert (guard[need:] == 77).all()
        with pytest.raises(av.AvsaError):
            av.avsa_prefix_attn(q, pool, pool, table, ints([1] * B), prefix_pages=prefix, ws=guard[:need - 32])
