"""The paged cache held in 4 bits, against the plain statements in oracle/q4_oracle.py and oracle/cache_oracle.py.

What a page stands for is compared bit for bit: codes and scales are whole numbers that the format decides, and every value is a bf16 number.  Attention has the bars of
the other attention calls (parity_bars.py) against 64 bits on those values.
"""
import math
import random

import numpy as np
import pytest
import torch

from oracle import cache_oracle as corc
from oracle import q4_oracle as orc
from paper_2608_15522_b200 import binding as av
from paper_2608_15522_b200.continuation import ClipCache, continue_clip
from parity_bars import close_lse, close_o
from test_paged_cache import attention_case, cu, exact_on_gpu, ints, lengths_behind, random_state, status

gpu = pytest.mark.gpu


def held(pool):
    """A bf16 pool [pages,Hkv,page,d] as the cache holds it: uint8 pool, and the values as bf16."""
    code, scale = orc.quantise(pool)
    return orc.pack(code, scale), orc.values(code, scale).to(torch.bfloat16)


def held_case(*args, **kw):
    """attention_case in 4 bits; what no sequence holds is NaN."""
    q, k, v, table, length = attention_case(*args, **kw)
    (k4, kv), (v4, vv) = held(k), held(v)
    return (q, k4, v4, table, length), (q, kv, vv, table, length)


# ------------------------------------------------------------------------------------------------ the format itself
@pytest.mark.parametrize("d", [64, 128])
def test_every_value_is_a_bf16_number_near_what_was_written(d):
    x = (torch.randn((3, 2, 32, d)).double() * torch.exp2(torch.randint(-90, 90, (3, 2, 32, 1)).double())).bfloat16()
    code, scale = orc.quantise(x)
    y = orc.values(code, scale)
    assert torch.equal(y, y.bfloat16().double()) and code.abs().max() == 7
    assert (scale == scale.bfloat16().double()).all()
    assert ((y - x.double()).abs() <= scale.repeat_interleave(32, -1) / 2).all()
    pool = orc.pack(code, scale)
    assert pool.shape == (3, 2, 32, av.q4_token_bytes(d))
    again = orc.unpack(pool, d)
    assert torch.equal(again[0], code) and torch.equal(again[1], scale)


def test_ties_and_borders_of_the_format():
    """Scales halfway between two of five bits go up, codes halfway to the even one; groups that are too small are zeros, too large ones NaN."""
    row = torch.zeros(6, 32)
    row[0, :3] = torch.tensor([231.0, 115.5, 33.0])      # 231 / 7 = 33, halfway between 32 and 34: 34
    row[1, :5] = torch.tensor([7.0, 0.5, 1.5, 2.5, -2.5])
    row[2, 0] = 2.0 ** -101
    row[3, :2] = torch.tensor([2.0 ** -100, 2.0 ** -110])
    row[4, :2] = torch.tensor([2.0 ** 125, 1.0])
    row[5, :2] = torch.tensor([float("nan"), 1.0])
    code, scale = orc.quantise(row)
    assert scale[0] == 34 and code[0, :3].tolist() == [7, 3, 1]
    assert scale[1] == 1 and code[1, :5].tolist() == [7, 0, 2, 2, -2]
    assert scale[2] == 0 and (code[2] == 0).all() and scale[3] > 0 and torch.isnan(scale[4:]).all()


# ------------------------------------------------------------------------------------------------ refusals
_T = av._Bf16Tensor4(1 << 20, 64 * 64 * 4, 64 * 64, 64)
_P = av._Q4Pool(1 << 20, 36 * 64 * 4, 36 * 64)


@pytest.mark.parametrize("change,want", [
    (dict(n=-1), 1), (dict(Hkv=0), 1), (dict(T=-1), 1), (dict(pages=0), 1), (dict(width=0), 1), (dict(d=96), 2), (dict(page=48), 2), (dict(n=65536, seq=1 << 20), 2),
    (dict(seqs=1 << 16, width=1 << 16), 2), (dict(T=(1 << 30) + 1), 2), (dict(n=9), 1), (dict(table=None), 1), (dict(length=(1 << 20) + 2), 1), (dict(seq=(1 << 20) + 1), 1),
    (dict(count=(1 << 20) + 3), 1), (dict(k=av._Bf16Tensor4(None, 16384, 4096, 64)), 1), (dict(v=av._Bf16Tensor4(1 << 20, 16384, 4096, 60)), 1),
    (dict(kp=av._Q4Pool(None, 9216, 2304)), 1), (dict(kp=av._Q4Pool((1 << 20) + 8, 9216, 2304)), 1), (dict(vp=av._Q4Pool(1 << 20, 9216, 2288)), 1),
    (dict(vp=av._Q4Pool(1 << 20, 9216 + 8, 2304)), 1), (dict(vp=av._Q4Pool(1 << 20, 9216, 2304 + 8)), 1), (dict(n=0), 0), (dict(T=0), 0)])
def test_refusals_of_write_and_read(change, want):
    a = {**dict(n=2, Hkv=4, T=64, d=64, page=64, pages=10, seqs=8, width=5, k=_T, v=_T, kp=_P, vp=_P, table=1 << 20, length=1 << 20, seq=None, count=None), **change}
    lib = av.load_library()
    head = [a[x] for x in ("n", "Hkv", "T", "d", "page", "pages", "seqs", "width")]
    lists = [a[x] for x in ("table", "length", "seq", "count")]
    assert lib.avsa_cache_write_q4(*head, a["k"], a["v"], a["kp"], a["vp"], *lists, 0) == want
    assert lib.avsa_cache_read_q4(*head, a["kp"], a["vp"], *lists, a["k"], a["v"], 0) == want


@pytest.mark.parametrize("change,want", [
    (dict(B=-1), 1), (dict(pages=0), 1), (dict(H=3, Hkv=2), 1), (dict(flags=2), 1), (dict(prefix=6), 1), (dict(d=32), 2), (dict(page=8), 2), (dict(H=129 * 4), 2),
    (dict(B=9), 1), (dict(scale=-1.0), 1), (dict(scale=math.inf), 1), (dict(kp=av._Q4Pool(1 << 20, 9216, 2288)), 1), (dict(vp=av._Q4Pool(8, 9216, 2304)), 1),
    (dict(table=None), 1), (dict(o=None), 1), (dict(o=8), 1), (dict(log=(1 << 20) + 2), 1), (dict(ws=None), 3), (dict(ws_bytes=255), 3), (dict(ws=(1 << 20) + 16), 1),
    (dict(B=0), 0), (dict(L=0), 0)])
def test_refusals_of_attention(change, want):
    a = {**dict(B=2, H=4, Hkv=4, L=1, d=64, page=64, pages=10, seqs=8, width=5, q=_T, kp=_P, vp=_P, table=1 << 20, prefix=0, flags=0, scale=0.0, o=1 << 20, log=None,
                ws=1 << 20, ws_bytes=1 << 40), **change}
    got = av.load_library().avsa_prefix_attn_q4(a["B"], a["H"], a["Hkv"], a["L"], a["d"], a["page"], a["pages"], a["seqs"], a["width"], a["q"], a["kp"], a["vp"], a["table"],
                                                1 << 20, None, None, a["prefix"], a["flags"], a["scale"], a["o"], None, a["log"], a["ws"], a["ws_bytes"], 0)
    assert got == want


def test_workspace_query():
    """Few rows need what the bf16 cache needs of them; many also room for one layer in bf16; sizes that are not supported need none."""
    ask = av.avsa_prefix_attn_q4_workspace_bytes
    few, more, many = (ask(4, 8, 8, L, 128, 64, 50000, 40, 0) for L in (1, 64, 1000))
    assert 256 < few < 1 << 22 and 256 < more < 1 << 28 and many > 2 * 50000 * 8 * 64 * 128 * 2
    assert ask(4, 8, 8, 64, 96, 64, 500, 40, 0) == 0 and ask(4, 8, 8, 64, 128, 64, 0, 40, 0) == 0 and ask(2, 1, 1, 1, 64, 128, 5, 1 << 25, 5) == 0
    assert ask(1, 1, 1, 1000, 64, 128, (1 << 31) - 1, 4, 0) > 2 * ((1 << 31) - 1) * 128 * 64 * 2


def test_wrappers_take_device_tensors_only():
    pool, ints_ = torch.zeros((3, 2, 16, 36), dtype=torch.uint8), torch.zeros((2, 1), dtype=torch.int32)
    with pytest.raises(ValueError):
        av.avsa_cache_read_q4(pool, pool, ints_, ints_[:, 0], 4)
    with pytest.raises(ValueError):
        av.q4_token_bytes(96)


# ------------------------------------------------------------------------------------------------ writing and reading
def random_pool(gen, *size):
    return torch.randint(0, 256, size, generator=gen, dtype=torch.uint8).cuda()


@gpu
@pytest.mark.parametrize("layout", ["tokens", "heads", "gaps"])
@pytest.mark.parametrize("n,Hkv,L,d,page,ragged", [(1, 1, 1, 64, 16, False), (5, 3, 1, 128, 32, False), (4, 24, 37, 128, 64, True), (9, 8, 200, 64, 16, True),
                                                   (3, 2, 130, 128, 128, False), (2, 70, 3, 64, 32, False), (2, 1, 300, 128, 16, True)])
def test_write_and_read_back(n, Hkv, L, d, page, ragged, layout):
    """Codes, scales and whatever lies beside them, byte for byte; then the tokens and some in front of them as bf16."""
    rng, gen = random.Random(n * L), torch.Generator().manual_seed(n * L + d)
    most = L + 3 * page
    table, length, ref = random_state(rng, n + 2, page, (n + 2) * (most // page + 2), most)
    seq = rng.sample(range(n + 2), n)
    count = [min(int(length[s]), rng.randint(0, L) if ragged else L) for s in seq]
    if n > 3:
        seq[2] = -1
    pools = [held(torch.randn((len(ref), Hkv, page, d), generator=gen).cuda())[0] for _ in range(2)]
    new = []
    for _ in range(2):
        x = torch.randn((n, L, Hkv, d), generator=gen) * torch.exp2(torch.randint(-20, 20, (n, L, Hkv, 1), generator=gen).float())
        x = x.bfloat16().cuda()
        if layout == "gaps":          # rows of 16-byte alignment only
            x = torch.nn.functional.pad(x.flatten(2), (8, 16))[:, :, 8:-16].unflatten(2, (Hkv, d))
        x = x.transpose(1, 2)
        new.append(x.contiguous() if layout == "heads" else x)
    code_scale = [orc.quantise(x) for x in new]
    want = []
    for pool, (code, scale) in zip(pools, code_scale):
        c, s = orc.unpack(pool, d)
        for b, k in enumerate(count):
            for j in range(k if seq[b] >= 0 else 0):
                pos = int(length[seq[b]]) - k + j
                c[table[seq[b], pos // page], :, pos % page], s[table[seq[b], pos // page], :, pos % page] = code[b, :, j], scale[b, :, j]
        want.append((c, s))
    av.avsa_cache_write_q4(*new, *pools, cu(table), cu(length), seq=ints(seq), count=ints(count))
    for p, w in zip(pools, want):
        assert torch.equal(p, orc.pack(*w))
    back = [min(int(length[s]), k + 5) if s >= 0 else 9 for s, k in zip(seq, count)]
    k, v = av.avsa_cache_read_q4(*pools, cu(table), cu(length), L + 5, seq=ints(seq), count=ints(back))
    for got, pool in zip((k, v), pools):
        values = orc.values(*orc.unpack(pool, d)).to(torch.bfloat16)
        full = torch.zeros_like(got)
        for b, m in enumerate(back):
            if seq[b] >= 0:
                at = np.arange(int(length[seq[b]]) - m, int(length[seq[b]]))
                full[b, :, :m] = values[table[seq[b], at // page].astype(np.int64), :, at % page].transpose(0, 1)
        assert torch.equal(got, full)


@gpu
@pytest.mark.parametrize("d", [64, 128])
def test_write_of_extreme_groups(d):
    """Ties, the largest and the smallest that are held, infinities and NaN, zeros of both signs: each group for itself."""
    special = [0.0, -0.0, 2.0 ** -101, 2.0 ** -100, 2.0 ** 124, 1.99 * 2.0 ** 124, 2.0 ** 125, 3e38, math.inf, -math.inf, math.nan]
    gen = torch.Generator().manual_seed(3)
    x = torch.randn((1, 1, 16 * 40, d), generator=gen)
    for i, s in enumerate(special):
        x[0, 0, i, 5] = s
        x[0, 0, 20 + i] = 0.0
        x[0, 0, 20 + i, d - 1] = s
    # every mantissa as the largest, with every multiple of half a scale: exact ties
    top = torch.arange(128, 256).float()
    for i, t in enumerate(top):
        s = float(orc.quantise(torch.cat((t[None], torch.zeros(31))).double())[1])
        x[0, 0, 40 + i, :32] = torch.tensor([float(t)] + [(0.5 + j % 7) * s * (-1) ** j for j in range(31)]).clamp(-float(t), float(t))
    x = x.bfloat16().cuda()
    pool = torch.zeros((5, 1, 128, av.q4_token_bytes(d)), dtype=torch.uint8, device="cuda")
    v = pool.clone()
    table, length = ints([[3, 1, 0, 4, 2]]), ints([640])
    av.avsa_cache_write_q4(x, x, pool, v, table, length)
    assert torch.equal(pool, v)
    k, _ = av.avsa_cache_read_q4(pool, v, table, length, 640)
    code, scale = orc.quantise(x)
    want = orc.values(code, scale).to(torch.bfloat16)
    assert torch.equal(torch.isnan(k), torch.isnan(want)) and torch.equal(torch.nan_to_num(k), torch.nan_to_num(want))


@gpu
def test_tokens_without_a_page():
    """Before the sequence's begin, behind the table, of a page out of range: nothing is written there, and zeros are read."""
    page, d = 16, 64
    pool = torch.zeros((4, 1, page, 36), dtype=torch.uint8, device="cuda")
    v = pool.clone()
    new = torch.ones((4, 1, 20, d), dtype=torch.bfloat16, device="cuda")
    table, length = ints([[0, -1], [1, 9], [2, 3], [-1, -1]]), ints([5, 20, 40, 3])
    av.avsa_cache_write_q4(new, new, pool, v, table, length)
    want = torch.zeros((4, 1, page, d), dtype=torch.float64)
    want[0, 0, :5] = 1
    want[1] = 1
    want[3, 0, 4:] = 1
    one = orc.quantise(torch.ones(32))
    assert float(one[0][0] * one[1]) == 7 * 0.140625 and torch.equal(orc.values(*orc.unpack(pool.cpu(), d)), want * 7 * 0.140625) and torch.equal(pool, v)
    out = [torch.full((5, 1, 20, d), 77.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    k, _ = av.avsa_cache_read_q4(pool, v, table, length, 20, seq=ints([0, 1, 2, -1, 7]), k=out[0], v=out[1])
    assert k is out[0] and torch.equal(out[0], out[1])
    full = torch.zeros((5, 20))
    full[0, 15:], full[1, :16], full[2, :12] = 7 * 0.140625, 7 * 0.140625, 7 * 0.140625
    # sequence 0: 5 tokens, the 20 asked for begin 15 in front of them; 1: its page for tokens 16..19 is out of range; 2: positions 20..39, of which 32.. have no entry
    assert torch.equal(k[:, 0, :, 0].float().cpu() != 0, full != 0)
    k, _ = av.avsa_cache_read_q4(pool, v, table, length, 20, seq=ints([1, 0]), count=ints([50, -3]))
    assert (k[1] == 0).all() and torch.equal(k[0], out[0][1])


@gpu
def test_outputs_and_pools_with_strides():
    """Keys and values of one tensor side by side, pools as slices of a larger one; what lies between is left alone."""
    page, d, Hkv = 32, 128, 3
    gen = torch.Generator().manual_seed(8)
    big = random_pool(gen, 6, 2, Hkv + 1, page, 72)
    kp, vp = big[:, 0, :Hkv], big[:, 1, 1:]
    before = big.clone()
    new = torch.randn((2, 40, 2, Hkv, d), generator=gen).bfloat16().cuda()
    table, length = ints([[5, 0, -1], [2, 3, 1]]), ints([50, 90])
    av.avsa_cache_write_q4(new[:, :, 0].transpose(1, 2), new[:, :, 1].transpose(1, 2), kp, vp, table, length)
    assert torch.equal(big[:, 0, Hkv:], before[:, 0, Hkv:]) and torch.equal(big[:, 1, :1], before[:, 1, :1]) and torch.equal(big[4], before[4])
    out = torch.full((2, 40, 2, Hkv, d + 8), 5.0, dtype=torch.bfloat16, device="cuda")
    av.avsa_cache_read_q4(kp, vp, table, length, 40, k=out[:, :, 0, :, :d].transpose(1, 2), v=out[:, :, 1, :, :d].transpose(1, 2))
    assert (out[..., d:] == 5).all()
    assert torch.equal(out[..., :d], orc.values(*orc.quantise(new)).to(torch.bfloat16))


@gpu
def test_fork_and_compact_of_pages_in_4_bits():
    page, d, Hkv = 16, 128, 2
    pool = random_pool(torch.Generator().manual_seed(1), 4, 9, Hkv, page, 72)
    table, length, ref = np.array([[8, 6, 7], [-1] * 3, [3, -1, -1]], np.int32), np.array([40, 0, 5], np.int32), np.zeros(9, np.int32)
    ref[[8, 6, 7, 3]] = 1
    *want, moves, _ = corc.fork(table, length, ref, [0], [1], page)
    state = [cu(t) for t in (table, length, ref)]
    content = pool.clone()
    av.avsa_cache_fork(pool, *state, ints([0]), ints([1]))
    for a, b in moves:
        content[:, b] = content[:, a]
    for g, w in zip(state, want):
        assert np.array_equal(g.cpu().numpy(), w)
    assert torch.equal(pool, content)
    t, r, live, moves = corc.compact(want[0], want[2])
    n_live, ws = av.avsa_cache_compact(pool, *state)
    for a, b in moves:
        content[:, b] = content[:, a]
    assert int(n_live) == live and status(ws) == av.AVSA_OK and np.array_equal(state[0].cpu().numpy(), t) and torch.equal(pool[:, :live], content[:, :live])


# ------------------------------------------------------------------------------------------------ attention
def check(case, values, what, prefix_pages=0, seq=None, causal=False, scale=0.0, **kw):
    q, k4, v4, table, length = case
    o, lse, ws = av.avsa_prefix_attn_q4(q, k4, v4, cu(table), cu(length), prefix_pages=prefix_pages, seq=None if seq is None else ints(seq), causal=causal,
                                        softmax_scale=scale, want_lse=True, **kw)
    assert status(ws) == av.AVSA_OK
    want, want_lse = exact_on_gpu(*(values if not scale else ((values[0].double() * (scale * math.sqrt(q.shape[3]))), *values[1:])), seq, causal)
    empty = torch.isinf(want_lse)
    assert torch.equal(torch.isinf(lse), empty) and (o[empty] == 0).all(), what
    if not empty.all():
        close_o(o.double()[~empty].cpu().numpy(), want[~empty].cpu().numpy(), what)
        close_lse(lse.double()[~empty].cpu().numpy(), want_lse[~empty].cpu().numpy(), what)
    return o, lse, ws


@gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("n", [0, 1, 2, 15, 16, 17, 63, 65, 128, 129, 400])
def test_attention_lengths(n, page, d):
    """One token and forty against n of them, beside a longer sequence; what lies behind the last token is NaN."""
    for L in (1, 40):
        check(*held_case(2, 3, 3, L, d, page, [n, 300], seed=n), what=f"{n}, {L}")


@gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("H,Hkv", [(1, 1), (6, 2), (8, 1), (14, 2), (128, 1), (16, 16)])
@pytest.mark.parametrize("L", [1, 2, 7, 33])
@pytest.mark.parametrize("causal", [False, True])
def test_attention_heads_and_queries(H, Hkv, L, d, causal):
    check(*held_case(3, H, Hkv, L, d, 32, [200, 64, 131], seed=H + L, q_layout="blhd"), what="heads", causal=causal)


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
    (12, 10, 24, 8, 32, 4096, 200),       # 30 rows a sequence, gathered (three query heads to a key head)
    (12, 20, 8, 2, 32, 16384, 400),       # 80 rows: the tile kernel for both, pages made bf16 before it
    (4, 40, 8, 4, 64, 16384, 300),        # 80 rows, 320 stacked: tiles made in the kernel
    (4, 40, 8, 4, 16, 16384, 300),
    (5, 24, 16, 8, 128, 16384, 200),
    (24, 1, 32, 32, 64, 20480, 100)])      # 24 rows, so many keys that the tile kernel takes them
def test_attention_stacked(B, L, H, Hkv, page, tokens, most, d, causal):
    """The beginning is read for the rows of all sequences at once; the same call without saying that it is shared gives the same."""
    rng = random.Random(B + d)
    shared = tokens // page
    case = held_case(B, H, Hkv, L, d, page, lengths_behind(rng, B, shared, page, most), shared=shared, seed=B, q_layout="blhd")
    a = check(*case, "stacked", prefix_pages=shared, causal=causal)
    b = check(*case, "each by itself", causal=causal)
    assert torch.allclose(a[0].float(), b[0].float(), atol=2e-2, rtol=2e-2)


@gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B,L,H,Hkv,width,lengths", [
    (1, 1, 8, 8, 400, (6000,)),           # few items, long rows: parts that another kernel joins
    (1, 31, 4, 4, 300, (4700,)),
    (1, 1, 24, 24, 1100, (17000,)),       # parts of 24 items
    (1, 4, 32, 8, 700, (11001,)),
    (3, 1, 24, 24, 60, (900, 0, 17)),     # a cluster of CTAs an item
    (20, 2, 16, 16, 80, tuple(range(5, 1285, 64))),
    (70, 1, 32, 8, 300, tuple(range(1, 4700, 67))[:70]),
    (1, 700, 8, 8, 200, (3000,)),         # six row tiles: tiles made in the kernel
    (3, 200, 24, 8, 100, (1000, 0, 640)),
    (9, 20, 8, 8, 470, (7500,) + (300,) * 8),      # 20 rows of a table with room for so many keys
    (2, 900, 4, 4, 200, (3000, 1111)),    # more: pages made bf16 before it
    (3, 333, 24, 8, 80, (1000, 1, 640))])
def test_attention_ways_of_cutting(B, L, H, Hkv, width, lengths, d):
    case = held_case(B, H, Hkv, L, d, 16, list(lengths), seed=B, width=width)
    for causal in (False, True):
        check(*case, "cut", causal=causal)


@gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B,L,H,Hkv,page,shared,lengths", [
    (1, 17, 3, 3, 16, 0, (11000,)),                      # parts of three items
    (2, 6, 12, 3, 16, 0, (1200, 0)),                     # 24 rows of a cluster's CTAs
    (3, 7, 24, 8, 32, 0, (6, 23, 2049)),
    (60, 3, 48, 8, 64, 0, tuple(range(1, 1500, 25))),
    (20, 1, 4, 4, 64, 40, tuple(range(2560, 2580))),     # stacked to 20 rows, or to 24, 22 and 17 in front of own ones of 8, 11 and 17
    (3, 8, 8, 8, 64, 160, (10240, 10300, 10999)),
    (2, 11, 2, 2, 128, 600, (76800, 76900)),
    (1, 17, 8, 8, 64, 160, (10700,)),
    (1, 26, 3, 3, 16, 0, (11000,)),
    (2, 8, 12, 3, 16, 0, (1200, 0)),
    (60, 1, 108, 4, 64, 0, tuple(range(1, 1500, 25))),
    (4, 8, 8, 8, 64, 160, (10240, 10300, 10999, 10247)),
    (28, 1, 4, 4, 64, 40, tuple(range(2560, 2588))),
    (9, 20, 8, 8, 128, 0, (10200,) + (300,) * 8)])       # 20 rows of a table with room for many keys
def test_attention_of_17_to_32_rows(B, L, H, Hkv, page, shared, lengths, d):
    case = held_case(B, H, Hkv, L, d, page, list(lengths), shared=shared, seed=B + d)
    for causal in (False, True):
        first = check(*case, "rows", prefix_pages=shared, causal=causal)
        again = check(*case, "rows", prefix_pages=shared, causal=causal)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


@gpu
@pytest.mark.parametrize("L", [1, 40])
def test_attention_of_chosen_sequences_counts_and_scales(L):
    case, values = held_case(5, 4, 2, L, 64, 16, [140, 177, 0, 230, 116, 99, 164], seed=5)
    for causal in (False, True):
        check(case, values, "chosen", seq=[6, -1, 3, 2, 0], causal=causal, scale=0.3)
    if L > 1:
        count = [3, L, 0, 1, 7]
        q, k4, v4, table, length = case
        o, lse, ws = av.avsa_prefix_attn_q4(q, k4, v4, cu(table), cu(length), seq=ints([6, 0, 3, 2, 1]), causal=True, want_lse=True, count=ints(count))
        f64 = lambda t: t.double().cpu().numpy()
        want, want_lse = corc.prefix_attention(f64(q), *(np.nan_to_num(f64(x)) for x in values[1:3]), table, length, [6, 0, 3, 2, 1], True, None, count)
        empty = np.isneginf(want_lse)
        assert status(ws) == av.AVSA_OK and np.array_equal(np.isneginf(f64(lse)), empty) and (f64(o)[empty] == 0).all()
        close_o(f64(o)[~empty], want[~empty], "counts")


@gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B,L,H,Hkv,tokens", [(2, 1, 4, 4, 0), (16, 1, 24, 24, 2048), (40, 1, 32, 8, 2048), (1, 300, 4, 4, 0)])
def test_attention_rows_that_outgrow_their_reference(B, L, H, Hkv, tokens, d):
    """Logits that rise along the keys, by 300 as powers of e: every reference is outgrown."""
    page, shared = 64, tokens // 64
    q, k, v, table, length = attention_case(B, H, Hkv, L, d, page, [tokens + 700 + b for b in range(B)], shared=shared, seed=4, poison=False)
    one = torch.zeros(d, device="cuda")
    one[0] = 1.0
    q = (q.float() * (1 - one) + one * 4.0).bfloat16()
    k = k.clone()
    for s in range(B):
        at = torch.arange(int(length[s]), device="cuda")
        k[cu(table)[s].long()[at // page], :, at % page, 0] = (300.0 * math.sqrt(d) / 4.0 * at / (tokens + 800)).bfloat16()[:, None].expand(-1, Hkv)
    (k4, kv), (v4, vv) = held(k), held(v)
    check((q, k4, v4, table, length), (q, kv, vv, table, length), "growing", prefix_pages=shared)


@gpu
@pytest.mark.parametrize("B,L,H,Hkv,shared", [(3, 2, 8, 4, 0), (20, 2, 8, 4, 20), (40, 1, 32, 8, 32), (2, 150, 4, 4, 0), (2, 900, 4, 4, 0)])
def test_attention_is_that_over_what_is_read_back(B, L, H, Hkv, shared):
    """The same keys and values in a bf16 cache: the same up to the order of sums; bit for bit where the tile kernel does all the work."""
    (q, k4, v4, table, length), (_, k, v, _, _) = held_case(B, H, Hkv, L, 128, 64, [64 * shared + 500 + 13 * i for i in range(B)], shared=shared, seed=9)
    o4, lse4, _ = av.avsa_prefix_attn_q4(q, k4, v4, cu(table), cu(length), prefix_pages=shared, causal=True, want_lse=True)
    o, lse, _ = av.avsa_prefix_attn(q, k, v, cu(table), cu(length), prefix_pages=shared, causal=True, want_lse=True)
    empty = torch.isinf(lse)          # (queries in front of the sequence's first token)
    assert torch.equal(torch.isinf(lse4), empty) and (o4[empty] == 0).all()
    close_o(o4[~empty].double().cpu().numpy(), o[~empty].double().cpu().numpy(), "read back")
    close_lse(lse4[~empty].double().cpu().numpy(), lse[~empty].double().cpu().numpy(), "read back")


@gpu
@pytest.mark.parametrize("B,L,H,Hkv,shared", [(20, 2, 8, 4, 20), (40, 1, 32, 8, 32), (2, 150, 4, 4, 0), (2, 900, 4, 4, 0), (1, 1, 4, 4, 0)])
def test_attention_reproduces_and_ignores_old_memory(B, L, H, Hkv, shared):
    """Bit for bit: run after run, whatever workspace and outputs held, on another stream, and as a replayed graph."""
    q, k, v, table, length = held_case(B, H, Hkv, L, 128, 64, [64 * shared + 1500 + 13 * i for i in range(B)], shared=shared, seed=9)[0]
    t, n = cu(table), cu(length)
    first = av.avsa_prefix_attn_q4(q, k, v, t, n, prefix_pages=shared, want_lse=True)
    for fill in (0, 255):
        ws = torch.full_like(first[2], fill)
        o, lse = torch.full_like(first[0], float("nan")), torch.full_like(first[1], float("nan"))
        av.avsa_prefix_attn_q4(q, k, v, t, n, prefix_pages=shared, want_lse=True, o=o, lse=lse, ws=ws)
        assert torch.equal(o, first[0]) and torch.equal(lse, first[1])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        o3 = av.avsa_prefix_attn_q4(q, k, v, t, n, prefix_pages=shared)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(o3[0], first[0])
    graph = torch.cuda.CUDAGraph()
    o, lse, ws = torch.empty_like(first[0]), torch.empty_like(first[1]), torch.empty_like(first[2])
    with torch.cuda.graph(graph):
        av.avsa_prefix_attn_q4(q, k, v, t, n, prefix_pages=shared, want_lse=True, o=o, lse=lse, ws=ws)
    for _ in range(3):
        o.zero_()
        graph.replay()
        assert torch.equal(o, first[0]) and torch.equal(lse, first[1])


@gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B,L,H,Hkv,page,shared,most", [(4, 64, 64, 8, 128, 3, 1400), (8, 33, 48, 3, 64, 6, 1500), (2, 200, 8, 8, 16, 0, 3000)])
def test_attention_of_codes_that_land_in_any_order(B, L, H, Hkv, page, shared, most, d):
    """The tile kernel with nothing in L2: values may be there before the keys in front of them, and the other way round."""
    draw = random.Random(d + B)
    flush = torch.empty(1 << 28, dtype=torch.uint8, device="cuda")
    for seed in range(8):
        case = held_case(B, H, Hkv, L, d, page, [shared * page + draw.randint(0, most) for _ in range(B)], shared=shared, seed=seed)
        flush.zero_()
        first = check(*case, "cold")
        for _ in range(2):
            flush.zero_()
            again = check(*case, "cold again")
            assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


@gpu
@pytest.mark.parametrize("L", [1, 33, 400])
def test_outputs_of_a_call_lie_apart(L):
    """The outputs and the workspace of one call overlap nowhere, begin on 512 bytes, and keep no more memory than they need; q's strides go over to o."""
    case = held_case(2, 6, 3, L, 64, 16, [100 + L, 9 + L], seed=21)[0]
    q, k, v, table, length = case
    wide = torch.zeros((2, L, 8, 64), dtype=torch.bfloat16, device="cuda").transpose(1, 2)
    wide[:, :6] = q
    for query in (q, wide[:, :6]):
        o, lse, ws = av.avsa_prefix_attn_q4(query, k, v, cu(table), cu(length), want_lse=True)
        assert o.stride() == query.stride()
        spans = []
        for t in (o, lse, ws):
            last = sum((n - 1) * s for n, s in zip(t.shape, t.stride()))
            spans.append((t.data_ptr(), t.data_ptr() + (last + 1) * t.element_size()))
            assert t.data_ptr() % 512 == 0 and t._version == 0
        spans.sort()
        assert all(a[1] <= b[0] for a, b in zip(spans, spans[1:]))
        held = {t.untyped_storage().data_ptr(): t.untyped_storage().nbytes() for t in (o, lse, ws)}
        assert sum(held.values()) <= sum(-(-(b - a) // 512) * 512 for a, b in spans)
        kept = o.clone(), lse.clone()
        ws.fill_(255)
        assert torch.equal(o, kept[0])
        lse.fill_(7.0)
        assert torch.equal(o, kept[0])
        o.fill_(3.0)
        assert (lse == 7).all()


@gpu
@pytest.mark.parametrize("L", [1, 40, 900])
def test_attention_reports_malformed_tables(L):
    """Pages out of range contribute nothing (zeros), lengths beyond the row are cut: reported, and the other sequences are right."""
    (q, k4, v4, table, length), values = held_case(3, 2, 2, L, 64, 16, [100, 100, 100], seed=1)
    want, _ = exact_on_gpu(*values)
    zero = [x.clone() for x in values[1:3]]
    for x in zero:
        x[table[1, 2]] = 0.0
    without, _ = exact_on_gpu(values[0], *zero, table, length)
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
        log = ints([0, 0, 0, 0])
        o, _, ws = av.avsa_prefix_attn_q4(q, k4, v4, cu(t), cu(n), seq=ints(seq), log=log)
        assert status(ws) == av.AVSA_ERR_BAD_TABLE and int(log[0]) == av.AVSA_ERR_BAD_TABLE, change
        close_o(o.double()[[0, 2]].cpu().numpy(), want[[0, 2]].cpu().numpy(), change)
        if change in ("page", "negative"):
            close_o(o.double()[1].cpu().numpy(), without[1].cpu().numpy(), change)


@gpu
@pytest.mark.parametrize("where", ["k", "v"])
@pytest.mark.parametrize("L", [1, 40, 900])
def test_attention_values_that_are_not_finite(L, where):
    """A group that reads as NaN reaches the rows that see its token, and no others."""
    q, k, v, table, length = attention_case(2, 2, 2, L, 64, 16, [100, 90], seed=1, poison=False)
    page = int(table[0, 6])
    (k if where == "k" else v)[page, 1, 3, 40] = float("inf")          # token 99, of which causal rows but the last see nothing
    (k4, kv), (v4, vv) = held(k), held(v)
    o, _, _ = av.avsa_prefix_attn_q4(q, k4, v4, cu(table), cu(length))
    bad = torch.isnan(o)
    assert not bad[1].any() and not bad[0, 0].any() and bad[0, 1].any(-1).all()
    if where == "v":
        assert torch.equal(bad[0, 1, 0], torch.arange(64, device="cuda") >= 32)


@gpu
def test_offsets_beyond_32_bits():
    """Pages whose distance from the pool's beginning passes 2^32 bytes, and a table row far into the pool: written, read and attended to."""
    page, d, pages = 64, 128, 6
    step = (1 << 30) + 64
    if torch.cuda.mem_get_info()[0] < 2 * (5 * step + page * 72) + (2 << 30):
        pytest.skip("too little free memory")
    pools = [torch.empty(5 * step + page * 72, dtype=torch.uint8, device="cuda").as_strided((pages, 1, page, 72), (step, page * 72, 72, 1)) for _ in range(2)]
    for p in pools:
        p.zero_()
    table, length = np.array([[5, 0, 4], [3, 2, 1]], np.int32), np.array([170, 192], np.int32)
    new = [torch.randn((2, 1, 170, d), device="cuda").bfloat16() for _ in range(2)]
    av.avsa_cache_write_q4(*new, *pools, cu(table), cu(length))
    values = [orc.values(*orc.quantise(x)).to(torch.bfloat16) for x in new]
    for got, want in zip(av.avsa_cache_read_q4(*pools, cu(table), cu(length), 170), values):
        assert torch.equal(got, want)
    for L in (1, 40, 900):
        q = torch.randn((2, 2, L, d), device="cuda").bfloat16()
        o, _, ws = av.avsa_prefix_attn_q4(q[:1], *pools, cu(table), cu(length))
        x = q[:1].double() @ values[0][:1].double().transpose(2, 3) / math.sqrt(d)
        close_o(o.double().cpu().numpy(), (torch.softmax(x, 3) @ values[1][:1].double()).cpu().numpy(), "far pages")


@gpu
def test_attention_workspaces_depend_on_the_shape_alone():
    """What the query says is enough for every call of the shape, whatever the lengths."""
    for B, L, H, Hkv, page, width, prefix in ((1, 1, 8, 8, 16, 400, 0), (16, 1, 24, 24, 64, 60, 32), (40, 1, 32, 8, 128, 40, 16), (3, 200, 32, 8, 64, 50, 0), (1, 100, 4, 4, 64, 30, 0)):
        need = av.avsa_prefix_attn_q4_workspace_bytes(B, H, Hkv, L, 64, page, width, width, prefix)
        assert need > 256
        q = torch.randn((B, H, L, 64), device="cuda").bfloat16()
        pool = held(torch.randn((width, Hkv, page, 64), device="cuda").bfloat16())[0]
        table = torch.arange(width, dtype=torch.int32, device="cuda").repeat(B, 1)
        guard = torch.full((need + 4096,), 77, dtype=torch.uint8, device="cuda")
        for n in (width * page, prefix * page, 1, 0):
            av.avsa_prefix_attn_q4(q, pool, pool, table, ints([n] * B), prefix_pages=prefix, ws=guard[:need])
            assert (guard[need:] == 77).all()
        with pytest.raises(av.AvsaError):
            av.avsa_prefix_attn_q4(q, pool, pool, table, ints([1] * B), prefix_pages=prefix, ws=guard[:need - 32])


@gpu
def test_wrapper_refusals():
    q, pool = torch.zeros((1, 2, 1, 64), device="cuda").bfloat16(), torch.zeros((3, 2, 16, 36), dtype=torch.uint8, device="cuda")
    table, length = ints([[0, 1, 2]]), ints([40])
    new = torch.zeros((1, 2, 5, 64), device="cuda").bfloat16()
    for bad in (pool.char(), pool[:, :, :, :35], torch.zeros((3, 2, 16, 72), dtype=torch.uint8, device="cuda"), pool.transpose(1, 2), pool[0]):
        with pytest.raises(ValueError):
            av.avsa_prefix_attn_q4(q, bad, bad, table, length)
        with pytest.raises(ValueError):
            av.avsa_cache_write_q4(new, new, bad, bad, table, length)
    for call in (lambda: av.avsa_prefix_attn_q4(q, pool, pool[:2], table, length), lambda: av.avsa_cache_write_q4(new, new[:, :1], pool, pool, table, length),
                 lambda: av.avsa_cache_read_q4(pool, pool, table, length, -1), lambda: av.avsa_cache_read_q4(pool, pool, table, length, 5, count=ints([1, 2])),
                 lambda: av.avsa_cache_read_q4(pool, pool, table, length, 5, k=new[:, :1]), lambda: av.avsa_prefix_attn_q4(q, pool, pool, table, length[:0]),
                 lambda: av.avsa_cache_read_q4(pool, pool, table.long(), length, 5)):
        with pytest.raises(ValueError):
            call()


# ------------------------------------------------------------------------------------------------ a run of them together
@gpu
@pytest.mark.parametrize("L,H,Hkv,d", [(1, 8, 2, 64), (40, 4, 4, 128)])
def test_clip_cache_in_4_bits(L, H, Hkv, d):
    """Branches, steps of turned queries and keys, pages given back, a compaction: against 64 bits on what the cache stands for."""
    page, seqs, shared = 16, 3, 4
    cache = ClipCache(2, Hkv, d, page, 60, seqs, 20, bits=4)
    assert cache.pool.dtype == torch.uint8
    gen = torch.Generator().manual_seed(5)
    sections, freq = (d // 4, d // 4), av.avsa_rope_frequencies((d // 4, d // 4))
    kept = {}

    def step(ids, n, prefix):
        cache.begin_step(ids, [n] * len(ids))
        for layer in range(2):
            q, k, v = (torch.randn((len(ids), h, n, d), generator=gen).bfloat16().cuda() for h in (H, Hkv, Hkv))
            first = [kept[s][layer][0].shape[1] if s in kept and len(kept[s]) > layer else 0 for s in ids]
            pos = torch.stack([torch.stack((torch.arange(n) + f, (torch.arange(n) + f) % 7), 1) for f in first]).int().cuda()
            q, k = av.avsa_rope(q, k, pos, freq, sections)
            o = cache.attend(layer, q, k, v, prefix, causal=True)
            for b, s in enumerate(ids):
                new = [orc.values(*orc.quantise(x[b])) for x in (k, v)]
                mine = kept.setdefault(s, [])
                if len(mine) <= layer:
                    mine.append(new)
                else:
                    mine[layer] = [torch.cat(p, 1) for p in zip(mine[layer], new)]
                kk, vv = (x.repeat_interleave(H // Hkv, 0) for x in mine[layer])
                x = q[b].double() @ kk.transpose(1, 2) / math.sqrt(d)
                N = kk.shape[1]
                x = x.masked_fill((torch.arange(N)[None] > torch.arange(N - n, N)[:, None]).cuda(), -math.inf)
                close_o(o[b].double().cpu().numpy(), (torch.softmax(x, -1) @ vv).cpu().numpy(), f"sequence {s}, layer {layer}")

    step([0], shared * page + 3, 0)
    cache.branch([0, 0], [1, 2])
    kept[1], kept[2] = [list(x) for x in kept[0]], [list(x) for x in kept[0]]
    step([2, 0, 1], L, shared)
    cache.drop([0])
    cache.compact()
    step([1, 2], L, shared)
    cache.check()
    k, v = av.avsa_cache_read_q4(cache.pool[2], cache.pool[3], cache.table, cache.length, kept[1][1][0].shape[1], seq=ints([1]))
    assert torch.equal(k[0].double(), kept[1][1][0]) and torch.equal(v[0].double(), kept[1][1][1])


@gpu
@pytest.mark.parametrize("L", [1, 40])
def test_step_in_4_bits_as_a_graph(L):
    """Lengths and pages are read on the device only: a step captured once goes on where the last replay ended."""
    page, H, d = 16, 4, 64

    def begin():
        cache = ClipCache(2, H, d, page, 120, 3, 40, bits=4)
        gen = torch.Generator().manual_seed(5)
        draw = lambda n, m: torch.randn((n, H, m, d), generator=gen).bfloat16().cuda()
        cache.begin_step([0], [70])
        for layer in range(2):
            cache.attend(layer, *(draw(1, 70) for _ in range(3)), causal=True)
        cache.branch([0, 0], [1, 2])
        return cache, [[draw(3, L) for _ in range(3)] for _ in range(2)]

    seq, count = ints([2, 0, 1]), ints([L, L - 1, L])

    def step(cache, inputs):
        cache.begin_step(seq, count)
        return [cache.attend(i, *x, 4, causal=True) for i, x in enumerate(inputs)]

    plain, inputs = begin()
    want = [[o.clone() for o in step(plain, inputs)] for _ in range(5)]
    plain.check()
    cache, inputs = begin()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(cache, inputs)
    for n in range(5):
        graph.replay()
        for a, b in zip(got, want[n]):
            assert torch.equal(a, b), n
    cache.check()


def test_clip_cache_refuses_other_widths():
    with pytest.raises(ValueError):
        ClipCache(1, 1, 64, 16, 2, 2, 8, "cpu", calls=av, bits=8)
    with pytest.raises(ValueError):
        ClipCache(1, 1, 96, 16, 2, 2, 8, "cpu", calls=av, bits=4)


@gpu
def test_command_in_4_bits():
    said = []
    cache, live = continue_clip(layers=2, heads=4, heads_kv=2, d=64, width=128, beginning=200, chunk=24, audio=3, candidates=3, rounds=2, page=16, bits=4, rotary=True,
                                report=said.append)
    assert live == -(-(200 + 2 * 27) // 16) and len(said) == 3 and cache.pool.dtype == torch.uint8
