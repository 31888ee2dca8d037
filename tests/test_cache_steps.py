"""Steps over the paged cache in which something is refused: the calls after one another, and ``ClipCache``, on the CPU by the plain statement and on the GPU."""
import random

import numpy as np
import pytest
import torch

from oracle import cache_oracle as orc
from paper_2608_15522_b200 import binding as av
from paper_2608_15522_b200.continuation import ClipCache
from parity_bars import close_lse, close_o
from test_continuation import OracleCalls
from test_paged_cache import SIZES, attention_case, cu, ints, lengths_behind, nump, random_state, status

gpu = pytest.mark.gpu


class StepCalls(OracleCalls):
    """``OracleCalls`` with what the calls say on the device."""

    def avsa_cache_extend(self, table, length, ref, seq, count, page, out=None, ws=None, granted=None):
        refused = orc.extend(table.numpy(), length.numpy(), ref.numpy(), seq.tolist(), count.tolist(), page)[3]
        granted.copy_(torch.tensor(granted_of(seq.tolist(), count.tolist(), refused)))
        return super().avsa_cache_extend(table, length, ref, seq, count, page)

    def avsa_prefix_attn(self, q, k, v, table, length, prefix_pages=0, seq=None, causal=False, softmax_scale=0.0, count=None):
        f64 = lambda t: t.double().numpy()
        o, lse = orc.prefix_attention(f64(q), f64(k), f64(v), table.numpy(), length.numpy(), seq.tolist(), causal, softmax_scale or None, count.tolist())
        return torch.from_numpy(o).bfloat16(), None, av.AVSA_OK


def granted_of(seq, count, refused):
    return [0 if s < 0 or k in refused else c for k, (s, c) in enumerate(zip(seq, count))]


WHERE = [pytest.param("cpu", id="plain"), pytest.param("cuda", id="gpu", marks=gpu)]


def clip_cache(where, *sizes):
    return ClipCache(*sizes, device=where, calls=StepCalls() if where == "cpu" else None)


def plain_rows(q, k, v, lim):
    """softmax(q k / sqrt(d)) v in 64 bits: q [H,L,d], k and v [Hkv,n,d], row i sees lim[i] tokens; empty rows are zero."""
    group = q.shape[0] // k.shape[0]
    k, v = (x.double().repeat_interleave(group, 0) for x in (k, v))
    x = (q.double() @ k.transpose(1, 2) * q.shape[2] ** -0.5).masked_fill(torch.arange(k.shape[1]) >= torch.as_tensor(lim)[:, None], -float("inf"))
    return torch.nan_to_num(torch.softmax(x, -1)) @ v


# ------------------------------------------------------------------------------------------------ what was granted
@pytest.mark.parametrize("where", WHERE)
@pytest.mark.parametrize("seq,count", [([0, 1], [16, 40]), ([1, 0], [40, 16]), ([1, 1], [3, 9]), ([0, 1], [0, 200]), ([1, 0], [64, 1])])
def test_a_refused_step_leaves_the_tokens_that_are_there(where, seq, count):
    """A parent and a branch share 32 tokens in two pages of four.  What cannot be had (pages, room in the row, a sequence twice) changes no token of
    anybody, and the others attend to what they have."""
    page, d, L = 16, 64, max(count)
    cache = clip_cache(where, 1, 1, d, page, 4, 2, 8)
    gen = torch.Generator().manual_seed(0)
    draw = lambda n, L: torch.randn((n, 1, L, d), generator=gen).bfloat16()
    cache.begin_step([0], [32])
    old = draw(1, 32), draw(1, 32)
    cache.attend(0, *(x.to(where) for x in (old[0], *old)))
    cache.branch([0], [1])
    before, table, length, ref = (nump(t).copy() for t in (cache.pool.float(), cache.table, cache.length, cache.ref))
    *_, refused = orc.extend(table, length, ref, seq, count, page)
    granted = granted_of(seq, count, refused)
    assert 0 in granted
    cache.begin_step(seq, count)
    q, k, v = draw(len(seq), L), draw(len(seq), L), draw(len(seq), L)
    o = cache.attend(0, *(x.to(where) for x in (q, k, v))).cpu()
    for p in nump(cache.table)[:, :2].ravel():
        assert np.array_equal(nump(cache.pool.float())[:, p], before[:, p])
    for b, (s, c, g) in enumerate(zip(seq, count, granted)):
        if c and g == c:
            kk, vv = (torch.cat([x[0], y[b, :, :c]], 1) for x, y in zip(old, (k, v)))
            close_o(o[b].double().numpy(), plain_rows(q[b], kk, vv, [32 + c] * L).numpy(), f"sequence {s}")
    for s in range(2):
        assert int(cache.length[s]) == 32 + sum(g for t, g in zip(seq, granted) if t == s)
    with pytest.raises(av.AvsaError, match="extend"):
        cache.check()


@gpu
@pytest.mark.parametrize("out", [False, True])
@pytest.mark.parametrize("seqs,page,pages,most", SIZES)
def test_extend_says_what_it_granted(seqs, page, pages, most, out):
    rng = random.Random(seqs)
    table, length, ref = random_state(rng, seqs, page, pages, most)
    for more in (1, 3 * pages):
        seq = [rng.randint(-1, seqs) for _ in range(seqs + 3)]
        count = [rng.choice((0, 1, page, rng.randint(0, 1 + more * page // seqs))) for _ in seq]
        *want, refused = orc.extend(table, length, ref, seq, count, page)
        state = [cu(x) for x in (table, length, ref)]
        target = tuple(torch.full_like(x, 77) for x in state) if out else None
        granted = torch.full((len(seq) + 2,), 77, dtype=torch.int32, device="cuda")
        got = av.avsa_cache_extend(*state, ints(seq), ints(count), page, out=target, granted=granted[:-2])
        assert granted.tolist() == granted_of(seq, count, refused) + [77, 77]
        for g, w in zip(got, want):
            assert np.array_equal(nump(g), w)
        assert (status(got[3]) == av.AVSA_OK) == (not refused)


def test_what_is_granted_overlaps_nothing():
    lib = av.load_library()
    state = dict(table=1 << 20, length=2 << 20, ref=3 << 20, table_out=4 << 20, length_out=5 << 20, ref_out=6 << 20, seqs=4, width=8, pages=100, page=16)
    call = lambda granted: lib.avsa_cache_extend_step(av._Cache(**state), 8192, 16384, 2, granted, None, 1 << 16, 1 << 30, 0)
    for name in ("table", "length", "ref", "table_out", "length_out", "ref_out"):
        assert call(state[name]) == av.AVSA_ERR_INVALID_ARG, name
    for granted in (8196, 16380, 32770):
        assert call(granted) == av.AVSA_ERR_INVALID_ARG, granted


@gpu
def test_wrapper_refuses_another_number_of_granted_entries():
    i = ints([0] * 4)
    with pytest.raises(ValueError, match="granted"):
        av.avsa_cache_extend(ints([[0, 0]] * 4), i, ints([0] * 5), ints([0, 1]), ints([1, 1]), 16, granted=ints([0]))
    with pytest.raises(ValueError, match="granted"):
        av.avsa_cache_extend(ints([[0, 0]] * 4), i, ints([0] * 5), ints([0, 1]), ints([1, 1]), 16, granted=torch.zeros(2, device="cuda"))


# ------------------------------------------------------------------------------------------------ different numbers of tokens
def test_oracle_counts_closed_forms():
    """Two sequences, three queries each, of which the second one has two."""
    assert orc.limits(np.array([3, 2, 9]), [0, 1, 2], 3, 3, True, [3, 2, 0]).tolist() == [[1, 2, 3], [1, 2, 0], [0, 0, 0]]
    assert orc.limits(np.array([5, 2]), [0, 1], 2, 3, True, [2, 3]).tolist() == [[4, 5, 0], [0, 1, 2]]
    assert orc.limits(np.array([5, 2]), [0, 1], 2, 3, False, [2, 3]).tolist() == [[5] * 3, [2] * 3]


@pytest.mark.parametrize("where", WHERE)
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("H,Hkv,L,shared", [(1, 1, 3, 0), (4, 2, 5, 2), (2, 2, 40, 2), (6, 2, 23, 0)])
def test_a_ragged_step(where, H, Hkv, L, shared, causal):
    """Sequences of a step get none, one, some and all of its tokens: what each of them adds sees the tokens up to itself."""
    page, d, n = 16, 64, 5
    cache = clip_cache(where, 1, Hkv, d, page, 80, n, 12)
    gen = torch.Generator().manual_seed(L)
    draw = lambda h, n, L: torch.randn((n, h, L, d), generator=gen).bfloat16()
    kept = [torch.zeros((2, Hkv, 0, d), dtype=torch.bfloat16)] * n

    def step(seq, count, L, shared):
        q, k, v = draw(H, len(seq), L), draw(Hkv, len(seq), L), draw(Hkv, len(seq), L)
        cache.begin_step(seq, count)
        o = cache.attend(0, *(x.to(where) for x in (q, k, v)), shared, causal).cpu()
        for b, (s, c) in enumerate(zip(seq, count)):
            kept[s] = torch.cat([kept[s], torch.stack([k[b, :, :c], v[b, :, :c]])], 2)
            all_ = kept[s].shape[2]
            lim = [all_ - c + i + 1 if i < c else 0 for i in range(L)] if causal else [all_] * L
            want = plain_rows(q[b], *kept[s], lim)
            empty = torch.tensor(lim) == 0
            assert (o[b][:, empty] == 0).all()
            if not empty.all():
                close_o(o[b][:, ~empty].double().numpy(), want[:, ~empty].numpy(), f"sequence {s}")

    if shared:
        step([0], [shared * page], shared * page, 0)
        cache.branch([0] * (n - 1), list(range(1, n)))
        kept[1:] = [kept[0]] * (n - 1)
    step([2, 0, 4, 1, 3], [L, L - 1, 0, 1, (L + 1) // 2], L, shared)
    step([4, 1, 0], [L // 2, L, 1], L, shared)
    step([3, 2, 1, 0, 4], [1] * 5, 1, shared)
    cache.check()


def exact_counts(q, k, v, table, length, count, causal):
    """orc.prefix_attention in 64 bits on the GPU."""
    B, H, L, d = q.shape
    page, group = k.shape[2], H // k.shape[1]
    lim = orc.limits(length, range(B), B, L, causal, count)
    o, lse = torch.zeros((B, H, L, d), dtype=torch.float64, device="cuda"), torch.full((B, H, L), -float("inf"), dtype=torch.float64, device="cuda")
    for b in range(B):
        n = int(length[b])
        if n == 0:
            continue
        at = torch.arange(n, device="cuda")
        pages = cu(table)[b].long()[at // page]
        kk, vv = (x[pages, :, at % page].double().transpose(0, 1) for x in (k, v))
        x = q[b].double().reshape(-1, group * L, d) @ kk.transpose(1, 2) * d ** -0.5
        x.masked_fill_(at >= cu(lim[b]).repeat(group)[:, None], -float("inf"))
        z = torch.logsumexp(x, 2)
        o[b], lse[b] = (torch.exp(x - torch.where(torch.isinf(z), 0.0, z)[..., None]) @ vv).reshape(H, L, d), z.reshape(H, L)
    return o, lse


WAYS = [(1, 3, 8, 2, 16, 0, (6400,)),                        # parts that another kernel joins
        (3, 5, 24, 24, 16, 0, (900, 0, 17)),                 # a cluster of CTAs an item
        (8, 2, 16, 16, 32, 2048, 300),                       # the beginning by the stream kernel: 16 stacked rows
        (4, 7, 24, 24, 64, 4096, 90),                        # 28
        (12, 10, 24, 8, 32, 4096, 200),                      # the beginning by the tile kernel, own keys by warps
        (12, 20, 8, 2, 32, 16384, 400),                      # the tile kernel for both
        (9, 50, 24, 8, 64, 16384, 333),                      # two row tiles of own rows, gathered
        (1, 700, 32, 32, 64, 0, (3000,)),                    # whole items off a queue, the last ones cut
        (3, 509, 32, 8, 64, 0, (509, 3000, 1754)),
        (2, 300, 6, 6, 16, 0, (2000, 299))]                  # fewer items than SMs


@gpu
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B,L,H,Hkv,page,tokens,most", WAYS)
def test_attention_of_counts(B, L, H, Hkv, page, tokens, most, d, causal):
    """Every way that the work is cut; with the full count the bits of the call without one."""
    rng = random.Random(B + d)
    shared = tokens // page
    lengths = list(most) if isinstance(most, tuple) else lengths_behind(rng, B, shared, page, most)
    q, k, v, table, length = attention_case(B, H, Hkv, L, d, page, lengths, shared=shared, seed=B, q_layout="blhd")
    call = lambda count: av.avsa_prefix_attn(q, k, v, cu(table), cu(length), prefix_pages=shared, causal=causal, want_lse=True, count=count)
    plain, full = call(None), call(ints([L] * B))
    assert torch.equal(plain[0], full[0]) and torch.equal(plain[1], full[1])
    for counts in ([rng.randint(0, L) for _ in range(B)], [(0, 1, L - 1)[(b + 1) % 3] for b in range(B)], [min(L, L // 3 + 1)] * B):
        o, lse, ws = call(ints(counts))
        assert status(ws) == av.AVSA_OK
        if not causal:
            assert torch.equal(o, plain[0]) and torch.equal(lse, plain[1])
            continue
        want, want_lse = exact_counts(q, k, v, table, length, counts, causal)
        empty = torch.isinf(want_lse)
        assert torch.equal(torch.isinf(lse), empty) and (o[empty] == 0).all(), counts
        if not empty.all():
            close_o(o.double()[~empty].cpu().numpy(), want[~empty].cpu().numpy(), counts)
            close_lse(lse.double()[~empty].cpu().numpy(), want_lse[~empty].cpu().numpy(), counts)


@gpu
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("B,L,H,Hkv,page,tokens,most", WAYS)
def test_counts_out_of_range_are_reported(B, L, H, Hkv, page, tokens, most, causal):
    """More queries than there are, or less than none: reported, and cut."""
    shared = tokens // page
    lengths = list(most) if isinstance(most, tuple) else [tokens + most] * B
    q, k, v, table, length = attention_case(B, H, Hkv, L, 64, page, lengths, shared=shared, seed=B)
    call = lambda count: av.avsa_prefix_attn(q, k, v, cu(table), cu(length), prefix_pages=shared, causal=causal, want_lse=True, count=ints(count))
    for bad, cut in ((L + 1, L), (2 ** 31 - 1, L), (-1, 0), (-2 ** 31, 0)):
        got, want = call([L] * (B - 1) + [bad]), call([L] * (B - 1) + [cut])
        assert status(got[2]) == av.AVSA_ERR_BAD_TABLE and status(want[2]) == av.AVSA_OK
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@gpu
def test_wrapper_refuses_other_counts():
    q, k, v, table, length = attention_case(3, 2, 2, 4, 64, 16, [100, 100, 100], seed=1)
    for count in (ints([1, 2]), torch.ones(3, device="cuda"), ints([[1, 2, 3]]), ints([1, 0, 2, 0, 3, 0])[::2]):
        with pytest.raises(ValueError, match="count"):
            av.avsa_prefix_attn(q, k, v, cu(table), cu(length), count=count)


def test_counts_off_their_grid_are_refused():
    t = av._Bf16Tensor4(1 << 24, 2 * 64 * 64, 64 * 64, 64)
    assert av.load_library().avsa_prefix_attn_step(4, 4, 2, 3, 64, 64, 10, 4, 8, t, t, t, 8192, 8192, None, 8194, 2, 0, 0.0, 1 << 25, None, None, 1 << 16, 1 << 40,
                                                   0) == av.AVSA_ERR_INVALID_ARG


# ------------------------------------------------------------------------------------------------ errors that nobody reads at once
class LogCalls(StepCalls):
    """``StepCalls`` with the log of extend and attention."""

    def avsa_cache_extend(self, table, length, ref, seq, count, page, out=None, ws=None, granted=None, log=None):
        done = super().avsa_cache_extend(table, length, ref, seq, count, page, granted=granted)
        if done[3] != av.AVSA_OK and log[0] == 0:
            log[0] = done[3]
        return done

    def avsa_prefix_attn(self, *args, count=None, log=None, **kw):
        return super().avsa_prefix_attn(*args, count=count, **kw)


@pytest.mark.parametrize("where", WHERE)
def test_errors_stay_until_they_are_read(where):
    """A step that is refused, steps and drops that are not: check says so, once."""
    cache = ClipCache(1, 1, 64, 16, 4, 2, 8, device=where, calls=LogCalls() if where == "cpu" else None)
    x = torch.ones((1, 1, 1, 64), dtype=torch.bfloat16, device=where)
    cache.begin_step([0], [16])
    cache.check()
    cache.begin_step([1], [100])
    for _ in range(3):
        cache.begin_step([0], [1])
        cache.attend(0, x, x, x)
    cache.drop([0])
    with pytest.raises(av.AvsaError, match="extend") as e:
        cache.check()
    assert e.value.status == av.AVSA_ERR_NO_PAGES
    cache.check()
    cache.begin_step([0], [64])
    cache.check()


@gpu
def test_errors_of_replays_and_of_every_layer_are_read():
    """A captured step runs out of pages in one of its replays; in another cache only the first of two layers leaves tokens out, the fork and the drop are refused."""
    cache = ClipCache(1, 1, 64, 16, 4, 2, 8)
    seq, count, x = ints([0, 1]), ints([9, 3]), torch.ones((2, 1, 9, 64), dtype=torch.bfloat16, device="cuda")

    def step():
        cache.begin_step(seq, count)
        return cache.attend(0, x, x, x, causal=True)

    step()
    cache.drop([0, 1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(4):
        graph.replay()
    cache.check()
    assert cache.length.tolist() == [36, 12]
    for _ in range(2):
        graph.replay()          # 45 and 15 tokens fill four pages up to 3 and 1: of the step behind that neither sequence gets anything
    assert cache.length.tolist() == [45, 15]
    with pytest.raises(av.AvsaError, match="extend"):
        cache.check()
    cache.drop([0, 1])
    graph.replay()
    cache.check()

    cache = ClipCache(2, 1, 64, 16, 4, 3, 8)
    cache.begin_step(ints([0]), ints([9]))
    cache.attend(0, x[:1, :, :8], x[:1, :, :8], x[:1, :, :8])
    cache.attend(1, x[:1], x[:1], x[:1])
    cache.branch([0, 0], [0, 1])          # 0 is not empty
    cache.drop([2, 3])
    cache.compact()
    with pytest.raises(av.AvsaError, match="attention.*fork.*free") as e:
        cache.check()
    assert e.value.status == av.AVSA_ERR_BAD_TABLE and "extend" not in str(e.value) and "compact" not in str(e.value)
    cache.check()


@gpu
@pytest.mark.parametrize("B,L,H,Hkv,page,tokens,most", WAYS)
def test_log_of_the_attention(B, L, H, Hkv, page, tokens, most):
    """Whatever kernel finds it: the first error stays, with the status record's words."""
    shared = tokens // page
    lengths = list(most) if isinstance(most, tuple) else [tokens + most] * B
    q, k, v, table, length = attention_case(B, H, Hkv, L, 64, page, lengths, shared=shared, seed=B)
    log, n = torch.zeros(4, dtype=torch.int32, device="cuda"), length.copy()
    call = lambda length, log: av.avsa_prefix_attn(q, k, v, cu(table), cu(length), prefix_pages=shared, log=log)[2]
    assert status(call(length, log)) == av.AVSA_OK and log.tolist() == [0] * 4
    n[-1] = -7
    code, detail = av.avsa_read_status(call(n, log))
    assert log.tolist() == [code, *detail] and code == av.AVSA_ERR_BAD_TABLE
    call(length, log)
    assert log.tolist() == [code, *detail]
    mine = ints([av.AVSA_ERR_NO_PAGES, 1, 2, 3])
    call(n, mine)
    assert mine.tolist() == [av.AVSA_ERR_NO_PAGES, 1, 2, 3]


@gpu
@pytest.mark.parametrize("pages", [6, 20000])
def test_log_of_the_cache_calls(pages):
    """A CTA's own work and a cluster's; free, fork, extend and compact one after the other."""
    pool = torch.zeros((1, pages, 1, 16, 64), dtype=torch.bfloat16, device="cuda")
    ref = np.zeros(pages, np.int32)
    ref[[2, 5]] = 1
    state = lambda bad=False: (ints([[2, pages if bad else 5], [-1, -1]]), ints([20, 0]), cu(ref))
    calls = {"free": lambda bad, **kw: av.avsa_cache_free(*state(bad), ints([0]), **kw)[3],
             "fork": lambda bad, **kw: av.avsa_cache_fork(pool, *state(bad), ints([0]), ints([1]), **kw)[3],
             "extend": lambda bad, **kw: av.avsa_cache_extend(*state(), ints([1]), ints([100 if bad else 3]), 16, **kw)[3],
             "compact": lambda bad, **kw: av.avsa_cache_compact(pool, *state(bad), **kw)[1]}
    for name, call in calls.items():
        log = torch.zeros(4, dtype=torch.int32, device="cuda")
        assert status(call(False, log=log)) == av.AVSA_OK and log.tolist() == [0] * 4, name
        code, detail = av.avsa_read_status(call(True, log=log))
        assert code != av.AVSA_OK and log.tolist() == [code, *detail], name
        for again in calls.values():
            again(False, log=log)
            again(True, log=log)
        assert log.tolist() == [code, *detail], name


@gpu
@pytest.mark.parametrize("seqs,pages", [(900, 50), (900, 20000)])
def test_log_of_many_errors_at_once(seqs, pages):
    """Of errors that hundreds of threads report at the same time the log has the one that the status record has."""
    table, length, ref = (torch.full((seqs, 4), -1, dtype=torch.int32, device="cuda"), ints([0] * seqs), ints([0] * pages))
    for k in range(40):
        log = torch.zeros(4, dtype=torch.int32, device="cuda")
        count = ints([(-1, 70, 64, 30)[(s * 7 + k) % 4] for s in range(seqs)])          # below 0, beyond the row, beyond the pool or not
        ws = av.avsa_cache_extend(table.clone(), length.clone(), ref.clone(), ints(list(range(seqs))), count, 16, log=log)[3]
        code, detail = av.avsa_read_status(ws)
        assert code != av.AVSA_OK and log.tolist() == [code, *detail]


def test_logs_that_are_refused():
    """Off their grid, or a part of what a call reads or writes."""
    lib, t = av.load_library(), av._Bf16Tensor4(1 << 24, 2 * 64 * 64, 64 * 64, 64)
    state = dict(table=1 << 20, length=2 << 20, ref=3 << 20, table_out=4 << 20, length_out=5 << 20, ref_out=6 << 20, seqs=4, width=8, pages=100, page=16)
    c, p, big = av._Cache(**state), av._Pages(ptr=1 << 24, planes=2, page_bytes=4096, stride_plane=409600, stride_page=4096), (1 << 16, 1 << 30, 0)
    for log in (8194, (1 << 20) + 4, (2 << 20) - 12, (6 << 20) + 396):
        assert lib.avsa_cache_extend_step(c, 8192, 16384, 2, None, log, *big) == av.AVSA_ERR_INVALID_ARG, log
        assert lib.avsa_cache_fork_step(c, p, 8192, 16384, 2, log, *big) == av.AVSA_ERR_INVALID_ARG, log
        assert lib.avsa_cache_free_step(c, 8192, 2, log, *big) == av.AVSA_ERR_INVALID_ARG, log
        assert lib.avsa_cache_compact_step(c, p, 8192, log, *big) == av.AVSA_ERR_INVALID_ARG, log
    assert lib.avsa_prefix_attn_step(4, 4, 2, 3, 64, 64, 10, 4, 8, t, t, t, 8192, 8192, None, None, 2, 0, 0.0, 1 << 25, None, 8194, 1 << 16, 1 << 40,
                                     0) == av.AVSA_ERR_INVALID_ARG


@gpu
def test_wrappers_refuse_other_logs():
    i, t, ref = ints([0] * 4), ints([[0, 0]] * 4), ints([0] * 5)
    for log in (ints([0] * 3), torch.zeros(4, device="cuda"), ints([[0] * 4])):
        with pytest.raises(ValueError, match="log"):
            av.avsa_cache_free(t, i, ref, i, log=log)
        with pytest.raises(ValueError, match="log"):
            av.avsa_cache_extend(t, i, ref, i, i, 16, log=log)


# ------------------------------------------------------------------------------------------------ fewer tokens than there is room for
@pytest.mark.parametrize("where", WHERE)
def test_a_step_of_fewer_tokens_than_it_made_room_for(where):
    """Counts in a list are looked at before anything is written."""
    cache = ClipCache(1, 1, 64, 16, 8, 2, 8, device=where, calls=LogCalls() if where == "cpu" else None)
    x = torch.ones((2, 1, 5, 64), dtype=torch.bfloat16, device=where)
    cache.begin_step([0, 1], [6, 2])
    before = cache.pool.view(torch.int16).clone()
    with pytest.raises(ValueError, match="5 tokens.*room for 6"):
        cache.attend(0, x, x, x)
    assert torch.equal(cache.pool.view(torch.int16), before)
    x = torch.ones((2, 1, 6, 64), dtype=torch.bfloat16, device=where)
    assert (cache.attend(0, x, x, x) == 1).all()
    cache.begin_step([0, -1], [1, 99])          # an entry that is left out needs none
    cache.attend(0, x, x, x)
    cache.begin_step([], [])
    cache.check()


@gpu
def test_a_tensor_of_more_counts_than_tokens_is_reported():
    cache = ClipCache(1, 1, 64, 16, 8, 2, 8)
    x = torch.ones((2, 1, 5, 64), dtype=torch.bfloat16, device="cuda")
    for count, good in (([5, 2], True), ([6, 2], False)):
        cache.begin_step(ints([0, 1]), ints(count))
        cache.attend(0, x, x, x, causal=True)
        if good:
            cache.check()
        else:
            with pytest.raises(av.AvsaError, match="attention"):
                cache.check()


# ------------------------------------------------------------------------------------------------ several passes over the tokens of a step
@pytest.mark.parametrize("where", WHERE)
@pytest.mark.parametrize("causal", [False, True])
def test_passes_of_a_step_replace_its_tokens(where, causal):
    """One begin_step, attend once for every denoising pass: each pass sees the beginning and its own tokens, the last one's stay."""
    page, d, H, Hkv, L = 16, 64, 4, 2, 21
    cache = ClipCache(2, Hkv, d, page, 20, 3, 8, device=where, calls=LogCalls() if where == "cpu" else None)
    gen = torch.Generator().manual_seed(3)
    draw = lambda h, n, L: torch.randn((n, h, L, d), generator=gen).bfloat16()
    attend = lambda layer, x, shared=0: cache.attend(layer, *(t.to(where) for t in x), shared, causal).cpu()
    old = [[draw(h, 1, 40) for h in (H, Hkv, Hkv)] for _ in range(2)]
    cache.begin_step([0], [40])
    for layer in range(2):
        attend(layer, old[layer])
    cache.branch([0, 0], [1, 2])
    cache.begin_step([0, 1, 2], [L, L, 4])
    for _ in range(3):
        for layer in range(2):
            x = [draw(h, 3, L) for h in (H, Hkv, Hkv)]
            o = attend(layer, x, 2)
            for b, c in enumerate((L, L, 4)):
                k, v = (torch.cat([a[0], y[b, :, :c]], 1) for a, y in zip(old[layer][1:], x[1:]))
                lim = [40 + i + 1 if causal else 40 + c for i in range(c)]
                close_o(o[b][:, :c].double().numpy(), plain_rows(x[0][b][:, :c], k, v, lim).numpy(), f"sequence {b}, layer {layer}")
    cache.check()
    assert cache.length.tolist() == [40 + L, 40 + L, 44]


def test_stand_ins_of_some_calls_alone():
    """Calls that are not there, or that do not say what they take, are missed when they are made."""
    class Some:
        avsa_cache_extend = staticmethod(lambda *a: (*a[:3], av.AVSA_OK))
        avsa_cache_free = print          # (a builtin)
        avsa_read_status = staticmethod(lambda ws: (ws, (0, 0, 0)))

    cache = ClipCache(1, 1, 64, 16, 4, 2, 4, device="cpu", calls=Some())
    cache.begin_step([0], [3])
    cache.check()
    with pytest.raises(AttributeError):
        cache.branch([0], [1])
