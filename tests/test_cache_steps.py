"""Steps over the paged cache in which something is refused: the calls after one another, and ``ClipCache``, on the CPU by the plain statement and on the GPU."""
import random

import numpy as np
import pytest
import torch

from oracle import cache_oracle as orc
from paper_2608_15522_b200 import binding as av
from paper_2608_15522_b200.continuation import ClipCache
from parity_bars import close_o
from test_continuation import OracleCalls
from test_paged_cache import SIZES, cu, ints, nump, random_state, status

gpu = pytest.mark.gpu


class StepCalls(OracleCalls):
    """``OracleCalls`` with what the calls say on the device."""

    def avsa_cache_extend(self, table, length, ref, seq, count, page, out=None, ws=None, granted=None):
        refused = orc.extend(table.numpy(), length.numpy(), ref.numpy(), seq.tolist(), count.tolist(), page)[3]
        granted.copy_(torch.tensor(granted_of(seq.tolist(), count.tolist(), refused)))
        return super().avsa_cache_extend(table, length, ref, seq, count, page)


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
    call = lambda granted: lib.avsa_cache_extend_step(av._Cache(**state), 8192, 16384, 2, granted, 1 << 16, 1 << 30, 0)
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
