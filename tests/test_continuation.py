"""A clip continued over the paged cache: the sequencing of ``ClipCache`` on the CPU, its results against plain attention on the GPU."""
import numpy as np
import pytest
import torch

from oracle import cache_oracle as orc
from paper_2608_15522_b200 import binding as av
from paper_2608_15522_b200.continuation import ClipCache, continue_clip, main
from parity_bars import close_o

gpu = pytest.mark.gpu


class OracleCalls:
    """The cache calls of ``binding`` on the CPU, by the plain statement."""

    def _put(self, targets, arrays):
        for t, a in zip(targets, arrays):
            t.copy_(torch.from_numpy(np.ascontiguousarray(a)))

    def avsa_cache_extend(self, table, length, ref, seq, count, page, out=None, ws=None):
        state = (table, length, ref)
        *new, refused = orc.extend(*(t.numpy() for t in state), seq.tolist(), count.tolist(), page)
        self._put(state, new)
        return (*state, av.AVSA_ERR_NO_PAGES if refused else av.AVSA_OK)

    def avsa_cache_write(self, k_new, v_new, k_pool, v_pool, table, length, seq=None, count=None):
        k, v = k_pool.float().numpy(), v_pool.float().numpy()
        orc.write(k_new.float().numpy(), v_new.float().numpy(), k, v, table.numpy(), length.numpy(), seq.tolist(), count.tolist())
        k_pool.copy_(torch.from_numpy(k))
        v_pool.copy_(torch.from_numpy(v))

    def avsa_prefix_attn(self, q, k, v, table, length, prefix_pages=0, seq=None, causal=False, softmax_scale=0.0):
        f64 = lambda t: t.double().numpy()
        o, lse = orc.prefix_attention(f64(q), f64(k), f64(v), table.numpy(), length.numpy(), seq.tolist(), causal, softmax_scale or None)
        return torch.from_numpy(o).bfloat16(), None, av.AVSA_OK

    def avsa_cache_fork(self, pool, table, length, ref, parent, child):
        state = (table, length, ref)
        *new, moves, refused = orc.fork(*(t.numpy() for t in state), parent.tolist(), child.tolist(), pool.shape[3])
        self._put(state, new)
        for a, b in moves:
            pool[:, b] = pool[:, a]
        return (*state, av.AVSA_ERR_NO_PAGES if refused else av.AVSA_OK)

    def avsa_cache_free(self, table, length, ref, seq):
        state = (table, length, ref)
        self._put(state, orc.free(*(t.numpy() for t in state), seq.tolist())[:3])
        return (*state, av.AVSA_OK)

    def avsa_cache_compact(self, pool, table, length, ref):
        *new, live, moves = orc.compact(table.numpy(), ref.numpy())
        self._put((table, ref), new)
        for a, b in moves:
            pool[:, b] = pool[:, a]
        return torch.tensor([live]), av.AVSA_OK

    def avsa_read_status(self, ws):
        return ws, (0, 0, 0)


def drive(cache, H, Hkv, d, page, seed, dtype=torch.float64):
    """Branches, steps of several lengths, drops, a compaction; beside the cache every sequence's tokens in plain lists, whose attention it has to give."""
    gen = torch.Generator().manual_seed(seed)
    dev = cache.table.device
    kept = {}          # sequence -> [layers] of (k, v) [Hkv, n, d]

    def step(seqs, L, shared, causal):
        n = len(seqs)
        cache.begin_step(seqs, [L] * n)
        for layer in range(cache.layers):
            q, k, v = (torch.randn((n, h, L, d), generator=gen).bfloat16() for h in (H, Hkv, Hkv))
            o = cache.attend(layer, q.to(dev), k.to(dev), v.to(dev), shared, causal).cpu().double()
            for b, s in enumerate(seqs):
                now = kept.setdefault(s, [torch.zeros((2, Hkv, 0, d))] * cache.layers)
                now = kept[s] = list(now)
                now[layer] = torch.cat([now[layer], torch.stack([k[b].float(), v[b].float()])], 2)
                kk, vv = now[layer].to(dtype).repeat_interleave(H // Hkv, 1)
                x = q[b].to(dtype) @ kk.transpose(1, 2) * d ** -0.5
                if causal:
                    N = kk.shape[1]
                    x = x.masked_fill(torch.arange(N) > torch.arange(N - L, N)[:, None], -float("inf"))
                close_o(o[b].numpy(), (torch.softmax(x, -1) @ vv).numpy(), f"sequence {s}, layer {layer}")

    def branch(parent, children):
        cache.branch([parent] * len(children), children)
        for c in children:
            kept[c] = kept[parent]

    def drop(seqs):
        cache.drop(seqs)
        for s in seqs:
            kept.pop(s)

    step([0], 2 * page + 5, 0, True)
    step([0], 1, 0, False)
    branch(0, [1, 2, 3])
    step([0, 1, 2, 3], 7, 2, True)
    step([0, 1, 2, 3], 1, 2, False)
    drop([0, 2])
    step([3, 1], page, 2, False)
    live = int(cache.compact())
    branch(3, [0])
    step([3, 0], 1, 3, True)
    cache.check()
    assert int((cache.ref > 0).sum()) == live + 1          # the branch's copy of the page that its parent had begun
    held = torch.zeros_like(cache.ref)
    for s, n in enumerate(cache.length.tolist()):
        row = cache.table[s, :-(-n // page)]
        held.index_add_(0, row.long(), torch.ones_like(row))
        assert n == (kept[s][0].shape[2] if s in kept else 0)
    assert torch.equal(held, cache.ref)


def test_sequencing_with_plain_calls():
    drive(ClipCache(2, 1, 64, 16, 40, 4, 8, "cpu", OracleCalls()), 2, 1, 64, 16, 0)


def test_errors_reach_the_host():
    cache = ClipCache(1, 1, 64, 16, 2, 2, 8, "cpu", OracleCalls())
    with pytest.raises(ValueError):
        cache.attend(0, None, None, None)
    cache.begin_step([0], [40])
    with pytest.raises(av.AvsaError) as e:
        cache.check()
    assert e.value.status == av.AVSA_ERR_NO_PAGES and "extend" in str(e.value)


@gpu
@pytest.mark.parametrize("H, Hkv, d, page", [(4, 4, 64, 16), (8, 2, 128, 64), (24, 4, 128, 128)])
def test_clip_cache(H, Hkv, d, page):
    drive(ClipCache(2, Hkv, d, page, 40, 4, 8), H, Hkv, d, page, 1)


@gpu
def test_errors_reach_the_host_from_the_device():
    cache = ClipCache(1, 1, 64, 16, 2, 2, 8)
    cache.begin_step([0], [40])
    with pytest.raises(av.AvsaError) as e:
        cache.check()
    assert e.value.status == av.AVSA_ERR_NO_PAGES and "extend" in str(e.value)


@gpu
def test_command(capsys):
    cache, live = continue_clip(layers=2, heads=4, heads_kv=2, d=64, width=128, beginning=200, chunk=24, audio=3, candidates=3, rounds=2, page=16)
    span = 200 + 2 * 27
    assert live == -(-span // 16) and sorted(cache.length.tolist()) == [0, 0, 0, span]
    assert int(cache.table.max()) == live - 1
    main("--layers 1 --heads 2 --heads-kv 1 --d 64 --beginning 64 --chunk 16 --audio 1 --candidates 2 --rounds 1 --page 32".split())
    assert "compacted: pages 0..2" in capsys.readouterr().out


@gpu
@pytest.mark.parametrize("L, H, Hkv", [(1, 8, 2), (40, 4, 4)])
def test_step_as_a_graph(L, H, Hkv):
    """Lengths and pages are read on the device only: a step captured once goes on where the last replay ended."""
    d, page, seqs, shared, steps = 64, 16, 3, 4, 9

    def begin():
        cache = ClipCache(2, Hkv, d, page, 120, seqs, 40)
        gen = torch.Generator().manual_seed(5)
        draw = lambda n, h, m: torch.randn((n, h, m, d), generator=gen).bfloat16().cuda()
        cache.begin_step([0], [shared * page + 3])
        for layer in range(2):
            cache.attend(layer, *(draw(1, h, shared * page + 3) for h in (H, Hkv, Hkv)), causal=True)
        cache.branch([0, 0], [1, 2])
        return cache, [[draw(seqs, h, L) for h in (H, Hkv, Hkv)] for _ in range(2)]

    seq, count = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([2, 0, 1], [L, L - 1, L]))

    def step(cache, inputs):
        cache.begin_step(seq, count)
        return [cache.attend(i, *x, shared, causal=True) for i, x in enumerate(inputs)]

    plain, inputs = begin()
    want = [[o.clone() for o in step(plain, inputs)] for _ in range(steps)]
    plain.check()
    cache, inputs = begin()
    graph = torch.cuda.CUDAGraph()
    state = [t.clone() for t in cache._state()]
    with torch.cuda.graph(graph):
        got = step(cache, inputs)
    assert all(torch.equal(a, b) for a, b in zip(state, cache._state()))          # captured, not run
    for n in range(steps):
        graph.replay()
        for a, b in zip(got, want[n]):
            assert torch.equal(a, b), n
    cache.check()
    assert all(torch.equal(a, b) for a, b in zip(plain._state(), cache._state()))
