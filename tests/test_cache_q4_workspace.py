"""Room that the attention over a cache held in 4 bits takes beside it: for the pages that its batch can name, however large the pool is."""
import numpy as np
import pytest
import torch

from paper_2608_15522_b200 import binding as av
from test_cache_q4 import held_case
from test_paged_cache import cu, exact_on_gpu, ints, status
from parity_bars import close_lse, close_o

gpu = pytest.mark.gpu


@pytest.mark.parametrize("B,H,L,page,width,shared", [(4, 8, 1000, 64, 40, 0), (4, 8, 1000, 64, 40, 17), (1, 8, 2000, 16, 300, 300), (20, 32, 40, 16, 1030, 1024)])
def test_a_call_asks_for_no_more_than_its_table_can_name(B, H, L, page, width, shared):
    """Room for prefix_pages pages and each sequence's others is enough, of any pool; of a pool that has fewer, for its pages."""
    Hkv, d = 8, 128
    ask = lambda pages: av.avsa_prefix_attn_q4_workspace_bytes(B, H, Hkv, L, d, page, pages, width, shared)
    named = shared + B * (width - shared)
    t, pool = av._Bf16Tensor4(1 << 20, L * H * d, L * d, d), av._Q4Pool(1 << 20, 72 * page * Hkv, 72 * page)

    def room(pages, ws_bytes):
        """Whether so many bytes are enough; the workspace's address is off its grid, so nothing runs."""
        got = av.load_library().avsa_prefix_attn_q4(B, H, Hkv, L, d, page, pages, B, width, t, pool, pool, 1 << 20, 1 << 20, None, None, shared, 0, 0.0, 1 << 20, None, None,
                                                    (1 << 20) + 16, ws_bytes, 0)
        assert got in (av.AVSA_ERR_INVALID_ARG, av.AVSA_ERR_WORKSPACE)
        return got == av.AVSA_ERR_INVALID_ARG

    assert ask(named) > 2 * named * Hkv * page * d * 2
    for pages in (named, named + 1, 50 * named, (1 << 31) - 1):
        assert room(pages, ask(named)) and not room(pages, ask(named) - 1)
    half = named // 2
    assert ask(half) < ask(named) and room(half, ask(half)) and not room(half, ask(half) - 1)


@gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B,L,H,Hkv,page,shared,lengths", [
    (2, 900, 4, 4, 32, 0, (3000, 1111)),                                      # each its own
    (3, 900, 6, 2, 16, 40, (1700, 640, 651)),                                 # a beginning that every row tile meets with its sequence's others
    (4, 333, 24, 8, 64, 3, (1000, 0, 130, 640)),                              # a sequence that holds nothing, one that ends in the beginning
    (20, 40, 4, 1, 16, 1024, tuple(16384 + 90 - 4 * b for b in range(20))),   # a beginning that is read for all rows at once, and own pages
    (60, 1, 32, 1, 32, 800, tuple(25600 + 9 * b for b in range(60)))])       # ... and own ones that the stream kernel reads as codes
def test_large_pools(B, L, H, Hkv, page, shared, lengths, d):
    """The same pages in a pool of just so many and far apart in a large one: the same bits, from a workspace that does not grow with the pool."""
    (q, k, v, table, length), values = held_case(B, H, Hkv, L, d, page, list(lengths), shared=shared, seed=B)
    pages, width = k.shape[0], table.shape[1]
    named = shared + B * (width - shared)
    many = 3 * named + 2 * pages
    place = torch.randperm(many, generator=torch.Generator().manual_seed(1))[:pages].cuda()
    far = [torch.full((many, *x.shape[1:]), 255, dtype=torch.uint8, device="cuda") for x in (k, v)]      # (codes of NaN)
    for x, y in zip(far, (k, v)):
        x[place] = y
    moved = np.where(table >= 0, place.cpu().numpy()[table], -1).astype(np.int32)
    for causal in (False, True):
        a = av.avsa_prefix_attn_q4(q, k, v, cu(table), cu(length), prefix_pages=shared, causal=causal, want_lse=True)
        b = av.avsa_prefix_attn_q4(q, *far, cu(moved), cu(length), prefix_pages=shared, causal=causal, want_lse=True)
        assert status(a[2]) == status(b[2]) == av.AVSA_OK
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
        assert b[2].numel() <= av.avsa_prefix_attn_q4_workspace_bytes(B, H, Hkv, L, d, page, named, width, shared)
        # another workspace, whatever it holds
        o, lse, _ = av.avsa_prefix_attn_q4(q, *far, cu(moved), cu(length), prefix_pages=shared, causal=causal, want_lse=True, ws=torch.full_like(b[2], 255))
        assert torch.equal(o, b[0]) and torch.equal(lse, b[1])
        want, want_lse = exact_on_gpu(*values, causal=causal)
        seen = ~torch.isinf(want_lse)
        close_o(b[0].double()[seen].cpu().numpy(), want[seen].cpu().numpy(), "large pool")
        close_lse(b[1].double()[seen].cpu().numpy(), want_lse[seen].cpu().numpy(), "large pool")


@gpu
def test_large_pool_of_chosen_sequences():
    """Any sequences in any order, one of them twice, one left out; rows that share pages without saying so."""
    (q, k, v, table, length), values = held_case(5, 4, 4, 900, 64, 16, [1400, 1777, 0, 930, 1160, 990, 1640], seed=5)
    table[6, :80] = table[1, :80]
    pages, width, seq = k.shape[0], table.shape[1], [6, -1, 1, 6, 3]
    many = 8 * width * 5
    far = [torch.full((many, *x.shape[1:]), 255, dtype=torch.uint8, device="cuda") for x in (k, v)]
    for x, y in zip(far, (k, v)):
        x[many - pages:] = y
    moved = np.where(table >= 0, table + many - pages, -1).astype(np.int32)
    o, lse, ws = av.avsa_prefix_attn_q4(q, *far, cu(moved), cu(length), seq=ints(seq), causal=True, want_lse=True)
    assert status(ws) == av.AVSA_OK and ws.numel() <= av.avsa_prefix_attn_q4_workspace_bytes(5, 4, 4, 900, 64, 16, 5 * width, width, 0)
    want, want_lse = exact_on_gpu(values[0], *values[1:3], table, length, seq, True)
    seen = ~torch.isinf(want_lse)
    assert torch.equal(torch.isinf(lse), ~seen) and (o[~seen] == 0).all()
    close_o(o.double()[seen].cpu().numpy(), want[seen].cpu().numpy(), "chosen")
    close_lse(lse.double()[seen].cpu().numpy(), want_lse[seen].cpu().numpy(), "chosen")


@gpu
@pytest.mark.parametrize("row", [0, 1, 2])
def test_large_pool_with_a_bad_page(row):
    """A page out of range in any row: reported, zeros, and nothing that the workspace held; sequence 1 is the longest, whose row the shared pages are read by."""
    B, page, shared = 3, 16, 40
    (q, k, v, table, length), values = held_case(B, 2, 2, 900, 64, page, [1000, 1300, 900], shared=shared, seed=4)
    pages = 6 * (shared + B * table.shape[1])
    far = [torch.zeros((pages, *x.shape[1:]), dtype=torch.uint8, device="cuda") for x in (k, v)]
    for x, y in zip(far, (k, v)):
        x[pages - y.shape[0]:] = y
    moved = np.where(table >= 0, table + pages - k.shape[0], -1).astype(np.int32)
    call = lambda t, ws=None: av.avsa_prefix_attn_q4(q, *far, cu(t), cu(length), prefix_pages=shared, want_lse=True, ws=ws)
    good = call(moved)
    assert status(good[2]) == av.AVSA_OK
    for at, bad in ((7, -1), (39, pages), (50, 1 << 30)):      # two shared ones and one of its own
        t = moved.copy()
        t[row, at] = bad
        o, lse, ws = call(t, torch.full_like(good[2], 255))
        assert status(ws) == av.AVSA_ERR_BAD_TABLE and torch.isfinite(o.float()).all() and torch.isfinite(lse).all()
        # without that page: zeros for whoever goes by it
        hit = [b for b in range(B) if b == row or (at < shared and row == 1)]
        zero = [x.clone() for x in values[1:3]]
        for x in zero:
            x[table[row, at]] = 0.0
        want, want_lse = exact_on_gpu(values[0], *zero, table, length)
        for b in range(B):
            if b not in hit:
                assert torch.equal(o[b], good[0][b]) and torch.equal(lse[b], good[1][b])
            else:
                close_o(o[b].double().cpu().numpy(), want[b].cpu().numpy(), "zeros")
                close_lse(lse[b].double().cpu().numpy(), want_lse[b].cpu().numpy(), "zeros")
