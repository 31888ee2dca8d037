"""Tables that are not as they should be, at every place of a row and in every way that the attention over a paged cache reads them."""
import pytest
import torch

from paper_2608_15522_b200 import binding as av
from test_cache_q4 import held
from test_paged_cache import attention_case, cu, ints, status

gpu = pytest.mark.gpu


@gpu
@pytest.mark.parametrize("way,B,L,Hkv", [
    ("bf16", 1, 1000, 37),     # the tile kernel by TMA
    ("codes", 1, 700, 74),     # tiles made of codes in the kernel
    ("codes", 1, 1000, 37),    # pages of codes made bf16 before it
    ("codes", 4, 1, 8)])       # the stream kernel
def test_the_first_page_number_out_of_range(way, B, L, Hkv):
    """An entry that equals the number of pages is out of range like any other: wherever in a row it stands, it is reported and its tokens read as zeros.

    Rows of 569 pages, of which 32 come with an item of the tile kernel; its items are whole ones here (a multiple of 148), so the others are looked up behind these."""
    page, n = 16, 9100
    q, k, v, table, length = attention_case(B, Hkv, Hkv, L, 64, page, [n] * B, seed=3, poison=False)
    call = av.avsa_prefix_attn
    if way == "codes":
        (k, kv), (v, vv) = held(k), held(v)
        call = av.avsa_prefix_attn_q4
    pages = k.shape[0]
    t, lengths, log = cu(table), cu(length), ints([0, 0, 0, 0])
    good = call(q, k, v, t, lengths, log=log)[0]
    assert int(log[0]) == av.AVSA_OK
    row = B - 1
    zero = (k.clone(), v.clone())
    for at in (3, 31, 32, 33, 100, 303, 567, 568):
        bad, log = t.clone(), ints([0, 0, 0, 0])
        bad[row, at] = pages
        o, _, ws = call(q, k, v, bad, lengths, log=log)
        assert status(ws) == av.AVSA_ERR_BAD_TABLE and int(log[0]) == av.AVSA_ERR_BAD_TABLE, at
        # the same page, with zeros in it: no sequence but this one has it
        kept = [x[table[row, at]].clone() for x in zero]
        for x in zero:
            x[table[row, at]] = 0
        want = call(q, *zero, t, lengths)[0]
        for x, old in zip(zero, kept):
            x[table[row, at]] = old
        assert torch.equal(o, want), at
        assert torch.equal(o[:row], good[:row])


@gpu
@pytest.mark.parametrize("way", ["bf16", "codes"])
@pytest.mark.parametrize("L,Hkv", [(40, 1), (1, 4)])
def test_of_equally_long_sequences_the_first_names_the_shared_pages(L, Hkv, way):
    """The longest sequence's row says which pages are shared; of several the first one's, for everything that the call does.

    Rows that differ are malformed.  What the first one lacks reads as zeros and is reported, whatever the workspace held; what another one lacks is not looked at.
    With forty queries the pages of codes are made bf16 before the products, and a sequence has two row tiles."""
    B, group, page, shared = 20, 4, 16, 1024
    lengths = [shared * page + (90 if b in (1, 16, 19) else 1 + 3 * b) for b in range(B)]
    q, k, v, table, length = attention_case(B, group * Hkv, Hkv, L, 64, page, lengths, shared=shared, seed=2, poison=False)
    call, query = av.avsa_prefix_attn, av.avsa_prefix_attn_workspace_bytes(B, group * Hkv, Hkv, L, 64, page, table.shape[1], shared)
    if way == "codes":
        (k, _), (v, _) = held(k), held(v)
        call, query = av.avsa_prefix_attn_q4, av.avsa_prefix_attn_q4_workspace_bytes(B, group * Hkv, Hkv, L, 64, page, k.shape[0], table.shape[1], shared)
    n = cu(length)

    def run(t, k=k, v=v):
        ws = torch.full((query,), 255, dtype=torch.uint8, device="cuda")      # (as bf16 or fp32: NaN)
        o, lse, _ = call(q, k, v, cu(t), n, prefix_pages=shared, want_lse=True, ws=ws)
        return o, lse, status(ws)

    good = run(table)
    assert good[2] == av.AVSA_OK and torch.isfinite(good[0].float()).all()
    for at in (5, 700):
        bad = table.copy()
        bad[16, at] = -1 if at == 5 else k.shape[0]
        o, lse, st = run(bad)
        assert st == av.AVSA_OK and torch.equal(o, good[0]) and torch.equal(lse, good[1])
        bad = table.copy()
        bad[1, at] = -1 if at == 5 else k.shape[0]
        o, lse, st = run(bad)
        zero = [x.clone() for x in (k, v)]
        for x in zero:
            x[table[1, at]] = 0
        want = run(table, *zero)
        assert st == av.AVSA_ERR_BAD_TABLE and torch.equal(o, want[0]) and torch.equal(lse, want[1])
