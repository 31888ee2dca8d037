"""Attention over a cache held in 4 bits: what of its numbers is exact, and how far off the others may be where the softmax is sharp."""
import pytest
import torch

from paper_2608_15522_b200 import binding as av
from test_cache_q4 import held, held_case
from test_paged_cache import attention_case, cu, status

gpu = pytest.mark.gpu


@gpu
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B,L,H,Hkv,page,shared,own", [
    (2, 150, 4, 4, 64, 0, 513),         # tiles made of codes in the kernel
    (3, 70, 16, 4, 16, 0, 1297),
    (4, 40, 8, 4, 32, 512, 200),        # ... behind a beginning that is read for all rows at once
    (2, 900, 4, 4, 64, 0, 513),         # pages made bf16 before it
    (3, 1000, 2, 1, 128, 3, 700)])
def test_the_tile_kernel_has_the_bits_of_the_one_over_bf16(B, L, H, Hkv, page, shared, own, d, causal):
    """Every value that a page of codes stands for is a bf16 number, and more than 32 query rows are cut alike whatever their keys come from: the same cache in bf16 gives the same bits."""
    lengths = [page * shared + own - 61 * i for i in range(B)]
    (q, k4, v4, table, length), (_, k, v, _, _) = held_case(B, H, Hkv, L, d, page, lengths, shared=shared, seed=9)
    got = av.avsa_prefix_attn_q4(q, k4, v4, cu(table), cu(length), prefix_pages=shared, causal=causal, want_lse=True)
    want = av.avsa_prefix_attn(q, k, v, cu(table), cu(length), prefix_pages=shared, causal=causal, want_lse=True)
    assert status(got[2]) == status(want[2]) == av.AVSA_OK
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@gpu
@pytest.mark.parametrize("L", [2, 40, 900])
def test_keys_that_a_causal_row_does_not_see_may_be_anything(L):
    """A group of a key that reads as NaN: the row that sees its token has no numbers, those in front of it the bits that they have without it."""
    q, k, v, table, length = attention_case(2, 2, 2, L, 64, 16, [100, 90], seed=1, poison=False)
    v4 = held(v)[0]
    clean = av.avsa_prefix_attn_q4(q, held(k)[0], v4, cu(table), cu(length), causal=True, want_lse=True)
    k[int(table[0, 6]), 1, 3, 40] = float("inf")          # token 99, the last one
    o, lse, _ = av.avsa_prefix_attn_q4(q, held(k)[0], v4, cu(table), cu(length), causal=True, want_lse=True)
    assert torch.isnan(o[0, 1, -1]).all() and torch.isnan(lse[0, 1, -1])
    for got, want in ((o, clean[0]), (lse, clean[1])):
        assert torch.equal(got[1], want[1]) and torch.equal(got[0, 0], want[0, 0]) and torch.equal(got[0, 1, :-1], want[0, 1, :-1])


@gpu
@pytest.mark.parametrize("way", ["bf16", "codes"])
@pytest.mark.parametrize("B,L,H,Hkv,d", [(16, 1, 24, 24, 128), (4, 1, 64, 8, 64), (4, 64, 64, 8, 128), (2, 900, 4, 4, 128), (2, 300, 8, 8, 64)])
def test_a_sharp_softmax(B, L, H, Hkv, d, way):
    """Logits of standard deviation sqrt(d): most of a row's weight is one key's, whose rounding no other one evens out.

    A weight that goes into the second product is bf16 (off by 2^-8 of itself at most), their sum is of the unrounded ones, and the result is bf16: with A the weighted mean of |v|,
    2^-8 A + 2^-8 |o|.  The logits are fp32 sums of d exact products: eight steps of sixteen, each off by 2^-23 of what is summed, and what a step sums inside likewise, 24 * 2^-23
    of the sum of |q k| (100 here, 160 at most): 5e-4 of each weight, above and below the line 1e-3 A, in which the exponentials' 2^-22 and the second sums are as well."""
    for seed in range(3):
        case, values = held_case(B, H, Hkv, L, d, 64, [700 - 31 * b for b in range(B)], seed=seed)
        q, k, v, table, length = values
        pools = case[1:3] if way == "codes" else (torch.nan_to_num(k), torch.nan_to_num(v))
        call = av.avsa_prefix_attn_q4 if way == "codes" else av.avsa_prefix_attn
        o, lse, ws = call(q, *pools, cu(table), cu(length), softmax_scale=1.0, want_lse=True)
        assert status(ws) == av.AVSA_OK
        for b in range(B):
            n = int(length[b])
            at = torch.arange(n, device="cuda")
            pages = cu(table)[b].long()[at // 64]
            kk, vv = (x[pages, :, at % 64].double().transpose(0, 1).repeat_interleave(H // Hkv, 0) for x in (k, v))
            x = q[b].double() @ kk.transpose(1, 2)
            assert float((q[b].double().abs() @ kk.abs().transpose(1, 2)).amax()) < 160
            w = torch.softmax(x, 2)
            want, spread = w @ vv, w @ vv.abs()
            error = (o[b].double() - want).abs()
            assert (error <= 2.0 ** -8 * (spread + want.abs()) + 1e-3 * spread).all(), (seed, b, float((error / spread).max()))
            assert (lse[b].double() - torch.logsumexp(x, 2)).abs().max() <= 1e-3
