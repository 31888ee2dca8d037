"""Attention over the paged cache: infinities and NaN in keys and values that are seen, and tables with room."""
import math
import random

import numpy as np
import pytest
import torch

from oracle import cache_oracle as orc
from paper_2608_15522_b200 import binding as av
from parity_bars import close_lse, close_o
from test_cache_steps import WAYS
from test_paged_cache import attention_case, check_on_gpu, cu, lengths_behind, status

pytestmark = pytest.mark.gpu


def case(B, H, Hkv, L, d, page, tokens, most, **kw):
    shared = tokens // page
    lengths = list(most) if isinstance(most, tuple) else lengths_behind(random.Random(B + d), B, shared, page, most)
    return attention_case(B, H, Hkv, L, d, page, lengths, shared=shared, seed=B, q_layout="blhd", **kw), shared


def tokens_at(table, length, page, positions):
    """Pages and places of positions of each sequence, those that it has: a list a sequence."""
    return [[(int(table[s, t // page]), t % page) for t in positions if t < n] for s, n in enumerate(length)]


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B,L,H,Hkv,page,tokens,most", WAYS)
def test_first_keys_of_no_weight(B, L, H, Hkv, page, tokens, most, d, causal):
    """The logits of the first 300 keys are -inf, those behind them so far below 0 that only a reference of their own gives them a weight."""
    (q, k, v, table, length), shared = case(B, H, Hkv, L, d, page, tokens, most, poison=False)
    one = torch.zeros(d, device="cuda")
    one[0] = 1.0
    q = (q.float() * (1 - one) + one).bfloat16()
    k = k.clone()
    k[..., 0] = -300.0 * math.sqrt(d)
    first = {at for row in tokens_at(table, length, page, range(300)) for at in row}
    for p, i in first:
        k[p, :, i] = 0.0
        k[p, :, i, 0] = -math.inf
    check_on_gpu(q, k, v, table, length, "first keys of no weight", prefix_pages=shared, causal=causal)


def exact(q, k, v, table, length, causal):
    """softmax by its definition in 64 bits: exp(x - max) over its sum, NaN where the maximum is +inf; an empty row is 0 and -inf."""
    B, H, L, d = q.shape
    page, group = k.shape[2], H // k.shape[1]
    lim = orc.limits(length, range(B), B, L, causal)
    o, lse = torch.zeros((B, H, L, d), dtype=torch.float64, device="cuda"), torch.full((B, H, L), -math.inf, dtype=torch.float64, device="cuda")
    for b in range(B):
        at = torch.arange(int(length[b]), device="cuda")
        if len(at) == 0:
            continue
        pages = cu(table)[b].long()[at // page]
        kk, vv = (x[pages, :, at % page].double().transpose(0, 1) for x in (k, v))
        x = (q[b].double().reshape(-1, group * L, d) @ kk.transpose(1, 2) * d ** -0.5).masked_fill_(at >= cu(lim[b]).repeat(group)[:, None], -math.inf)
        top = x.amax(2, keepdim=True)
        top = torch.where(torch.isneginf(top), 0.0, top)
        w = torch.exp(x - top)
        z = w.sum(2, keepdim=True)
        o[b] = torch.where(z == 0, 0.0, (w @ vv) / z).reshape(H, L, d)
        lse[b] = (top + torch.log(z))[..., 0].reshape(H, L)
    return o, lse


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("what", ["nan", "inf", "-inf"])
@pytest.mark.parametrize("B,L,H,Hkv,page,tokens,most", WAYS)
def test_keys_that_are_no_numbers(B, L, H, Hkv, page, tokens, most, what, d, causal):
    """One key of one key head: rows that see it and whose logit is NaN or +inf become NaN, -inf weighs nothing, and no other row notices."""
    (q, k, v, table, length), shared = case(B, H, Hkv, L, d, page, tokens, most, poison=False)
    k = k.clone()
    s = int(np.argmax(length))
    p, i = int(table[s, 40 // page]), 40 % page
    k[p, Hkv - 1, i] = 0.0
    k[p, Hkv - 1, i, 0] = float(what)
    o, lse, ws = av.avsa_prefix_attn(q, k, v, cu(table), cu(length), prefix_pages=shared, causal=causal, want_lse=True)
    assert status(ws) == av.AVSA_OK
    want, want_lse = exact(q, k, v, table, length, causal)
    bad = torch.isnan(want).any(-1)
    assert bool(bad.any()) and torch.equal(torch.isnan(o).any(-1), bad) and torch.isnan(o[bad]).all()
    empty, good = torch.isneginf(want_lse), ~bad & ~torch.isneginf(want_lse)
    assert torch.equal(torch.isneginf(lse), empty) and (o[empty] == 0).all() and not torch.isfinite(lse[bad]).any()
    close_o(o.double()[good].cpu().numpy(), want[good].cpu().numpy(), what)
    close_lse(lse.double()[good].cpu().numpy(), want_lse[good].cpu().numpy(), what)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("what", ["nan", "inf"])
@pytest.mark.parametrize("B,L,H,Hkv,page,tokens,most", WAYS)
def test_values_that_are_no_numbers(B, L, H, Hkv, page, tokens, most, what, d):
    """One value of a token that all see: its channel, and no other."""
    (q, k, v, table, length), shared = case(B, H, Hkv, L, d, page, tokens, most, poison=False)
    v = v.clone()
    s = int(np.argmax(length))
    p, i = int(table[s, 10 // page]), 10 % page
    v[p, 0, i, 5] = float(what)
    sees = torch.tensor([int(table[b, 10 // page]) == p and int(length[b]) > 10 for b in range(B)], device="cuda")
    plain = v.clone()
    plain[p, 0, i, 5] = 0.0
    o, lse, _ = av.avsa_prefix_attn(q, k, v, cu(table), cu(length), prefix_pages=shared, want_lse=True)
    o0, lse0, _ = av.avsa_prefix_attn(q, k, plain, cu(table), cu(length), prefix_pages=shared, want_lse=True)
    group = H // Hkv
    hit = torch.zeros_like(o, dtype=torch.bool)
    hit[sees, :group, :, 5] = True
    got = torch.isnan(o) if what == "nan" else torch.isinf(o)
    assert torch.equal(got, hit) and torch.equal(o[~hit], o0[~hit]) and torch.equal(lse, lse0)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("room", [1, 64, 512])
@pytest.mark.parametrize("B,L,H,Hkv,page,tokens,most", WAYS)
def test_tables_with_room(B, L, H, Hkv, page, tokens, most, room, d, causal):
    """Rows far longer than what the sequences hold, as a cache that grows has them."""
    longest = max(most) if isinstance(most, tuple) else tokens + most
    c, shared = case(B, H, Hkv, L, d, page, tokens, most, width=-(-longest // page) + room)
    check_on_gpu(*c, f"{room} pages of room", prefix_pages=shared, causal=causal)
