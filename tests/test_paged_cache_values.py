"""Attention over the paged cache: infinities in keys that are seen."""
import math
import random

import pytest
import torch

from test_cache_steps import WAYS
from test_paged_cache import attention_case, check_on_gpu, lengths_behind

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
