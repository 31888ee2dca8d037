"""What a call's outputs keep alive."""
import pytest
import torch

from paper_2608_15522_b200 import binding as av
from test_paged_cache import attention_case, cu

gpu = pytest.mark.gpu

MOST = 2 << 20      # what the outputs of one call may share


@gpu
@pytest.mark.parametrize("L", [1, 200, 700])
def test_one_output_keeps_little_of_the_others(L):
    """An lse does not keep a large o, nor o a large workspace: who keeps an output keeps 2 MB in all, or what it has itself."""
    q, k, v, table, length = attention_case(2, 16, 4, L, 128, 64, [900, 800], seed=1)
    for o in av.avsa_prefix_attn(q, k, v, cu(table), cu(length), want_lse=True):
        assert o.untyped_storage().nbytes() <= max(MOST, o.numel() * o.element_size() + 512)


@gpu
@pytest.mark.parametrize("N", [1, 333, 1009])
def test_keys_that_are_kept_do_not_keep_the_queries(N):
    q, k = torch.randn((1, 32, N, 128), device="cuda").bfloat16(), torch.randn((1, 8, N, 128), device="cuda").bfloat16()
    sections = (22, 21, 21)
    pos = torch.arange(3 * N, dtype=torch.int32, device="cuda").view(N, 3)
    for x in av.avsa_rope(q, k, pos, av.avsa_rope_frequencies(sections), sections):
        assert x.untyped_storage().nbytes() <= max(MOST, x.numel() * x.element_size() + 512)


@gpu
def test_more_tokens_than_63_bits_count_are_refused():
    """32768 sequences x 32768 heads x 2^30 tokens x 64 channels are 2^66 values: no size that wrapped around is allocated, and nothing runs."""
    pool = torch.zeros((1, 32768, 16, 36), dtype=torch.uint8, device="cuda")
    table, length = torch.zeros((32768, 1), dtype=torch.int32, device="cuda"), torch.zeros(32768, dtype=torch.int32, device="cuda")
    with pytest.raises(RuntimeError):
        av.avsa_cache_read_q4(pool, pool, table, length, 1 << 30)


@gpu
@pytest.mark.parametrize("tokens", [1, 300, 3000])
def test_keys_that_are_kept_keep_no_more_than_the_values(tokens):
    """Two outputs of one size: as much again at most, and nothing of the other one's beyond 16 MB."""
    pool = torch.zeros((400, 8, 16, 72), dtype=torch.uint8, device="cuda")
    table, length = torch.arange(400, dtype=torch.int32, device="cuda").view(2, 200), torch.full((2,), 3000, dtype=torch.int32, device="cuda")
    for x in av.avsa_cache_read_q4(pool, pool, table, length, tokens):
        own = x.numel() * x.element_size()
        assert x.untyped_storage().nbytes() <= (own if 2 * own > 16 << 20 else 2 * own) + 1024
