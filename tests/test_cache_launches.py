"""Launches of the paged cache's calls that one CTA takes alone, by the shared memory that they ask for; lengths of 31 bits."""
import os
import subprocess
import sys
import threading

import pytest
import torch

from paper_2608_15522_b200 import binding as av

gpu = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

# Every second page is in use: as many moves as a pool can have, and plenty of free pages.
POOLS = """if True:
    import numpy as np, torch
    from oracle import cache_oracle as orc
    from paper_2608_15522_b200 import binding as av
    cu = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")

    def state(pages, seqs, width, held):
        ref, table, length = np.zeros(pages, np.int32), np.full((seqs, width), -1, np.int32), np.zeros(seqs, np.int32)
        table[0, :len(held)], length[0], ref[held] = held, 16 * len(held) - 5, 1
        return table, length, ref

    def same(got, want, what):
        for g, w in zip(got, want):
            assert np.array_equal(g.cpu().numpy(), w), what

    # 48 KB of shared memory are a CTA's without asking, the kernels' own arrays of 1 KB among them
    for pages in (8020, 8022, 8192, 8194, 16384):
        table, length, ref = state(pages, 1, pages // 2, list(range(1, pages, 2)))
        pool = torch.arange(pages, device="cuda").to(torch.int16).view(1, pages, 1, 1, 1).expand(1, pages, 1, 16, 64).contiguous().view(torch.bfloat16)
        t, n, r = cu(table), cu(length), cu(ref)
        live, ws = av.avsa_cache_compact(pool, t, n, r)
        want_table, want_ref, want_live, moves = orc.compact(table, ref)
        assert int(live) == want_live and av.avsa_read_status(ws)[0] == 0, pages
        same((t, r), (want_table, want_ref), pages)
        content = np.arange(pages)
        for a, b in moves:
            content[b] = a
        assert np.array_equal(pool.view(torch.int16)[0, :, 0, 7, 63].cpu().numpy(), content.astype(np.int16)), pages
    for pages in (12012, 12013, 12268, 12269, 16380):
        table, length, ref = state(pages, 4, 9, [5, 3])
        *want, refused = orc.extend(table, length, ref, [0, 2], [40, 3], 16)
        got = av.avsa_cache_extend(*map(cu, (table, length, ref)), ints([0, 2]), ints([40, 3]), 16)
        assert not refused and av.avsa_read_status(got[3])[0] == 0, pages
        same(got, want, pages)
        pool = torch.zeros((1, pages, 1, 16, 64), dtype=torch.bfloat16, device="cuda")
        *want, moves, refused = orc.fork(table, length, ref, [0, 0], [2, 3], 16)
        got = av.avsa_cache_fork(pool, *map(cu, (table, length, ref)), ints([0, 0]), ints([2, 3]))
        assert not refused and av.avsa_read_status(got[3])[0] == 0, pages
        same(got, want, pages)
"""


@gpu
def test_pools_around_the_shared_memory_that_needs_no_asking():
    """In a process of its own, smallest first: a larger call before would leave the limit raised."""
    r = subprocess.run([sys.executable, "-c", POOLS], cwd=ROOT, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert r.returncode == 0, r.stdout


@gpu
def test_threads_with_pools_of_different_sizes():
    """Two threads, streams and workspaces; what the kernels of both need lies above what they get without asking."""
    refused = []

    def work(pages):
        ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
        with torch.cuda.stream(torch.cuda.Stream()):
            table, length, ref = torch.full((2, 4), -1, dtype=torch.int32, device="cuda"), ints([0, 0]), torch.zeros(pages, dtype=torch.int32, device="cuda")
            pool = torch.zeros((1, pages, 1, 16, 64), dtype=torch.bfloat16, device="cuda")
            seq, count = ints([0]), ints([0])
            try:
                for _ in range(4000):
                    av.avsa_cache_extend(table, length, ref, seq, count, 16)
                    av.avsa_cache_fork(pool, table, length, ref, seq, seq)
                    av.avsa_cache_compact(pool, table, length, ref)
            except av.AvsaError as e:
                refused.append((pages, str(e)))
            torch.cuda.current_stream().synchronize()

    threads = [threading.Thread(target=work, args=(pages,)) for pages in (12500, 16000)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not refused


@gpu
def test_extend_lengths_up_to_31_bits():
    """A row that could hold 2^31 tokens: pages are counted without wrapping, what a length cannot say is refused."""
    page, width, top = 128, 1 << 24, (1 << 31) - 1
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    table = torch.full((2, width), -1, dtype=torch.int32, device="cuda")
    for length, count, want, code in (([top - 5, 0], [3, 1], [top - 2, 1], av.AVSA_OK),
                                      ([top - 128, 0], [2, 1], [top - 126, 1], av.AVSA_OK),          # one page more
                                      ([top - 5, 0], [6, 1], [top - 5, 1], av.AVSA_ERR_NO_PAGES),
                                      ([0, 0], [top, 1], [0, 0], av.AVSA_ERR_NO_PAGES)):             # 2^24 pages: there are four, and who is behind gets none
        table.fill_(-1)
        n, ref = ints(length), ints([0, 1, 0, 0])
        ws = av.avsa_cache_extend(table, n, ref, ints([0, 1]), ints(count), page)[3]
        assert av.avsa_read_status(ws)[0] == code and n.tolist() == want
        crossing = length[0] == top - 128
        assert int(table[0, -1]) == (0 if crossing else -1)
        assert int(table[1, 0]) == (-1 if want[1] == 0 else 2 if crossing else 0)
        assert int((ref > 0).sum()) == 1 + int(crossing) + int(want[1] == 1)
