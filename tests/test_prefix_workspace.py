"""The workspace query of the attention over a paged cache at sizes out of its range (no GPU needed).

In processes of their own: a division by 0 ends them."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def run(code):
    r = subprocess.run([sys.executable, "-c", "if True:\n" + code], cwd=ROOT, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert r.returncode == 0, (r.returncode, r.stdout)


def test_rows_of_more_keys_than_32_bits_count():
    """2^32 keys wrap to 0, which the plan divides by: the query says 0 (not supported), the call AVSA_ERR_UNSUPPORTED."""
    run("""
        from paper_2608_15522_b200 import binding as av
        for b, width, prefix in ((2, 1 << 25, 1 << 25), (2, 1 << 25, 1 << 24), (1, 1 << 24, 5), (3, (1 << 25) + 3, (1 << 25) + 1)):
            assert av.avsa_prefix_attn_workspace_bytes(b, 1, 1, 1, 64, 128, width, prefix) == 0, (b, width, prefix)
        assert av.avsa_prefix_attn_workspace_bytes(2, 1, 1, 1, 64, 128, (1 << 24) - 1, (1 << 24) - 1) > 0
        assert av.avsa_prefix_attn_workspace_bytes(2, 1, 1, 1, 64, 16, (1 << 27) - 1, (1 << 27) - 1) == 0          # (a tile's end would be 2^31)
        t = av._Bf16Tensor4(1 << 24, 8192, 4096, 64)
        assert av.load_library().avsa_prefix_attn(2, 1, 1, 1, 64, 128, 10, 2, 1 << 25, t, t, t, 8192, 8192, None, 1 << 25, 0, 0.0, 1 << 25, None, 1 << 16, 1 << 40,
                                                  0) == av.AVSA_ERR_UNSUPPORTED
    """)


def test_any_sizes_are_planned_or_refused():
    """Sizes over the whole range of int, many of them at powers of two: no plan overflows into a division by 0."""
    run("""
        import random
        from paper_2608_15522_b200 import binding as av
        rng = random.Random(1)
        size = lambda: max(1, min((1 << 31) - 1, (1 << rng.randint(0, 31)) + rng.choice((-1, 0, 0, 1, rng.randint(0, 1000)))))
        planned = 0
        for _ in range(20000):
            Hkv, G = rng.choice((1, 2, 8, 24, size())), rng.choice((1, 3, 8, 128))
            H, width = min(Hkv * G, (1 << 31) - 1), size()
            planned += av.avsa_prefix_attn_workspace_bytes(rng.choice((1, 2, 16, 64, size())), H, Hkv, rng.choice((1, 7, 500, size())), rng.choice((64, 128)),
                                                           rng.choice((16, 32, 64, 128)), width, rng.choice((0, width, width // 2, rng.randint(0, width)))) > 0
        assert planned > 2000, planned
    """)
