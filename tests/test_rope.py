"""Rotary positions with several axes, against the plain statement in oracle/q4_oracle.py.

Bound of an output y of the pair (a, b): half a step of bf16, 2^-8 |y|, and what fp32 leaves of y: the fraction of a turn to 2^-26 (2^-23.3 of a radian), sine and cosine
to 2 units of 2^-24, two products and a sum, together below 2^-21 (|a| + |b|).
"""
import ctypes
import math

import pytest
import torch

from oracle import q4_oracle as orc
from paper_2608_15522_b200 import binding as av

gpu = pytest.mark.gpu


def check(got, x, pos, freq, sections, halves, inverse):
    want = orc.rope(x, pos, freq, sections, halves, inverse)
    a = x.double().abs()
    a, b = (a[..., :a.shape[-1] // 2], a[..., a.shape[-1] // 2:]) if halves else (a[..., 0::2], a[..., 1::2])
    size = torch.cat((a + b, a + b), -1) if halves else (a + b).repeat_interleave(2, -1)
    assert got.dtype == torch.bfloat16 and got.shape == x.shape
    excess = (got.double() - want).abs() - (2.0 ** -8 * want.abs() + 2.0 ** -21 * size)
    assert excess.max() <= 0, excess.max()


def positions(B, N, axes, far, seed=0):
    gen = torch.Generator().manual_seed(seed)
    return torch.randint(-far, far + 1, (B, N, axes), generator=gen, dtype=torch.int32)


SECTIONS = {(64, 1): (32,), (64, 2): (20, 12), (64, 3): (12, 10, 10), (64, 4): (8, 0, 23, 1), (128, 1): (64,), (128, 2): (0, 64), (128, 3): (22, 21, 21), (128, 4): (1, 61, 1, 1)}


# ------------------------------------------------------------------------------------------------ the oracle itself, refusals
def test_oracle_closed_forms():
    """A quarter of a turn, a whole one, the other axis alone, and back again."""
    x = torch.randn(1, 2, 3, 64).double()
    freq = torch.full((32,), 0.25, dtype=torch.float64)
    pos = torch.tensor([[1, 0], [4, 1], [0, 0]])
    y = orc.rope(x, pos, freq, (30, 2))
    assert torch.allclose(y[:, :, 0, 0:60:2], -x[:, :, 0, 1:60:2], atol=1e-12) and torch.allclose(y[:, :, 0, 1:60:2], x[:, :, 0, 0:60:2], atol=1e-12)
    assert torch.allclose(y[:, :, 0, 60:], x[:, :, 0, 60:]) and torch.allclose(y[:, :, 1, :60], x[:, :, 1, :60], atol=1e-12)
    assert torch.allclose(y[:, :, 1, 60::2], -x[:, :, 1, 61::2], atol=1e-12) and torch.equal(y[:, :, 2], x[:, :, 2])
    h = orc.rope(x, pos, freq, (30, 2), halves=True)
    assert torch.allclose(h[:, :, 0, :30], -x[:, :, 0, 32:62], atol=1e-12)
    assert torch.allclose(orc.rope(h, pos, freq, (30, 2), halves=True, inverse=True), x, atol=1e-12)


def test_frequencies():
    f = av.avsa_rope_frequencies((22, 21, 21), device="cpu")
    assert f.dtype == torch.float64 and f.shape == (64,)
    assert f[0] == f[22] == f[43] == 1 / (2 * math.pi)
    assert math.isclose(f[1], 10000.0 ** (-2 / 44) / (2 * math.pi)) and math.isclose(f[63], 10000.0 ** (-40 / 42) / (2 * math.pi))


_T = av._Bf16Tensor4(1 << 20, 64 * 64 * 4, 64 * 64, 64)


@pytest.mark.parametrize("change,want", [
    (dict(B=-1), 1), (dict(N=-1), 1), (dict(H=-1), 1), (dict(d=96), 2), (dict(d=32), 2), (dict(axes=0), 1), (dict(axes=5, sections=(8, 8, 8, 4, 4)), 2),
    (dict(sections=(32, 1)), 1), (dict(sections=(30, 1)), 1), (dict(sections=(33, -1)), 1), (dict(sections=None), 1), (dict(flags=4), 1), (dict(pos=None), 1),
    (dict(pos=(1 << 20) + 2), 1), (dict(freq=(1 << 20) + 4), 1), (dict(freq=None), 1), (dict(pos_stride=-1), 1), (dict(B=65536), 2),
    (dict(B=65535, N=1 << 20), 2), (dict(q=av._Bf16Tensor4(None, 16384, 4096, 64)), 1), (dict(k_out=av._Bf16Tensor4((1 << 20) + 8, 16384, 4096, 64)), 1),
    (dict(q=av._Bf16Tensor4(1 << 20, 16384, 4096, 60)), 1), (dict(q_out=av._Bf16Tensor4(1 << 20, 16384, 4096, 128)), 1),       # in place with other strides
    (dict(B=0), 0), (dict(N=0), 0), (dict(H=0, Hk=0), 0)])
def test_refusals(change, want):
    a = {**dict(B=2, H=4, Hk=4, N=64, d=64, q=_T, k=_T, q_out=_T, k_out=_T, pos=1 << 20, pos_stride=0, axes=2, sections=(16, 16), freq=1 << 20, flags=0), **change}
    sections = None if a["sections"] is None else (ctypes.c_int * len(a["sections"]))(*a["sections"])
    got = av.load_library().avsa_rope(a["B"], a["H"], a["Hk"], a["N"], a["d"], a["q"], a["k"], a["q_out"], a["k_out"], a["pos"], a["pos_stride"], a["axes"],
                                      sections, a["freq"], a["flags"], 0)
    assert got == want


def test_wrapper_takes_device_tensors_only():
    x = torch.zeros((1, 2, 3, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        av.avsa_rope(x, None, torch.zeros((3, 1), dtype=torch.int32), torch.zeros(32, dtype=torch.float64), (32,))


# ------------------------------------------------------------------------------------------------ on the GPU
@gpu
@pytest.mark.parametrize("halves", [False, True])
@pytest.mark.parametrize("d,axes", list(SECTIONS))
@pytest.mark.parametrize("B,H,Hk,N", [(1, 1, 1, 1), (2, 24, 24, 1), (1, 24, 8, 77), (3, 5, 2, 130), (1, 16, 0, 1009), (7, 9, 9, 333)])
def test_rotation(B, H, Hk, N, d, axes, halves):
    gen = torch.Generator().manual_seed(N + d)
    draw = lambda heads: torch.randn((B, N, heads, d), generator=gen).bfloat16().cuda().transpose(1, 2)
    q, k = draw(H), draw(Hk) if Hk else None
    pos, freq = positions(B, N, axes, 100000, N).cuda(), av.avsa_rope_frequencies(SECTIONS[d, axes])
    for inverse in (False, True):
        got = av.avsa_rope(q, k, pos, freq, SECTIONS[d, axes], halves=halves, inverse=inverse)
        assert got[0].stride() == q.stride()
        for y, x in zip(got, (q, k)):
            if x is not None:
                check(y, x, pos, freq, SECTIONS[d, axes], halves, inverse)
        assert (got[1] is None) == (k is None)


@gpu
@pytest.mark.parametrize("halves", [False, True])
def test_positions_over_the_whole_range_of_int(halves):
    """Angles of 2^31 steps, both signs: turns are counted in 64 bits."""
    x = torch.randn((1, 2, 6, 128), device="cuda").bfloat16()
    pos = torch.tensor([[2 ** 31 - 1], [-2 ** 31], [0], [1], [1 << 24], [-(1 << 24) - 1]], dtype=torch.int32, device="cuda")
    freq = av.avsa_rope_frequencies((64,))
    y, _ = av.avsa_rope(x, None, pos, freq, (64,), halves=halves)
    # (here fp64 itself leaves 2^31 / (2 pi) * 2^-53 of a turn, 2^-22 of a radian, in both)
    want = orc.rope(x, pos, freq, (64,), halves)
    assert ((y.double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -19 * x.double().abs().amax()).all()
    assert torch.equal(y[:, :, 2], x[:, :, 2])


@gpu
@pytest.mark.parametrize("halves", [False, True])
def test_in_place_slices_and_shared_positions(halves):
    """q and k as slices of one projection [B,N,(q,k,v),H,d], rotated where they are; positions that all batch entries share, and their own ones, equal."""
    B, N, H, d = 3, 50, 6, 64
    qkv = torch.randn((B, N, 3, H, d), device="cuda").bfloat16()
    before = qkv.clone()
    q, k = (qkv[:, :, i].transpose(1, 2) for i in range(2))
    pos, freq = positions(1, N, 2, 500)[0].cuda(), av.avsa_rope_frequencies((16, 16))
    fresh = av.avsa_rope(q, k, pos, freq, (16, 16), halves=halves)
    assert fresh[0].stride() == fresh[1].stride() == (N * H * d, d, H * d, 1)          # in the order of q's dimensions, without the gaps
    own = av.avsa_rope(q, k, pos.repeat(B, 1, 1), freq, (16, 16), halves=halves)
    got = av.avsa_rope(q, k, pos, freq, (16, 16), halves=halves, q_out=q, k_out=k)
    assert got[0] is q and got[1] is k
    for y, f, o, i in zip(got, fresh, own, range(2)):
        check(y, before[:, :, i].transpose(1, 2), pos, freq, (16, 16), halves, False)
        assert torch.equal(y, f) and torch.equal(y, o)
    assert torch.equal(qkv[:, :, 2], before[:, :, 2])


@gpu
def test_pairs_that_never_turn_and_values_that_are_not_finite():
    """A frequency of 0 leaves its channels as they are, bit for bit; an infinity or NaN stays in its pair."""
    x = torch.randn((1, 3, 20, 128), device="cuda").bfloat16()
    freq = av.avsa_rope_frequencies((64,))
    freq[40:] = 0.0
    pos = torch.arange(20, dtype=torch.int32, device="cuda")[:, None]
    y, _ = av.avsa_rope(x, None, pos, freq, (64,))
    assert torch.equal(y[..., 80:], x[..., 80:]) and not torch.equal(y[..., :80], x[..., :80])
    z = x.clone()
    z[0, 1, 7, 10], z[0, 2, 3, 21] = float("inf"), float("nan")
    w, _ = av.avsa_rope(z, None, pos, freq, (64,))
    differ = (w.view(torch.int16) != y.view(torch.int16)).nonzero().tolist()
    assert {tuple(i[:3]) + (i[3] // 2,) for i in differ} == {(0, 1, 7, 5), (0, 2, 3, 10)} and torch.isnan(w[0, 2, 3, 20:22]).all()


@gpu
@pytest.mark.parametrize("halves", [False, True])
def test_inverse_is_the_gradient(halves):
    """The rotation is linear: its differences along the unit vectors are the columns of a matrix, whose transpose the inverse is."""
    d = 64
    e = torch.eye(d, device="cuda").bfloat16().reshape(d, 1, 1, d)
    pos, freq = torch.tensor([[3, 9]], dtype=torch.int32, device="cuda"), av.avsa_rope_frequencies((20, 12))
    step = lambda x, **kw: av.avsa_rope(x, None, pos, freq, (20, 12), halves=halves, **kw)[0].double().reshape(d, d)
    jacobian = (step(e) - step(-e)) / 2            # [input channel, output channel]
    back = step(e, inverse=True)                   # row i: the gradient of output channel i
    # both hold sines and cosines rounded to bf16 (2^-9 at most, as their magnitudes are below 1), from fp32 values that agree to 2^-22
    assert (jacobian.T - back).abs().max() <= 2 * 2.0 ** -9 + 2.0 ** -21
    want = orc.rope(e, pos, freq, (20, 12), halves).reshape(d, d)
    assert (jacobian - want).abs().max() <= 2.0 ** -9 + 2.0 ** -21


@gpu
def test_streams_graphs_and_reproduction():
    q, k = torch.randn((2, 4, 300, 128), device="cuda").bfloat16(), torch.randn((2, 2, 300, 128), device="cuda").bfloat16()
    pos, freq = positions(2, 300, 3, 4000).cuda(), av.avsa_rope_frequencies((22, 21, 21))
    want = av.avsa_rope(q, k, pos, freq, (22, 21, 21))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = av.avsa_rope(q, k, pos, freq, (22, 21, 21))
    torch.cuda.current_stream().wait_stream(side)
    out = [torch.empty_like(x) for x in (q, k)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        av.avsa_rope(q, k, pos, freq, (22, 21, 21), q_out=out[0], k_out=out[1])
    graph.replay()
    for a, b, c in zip(want, other, out):
        assert torch.equal(a, b) and torch.equal(a, c)


@gpu
def test_wrapper_refusals():
    q, freq = torch.zeros((1, 2, 5, 64), device="cuda").bfloat16(), av.avsa_rope_frequencies((32,))
    pos = torch.zeros((5, 1), dtype=torch.int32, device="cuda")
    k = lambda *s: torch.zeros(s, device="cuda").bfloat16()
    for bad in (dict(pos=pos.long()), dict(pos=pos[:4]), dict(pos=pos.repeat(2, 1, 1)), dict(freq=freq.float()), dict(freq=freq[:31]), dict(sections=(16, 16)),
                dict(sections=(64,)), dict(k=k(1, 2, 4, 64)), dict(k=k(1, 2, 5, 128)), dict(q=q.float()), dict(q_out=k(1, 2, 5, 128)), dict(k_out=k(1, 2, 5, 64)),
                dict(pos=torch.zeros((5, 2), dtype=torch.int32, device="cuda")[:, :1])):
        with pytest.raises(ValueError):
            av.avsa_rope(**{**dict(q=q, k=None, pos=pos, freq=freq, sections=(32,)), **bad})
    with pytest.raises(av.AvsaError):
        av.avsa_rope(q, None, pos, freq, (31,))
    with pytest.raises(av.AvsaError):
        av.avsa_rope(q.expand(4, 2, 5, 64), None, pos, freq, (32,))          # (a batch axis without a stride)
