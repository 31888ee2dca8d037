"""Plain statement of the cache held in 4 bits and of rotary positions, in 64 bits (torch, on whatever device the arguments are).

A token of a head is d/2 bytes of codes and d/32 bf16 scales; 16 tokens keep their codes together and their scales behind them.
"""
from __future__ import annotations

import math

import torch

GROUP, BLOCK = 32, 16


def quantise(x):
    """x [..., d] -> (codes -7..7, scales [..., d/32]) in fp64; a scale of NaN: the group has something that is not finite, or 2^125 and more."""
    g = x.double().unflatten(-1, (-1, GROUP))
    top = g.abs().amax(-1)
    part, power = torch.frexp(torch.where(torch.isfinite(top), top, 0.0) / 7)          # part in [1/2, 1)
    scale = torch.ldexp(torch.floor(part * 32 + 0.5) / 32, power)                        # five significant bits, halfway up
    scale = torch.where(top < 2.0 ** -100, 0.0, scale)
    scale = torch.where(top < 2.0 ** 125, scale, math.nan)
    safe = torch.where(scale > 0, scale, 1.0)[..., None]
    code = torch.where((scale > 0)[..., None], torch.round(torch.where(torch.isfinite(g), g, 0.0) / safe), 0.0)      # halfway to even
    return code.flatten(-2), scale


def values(code, scale):
    return (code.unflatten(-1, (-1, GROUP)) * scale[..., None]).flatten(-2)


def pack(code, scale):
    """Codes [pages,Hkv,page,d], scales [pages,Hkv,page,d/32] -> uint8 [pages,Hkv,page,d/2 + d/16]."""
    pages, heads, page, d = code.shape
    u = (code.long() + 8).unflatten(-1, (-1, 8))
    word = sum(u[..., c] << (4 * (c // 2) + 16 * (c % 2)) for c in range(8))
    codes = torch.stack([word >> (8 * b) & 255 for b in range(4)], -1).flatten(-2)
    bits = scale.to(torch.bfloat16).view(torch.int16).long()
    scales = torch.stack([bits & 255, bits >> 8 & 255], -1).flatten(-2)
    parts = [t.unflatten(2, (-1, BLOCK)).flatten(3) for t in (codes, scales)]
    return torch.cat(parts, -1).reshape(pages, heads, page, d // 2 + d // 16).to(torch.uint8)


def unpack(pool, d):
    """The other way: (codes, scales) in fp64."""
    pages, heads, page, _ = pool.shape
    block = pool.reshape(pages, heads, page // BLOCK, BLOCK * (d // 2 + d // 16)).long()
    codes = block[..., :BLOCK * d // 2].unflatten(-1, (BLOCK, d // 8, 4)).flatten(2, 3)
    word = sum(codes[..., b] << (8 * b) for b in range(4))
    code = torch.stack([(word >> (4 * (c // 2) + 16 * (c % 2)) & 15) - 8 for c in range(8)], -1).flatten(-2)
    scales = block[..., BLOCK * d // 2:].unflatten(-1, (BLOCK, d // GROUP, 2)).flatten(2, 3)
    bits = scales[..., 0] | scales[..., 1] << 8
    return code.double(), torch.where(bits > 32767, bits - 65536, bits).to(torch.int16).view(torch.bfloat16).double()


def rope(x, pos, freq, sections, halves=False, inverse=False):
    """x [B,H,N,d] -> fp64; pos [B,N,axes] or [N,axes], freq [d/2] turns."""
    d = x.shape[-1]
    pos = pos.double() if pos.dim() == 3 else pos.double()[None]
    axis = [i for i, n in enumerate(sections) for _ in range(n)]
    turns = torch.stack([torch.remainder(pos[:, :, a] * freq[i].double(), 1.0) for i, a in enumerate(axis)], -1)[:, None]
    angle = turns * (2 * math.pi) * (-1 if inverse else 1)
    a, b = (x.double()[..., :d // 2], x.double()[..., d // 2:]) if halves else (x.double()[..., 0::2], x.double()[..., 1::2])
    y = (a * torch.cos(angle) - b * torch.sin(angle), a * torch.sin(angle) + b * torch.cos(angle))
    return torch.cat(y, -1) if halves else torch.stack(y, -1).flatten(-2)
