"""Continuing a clip: several candidates of one beginning, kept in a paged cache and thinned out as they grow.

A generation that continues a clip chunk by chunk attends to everything it has produced.  ``ClipCache`` owns the keys and values of
all layers (one pool of pages, a table of pages for each candidate) and sequences the library's calls: candidates begin as branches that
share the pages of the beginning, every step writes the new tokens of each and attends to the beginning (read once for all of them)
and to the candidate's own continuation, rejected candidates give their pages back, and the pool is compacted so that its end
can be handed on.  A chunk that takes several passes (the denoising steps of a diffusion model) begins its step once and attends in every pass: each one's
tokens replace those of the pass before.  Of ``ClipCache`` only ``check`` waits for the GPU, and whatever is given sequence numbers or counts in a list, for the
copy of it; int32 tensors on the device are taken as they are.

    python -m paper_2608_15522_b200.continuation        # a toy generator on random weights: branch, grow, prune, compact
"""
from __future__ import annotations

import argparse
import inspect
from typing import Optional, Sequence

import torch


def _takes(call, name: str) -> bool:
    """Whether a call has a parameter of this name."""
    try:
        return name in inspect.signature(call).parameters
    except (TypeError, ValueError):          # there is no such call, or it does not say
        return False


class ClipCache:
    """Keys and values of up to ``seqs`` candidates of up to ``width`` pages each, for ``layers`` layers.

    ``calls`` has the cache calls of ``binding`` (injectable, so that the sequencing can be exercised without a GPU; a stand-in whose extend takes no
    ``granted`` is taken to grant everything, one whose attention takes no ``count`` gets full steps only, and of calls that take no ``log`` the
    last one's workspace is read).  Sequence numbers are given as int32 tensors on the device, or as lists, which are copied there.

    A sequence that cannot have its pages is left as it was: a step writes nothing to it, and ``check`` says so.
    """

    def __init__(self, layers: int, heads: int, d: int, page: int, pages: int, seqs: int, width: int, device="cuda", calls=None):
        if calls is None:
            from . import binding as calls
        self.calls, self.layers, self.page = calls, layers, page
        kinds = {"extend": "avsa_cache_extend", "attention": "avsa_prefix_attn", "fork": "avsa_cache_fork", "free": "avsa_cache_free",
                 "compact": "avsa_cache_compact"}
        kinds = {kind: getattr(calls, name, None) for kind, name in kinds.items()}
        self._grants, self._counts = _takes(kinds["extend"], "granted"), _takes(kinds["attention"], "count")
        # the first error of each kind of call since the last check(), which replays of a captured step report as well
        self._errors = torch.zeros((len(kinds), 4), dtype=torch.int32, device=device)
        self._log = {kind: {"log": log} if _takes(call, "log") else {} for (kind, call), log in zip(kinds.items(), self._errors)}
        self._attention = self._log["attention"]          # what the step under way gives the attention besides
        # plane 2i: keys of layer i, plane 2i + 1: its values (what no token has been written to is never used)
        self.pool = torch.empty((2 * layers, pages, heads, page, d), dtype=torch.bfloat16, device=device)
        self.table = torch.full((seqs, width), -1, dtype=torch.int32, device=device)
        self.length = torch.zeros(seqs, dtype=torch.int32, device=device)
        self.ref = torch.zeros(pages, dtype=torch.int32, device=device)
        self._step = None          # sequences of the step under way, and the tokens that each of them was granted
        self._tokens = 0           # the most of them, where they came in lists
        self._ws = {}              # without a log: the last call's workspace, by kind

    def ints(self, x) -> torch.Tensor:
        return x if isinstance(x, torch.Tensor) else torch.tensor(x, dtype=torch.int32, device=self.table.device)

    def _state(self):
        return self.table, self.length, self.ref

    def _keep(self, kind, ws):
        if not self._log[kind]:
            self._ws[kind] = ws

    def begin_step(self, seq: Sequence[int], count: Sequence[int]) -> None:
        """Room for count[k] more tokens in sequence seq[k]; ``attend`` then writes and attends, layer by layer, with at least so many tokens (where they were
        fewer, and seq or count is a tensor, ``check`` says it)."""
        lists = not (isinstance(seq, torch.Tensor) or isinstance(count, torch.Tensor))
        self._tokens = max((c for s, c in zip(seq, count) if s >= 0), default=0) if lists else 0
        seq, count = self.ints(seq), self.ints(count)
        granted = {"granted": torch.empty_like(count)} if self._grants else {}
        self._keep("extend", self.calls.avsa_cache_extend(*self._state(), seq, count, self.page, **granted, **self._log["extend"])[3])
        self._step = seq, count = seq, granted.get("granted", count)
        if self._counts:
            self._attention = {"count": count, **self._log["attention"]}

    def attend(self, layer: int, q, k_new, v_new, prefix_pages: int = 0, causal: bool = False, softmax_scale: float = 0.0):
        """One layer of the step: the first count[k] of the L tokens of k_new/v_new [n,Hkv,L,d] go into the pages, q [n,H,L,d] attends to all tokens of its
        sequence (causal: up to its own, and rows behind the first count[k] are zero).  The first prefix_pages pages of the step's sequences are the same
        ones.  Returns o."""
        if self._step is None:
            raise ValueError("begin_step first")
        if self._tokens and k_new.shape[2] < self._tokens:
            raise ValueError(f"{k_new.shape[2]} tokens, where begin_step made room for {self._tokens}")
        seq, count = self._step
        k, v = self.pool[2 * layer], self.pool[2 * layer + 1]
        self.calls.avsa_cache_write(k_new, v_new, k, v, self.table, self.length, seq, count)
        o, _, ws = self.calls.avsa_prefix_attn(q, k, v, self.table, self.length, prefix_pages=prefix_pages, seq=seq, causal=causal,
                                               softmax_scale=softmax_scale, **self._attention)
        if "log" not in self._attention:
            self._ws["attention"] = ws
        return o

    def branch(self, parent: Sequence[int], child: Sequence[int]) -> None:
        """Sequence child[k], which is empty, becomes a copy of parent[k] that shares its full pages."""
        parent, child = self.ints(parent), self.ints(child)
        self._keep("fork", self.calls.avsa_cache_fork(self.pool, *self._state(), parent, child, **self._log["fork"])[3])

    def drop(self, seq: Sequence[int]) -> None:
        """Sequences seq give their pages back."""
        self._keep("free", self.calls.avsa_cache_free(*self._state(), self.ints(seq), **self._log["free"])[3])

    def compact(self) -> torch.Tensor:
        """The pages in use become the first ones of the pool; their number, int32 [1] on the device."""
        n_live, ws = self.calls.avsa_cache_compact(self.pool, *self._state(), **self._log["compact"])
        self._keep("compact", ws)
        return n_live

    def check(self) -> None:
        """Waits for the stream and raises for the first error of each kind of call that the device has met since the last check."""
        from .binding import AVSA_OK, AvsaError, status_string
        found = [(kind, code, tuple(detail)) for kind, (code, *detail) in zip(self._log, self._errors.tolist())]
        found += [(kind, *self.calls.avsa_read_status(ws)) for kind, ws in self._ws.items()]
        found = [(kind, code, detail) for kind, code, detail in found if code != AVSA_OK]
        if found:
            self._errors.zero_()
            (kind, code, detail), more = found[0], found[1:]
            also = "".join(f"; {kind}: {status_string(c)}, detail {d}" for kind, c, d in more)
            raise AvsaError(code, f"ClipCache: {kind}, detail {detail}{also}")


class ToyGenerator:
    """Random projections in place of a trained branch: per layer q, k and v of a chunk's tokens, attention over the cache, a residual."""

    def __init__(self, cache: ClipCache, width: int, heads: int, heads_kv: int, d: int, seed: int = 0):
        gen = torch.Generator().manual_seed(seed)
        device = cache.table.device
        self.cache, self.heads, self.heads_kv, self.d = cache, heads, heads_kv, d
        draw = lambda rows, cols: (torch.randn((rows, cols), generator=gen) / rows ** 0.5).bfloat16().to(device)
        self.layers = [(draw(width, heads * d), draw(width, heads_kv * d), draw(width, heads_kv * d), draw(heads * d, width)) for _ in range(cache.layers)]

    def step(self, x, seq, prefix_pages: int = 0, causal: bool = False):
        """x [n,L,width]: the next L tokens of sequences seq (an int32 tensor); returns what the last layer makes of them."""
        n, L, _ = x.shape
        # (the same number of tokens each: a full tensor is made on the device, where a list would be copied there)
        self.cache.begin_step(seq, torch.full((n,), L, dtype=torch.int32, device=x.device))
        for i, (wq, wk, wv, wo) in enumerate(self.layers):
            y = torch.nn.functional.layer_norm(x, x.shape[-1:])
            split = lambda t, heads: t.view(n, L, heads, self.d).transpose(1, 2)
            o = self.cache.attend(i, split(y @ wq, self.heads), split(y @ wk, self.heads_kv), split(y @ wv, self.heads_kv), prefix_pages, causal)
            x = x + o.transpose(1, 2).reshape(n, L, self.heads * self.d) @ wo
        return x


def continue_clip(layers=4, heads=16, heads_kv=4, d=128, width=1024, beginning=4096, chunk=256, audio=16, candidates=8, rounds=4, page=64, device="cuda",
                  seed=0, report=print):
    """A beginning in chunks, then rounds of: branch the best candidate, a chunk of video tokens at once and audio tokens one by one for all
    candidates, keep the one whose last state is largest, give the others' pages back; at the end compact.  Returns the cache and its pages in use."""
    span = beginning + rounds * (chunk + audio)
    pages = -(-span // page) + candidates * (-(-(chunk + audio) // page) + 2)
    cache = ClipCache(layers, heads_kv, d, page, pages, candidates + 1, -(-span // page) + 1, device)
    model = ToyGenerator(cache, width, heads, heads_kv, d, seed)
    gen = torch.Generator(device=device).manual_seed(seed)
    noise = lambda n, L: torch.randn((n, L, width), generator=gen, device=device).bfloat16()
    best, tokens = 0, 0
    for at in range(0, beginning, chunk):
        model.step(noise(1, min(chunk, beginning - at)), cache.ints([best]))
    tokens = beginning
    for r in range(rounds):
        others = [s for s in range(candidates + 1) if s != best]
        cache.branch([best] * candidates, others)
        cache.drop([best])
        seq, shared = cache.ints(others), tokens // page
        x = model.step(noise(candidates, chunk), seq, shared)[:, -1:]
        for _ in range(audio):
            x = model.step(x, seq, shared, causal=True)
        tokens += chunk + audio
        worth = x.float().square().mean((1, 2))
        keep = int(worth.argmax())          # (the decision is the host's: it waits here)
        best = others[keep]
        cache.drop([s for s in others if s != best])
        cache.check()
        report(f"round {r}: {tokens} tokens, candidate {best} kept ({worth[keep].item():.3f}), {int((cache.ref > 0).sum())} of {pages} pages in use")
    live = int(cache.compact())
    cache.check()
    report(f"compacted: pages 0..{live - 1} of {pages}")
    return cache, live


def main(argv: Optional[Sequence[str]] = None) -> None:
    p = argparse.ArgumentParser(description=continue_clip.__doc__)
    for name, value in (("layers", 4), ("heads", 16), ("heads-kv", 4), ("d", 128), ("beginning", 4096), ("chunk", 256), ("audio", 16), ("candidates", 8),
                        ("rounds", 4), ("page", 64), ("seed", 0)):
        p.add_argument(f"--{name}", type=int, default=value)
    continue_clip(**vars(p.parse_args(argv)))


if __name__ == "__main__":
    main()
