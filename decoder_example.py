"""A small decoder whose layers are the library's attention block, its norms and its MoE layer, served as a serving loop does: prompts of
different lengths in one prefill batch, further chunks of them on what the cache holds, decode steps of one token a sequence.

    python decoder_example.py [--fp8] [--w4] [--scored]

--fp8: an 8-bit cache.  --w4: projections with 4-bit weights (the library's; else bfloat16 and plain PyTorch).  --scored: experts chosen by sigmoid
scores with a bias for the choice, out of the best groups.  Weights and token embeddings are random.  tests/test_gpu_decoder.py and
tests/test_gpu_decoder_dense.py check that decoding token by token, and prefilling in chunks, give what one prefill of the whole sequences gives.
"""
from __future__ import annotations

import math
import sys
import time
from dataclasses import dataclass
from typing import Optional

import torch

import paper_2503_09304_amd as q

DEV = "cuda:0"


@dataclass
class Shape:
    H: int = 1024           # hidden size
    Hq: int = 16            # query heads
    Hk: int = 4             # key/value heads
    D: int = 64             # elements of a head
    E: int = 8              # experts
    k: int = 2              # experts a token
    F: int = 512            # size of an expert
    layers: int = 2
    page: int = 64          # tokens of a cache page


class Layer:
    def __init__(self, s: Shape, g, cache: q.AttnCache, w4: bool):
        def rnd(*shape):
            return (torch.randn(*shape, generator=g, device=DEV) * shape[-2 if len(shape) == 2 else -1] ** -0.5).to(torch.bfloat16)

        def four_bits(cols, rows):
            """Elements of e2m1 are 3 at the root of their mean square: the scale is the power of two next to a third of cols^-0.5."""
            codes = torch.randint(0, 256, (rows, cols // 2), generator=g, device=DEV, dtype=torch.uint8)
            return q.DenseMatrix4(codes, torch.full((rows, cols // 32), 127 - round(math.log2(3 * cols ** 0.5)), dtype=torch.uint8, device=DEV))

        self.cache = cache
        project = four_bits if w4 else rnd
        self.qkv, self.out = project(s.H, (s.Hq + 2 * s.Hk) * s.D), project(s.Hq * s.D, s.H)
        self.moe = [rnd(s.H, s.E), rnd(s.E, s.F, s.H), rnd(s.E, s.F, s.H), rnd(s.E, s.H, s.F)]
        self.w = q.Context.weights(*self.moe)


def norm(x, add=None):
    """The residual stream x + add, and its norm."""
    h = torch.empty_like(x)
    if add is None:
        q.dense_norm(x, None, h)
        return x, h
    total = torch.empty_like(x)
    q.dense_norm(add, None, h, add=x, total=total)
    return total, h


def product(x, w):
    if not isinstance(w, q.DenseMatrix4):
        return x @ w
    y = torch.empty((len(x), w.rows), dtype=torch.bfloat16, device=DEV)
    q.dense_linear(x, w, y)
    return y


class Decoder:
    """Up to `max_seqs` sequences of `seq_pages` pages each; every sequence's pages are taken from the pool when they are needed."""

    def __init__(self, s: Shape, max_seqs: int, seq_pages: int, max_tokens: int, fp8: bool = False, seed: int = 1, w4: bool = False,
                 scoring: Optional[q.MoeScoring] = None):
        g = torch.Generator(device=DEV)
        g.manual_seed(seed)
        self.s, self.n_pages, self.scoring = s, max_seqs * seq_pages, scoring
        self.layers = [Layer(s, g, q.AttnCache.empty(self.n_pages, s.Hk, s.page, s.D, fp8), w4) for _ in range(s.layers)]
        f, m = q.attn_rope_frequencies(s.D)
        self.rope = q.AttnRope(torch.tensor(f, dtype=torch.float64, device=DEV), "half", m)
        self.pages = torch.full((max_seqs, seq_pages), -1, dtype=torch.int32, device=DEV)
        self.lens = [0] * max_seqs
        self.free = list(range(self.n_pages))
        self.ctx = q.Context(s.E, s.k, s.H, s.F, q.MOE_BF16, 256, max_tokens)
        self.ws = q.attn_decode_workspace(self.layers[0].cache, max_seqs, s.Hq)

    def _place(self, lens):
        """Room for lens[b] more tokens of sequence b: their sequences and positions."""
        seq, pos = [], []
        for b, n in enumerate(lens):
            have, need = -(-self.lens[b] // self.s.page), -(-(self.lens[b] + n) // self.s.page)
            if need > have:
                self.pages[b, have:need] = torch.tensor([self.free.pop() for _ in range(need - have)], dtype=torch.int32, device=DEV)
            seq += [b] * n
            pos += range(self.lens[b], self.lens[b] + n)
            self.lens[b] += n
        return (torch.tensor(v, dtype=torch.int32, device=DEV) for v in (seq, pos))

    def _qkv(self, layer, h):
        s = self.s
        return product(h, layer.qkv).view(-1, s.Hq + 2 * s.Hk, s.D).split([s.Hq, s.Hk, s.Hk], 1)

    def _moe(self, layer, h, prio):
        y = torch.empty_like(h)
        if self.scoring is None:
            self.ctx.route(h, layer.w)
        else:
            self.ctx.route_scored(h, layer.w, self.scoring)
        self.ctx.permute(prio)
        self.ctx.expert_run(h, layer.w)
        self.ctx.combine(y)
        return y

    def prefill(self, x, lens, prio):
        """The next lens[b] tokens of each sequence, packed in x [tokens, H]; prio [tokens]: 1 for latency-sensitive ones."""
        s, before = self.s, list(self.lens)
        seq, pos = self._place(lens)
        offsets = lambda n: torch.tensor([0] + list(torch.tensor(n).cumsum(0)), dtype=torch.int32, device=DEV)  # noqa: E731
        cu_q, cu_k = offsets(lens), offsets(self.lens[:len(lens)])
        whole = any(before[:len(lens)])              # somebody has keys in the cache already: all keys are read from there
        if whole:
            all_seq = torch.tensor([b for b, n in enumerate(lens) for _ in range(self.lens[b])], dtype=torch.int32, device=DEV)
            all_pos = torch.tensor([i for b, n in enumerate(lens) for i in range(self.lens[b])], dtype=torch.int32, device=DEV)
        y = None
        for layer in self.layers:
            x, h = norm(x, y)
            qq, k, v = self._qkv(layer, h)
            q_out, k_out, o = (torch.empty((len(x), h, s.D), dtype=torch.bfloat16, device=DEV) for h in (s.Hq, s.Hk, s.Hq))
            q.attn_append(layer.cache, qq, k, v, seq, pos, self.pages, self.rope, q_out, k_out)
            if whole:
                k_out, v = (torch.empty((len(all_seq), s.Hk, s.D), dtype=torch.bfloat16, device=DEV) for _ in range(2))
                q.attn_read(layer.cache, all_seq, all_pos, self.pages, k_out, v)
            q.attn_prompt(q_out, k_out, v, cu_q, cu_k, o)
            x, h = norm(x, product(o.view(len(x), -1), layer.out))
            y = self._moe(layer, h, prio)
        return x + y

    def decode(self, x, prio):
        """One token of each sequence: x [sequences, H]."""
        s, n = self.s, len(x)
        _, pos = self._place([1] * n)
        pages, lens = self.pages[:n], pos + 1
        y = None
        for layer in self.layers:
            x, h = norm(x, y)
            qq, k, v = self._qkv(layer, h)
            q_out, o = (torch.empty((n, s.Hq, s.D), dtype=torch.bfloat16, device=DEV) for _ in range(2))
            q.attn_append(layer.cache, qq, k, v, None, pos, pages, self.rope, q_out)
            q.attn_decode(layer.cache, q_out, pages, lens, o, self.ws)
            x, h = norm(x, product(o.view(n, -1), layer.out))
            y = self._moe(layer, h, prio)
        return x + y


def main(fp8: bool, w4: bool = False, scored: bool = False) -> None:
    s = Shape(H=2048, Hq=16, Hk=4, D=128, E=64, k=8, F=1408)
    prompts, steps = [300, 17, 1024, 1, 509, 128, 77, 640], 64
    g = torch.Generator(device=DEV)
    g.manual_seed(2)
    bias = torch.randn(s.E, generator=g, device=DEV) * 0.05
    m = Decoder(s, len(prompts), 32, sum(prompts), fp8, w4=w4, scoring=q.MoeScoring(choice_bias=bias, score="sigmoid", groups=8, top_groups=4, group_best=2, factor=2.5) if scored else None)
    bank = torch.randn(4096, s.H, generator=g, device=DEV).to(torch.bfloat16)
    prio = (torch.arange(sum(prompts), device=DEV) < 317).to(torch.uint8)          # the first two prompts are latency-sensitive
    torch.cuda.synchronize()
    t = time.perf_counter()
    m.prefill(bank[:sum(prompts)], prompts, prio)
    torch.cuda.synchronize()
    first = time.perf_counter() - t
    t = time.perf_counter()
    for i in range(steps):
        x = m.decode(bank[i * len(prompts):(i + 1) * len(prompts)], prio[:len(prompts)])
    torch.cuda.synchronize()
    step = (time.perf_counter() - t) / steps
    assert torch.isfinite(x).all()
    print(f"{s.layers} layers, {'fp8' if fp8 else 'bf16'} cache{', 4-bit projections' if w4 else ''}{', scored experts' if scored else ''}: prefill of {sum(prompts)} tokens in {len(prompts)} prompts {first * 1e3:.2f} ms (first call), "
          f"decode step of {len(prompts)} sequences {step * 1e3:.3f} ms")


if __name__ == "__main__":
    main(*(flag in sys.argv[1:] for flag in ("--fp8", "--w4", "--scored")))
