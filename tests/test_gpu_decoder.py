"""decoder_example.py: the attention calls and the MoE layer together (-m gpu).

One prefill of whole sequences, prefill in chunks and decoding token by token compute the same hidden states by different kernels: other orders of
sums, weights of the softmax rounded relative to other maxima.  Each of a layer's 10 roundings to bf16 that may differ (qkv, rotation, weights, output,
projection, residual, norm, activation, expert sum, residual) leaves RHO = 1.66e-3 of a value's RMS; two paths of two layers that differ in all of them
are sqrt(2 * 2 * 10) * RHO = 1.05e-2 apart, and the bar is three times that.  All experts are chosen (k = E), so that no choice can flip."""
import math

import pytest
import torch

from decoder_example import DEV, Decoder, Shape, main
from gpu_util import RHO

pytestmark = pytest.mark.gpu
BAR = 3 * math.sqrt(2 * 2 * 10) * RHO


def run(plan, lens, bank, fp8):
    """Hidden states of every sequence's tokens, by `plan`: per call the tokens of each sequence; a call of one token each decodes."""
    s = Shape(H=256, Hq=8, Hk=2, D=32, E=4, k=4, F=128, page=16)
    m = Decoder(s, len(lens), 8, 512, fp8)
    at, got = [0] * len(lens), [[] for _ in lens]
    for counts, decode in plan:
        x = torch.cat([bank[b, at[b]:at[b] + n] for b, n in enumerate(counts)])
        prio = (torch.arange(len(x), device=DEV) % 3 == 0).to(torch.uint8)
        y = m.decode(x, prio) if decode else m.prefill(x, counts, prio)
        for b, part in enumerate(y.split(counts)):
            got[b].append(part)
            at[b] += counts[b]
    assert at == lens
    return torch.cat([torch.cat(v) for v in got]).double()


@pytest.mark.parametrize("fp8", [False, True])
def test_chunks_and_single_tokens_are_one_prefill(fp8):
    lens = [70, 33, 19, 100]
    g = torch.Generator(device=DEV)
    g.manual_seed(5)
    bank = torch.randn(len(lens), 128, 256, generator=g, device=DEV).to(torch.bfloat16)
    # With an fp8 cache a whole prefill attends to the keys before they are rounded; a first empty-handed call of one token makes it read them back.
    first = [([1] * 4, False)] if fp8 else []
    used = 1 if fp8 else 0
    whole = run(first + [([n - used for n in lens], False)], lens, bank, fp8)
    short = [n - 12 for n in lens]
    cut = [n // 2 for n in short]
    chunks = run(first + [([n - used for n in cut], False), ([n - c for n, c in zip(short, cut)], False), ([12] * 4, False)], lens, bank, fp8)
    tokens = run(first + [([n - used for n in short], False)] + [([1] * 4, True)] * 12, lens, bank, fp8)
    size = whole.norm()
    assert float((chunks - whole).norm() / size) < BAR and float((tokens - whole).norm() / size) < BAR
    rows = whole.norm(dim=1)
    assert float(((tokens - whole).norm(dim=1) / rows).max()) < 3 * BAR


@pytest.mark.parametrize("fp8", [False, True])
def test_the_example_runs(fp8, capsys):
    main(fp8)
    assert "decode step" in capsys.readouterr().out
