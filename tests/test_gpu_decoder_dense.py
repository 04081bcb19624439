"""decoder_example.py with the dense calls: norms, 4-bit projections, experts by scores (-m gpu).

The same hidden states by different kernels, as in test_gpu_decoder.py, with its bar: each of a layer's 10 roundings to bf16 that may differ leaves RHO of a
value's RMS, two paths of two layers are sqrt(2 * 2 * 10) * RHO apart, and the bar is three times that.  4-bit weights are exact in bf16.  All experts are
chosen (k = E), so that no choice can flip."""
import math

import pytest
import torch

from decoder_example import DEV, Decoder, Shape, main
from gpu_util import RHO

import paper_2503_09304_amd as q

pytestmark = pytest.mark.gpu
BAR = 3 * math.sqrt(2 * 2 * 10) * RHO
SHAPE = Shape(H=256, Hq=8, Hk=2, D=32, E=4, k=4, F=128, page=16)
LENS = [70, 33, 19, 100]


def inputs():
    g = torch.Generator(device=DEV)
    g.manual_seed(5)
    return torch.randn(len(LENS), 128, SHAPE.H, generator=g, device=DEV).to(torch.bfloat16)


def run(m, plan, bank):
    """Hidden states of every sequence's tokens; per call of `plan` the tokens of each sequence, a call of one token each decodes."""
    at, got = [0] * len(LENS), [[] for _ in LENS]
    for counts, decode in plan:
        x = torch.cat([bank[b, at[b]:at[b] + n] for b, n in enumerate(counts)])
        kept = x.clone()
        prio = (torch.arange(len(x), device=DEV) % 3 == 0).to(torch.uint8)
        y = m.decode(x, prio) if decode else m.prefill(x, counts, prio)
        assert torch.equal(x, kept)
        for b, part in enumerate(y.split(counts)):
            got[b].append(part)
            at[b] += counts[b]
    assert at == LENS
    return torch.cat([torch.cat(v) for v in got]).double()


def apart(a, b):
    return float((a - b).norm() / b.norm()), float(((a - b).norm(dim=1) / b.norm(dim=1)).max())


WHOLE = [(LENS, False)]
TOKENS = [([n - 12 for n in LENS], False)] + [([1] * 4, True)] * 12


@pytest.mark.parametrize("scored", [False, True])
def test_four_bit_projections(scored):
    """Token by token, in one prefill, and with the same weights in bf16."""
    bank = inputs()
    scoring = q.MoeScoring("sigmoid", None, None, 2, 2, 1, True, 2.0) if scored else None
    four = lambda: Decoder(SHAPE, len(LENS), 8, 512, w4=True, scoring=scoring)  # noqa: E731
    m = four()
    whole, tokens = run(m, WHOLE, bank), run(four(), TOKENS, bank)
    wide = four()
    for layer in wide.layers:
        for name in ("qkv", "out"):
            w = getattr(layer, name)
            eye = torch.eye(w.cols, dtype=torch.bfloat16, device=DEV)
            back = torch.empty((w.cols, w.rows), dtype=torch.float32, device=DEV)
            assert q.dense_linear(eye, w, back) == q.MOE_OK          # one product a sum: exact
            assert torch.equal(back.bfloat16().float(), back) and 0.5 < float(back.square().mean().sqrt()) * w.cols ** 0.5 < 2
            setattr(layer, name, back.bfloat16())
    plain = run(wide, WHOLE, bank)
    for other in (tokens, plain):
        mean, worst = apart(other, whole)
        assert mean < BAR and worst < 3 * BAR


def test_scores_change_the_weights_of_experts():
    """Without a choice bias sigmoid scores are another mixture than the softmax's; with one that bars an expert the result is another again."""
    bank = inputs()
    soft, same, sig, barred = (run(Decoder(SHAPE if s != 3 else Shape(**dict(vars(SHAPE), k=3)), len(LENS), 8, 512, scoring=sc), WHOLE, bank) for s, sc in enumerate(
        (None, q.MoeScoring("softmax"), q.MoeScoring("sigmoid"),
         q.MoeScoring("sigmoid", None, torch.tensor([0., 0., -math.inf, 0.], device=DEV)))))
    assert apart(same, soft)[0] < BAR
    assert apart(sig, soft)[0] > 0.01 and apart(barred, sig)[0] > 0.01


@pytest.mark.parametrize("fp8,w4,scored", [(False, True, False), (True, True, True)])
def test_the_example_runs(fp8, w4, scored, capsys):
    main(fp8, w4, scored)
    assert "decode step" in capsys.readouterr().out
