"""moe_route_scored's logits on ordinary inputs, whose sums are rounded (-m gpu).

Products of two bf16 numbers are exact in fp32; a sum of H of them in any order is off by at most (H + 16) 2^-24 of the sum of their sizes S (as for dense_linear), and the bias
adds a rounding, 2^-24 of the result.  What is chosen goes by those logits: it is compared with the definition in 64 bits on them."""
import numpy as np
import pytest
import torch

import paper_2503_09304_amd as q
from test_gpu_route_scored import DEV, context, reference

pytestmark = pytest.mark.gpu


def inputs(seed, N, H, E, dtype):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    x = torch.randn(N, H, generator=g, device=DEV) * torch.exp(torch.randn(N, 1, generator=g, device=DEV))
    return x.to(dtype), (torch.randn(H, E, generator=g, device=DEV) * H ** -0.5).to(dtype), torch.randn(E, generator=g, device=DEV) * 0.3, torch.randn(E, generator=g, device=DEV) * 0.1


@pytest.mark.parametrize("H,E,k,groups,take", [(64, 8, 2, 1, 1), (2048, 64, 8, 8, 4), (4096, 160, 6, 8, 3), (7168, 256, 8, 8, 4), (1600, 60, 4, 4, 2), (576, 255, 9, 5, 4)])
@pytest.mark.parametrize("N", [1, 37, 513, 3001])
@pytest.mark.parametrize("kind", ["rows", "packed", "fp32"])
def test_logits_and_choice(H, E, k, groups, take, N, kind):
    dtype = torch.float32 if kind == "fp32" else torch.bfloat16
    x, Wg, lb, cb = inputs(N + H, N, H, E, dtype)
    ctx, w, keep = context(N, H, E, k, Wg, dtype, kind == "packed")
    for score, choice in (("sigmoid", cb), ("softmax", None)):
        rule = q.MoeScoring(score, lb, choice, groups, take, 2, True, 2.5)
        ctx.route_scored(x, w, rule)
        logits, idx, wt = (ctx.get(n).clone() for n in ("logits", "topk_idx", "topk_w"))
        ref, S = x.double() @ Wg.double() + lb.double(), x.double().abs() @ Wg.double().abs()
        err = (H + 16 + (H if kind == "fp32" else 0)) * 2.0 ** -24 * S              # fp32: a product's rounding as well
        assert ((logits.double() - ref).abs() <= err + 2.0 ** -24 * (ref.abs() + err)).all()
        at, weight = reference(logits.cpu().numpy(), None if choice is None else choice.cpu().numpy(), score, groups, take, 2, True, 2.5, k)
        assert np.array_equal(idx.cpu().numpy(), at)
        assert (np.abs(wt.cpu().numpy() - weight) <= 2.0 ** -23 * np.abs(weight)).all()
        ctx.route_scored(x, w, rule)
        for name, old in (("logits", logits), ("topk_idx", idx), ("topk_w", wt)):
            assert torch.equal(ctx.get(name), old)


def test_other_tokens_values_change_nothing():
    for N, H, E in ((40, 2048, 256), (3000, 4096, 64)):
        x, Wg, lb, cb = inputs(7, N, H, E, torch.bfloat16)
        ctx, w, keep = context(N, H, E, 8, Wg, torch.bfloat16)
        rule = q.MoeScoring("sigmoid", lb, cb, 8, 4, 2)
        ctx.route_scored(x, w, rule)
        logits = ctx.get("logits").clone()
        x[1::2] = torch.randn_like(x[1::2].float()).to(x.dtype) * 100
        ctx.route_scored(x, w, rule)
        assert torch.equal(ctx.get("logits")[::2], logits[::2])
