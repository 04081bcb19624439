"""The routers on more tokens than one launch takes (-m gpu): rows on both sides of 2^25 and of 2^26, and the last."""
import pytest
import torch

import paper_2503_09304_amd as q

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("dtype,H", [(torch.bfloat16, 64), (torch.float32, 4)])
@pytest.mark.parametrize("scored", [False, True])
def test_tokens_behind_2_to_the_26(dtype, H, scored):
    N, E = (1 << 26) + 77, 2
    bf16 = dtype is torch.bfloat16
    g = torch.Generator(device=DEV)
    g.manual_seed(H)
    x = torch.empty((N, H), dtype=dtype, device=DEV)
    for r in range(0, N, 1 << 24):                                # on a grid that makes logits exact in any order
        x[r:r + (1 << 24)] = torch.randint(-8, 9, (min(1 << 24, N - r), H), generator=g, device=DEV, dtype=torch.int8)
    Wg = torch.randint(-8, 9, (H, E), generator=g, device=DEV).to(dtype)
    dummy = torch.empty(64, dtype=dtype, device=DEV)
    w = q.Context.weights(Wg, dummy, dummy, dummy)
    ctx = q.Context(E, 1, H, 64 if bf16 else 1, q.MOE_BF16 if bf16 else q.MOE_F32, 256, N, device=DEV)
    ctx.ws.fill_(0xFF)
    if scored:
        ctx.route_scored(x, w, q.MoeScoring("sigmoid", renormalise=False))
    else:
        ctx.route(x, w)
    torch.cuda.synchronize()
    for r in range(0, N, 1 << 24):
        logits = x[r:r + (1 << 24)].float() @ Wg.float()
        n = len(logits)
        assert torch.equal(ctx.get("logits")[r:r + n], logits), r
        score = 1.0 / (1.0 + torch.exp(-logits.double())) if scored else logits          # large ones are 1 in 64 bits: equal, the first is taken
        idx = (score[:, 1] > score[:, 0]).int()
        assert torch.equal(ctx.get("topk_idx")[r:r + n, 0], idx), r
        wt = ctx.get("topk_w")[r:r + n, 0]
        want = score.amax(1) if scored else torch.ones_like(wt)
        # 64 bits off by a few 2^-53 and one rounding to fp32: 2^-24 of the value, or, below 2^-126, where fp32's steps are 2^-149, half such a step
        assert ((wt.double() - want).abs() <= 2.0 ** -23 * want + 2.0 ** -150).all(), r
