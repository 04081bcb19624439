"""moe_route_scored against the definition in 64 bits (-m gpu).

Inputs lie on grids that make fp32 logits exact in any order of the sums (products are multiples of 2^-13, sums of their sizes stay below 2^10), so experts are
compared for equality, ties included.  Weights: 64-bit scores off by a few 2^-53 and one rounding, 2^-24; scores' own errors are far below."""
import math

import numpy as np
import pytest
import torch

import paper_2503_09304_amd as q

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def inputs(seed, N, H, E, dtype=torch.bfloat16, coarse=False):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    rnd = lambda *n: torch.randn(*n, generator=g, device=DEV)  # noqa: E731
    x = (rnd(N, H) * (1 if coarse else 16)).round().clamp(-96, 96) / (1 if coarse else 16)
    Wg = (rnd(H, E) * (1 if coarse else 1024 * H ** -0.5)).round().clamp(-255, 255) / (1 if coarse else 512)
    if coarse:                                     # few values: logits that are equal, often
        Wg *= (torch.rand(H, E, generator=g, device=DEV) < 4.0 / H)
    return x.to(dtype), Wg.to(dtype), (rnd(E) * 64).round() / 256, rnd(E) * 0.1


def context(N, H, E, k, Wg, dtype, packed=False):
    F = 64
    W = [torch.zeros((E, *n), dtype=dtype, device=DEV) for n in ((F, H), (F, H), (H, F))]
    w = q.Context.weights(Wg, *W)
    ctx = q.Context(E, k, H, F, q.MOE_BF16 if dtype is torch.bfloat16 else q.MOE_F32, 16, max(N, 1))
    keep = W
    if packed:
        P = [torch.empty_like(t) for t in W]
        pg = torch.empty(((E + 15) // 16 * 16, H), dtype=dtype, device=DEV)
        d = q.Context.weights(pg, *P)
        q.moe_pack_weights(ctx.cfg, w, d)
        w, keep = d, [W, P, pg]
    return ctx, w, keep


def reference(logits, choice, score, groups, take, best, renorm, factor, k):
    l = logits.astype(np.float64)
    if score == "sigmoid":
        s = 1.0 / (1.0 + np.exp(-l))
    else:
        s = np.exp(l - l.max(1, keepdims=True))
        s /= s.sum(1, keepdims=True)
    v = s if choice is None else s + choice.astype(np.float64)
    N, E = v.shape
    g = np.sort(v.reshape(N, groups, -1), 2)[:, :, ::-1][:, :, :best].sum(2)
    kept = np.argsort(-g, 1, kind="stable")[:, :take]
    allowed = np.zeros((N, groups), dtype=bool)
    np.put_along_axis(allowed, kept, True, 1)
    allowed = allowed.repeat(E // groups, 1)
    idx = np.stack([sorted(range(E), key=lambda e: (not a[e], -r[e], e))[:k] for a, r in zip(allowed, v)]) if N else np.zeros((0, k), int)
    w = np.take_along_axis(s, idx, 1)
    if renorm:
        total = w.sum(1, keepdims=True)
        w = np.where(total == 0, 1.0 / k, w / np.where(total == 0, 1.0, total))
    return idx, w * factor


def check(N, H, E, k, score="sigmoid", groups=1, take=1, best=1, renorm=True, factor=1.0, bias=True, choice=True, dtype=torch.bfloat16, packed=False, seed=0, coarse=False):
    x, Wg, lb, cb = inputs(seed + N + H + E + k, N, H, E, dtype, coarse)
    lb, cb = lb if bias else None, cb if choice else None
    ctx, w, keep = context(N, H, E, k, Wg, dtype, packed)
    ctx.route_scored(x, w, q.MoeScoring(score, lb, cb, groups, take, best, renorm, factor))
    torch.cuda.synchronize()
    logits = x.double() @ Wg.double() + (0 if lb is None else lb.double())
    got = ctx.get("logits").cpu().numpy()
    assert np.array_equal(got, logits.float().cpu().numpy())
    idx, wt = reference(got, None if cb is None else cb.cpu().numpy(), score, groups, take, best, renorm, factor, k)
    assert np.array_equal(ctx.get("topk_idx").cpu().numpy(), idx)
    assert (np.abs(ctx.get("topk_w").cpu().numpy() - wt) <= 2.0 ** -23 * np.abs(wt) + 1e-300).all()
    return ctx, w, x, keep


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("E,k,groups,take,best", [(8, 2, 1, 1, 1), (1, 1, 1, 1, 1), (16, 4, 4, 2, 2), (64, 8, 8, 3, 1), (64, 6, 64, 7, 1), (60, 5, 3, 2, 4), (60, 32, 1, 1, 1),
                                                  (96, 8, 6, 2, 3), (128, 8, 1, 1, 1), (160, 6, 8, 3, 1), (256, 8, 8, 4, 2), (256, 32, 2, 1, 2), (255, 9, 5, 4, 4), (200, 3, 50, 3, 2)])
def test_scores_and_groups(score, E, k, groups, take, best):
    for i, (renorm, bias, choice) in enumerate([(True, True, True), (False, False, True), (True, True, False)]):
        check(37, 256, E, k, score, groups, take, best, renorm, 2.5 if i else 1.0, bias, choice, seed=i)


@pytest.mark.parametrize("N", [1, 2, 15, 16, 17, 33, 64, 65, 130, 509, 1024, 1025, 2111])
@pytest.mark.parametrize("E,H", [(64, 2048), (256, 576), (8, 4096)])
def test_tokens(N, E, H):
    check(N, H, E, min(E, 8), groups=4, take=4 if E == 8 else 2, best=2, factor=2.5)


@pytest.mark.parametrize("E", [1, 2, 31, 32, 33, 64, 66, 96, 128, 150, 160, 192, 224, 255, 256])
@pytest.mark.parametrize("N", [1, 30, 2100])
def test_experts(N, E):
    """Waves, slices and ranges go by the experts; room for ranges by k and H."""
    for H, k in ((64, 1), (1024, min(E, 3))):
        check(N, H, E, k)
        check(N, H, E, k, "softmax", packed=True)


@pytest.mark.parametrize("H", [64, 128, 192, 576, 1024, 1600, 4096, 7168])
@pytest.mark.parametrize("packed", [False, True])
def test_inner_sizes(H, packed):
    check(70, H, 160, 6, "softmax", 8, 3, 1, False, 16.0, packed=packed)
    check(3, H, 24, 2, packed=packed)


@pytest.mark.parametrize("E", [4, 6, 9, 64, 250])
def test_fp32_context(E):
    check(41, 100, E, min(E, 5), dtype=torch.float32, groups=2 if E % 2 == 0 else 1, take=1 if E > 9 else 2 if E % 2 == 0 else 1)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_ties_go_to_the_lowest_index(score):
    for choice in (False, True):
        check(300, 64, 128, 16, score, 8, 3, 2, choice=choice, bias=False, coarse=True)
    ctx, w, x, keep = check(5, 64, 64, 8, score, 8, 2, 2, bias=False, choice=False)
    zero = torch.zeros_like(x)
    ctx.route_scored(zero, w, q.MoeScoring(score, groups=8, top_groups=2, group_best=2))
    assert (ctx.get("topk_idx") == torch.arange(8, device=DEV)).all() and (ctx.get("topk_w") == 0.125).all()


def test_barred_experts_and_vanishing_scores():
    N, H, E, k = 6, 64, 16, 4
    x, Wg, lb, cb = inputs(3, N, H, E)
    ctx, w, keep = context(N, H, E, k, Wg, torch.bfloat16)
    cb = torch.full((E,), -math.inf, device=DEV)
    cb[[3, 9, 15]] = 0.0
    ctx.route_scored(x, w, q.MoeScoring("sigmoid", choice_bias=cb))
    idx = ctx.get("topk_idx").sort(1)[0].tolist()
    assert all(r == [0, 3, 9, 15] for r in idx)                   # the barred one of lowest index fills the last slot
    cb[5] = float("nan")
    ctx.route_scored(x, w, q.MoeScoring("sigmoid", choice_bias=cb, groups=4, top_groups=2, group_best=4))
    idx = ctx.get("topk_idx")
    assert ((idx >= 0) & (idx < E)).all() and all(len(set(r)) == k for r in idx.tolist())
    low = torch.full((E,), -2000.0, device=DEV)
    ctx.route_scored(x, w, q.MoeScoring("sigmoid", logit_bias=low, factor=2.0))
    assert (ctx.get("topk_w") == 0.5).all() and (ctx.get("topk_idx") == torch.arange(k, device=DEV)).all()
    ctx.route_scored(x, w, q.MoeScoring("sigmoid", logit_bias=-low))
    assert (ctx.get("topk_w") == 0.25).all() and (ctx.get("topk_idx") == torch.arange(k, device=DEV)).all()


def test_softmax_renormalised_is_moe_route():
    """One group, no bias for the choice: the plain router's rule."""
    x, Wg, lb, _ = inputs(5, 200, 256, 64)
    ctx, w, keep = context(200, 256, 64, 8, Wg, torch.bfloat16)
    ctx.route(x, w, lb)
    idx, wt = ctx.get("topk_idx").clone(), ctx.get("topk_w").clone()
    ctx.route_scored(x, w, q.MoeScoring("softmax", logit_bias=lb))
    assert torch.equal(ctx.get("topk_idx"), idx) and ((ctx.get("topk_w") - wt).abs() <= 2.0 ** -20 * wt).all()


def test_a_layer_runs_behind_it():
    """route_scored -> permute -> experts -> combine, against the same layer's formula in 64 bits; and twice, the second batch smaller."""
    N, H, F, E, k = 90, 128, 192, 16, 4
    g = torch.Generator(device=DEV)
    g.manual_seed(8)
    x, Wg, lb, cb = inputs(8, N, H, E)
    W1, W3, W2 = ((torch.randn(E, *n, generator=g, device=DEV) * n[1] ** -0.5).to(torch.bfloat16) for n in ((F, H), (F, H), (H, F)))
    w = q.Context.weights(Wg, W1, W3, W2)
    ctx = q.Context(E, k, H, F, q.MOE_BF16, 16, N)
    prio = (torch.arange(N, device=DEV) % 3 == 0).to(torch.uint8)
    rule = q.MoeScoring("sigmoid", lb, cb, 4, 2, 2, True, 2.5)
    for n in (N, 17):
        ctx.route_scored(x, w, rule, n_tokens=n)
        ctx.permute(prio[:n].contiguous())
        ctx.expert_run(x, w)
        y = torch.empty((n, H), dtype=torch.float32, device=DEV)
        ctx.combine(y, q.MOE_CLASS_ALL | q.MOE_Y_F32)
        idx, wt = ctx.get("topk_idx").long(), ctx.get("topk_w").double()
        d, ref = x[:n].double(), torch.zeros((n, H), dtype=torch.float64, device=DEV)
        for e in range(E):
            h = torch.nn.functional.silu(d @ W1[e].double().t()) * (d @ W3[e].double().t())
            ref += ((idx == e) * wt).sum(1, keepdim=True) * (h @ W2[e].double().t())
        assert float((y - ref).norm() / ref.norm()) < 2.0 ** -8          # the activation's one rounding to bf16


def test_replayed_in_a_graph():
    x, Wg, lb, cb = inputs(9, 64, 512, 256)
    ctx, w, keep = context(64, 512, 256, 8, Wg, torch.bfloat16)
    rule = q.MoeScoring("sigmoid", lb, cb, 8, 4, 2, True, 2.5)
    ctx.route_scored(x, w, rule)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        ctx.route_scored(x, w, rule)
    for seed in range(4):
        x.copy_(inputs(20 + seed, 64, 512, 256)[0])
        cb.copy_(inputs(30 + seed, 64, 512, 256)[3])
        graph.replay()
        got = [ctx.get(n).clone() for n in ("logits", "topk_idx", "topk_w")]
        ctx.route_scored(x, w, rule)
        for a, n in zip(got, ("logits", "topk_idx", "topk_w")):
            assert torch.equal(a, ctx.get(n))


def test_refusals():
    x, Wg, lb, cb = inputs(10, 4, 64, 60)
    ctx, w, keep = context(4, 64, 60, 8, Wg, torch.bfloat16)
    for kw in (dict(groups=7), dict(groups=0), dict(groups=10, top_groups=1), dict(groups=4, top_groups=5), dict(group_best=5), dict(groups=30, top_groups=8, group_best=3),
               dict(factor=math.inf), dict(logit_bias=lb[:59].contiguous()), dict(choice_bias=torch.zeros(61, device=DEV))):
        with pytest.raises(q.MoeError):
            ctx.route_scored(x, w, q.MoeScoring("sigmoid", **kw))
    with pytest.raises(q.MoeError):
        q.MoeScoring("tanh")
    with pytest.raises(q.MoeError):
        q.MoeScoring(choice_bias=cb.double())


def test_two_contexts_on_two_streams():
    want, got, all_ = [], [[], []], []
    for i, N in enumerate((61, 700)):
        x, Wg, lb, cb = inputs(40 + i, N, 512, 160)
        ctx, w, keep = context(N, 512, 160, 8, Wg, torch.bfloat16)
        rule = q.MoeScoring("softmax" if i else "sigmoid", lb, cb, 8, 3, 2, True, 1.5)
        ctx.route_scored(x, w, rule)
        want.append([ctx.get(n).clone() for n in ("topk_idx", "topk_w")])
        all_.append((ctx, x, w, rule, keep))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(20):
        for i, (ctx, x, w, rule, keep) in enumerate(all_):
            with torch.cuda.stream(streams[i]):
                ctx.route_scored(x, w, rule)
                got[i].append([ctx.get(n).clone() for n in ("topk_idx", "topk_w")])
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        for c in b:
            assert torch.equal(a[0], c[0]) and torch.equal(a[1], c[1])


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("N,E,groups,take,best", [(20, 256, 8, 4, 2), (20, 48, 1, 1, 1), (5000, 160, 8, 3, 4)])
def test_rows_that_are_not_finite(score, N, E, groups, take, best):
    """Their experts are k different ones all the same, and other rows have what they have without them."""
    x, Wg, lb, cb = inputs(50, N, 256, E)
    ctx, w, keep = context(N, 256, E, 8, Wg, torch.bfloat16)
    rule = q.MoeScoring(score, lb, cb, groups, take, best, True, 1.0)
    ctx.route_scored(x, w, rule)
    idx, wt = ctx.get("topk_idx").clone(), ctx.get("topk_w").clone()
    for row, value in ((3, math.nan), (7, math.inf), (N - 1, -math.inf)):
        x[row, 5] = value
    ctx.route_scored(x, w, rule)
    got = ctx.get("topk_idx")
    assert ((got >= 0) & (got < E)).all() and (got.sort(1)[0].diff(dim=1) > 0).all()
    rest = torch.ones(N, dtype=torch.bool, device=DEV)
    rest[[3, 7, N - 1]] = False
    assert torch.equal(got[rest], idx[rest]) and torch.equal(ctx.get("topk_w")[rest], wt[rest])
    cursor = ctx.permute(torch.zeros(N, dtype=torch.uint8, device=DEV))
    assert cursor.n_units > 0 and int(ctx.get("counts").sum()) == 8 * N
