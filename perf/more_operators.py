"""Cases of the operators that stand beside attention and the experts in a served decoder layer, and their plain forms.

  norm     the residual's addition and the root-mean-square norm of each row, or of each head of a row: bf16 out
  linear   tokens times a matrix of 4-bit weights (e2m1 elements, a power-of-two scale byte for every 32 of a row)
  chain    both as a layer has them: the norm's output in 8 bits (e4m3, a power-of-two scale byte for every 32 elements), which
           the product takes as it is
  route    the router's logits, scores by softmax or sigmoid, a bias that counts for the choice alone, the best groups of
           experts, the k best of those, their weights

A case holds plain values:
  op            "norm" | "linear" | "chain" | "route"
  tokens        rows of the call
  H             elements of a row (norm), inner size of the product or of the router
  heads         norm: heads of a row, H elements each, slices of a wider row (0: the row is one vector)
  add           norm, chain: type of the residual that is added and kept: "bf16" | "fp32" | "none"
  shift         norm, chain: what is added to the norm's weights (1: weights are kept as differences from 1)
  wtype         norm, chain: type of those weights
  R             linear, chain: rows of the matrix
  out           linear, chain: type of the product (chain: bf16, as an element of the 8-bit rows that falls between two values may go either way)
  E, k          route: experts, how many a token gets
  score         route: "softmax" | "sigmoid"
  groups, take  route: groups of experts, how many of them a token may choose from
  best          route: how many of a group's experts its value is the sum of
  renorm        route: weights are divided by their sum
  factor        route: what they are multiplied with
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False
DEV = "cuda:0"
EPS = 1e-6
GROUP = 32               # elements that share a scale byte


def _norm(name, tokens, H, **kw):
    return dict(dict(name=name, op="norm", tokens=tokens, H=H, heads=0, add="bf16", shift=0.0, wtype="bf16"), **kw)


def _linear(name, tokens, H, R, **kw):
    return dict(dict(name=name, op="linear", tokens=tokens, H=H, R=R, out="bf16"), **kw)


def _chain(name, tokens, H, R, **kw):
    return dict(dict(name=name, op="chain", tokens=tokens, H=H, R=R, out="bf16", add="bf16", shift=0.0, wtype="bf16"), **kw)


def _route(name, tokens, H, E, k, **kw):
    return dict(dict(name=name, op="route", tokens=tokens, H=H, E=E, k=k, score="sigmoid", groups=8, take=4, best=2, renorm=True, factor=2.5), **kw)


def listed():
    return [
        # The next token of a single conversation, in front of its MoE layer: launch and latency are all there is.
        _norm("norm_1", 1, 4096),
        # The query heads of a prefill batch normalised head by head, out of the rows of one QKV product.
        _norm("norm_heads", 1531, 128, heads=32, add="none"),
        # A long prefill of prompts whose residual stream is kept in 32 bits.
        _norm("norm_prompts_fp32", 7919, 4096, add="fp32", shift=1.0, wtype="fp32"),
        # QKV projection of a single conversation's next token.
        _linear("linear_1", 1, 4096, 6144),
        # The logits of a decode step's eight conversations over a vocabulary.
        _linear("linear_8_vocabulary", 8, 2048, 32000, out="fp32"),
        # A dense layer's down projection for a decode step of 61 conversations.
        _linear("linear_61_down", 61, 14336, 4096),
        # QKV projection of the benchmark's long best-effort batch.
        _linear("linear_3584", 3584, 4096, 6144),
        # Norm and a dense layer's gate-up product in a decode step of 32 conversations (the evaluation's batch size).
        _chain("chain_32", 32, 2048, 2816),
        # The same for a long prefill, H 4096, F 14336.
        _chain("chain_4093", 4093, 4096, 28672, add="fp32"),
        # A single token's way to 8 of 64 experts.
        _route("route_1", 1, 2048, 64, 8, score="softmax", groups=1, take=1, best=1, factor=1.0),
        # A decode step of 61 conversations: 8 of 256 experts, out of 4 groups of 8.
        _route("route_61", 61, 4096, 256, 8),
        # A long prefill: 6 of 160 experts out of 3 groups, each valued by its best, weights as they are.
        _route("route_8192", 8192, 4096, 160, 6, score="softmax", take=3, best=1, renorm=False, factor=16.0),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case of the same ranges."""
    op = rng.choice(["norm", "linear", "linear", "chain", "route", "route"])
    tokens = _log_int(rng, 1, 8192)
    kw = dict(add=rng.choice(["bf16", "bf16", "fp32", "none"]), shift=rng.choice([0.0, 1.0]), wtype=rng.choice(["bf16", "fp32"]))
    if op == "norm":
        if rng.random() < 0.3:
            c = _norm("", _log_int(rng, 1, 4096), rng.choice([64, 80, 96, 128, 256]), heads=rng.choice([1, 4, 8, 16, 32]), **kw)
        else:
            c = _norm("", tokens, 8 * _log_int(rng, 8, 1024), **kw)
    elif op in ("linear", "chain"):
        H, R = GROUP * _log_int(rng, 2, 448), _log_int(rng, 16, 32768)
        while tokens * H * R > 4093 * 4096 * 28672 or tokens * R > 1 << 27:
            tokens = (tokens + 1) // 2
        c = _linear("", tokens, H, R) if op == "linear" else _chain("", tokens, min(H, 8192), R, **kw)
        c["out"] = rng.choice(["bf16", "bf16", "fp32"]) if op == "linear" else "bf16"
    else:
        E, groups, take, best = rng.choice([(8, 1, 1, 1), (16, 4, 2, 2), (32, 1, 1, 1), (60, 1, 1, 1), (64, 8, 3, 1), (64, 4, 1, 2), (96, 6, 2, 3),
                                            (128, 1, 1, 1), (160, 8, 3, 1), (256, 8, 4, 2), (256, 16, 5, 2)])
        k = rng.randint(1, min(32, max(1, take * E // groups // 2)))
        c = _route("", tokens, 64 * _log_int(rng, 2, 112), E, k, score=rng.choice(["softmax", "sigmoid"]), groups=groups, take=take, best=best,
                   renorm=rng.random() < 0.7, factor=rng.choice([1.0, 2.5]))
    del c["name"]
    return c


# ---- inputs ----

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV, dtype=torch.float32)


def _type(name):
    return torch.float32 if name == "fp32" else torch.bfloat16


def _matrix(g, R, K):
    """Codes [R, K/2] and scale bytes [R, K/32] of normally distributed weights, rows of different sizes among them."""
    codes = torch.empty((R, K // 2), dtype=torch.uint8, device=DEV)
    scales = torch.empty((R, K // GROUP), dtype=torch.uint8, device=DEV)
    edges = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], device=DEV)
    step = max(1, (1 << 24) // K)
    for r in range(0, R, step):
        n = min(step, R - r)
        w = (_randn(g, n, K) * (K ** -0.5 * torch.exp(0.4 * _randn(g, n, 1)))).view(n, K // GROUP, GROUP)
        e = (w.abs().amax(2).clamp(min=2.0 ** -60).view(torch.int32) >> 23) - 2          # the largest of 32 comes to 4 .. 8, held to 6
        m = torch.bucketize((w.abs() * ((254 - e) << 23).view(torch.float32)[:, :, None]), edges)
        c = (m + 8 * (w < 0)).view(n, K).to(torch.uint8)
        codes[r:r + n] = c[:, 0::2] | (c[:, 1::2] << 4)
        scales[r:r + n] = e.to(torch.uint8)
    return codes, scales


def prepare(case, seed):
    c, g = case, _gen(seed)
    T, H = c["tokens"], c["H"]
    s = {"case": c}
    if c["op"] == "route":
        # Activations and router weights on grids of 1/16 and 1/512, so that logits are exact in 32 bits in any order of their sums, and with them the choice.
        s["x"] = (_randn(g, T, H) * 16).round().clamp(-96, 96).div(16).to(torch.bfloat16)
        s["Wg"] = (_randn(g, H, c["E"]) * (512 * 2 * H ** -0.5)).round().clamp(-255, 255).div(512).to(torch.bfloat16)
        s["logit_bias"] = (_randn(g, c["E"]) * 64).round().div(256)
        s["choice_bias"] = _randn(g, c["E"]) * 0.1 if c["score"] == "sigmoid" else None
        return s
    if c["op"] != "linear":
        shape = (T, c["heads"], H) if c.get("heads") else (T, H)
        spread = torch.exp(0.5 * _randn(g, T, *[1] * (len(shape) - 1)))                  # rows of different sizes
        if c.get("heads"):
            s["x"] = (_randn(g, T, c["heads"] * 3 // 2 + 1, H) * spread).to(torch.bfloat16)[:, :c["heads"]]
        else:
            s["x"] = (_randn(g, *shape) * spread).to(torch.bfloat16)
        s["weight"] = (1.0 - c["shift"] + 0.2 * _randn(g, H)).to(_type(c["wtype"]))
        if c["add"] != "none":
            s["add"] = (_randn(g, *shape) * 3).to(_type(c["add"]))
            s["total"] = torch.empty_like(s["add"])
        if c["op"] == "norm":
            s["out"] = torch.empty(shape, dtype=torch.bfloat16, device=DEV)
            return s
        s["h"] = torch.empty((T, H), dtype=torch.float8_e4m3fn, device=DEV)
        s["h_scale"] = torch.empty((T, H // GROUP), dtype=torch.uint8, device=DEV)
    else:
        s["x"] = _randn(g, T, H).to(torch.bfloat16)
    s["codes"], s["scales"] = _matrix(g, c["R"], H)
    s["y"] = torch.empty((T, c["R"]), dtype=_type(c["out"]), device=DEV)
    return s


# ---- one pass ----

def run(state):
    return (_run_own if own else _run_plain)(state)


def _kept(s, *names):
    return {n: s[n] for n in names if s.get(n) is not None}


def _run_own(s):
    import paper_2503_09304_amd as q
    c = s["case"]
    if c["op"] == "route":
        if "ctx" not in s:                 # what a serving program sets up once; the router looks at none of the experts' weights
            F = 64
            s["experts"] = [torch.zeros((c["E"], *n), dtype=torch.bfloat16, device=DEV) for n in ((F, c["H"]), (F, c["H"]), (c["H"], F))]
            s["w"] = q.Context.weights(s["Wg"], *s["experts"])
            s["ctx"] = q.Context(c["E"], c["k"], c["H"], F, q.MOE_BF16, 256, c["tokens"])
            s["scoring"] = q.MoeScoring(c["score"], logit_bias=s["logit_bias"], choice_bias=s["choice_bias"], groups=c["groups"], top_groups=c["take"],
                                        group_best=c["best"], renormalise=c["renorm"], factor=c["factor"])
        s["ctx"].route_scored(s["x"], s["w"], s["scoring"])
        return {n: s["ctx"].get(n) for n in ("logits", "topk_idx", "topk_w")}
    x, scale = s["x"], None
    if c["op"] != "linear":
        x = s["out"] if c["op"] == "norm" else s["h"]
        scale = s.get("h_scale")
        q.dense_norm(s["x"], s["weight"], x, eps=EPS, add=s.get("add"), total=s.get("total"), scale=scale, shift=c["shift"])
        if c["op"] == "norm":
            return _kept(s, "out", "total")
    if "matrix" not in s:                  # laid out once, when a model is loaded
        s["matrix"] = q.DenseMatrix4(s["codes"], s["scales"])
    q.dense_linear(x, s["matrix"], s["y"], scale=scale)
    return _kept(s, "y", "total")


def _values(codes, scales):
    """The matrix in fp32."""
    table = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0], device=DEV)
    c = codes.int()
    w = table[torch.stack([c & 15, c >> 4], 2)].view(codes.shape[0], -1, GROUP)
    return (w * (scales.int() << 23).view(torch.float32)[:, :, None]).view(codes.shape[0], -1)


def _in_8_bits(x):
    """The values that rows stand for when every 32 elements share the smallest power of two, 2^-126 at least, for which none is over 448."""
    g = x.view(x.shape[0], -1, GROUP)
    b = g.abs().amax(2).view(torch.int32)
    e = ((b >> 23) - 8 + ((b & 0x7FFFFF) > 0x600000).to(torch.int32)).clamp(min=1)
    code = (g * ((254 - e) << 23).view(torch.float32)[:, :, None]).to(torch.float8_e4m3fn)
    return (code.float() * (e << 23).view(torch.float32)[:, :, None]).view(x.shape)


def _run_plain(s):
    c = s["case"]
    if c["op"] == "route":
        logits = s["x"].float() @ s["Wg"].float() + s["logit_bias"]
        l = logits.double()
        p = torch.sigmoid(l) if c["score"] == "sigmoid" else torch.exp(l - l.amax(1, keepdim=True))
        if c["score"] == "softmax":
            p = p / p.sum(1, keepdim=True)
        value = p if s["choice_bias"] is None else p + s["choice_bias"].double()
        T, E, n = c["tokens"], c["E"], c["groups"]
        if n > 1:
            worth = value.view(T, n, E // n).sort(dim=2, descending=True)[0][:, :, :c["best"]].sum(2)
            kept = worth.sort(dim=1, descending=True, stable=True)[1][:, :c["take"]]
            allowed = torch.zeros((T, n), dtype=torch.bool, device=DEV).scatter_(1, kept, True)
            value = value.masked_fill(~allowed.repeat_interleave(E // n, 1), -math.inf)
        idx = value.sort(dim=1, descending=True, stable=True)[1][:, :c["k"]]
        w = p.gather(1, idx)
        if c["renorm"]:
            w = w / w.sum(1, keepdim=True)
        return {"logits": logits, "topk_idx": idx.int(), "topk_w": (w * c["factor"]).float()}
    x = s["x"].float()
    if c["op"] != "linear":
        if c["add"] != "none":
            s["total"].copy_(x + s["add"].float())
            x = s["total"].float()
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * (s["weight"].float() + c["shift"])
        if c["op"] == "norm":
            s["out"].copy_(x)
            return _kept(s, "out", "total")
        x = _in_8_bits(x)
    s["y"].copy_(x @ _values(s["codes"], s["scales"]).t())
    return _kept(s, "y", "total")


# ---- what a pass cannot do without ----

def work(case):
    c = case
    T, H = c["tokens"], c["H"]
    if c["op"] == "route":
        return {"bytes": 2 * T * H + 2 * H * c["E"] + T * (4 * c["E"] + 8 * c["k"]) + 8 * c["E"], "flops": 2 * T * H * c["E"]}
    b = f = 0
    if c["op"] != "linear":
        n = T * H * (c.get("heads") or 1)
        b += n * 2 + {"none": 0, "bf16": 4, "fp32": 8}[c["add"]] * n + H * (4 if c["wtype"] == "fp32" else 2)
        f += 5 * n
        if c["op"] == "norm":
            return {"bytes": b + 2 * n, "flops": f}
        b += 2 * (T * H + T * H // GROUP)          # written in 8 bits, and read by the product
    else:
        b += 2 * T * H
    b += c["R"] * (H // 2 + H // GROUP) + T * c["R"] * (4 if c["out"] == "fp32" else 2)
    return {"bytes": b, "flops": f + 2 * T * H * c["R"]}


# ---- the definition in 64 bits ----

def exact(case, seed):
    s = prepare(case, seed)
    c = case
    T, H = c["tokens"], c["H"]
    if c["op"] == "route":
        x, wg = s["x"].double().cpu().numpy(), s["Wg"].double().cpu().numpy()
        logits = x @ wg + s["logit_bias"].double().cpu().numpy()
        if c["score"] == "sigmoid":
            p = 1.0 / (1.0 + np.exp(-logits))
        else:
            p = np.exp(logits - logits.max(1, keepdims=True))
            p /= p.sum(1, keepdims=True)
        v = p.copy() if s["choice_bias"] is None else p + s["choice_bias"].double().cpu().numpy()
        size = c["E"] // c["groups"]
        if c["groups"] > 1:
            worth = np.sort(v.reshape(T, c["groups"], size), axis=2)[:, :, size - c["best"]:].sum(2)
            out_of = np.argsort(-worth, axis=1, kind="stable")[:, c["take"]:]
            for t in range(T):
                for n in out_of[t]:
                    v[t, n * size:(n + 1) * size] = -np.inf
        idx = np.argsort(-v, axis=1, kind="stable")[:, :c["k"]]
        w = np.take_along_axis(p, idx, 1)
        if c["renorm"]:
            w = w / w.sum(1, keepdims=True)
        return {"logits": logits, "topk_idx": idx.astype(np.int32), "topk_w": w * c["factor"]}

    def power(n):
        return ((n.to(torch.int64) + 1023) << 52).view(torch.float64)

    def nearest(x, bits, least=-900):
        """To `bits` significant bits, half to even; steps no finer than those of the binade of 2^least."""
        step = power((torch.frexp(x)[1] - bits).clamp(min=least + 1 - bits))
        return torch.round(x / step) * step

    x, res = s["x"].double(), {}
    if c["op"] != "linear":
        if c["add"] != "none":
            res["total"] = x + s["add"].double()
            x = nearest(res["total"], 8) if c["add"] == "bf16" else res["total"]
        x = x / torch.sqrt((x * x).sum(-1, keepdim=True) / H + EPS)
        x = x * (s["weight"].double() + c["shift"])
        if c["op"] == "norm":
            return dict(res, out=x)
        groups = x.view(T, H // GROUP, GROUP)
        part, n = torch.frexp(groups.abs().amax(2, keepdim=True))          # 448 = 0.875 * 2^9
        unit = power((n - 9 + (part > 0.875).to(n.dtype)).clamp(min=-126))
        x = (nearest(groups / unit, 4, -6) * unit).view(T, H)
    y = torch.empty((T, c["R"]), dtype=torch.float64, device=DEV)
    size = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64, device=DEV)
    for r in range(0, c["R"], 4096):                                      # rows of the matrix at a time
        code, scale = s["codes"][r:r + 4096].long(), s["scales"][r:r + 4096]
        w = torch.empty((code.shape[0], H), dtype=torch.float64, device=DEV)
        for half in (0, 1):
            v = code >> 4 * half & 15
            w[:, half::2] = size[v & 7] * (1 - 2 * (v >> 3)).double()
        y[:, r:r + 4096] = x @ (w * power(scale.int() - 127).repeat_interleave(GROUP, 1)).t()
    return dict(res, y=y)
