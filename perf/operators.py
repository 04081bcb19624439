"""Cases of the attention operators between two MoE layers, and their plain forms.

A served layer's attention block does four things with the keys and values of a sequence; each is an operator:

  append   rotary positions on the queries and keys of a batch of tokens, keys and values written to a paged cache (bf16, or
           e4m3 with one power-of-two scale byte per token and head)
  read     keys and values of tokens read back from the pages as bf16
  prompt   causal attention over packed prompts of different lengths, heads grouped over shared keys; where a sequence has more
           keys than queries the queries are its last tokens, and a query without any key gives zero
  decode   attention of one token a sequence over the cache's pages

A case holds plain values:
  op           "append" | "read" | "prompt" | "decode"
  Hq, Hk, D    query heads, key/value heads, elements of a head
  fmt          cache elements: "bf16" | "fp8"
  page         tokens of a page
  lens         append, read: tokens of each sequence in the call; prompt: queries; decode: keys in the cache ("a,b,c")
  before       append, read: tokens that each sequence had before them; prompt: keys in front of the first query's own
  rot, layout  append: rotated elements of a head, "half" | "interleaved" pairs
  factor       append: how many times the trained context the positions reach over (1: plain frequencies)
  fused        append, prompt: q, k and v are slices of one product's rows (strided), not tensors of their own
  lse          prompt, decode: the logarithm of each row's sum of exponentials is an output too
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False
DEV = "cuda:0"
TRAINED = 4096          # trained context of the scaled frequencies
WIDE = dict(Hq=32, Hk=8, D=128)      # H 4096
FINE = dict(Hq=16, Hk=4, D=128)      # H 2048
SMALL = dict(Hq=16, Hk=16, D=64)     # H 1024, every head with keys of its own


def _text(v):
    return ",".join(str(int(x)) for x in v)


def _ints(t):
    return [int(x) for x in t.split(",")]


def _ragged(n, lo, hi, seed):
    """n lengths between lo and hi, spread over their logarithm, both ends among them."""
    r = np.random.default_rng(seed)
    v = np.exp(r.uniform(math.log(lo), math.log(hi + 1), n)).astype(int).clip(lo, hi)
    v[0], v[-1] = hi, lo
    return _text(v)


def _case(name, op, lens, **kw):
    n = len(_ints(lens))
    c = dict(name=name, op=op, lens=lens, before=_text([0] * n), fmt="bf16", page=64, **WIDE)
    if op == "append":
        c.update(rot=128, layout="half", factor=1.0, fused=True)
    if op == "prompt":
        c.update(fused=False, lse=False)
    if op == "decode":
        c.update(lse=False)
    c.update(kw)
    return c


def listed():
    return [
        # The next token of a single conversation: launch and latency are all there is.
        _case("append_1", "append", "1", before="1000"),
        # A decode step of 61 long conversations into an 8-bit cache, far beyond the trained context, half of each head rotated; read back.
        _case("append_61_far_fp8", "append", _text([1] * 61), before=_ragged(61, 900, 120001, 1), fmt="fp8", rot=64,
              layout="interleaved", factor=32.0, page=16),
        # A prefill batch of the serving loop: prompts of different lengths, 8192 tokens or so, from the rows of one QKV product.
        _case("append_prompts", "append", _ragged(29, 17, 1531, 2)),
        # The context of a preempted prompt fetched for its next chunk: a few hundred tokens.
        _case("read_509", "read", "509", **SMALL),
        # The contexts of a batch of long documents, 8-bit cache.
        _case("read_docs_fp8", "read", _ragged(12, 301, 16383, 3), fmt="fp8"),
        # One short question.
        _case("prompt_17", "prompt", "17"),
        # The long best-effort batch of the benchmark as prompts of any length, a token and an empty one among them.
        _case("prompt_3584_packed", "prompt", "512,1,1531,77,0,256,300,907", fused=True),
        # Chunked prefill: the next tokens of six conversations on what they have in the cache; one has lost its context (rows without keys).
        _case("prompt_chunks", "prompt", "512,509,1024,256,33,100", before="4096,1111,2048,7000,0,-40", lse=True, **SMALL),
        # One long document.
        _case("prompt_16384", "prompt", "16384"),
        # Decode step of 32 young conversations (the evaluation's batch size).
        _case("decode_32_young", "decode", _ragged(32, 1, 300, 4), **FINE),
        # Decode step of 64 conversations of any age, 8-bit cache.
        _case("decode_64_fp8", "decode", _ragged(64, 33, 16384, 5), fmt="fp8"),
        # One sequence with a book for context.
        _case("decode_1_book", "decode", "131071", lse=True, page=256),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case of the same ranges."""
    op = rng.choice(["append", "read", "prompt", "prompt", "decode", "decode"])
    heads = rng.choice([WIDE, WIDE, FINE, SMALL, dict(Hq=8, Hk=1, D=128), dict(Hq=24, Hk=8, D=64), dict(Hq=12, Hk=4, D=96),
                        dict(Hq=40, Hk=2, D=80), dict(Hq=5, Hk=5, D=112)])
    kw = dict(heads, fmt=rng.choice(["bf16", "fp8"]), page=rng.choice([16, 32, 64, 128, 256]))
    if op == "append":
        if rng.random() < 0.5:                       # a decode step
            n = _log_int(rng, 1, 256)
            lens, before = [1] * n, [_log_int(rng, 1, 32768) - 1 for _ in range(n)]
        else:
            total, lens = _log_int(rng, 2, 8192), []
            while total > 0:
                lens.append(min(total, _log_int(rng, 1, 4096)))
                total -= lens[-1]
            before = [rng.choice([0, 0, _log_int(rng, 1, 5000)]) for _ in lens]
        kw.update(rot=rng.choice([kw["D"], kw["D"] // 32 * 16]), layout=rng.choice(["half", "interleaved"]),
                  factor=rng.choice([1.0, 4.0, 32.0]), fused=rng.random() < 0.5)
        return _drop_name(_case("", op, _text(lens), **dict(kw, before=_text(before))))
    if op == "read":
        n = _log_int(rng, 1, 16)
        lens = [_log_int(rng, 1, 4096) for _ in range(n)]
        before = [rng.choice([0, 0, _log_int(rng, 1, 500)]) for _ in range(n)]
        return _drop_name(_case("", op, _text(lens), **dict(kw, before=_text(before))))
    if op == "prompt":
        total, lens, before = _log_int(rng, 1, 8192), [], []
        while total > 0:
            lens.append(min(total, _log_int(rng, 1, 8192)))
            total -= lens[-1]
            before.append(rng.choice([0, 0, 0, _log_int(rng, 1, 2048), -_log_int(rng, 1, lens[-1])]))
            if len(lens) >= 48:
                break
        while sum(lens) + sum(before) > 14000:
            before[before.index(max(before))] = 0
        del kw["fmt"], kw["page"]
        return _drop_name(_case("", op, _text(lens), **dict(kw, before=_text(before), fused=rng.random() < 0.5, lse=rng.random() < 0.5)))
    n, most = _log_int(rng, 1, 128), 131072
    lens = [_log_int(rng, 1, max(1, min(most, 400000 // n))) for _ in range(n)]
    if rng.random() < 0.3:
        lens[rng.randrange(n)] = 0                   # a sequence that has no key yet
    return _drop_name(_case("", op, _text(lens), **dict(kw, lse=rng.random() < 0.5)))


def _drop_name(c):
    del c["name"]
    return c


# ---- inputs ----

def frequencies(rot, factor, base=10000.0, fast=32.0, slow=1.0):
    """rot / 2 frequencies, and the factor on cos and sin.  factor > 1: those that turn more than `fast` times within the trained
    context stay, those that turn less than `slow` times are divided by the factor, a ramp in between; cos and sin times 0.1 ln factor + 1."""
    i = np.arange(rot // 2, dtype=np.float64)
    f = base ** (-2.0 * i / rot)
    if factor == 1.0:
        return f, 1.0
    at = lambda turns: rot * math.log(TRAINED / (turns * 2 * math.pi)) / (2 * math.log(base))  # noqa: E731
    lo, hi = max(0.0, math.floor(at(fast))), min(rot - 1.0, math.ceil(at(slow)))
    ramp = np.clip((i - lo) / max(hi - lo, 1e-3), 0.0, 1.0)
    return f * (1.0 - ramp) + f / factor * ramp, 0.1 * math.log(factor) + 1.0


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _rows(g, *shape, spread=1.0):
    return (torch.randn(*shape, generator=g, device=DEV, dtype=torch.float32) * spread).to(torch.bfloat16)


def _scale_byte(x):
    """e8m0 byte of the smallest power of two with max|row| <= 448 * 2^e (at least 2^-126)."""
    b = x.float().abs().amax(-1).view(torch.int32)
    return ((b >> 23) - 8 + ((b & 0x7FFFFF) > 0x600000).to(torch.int32)).clamp(min=1)


def _power(byte):
    return (byte.to(torch.int32) << 23).view(torch.float32)


def _quantised(x):
    """e4m3 codes of rows, and their scale bytes."""
    e = _scale_byte(x)
    return (x.float() * _power(254 - e).unsqueeze(-1)).to(torch.float8_e4m3fn), e.to(torch.uint8)


def _pools(c, n_pages, g, used):
    """K and V pools [pages, Hk, page, D]; slots that no sequence uses hold NaN, as memory that was never written may."""
    (k, ks), (v, vs) = _pool(c, n_pages, g, used), _pool(c, n_pages, g, used)
    return dict(k_pool=k, v_pool=v) if ks is None else dict(k_pool=k, v_pool=v, k_scale=ks, v_scale=vs)


def _pool(c, n_pages, g, used):
    x = _rows(g, n_pages, c["Hk"], c["page"], c["D"])
    free = ~used[:, None, :, None]
    if c["fmt"] == "bf16":
        return x.masked_fill_(free, float("nan")), None
    code, e = _quantised(x)
    code.view(torch.uint8).masked_fill_(free, 0x7F)
    return code, e


def _table(c, total, seed):
    """Pages of each sequence (drawn at random out of the pool, -1 behind its last), pages of the pool."""
    need = np.array([-(-t // c["page"]) for t in total])
    n_pages = int(need.sum()) + 3
    held = np.arange(max(1, need.max()))[None, :] < need[:, None]
    table = np.full(held.shape, -1, dtype=np.int32)
    table[held] = np.random.default_rng(seed).permutation(n_pages)[:need.sum()]
    return table, n_pages


def _split(g, c, tokens, heads, fused, spread):
    """Tensors [tokens, heads[i], D]: slices of one product's rows, or their own."""
    if not fused:
        return [_rows(g, tokens, h, c["D"], spread=s) for h, s in zip(heads, spread)]
    x = torch.cat([_rows(g, tokens, h, c["D"], spread=s) for h, s in zip(heads, spread)], 1)
    return list(x.split(heads, 1))


def prepare(case, seed):
    c, g = case, _gen(seed)
    lens, before = _ints(c["lens"]), _ints(c["before"])
    dev = lambda a, t: torch.from_numpy(np.ascontiguousarray(a, dtype=t)).to(DEV)  # noqa: E731
    s = {"case": c}
    if c["op"] in ("append", "read"):
        T = sum(lens)
        table, n_pages = _table(c, [a + b for a, b in zip(lens, before)], seed)
        seq = np.repeat(np.arange(len(lens)), lens)
        pos = np.concatenate([b + np.arange(n) for n, b in zip(lens, before)])
        s.update(seq=dev(seq, np.int32), pos=dev(pos, np.int32), pages=dev(table, np.int32))
        used = np.zeros((n_pages, c["page"]), dtype=bool)
        used[table[seq, pos // c["page"]], pos % c["page"]] = True
        for n in ("k_out", "v_out"):
            s[n] = torch.empty((T, c["Hk"], c["D"]), dtype=torch.bfloat16, device=DEV)
        if c["op"] == "read":
            s.update(_pools(c, n_pages, g, torch.from_numpy(used).to(DEV)))
            return s
        s["q"], s["k"], s["v"] = _split(g, c, T, [c["Hq"], c["Hk"], c["Hk"]], c["fused"], (1, 1, 1))
        shape = (n_pages, c["Hk"], c["page"], c["D"])
        for n in ("k", "v"):
            s[n + "_pool"] = torch.zeros(shape, dtype=torch.float8_e4m3fn if c["fmt"] == "fp8" else torch.bfloat16, device=DEV)
            if c["fmt"] == "fp8":
                s[n + "_scale"] = torch.zeros(shape[:3], dtype=torch.uint8, device=DEV)
        f, s["mscale"] = frequencies(c["rot"], c["factor"])
        s["freq"] = dev(f, np.float64)
        s["q_out"] = torch.empty((T, c["Hq"], c["D"]), dtype=torch.bfloat16, device=DEV)
        return s
    if c["op"] == "prompt":
        nk = [max(0, a + b) for a, b in zip(lens, before)]
        if c["fused"] and nk == lens:
            s["q"], s["k"], s["v"] = _split(g, c, sum(lens), [c["Hq"], c["Hk"], c["Hk"]], True, (1.5, 1, 1))
        else:
            s["q"] = _split(g, c, sum(lens), [c["Hq"]], False, (1.5,))[0]
            s["k"], s["v"] = _split(g, c, sum(nk), [c["Hk"], c["Hk"]], c["fused"], (1, 1))
        s["cu_q"], s["cu_k"] = (dev(np.concatenate([[0], np.cumsum(n)]), np.int32) for n in (lens, nk))
        s["out"] = torch.empty((sum(lens), c["Hq"], c["D"]), dtype=torch.bfloat16, device=DEV)
        s["lse"] = torch.empty((sum(lens), c["Hq"]), dtype=torch.float32, device=DEV) if c["lse"] else None
        return s
    table, n_pages = _table(c, lens, seed)
    used = np.zeros((n_pages, c["page"]), dtype=bool)
    for i, n in enumerate(lens):
        p = np.arange(n)
        used[table[i, p // c["page"]], p % c["page"]] = True
    s.update(_pools(c, n_pages, g, torch.from_numpy(used).to(DEV)))
    s["q"] = _rows(g, len(lens), c["Hq"], c["D"], spread=1.5)
    s.update(pages=dev(table, np.int32), lens=dev(lens, np.int32))
    s["out"] = torch.empty_like(s["q"])
    s["lse"] = torch.empty((len(lens), c["Hq"]), dtype=torch.float32, device=DEV) if c["lse"] else None
    return s


# ---- one pass ----

def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(s):
    import paper_2503_09304_amd as q
    c = s["case"]
    if c["op"] == "prompt":
        q.attn_prompt(s["q"], s["k"], s["v"], s["cu_q"], s["cu_k"], s["out"], lse=s["lse"])
        return _kept(s, "out", "lse")
    if "cache" not in s:                   # what a serving program sets up once
        s["cache"] = q.AttnCache(s["k_pool"], s["v_pool"], s.get("k_scale"), s.get("v_scale"))
        if c["op"] == "append":
            s["rope"] = q.AttnRope(s["freq"], c["layout"], s["mscale"])
        if c["op"] == "decode":
            s["ws"] = q.attn_decode_workspace(s["cache"], s["q"].shape[0], c["Hq"])
    if c["op"] == "decode":
        q.attn_decode(s["cache"], s["q"], s["pages"], s["lens"], s["out"], s["ws"], lse=s["lse"])
        return _kept(s, "out", "lse")
    if c["op"] == "append":
        q.attn_append(s["cache"], s["q"], s["k"], s["v"], s["seq"], s["pos"], s["pages"], s["rope"], s["q_out"])
        if c["fmt"] == "bf16":
            return _kept(s, "q_out", "k_pool", "v_pool")
    q.attn_read(s["cache"], s["seq"], s["pos"], s["pages"], s["k_out"], s["v_out"])
    return _kept(s, "q_out", "k_out", "v_out")


def _kept(s, *names):
    return {n: s[n] for n in names if s.get(n) is not None}


def _rotate(x, c, cos, sin):
    """x [T, heads, D] in fp32, rotated and rounded to bf16."""
    r = x[..., :c["rot"]]
    if c["layout"] == "half":
        a, b = r.chunk(2, -1)
    else:
        a, b = r[..., 0::2], r[..., 1::2]
    a, b = a * cos - b * sin, b * cos + a * sin
    r = torch.cat([a, b], -1) if c["layout"] == "half" else torch.stack([a, b], -1).flatten(-2)
    return torch.cat([r, x[..., c["rot"]:]], -1).to(torch.bfloat16)


def _value(pool, scale):
    x = pool.float()
    return x if scale is None else x * _power(scale).unsqueeze(-1)


def _attend(q, k, v, allowed):
    """q [Hk, n, D], k and v [Hk, m, D], allowed [n, m], all of them fp32: outputs, log of the sums of exponentials."""
    x = torch.bmm(q, k.transpose(1, 2).contiguous())
    x.mul_(1.0 / math.sqrt(q.shape[2]))
    x.masked_fill_(~allowed, float("-inf"))
    most = x.amax(2, keepdim=True) if x.shape[2] else x.new_full((*x.shape[:2], 1), float("-inf"))
    x.sub_(most.clamp(min=-1e30)).exp_()
    total = x.sum(2, keepdim=True)
    o = torch.bmm(x, v) / total.clamp(min=1e-30)
    return o, (most + total.log()).squeeze(2)


def _run_plain(s):
    c = s["case"]
    G = c["Hq"] // c["Hk"]
    if c["op"] == "prompt":
        T, M = s["q"].shape[0], s["k"].shape[0]
        n = s["cu_q"].shape[0]
        i, j = torch.arange(T, device=DEV), torch.arange(M, device=DEV)
        sq, sk = torch.bucketize(i, s["cu_q"].long(), right=True) - 1, torch.bucketize(j, s["cu_k"].long(), right=True) - 1
        last = i - s["cu_q"][1:n].long()[sq] + s["cu_k"][1:n].long()[sq]          # the query's own key
        allowed = (sq[:, None] == sk[None, :]) & (j[None, :] <= last[:, None])
        q = s["q"].float().view(T, c["Hk"], G, c["D"]).permute(1, 2, 0, 3).reshape(c["Hk"], G * T, c["D"])
        o, lse = _attend(q, s["k"].float().transpose(0, 1).contiguous(), s["v"].float().transpose(0, 1).contiguous(),
                         allowed.repeat(G, 1))
        s["out"].copy_(o.view(c["Hk"], G, T, c["D"]).permute(2, 0, 1, 3).reshape(T, c["Hq"], c["D"]))
        if s["lse"] is not None:
            s["lse"].copy_(lse.view(c["Hq"], T).t())
        return _kept(s, "out", "lse")
    if c["op"] == "decode":
        B, L = s["pages"].shape[0], s["pages"].shape[1] * c["page"]
        at = s["pages"].clamp(min=0).long()
        use = torch.arange(L, device=DEV)[None, :] < s["lens"][:, None]
        k, v = (_value(s[n + "_pool"][at], s[n + "_scale"][at] if n + "_scale" in s else None).transpose(2, 3).reshape(B, L, c["Hk"], c["D"])
                .masked_fill(~use[:, :, None, None], 0.0).transpose(1, 2).reshape(B * c["Hk"], L, c["D"]) for n in ("k", "v"))
        o, lse = _attend(s["q"].float().view(B * c["Hk"], G, c["D"]), k, v, use.repeat_interleave(c["Hk"], 0)[:, None, :])
        s["out"].copy_(o.view(B, c["Hq"], c["D"]))
        if s["lse"] is not None:
            s["lse"].copy_(lse.view(B, c["Hq"]))
        return _kept(s, "out", "lse")
    page = s["pages"][s["seq"].long(), s["pos"].long() // c["page"]].long()
    slot = s["pos"].long() % c["page"]
    if c["op"] == "append":
        a = s["pos"].double()[:, None] * s["freq"][None, :]
        cos, sin = ((f(a) * s["mscale"]).float().unsqueeze(1) for f in (torch.cos, torch.sin))
        s["q_out"].copy_(_rotate(s["q"].float(), c, cos, sin))
        _store(s, "k", page, slot, _rotate(s["k"].float(), c, cos, sin))
        _store(s, "v", page, slot, s["v"])
        if c["fmt"] == "bf16":
            return _kept(s, "q_out", "k_pool", "v_pool")
    s["k_out"].copy_(_fetch(s, "k", page, slot))
    s["v_out"].copy_(_fetch(s, "v", page, slot))
    return _kept(s, "q_out", "k_out", "v_out")


def _store(s, n, page, slot, x):
    pool = s[n + "_pool"]
    if pool.dtype == torch.bfloat16:
        pool[page, :, slot] = x
    else:
        code, e = _quantised(x)
        pool.view(torch.uint8)[page, :, slot] = code.view(torch.uint8)
        s[n + "_scale"][page, :, slot] = e


def _fetch(s, n, page, slot):
    pool = s[n + "_pool"]
    if pool.dtype == torch.bfloat16:
        return pool[page, :, slot]
    return _value(pool.view(torch.uint8)[page, :, slot].view(torch.float8_e4m3fn), s[n + "_scale"][page, :, slot])


# ---- what a pass cannot do without ----

def work(case):
    c = case
    lens, before = _ints(c["lens"]), _ints(c["before"])
    T, row = sum(lens), 2 * c["D"]
    held = c["D"] + 1 if c["fmt"] == "fp8" else row               # a key or value in the cache, its scale with it
    if c["op"] == "append":
        b = T * (row * (2 * c["Hq"] + 2 * c["Hk"]) + 2 * c["Hk"] * held + 8)
        if c["fmt"] == "fp8":
            b += T * 2 * c["Hk"] * (held + row)                   # read back
        return {"bytes": b, "flops": 3 * T * (c["Hq"] + c["Hk"]) * c["rot"]}
    if c["op"] == "read":
        return {"bytes": T * (2 * c["Hk"] * (held + row) + 8), "flops": 0}
    if c["op"] == "prompt":
        pairs, keys = 0, 0
        for n, b in zip(lens, before):
            m = max(0, n + b)
            seen = min(n, m)                                      # queries that see a key: the last of them all m
            pairs += seen * m - seen * (seen - 1) // 2
            keys += m
        return {"bytes": row * (2 * T * c["Hq"] + 2 * keys * c["Hk"]), "flops": 4 * pairs * c["Hq"] * c["D"]}
    return {"bytes": T * 2 * c["Hk"] * held + len(lens) * 2 * c["Hq"] * row, "flops": 4 * T * c["Hq"] * c["D"]}


# ---- the definition in 64 bits ----

def exact(case, seed):
    s = prepare(case, seed)
    c = case
    lens = _ints(c["lens"])
    G, D = c["Hq"] // c["Hk"], c["D"]

    def softmax_rows(q, k, v, seen):
        """q [n, D], k and v [m, D]; row i sees its first seen[i] keys."""
        x = (q @ k.t()) / math.sqrt(D)
        x = torch.where(torch.arange(k.shape[0], device=DEV)[None, :] < seen[:, None], x, torch.full_like(x, -math.inf))
        lse = torch.logsumexp(x, 1) if k.shape[0] else torch.full((q.shape[0],), -math.inf, dtype=torch.float64, device=DEV)
        p = torch.exp(x - torch.where(torch.isinf(lse), torch.zeros_like(lse), lse)[:, None])
        return p @ v, lse

    def pool_rows(n, pages, slots):
        """[tokens, Hk, D] of the pool `n` in 64 bits."""
        x = s[n + "_pool"]
        if c["fmt"] != "fp8":
            return x[pages, :, slots].double()
        return x.view(torch.uint8)[pages, :, slots].view(torch.float8_e4m3fn).double() * torch.pow(
            2.0, s[n + "_scale"][pages, :, slots].double() - 127.0).unsqueeze(-1)

    if c["op"] in ("prompt", "decode"):
        B = len(lens)
        out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
        lse = torch.full(s["q"].shape[:2], -math.inf, dtype=torch.float64, device=DEV)
        for b in range(B):
            if c["op"] == "prompt":
                (q0, q1), (k0, k1) = ([int(v) for v in s[n][b:b + 2]] for n in ("cu_q", "cu_k"))
                k, v = s["k"][k0:k1].double(), s["v"][k0:k1].double()
            else:
                q0, q1, k0, k1 = b, b + 1, 0, lens[b]
                p = torch.arange(k1, device=DEV)
                k, v = (pool_rows(n, s["pages"][b].long()[p // c["page"]], p % c["page"]) for n in ("k", "v"))
            if q1 == q0 or k1 == k0:
                continue
            for h in range(c["Hq"]):
                for r0 in range(q0, q1, 4096):                    # rows at a time, so that the largest fits
                    r1 = min(q1, r0 + 4096)
                    seen = torch.arange(r0 - q1, r1 - q1, device=DEV) + 1 + (k1 - k0)
                    out[r0:r1, h], lse[r0:r1, h] = softmax_rows(s["q"][r0:r1, h].double(), k[:, h // G], v[:, h // G], seen)
        return {"out": out, "lse": lse} if c["lse"] else {"out": out}

    pos, seq = s["pos"].long(), s["seq"].long()
    page, slot = s["pages"][seq, pos // c["page"]].long(), pos % c["page"]
    if c["op"] == "read":
        return {n + "_out": pool_rows(n, page, slot) for n in ("k", "v")}

    angle = pos.double()[:, None] * s["freq"][None, :]
    turn = torch.polar(torch.full_like(angle, s["mscale"]), angle)[:, None, :]

    def turned(x):
        x = x.double().clone()
        half = c["rot"] // 2
        first = slice(0, half) if c["layout"] == "half" else slice(0, c["rot"], 2)
        second = slice(half, c["rot"]) if c["layout"] == "half" else slice(1, c["rot"], 2)
        z = torch.complex(x[..., first], x[..., second]) * turn
        x[..., first], x[..., second] = z.real, z.imag
        return x

    k, v = turned(s["k"]), s["v"].double()
    out = {"q_out": turned(s["q"])}
    if c["fmt"] == "bf16":
        for n, x in (("k", k), ("v", v)):
            out[n + "_pool"] = torch.zeros(s[n + "_pool"].shape, dtype=torch.float64, device=DEV)
            out[n + "_pool"][page, :, slot] = x
        return out


    def power(n):
        return ((n.to(torch.int64) + 1023) << 52).view(torch.float64)

    def nearest(x, bits, least=-900):
        """To `bits` significant bits, half to even; steps no finer than those of the binade of 2^least."""
        step = power((torch.frexp(x)[1] - bits).clamp(min=least + 1 - bits))
        return torch.round(x / step) * step

    def held(x):
        """What the 8-bit cache holds for rows of bf16 values."""
        x = nearest(x, 8)
        part, n = torch.frexp(x.abs().amax(-1, keepdim=True))       # 448 = 0.875 * 2^9
        unit = power((n - 9 + (part > 0.875).to(n.dtype)).clamp(min=-126))
        return nearest(x / unit, 4, -6) * unit

    return dict(out, k_out=held(k), v_out=held(v))
