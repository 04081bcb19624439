"""The attention calls against a plain implementation in 64 bits (-m gpu).

Bars.  A rounding to bf16 is off by at most HALF = 2^-8 of the value.  Attention has two: of the weights exp(x - m), which are
a matrix operand, and of the output.  With A = sum_j p_j |v_j| the first moves an output by at most HALF * A, the second by HALF of
the value.  Scores are fp32 sums of D exact products: off by at most (D + 4) 2^-24 S, S = scale * sum |q k| at its largest in the row, and that
relative error goes into each weight and into the total; exponentials and fp32 sums add less than 2^-17.  So
    |o - o_ref| <= (HALF + 2^-17 + 2 (D + 4) 2^-24 S) A + HALF (|o_ref| + that)
    |lse - ref| <= (D + 4) 2^-24 S + 2^-17 + 2^-22 |ref|
Rotations are three fp32 roundings of values up to |a| + |b| with cos and sin off by 2^-22, then one to bf16.  What the cache holds and what
is read back is compared bit for bit."""
import math

import numpy as np
import pytest
import torch

import paper_2503_09304_amd as q

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
HALF = torch.finfo(torch.bfloat16).eps / 2
NAN = float("nan")


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def rows(g, T, heads, D, spread=1.0, pad=0, lead=0):
    """bf16 [T, heads, D]; pad, lead: elements between tokens and in front, all NaN."""
    x = torch.full((T * (heads * D + pad) + lead,), NAN, dtype=torch.bfloat16, device=DEV)
    x = x[lead:].view(T, heads * D + pad)[:, :heads * D].view(T, heads, D) if T else torch.empty((0, heads, D), dtype=torch.bfloat16, device=DEV)
    x.copy_(torch.randn(T, heads, D, generator=g, device=DEV) * spread)
    return x


def reference(qq, k, v, seen, scale):
    """qq [n, D], k, v [m, D] in 64 bits, row i sees its first seen[i] keys: output, lse, sum p|v|, largest scale*sum|qk|."""
    if k.shape[0] == 0:
        n = qq.shape[0]
        zero = torch.zeros((n, v.shape[1]), dtype=torch.float64, device=qq.device)
        return zero, torch.full((n,), -math.inf, dtype=torch.float64, device=qq.device), zero, zero[:, 0]
    x = scale * (qq @ k.t())
    hide = torch.arange(k.shape[0], device=qq.device)[None, :] >= seen[:, None]
    x = x.masked_fill(hide, -math.inf)
    lse = torch.logsumexp(x, 1)
    p = torch.exp(x - torch.where(torch.isinf(lse), torch.zeros_like(lse), lse)[:, None]).masked_fill(hide, 0.0)
    big = (scale * (qq.abs() @ k.abs().t())).masked_fill(hide, 0.0).amax(1)
    return p @ v, lse, p @ v.abs(), big


def check(o, lse, ref, D, what):
    ro, rl, A, S = ref
    rel = (D + 4) * 2.0 ** -24 * S
    slack = (HALF + 2.0 ** -17 + 2 * rel)[:, None] * A
    err = (o.double() - ro).abs()
    bar = slack + HALF * (ro.abs() + slack)
    assert torch.isfinite(o).all(), what
    assert (err <= bar).all(), (what, float((err - bar).max()), float((err / bar.clamp(min=1e-30)).max()))
    if lse is not None:
        none = torch.isinf(rl)
        assert torch.equal(torch.isinf(lse.double()), none) and (lse[none] < 0).all(), what
        ok = (lse.double() - rl).abs()[~none] <= (rel + 2.0 ** -17 + 2.0 ** -22 * rl.abs())[~none]
        assert ok.all(), what


def run_prompt(nq, nk, Hq, Hk, D, causal=True, seed=0, spread=1.0, scale=None, fused=False, lead=0):
    g = gen(seed)
    Tq, Tk = sum(nq), sum(nk)
    if fused:
        whole = rows(g, Tq, Hq + 2 * Hk, D, spread)
        qq, k, v = whole.split([Hq, Hk, Hk], 1)
    else:
        qq, k, v = rows(g, Tq, Hq, D, spread, pad=24, lead=lead), rows(g, Tk, Hk, D, spread, pad=8, lead=lead), rows(g, Tk, Hk, D, lead=lead)
    cq, ck = (torch.from_numpy(np.concatenate([[0], np.cumsum(n)]).astype(np.int32)).to(DEV) for n in (nq, nk))
    out = torch.full((Tq, Hq, D), NAN, dtype=torch.bfloat16, device=DEV)
    lse = torch.full((Tq, Hq), NAN, dtype=torch.float32, device=DEV)
    assert q.attn_prompt(qq, k, v, cq, ck, out, scale=scale, causal=causal, lse=lse) == q.MOE_OK
    torch.cuda.synchronize()
    G, q0, k0 = Hq // Hk, 0, 0
    for b, (n, m) in enumerate(zip(nq, nk)):
        for h in range(Hq):
            seen = torch.arange(n, device=DEV) + 1 + m - n if causal else torch.full((n,), m, device=DEV)
            ref = reference(qq[q0:q0 + n, h].double(), k[k0:k0 + m, h // G].double(), v[k0:k0 + m, h // G].double(), seen, scale or D ** -0.5)
            check(out[q0:q0 + n, h], lse[q0:q0 + n, h], ref, D, (b, h, n, m))
        q0, k0 = q0 + n, k0 + m
    return out, lse


@pytest.mark.parametrize("n", [1, 2, 15, 16, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 385, 515])
def test_prompt_lengths(n):
    run_prompt([n], [n], 4, 2, 128, seed=n)


@pytest.mark.parametrize("D", [16, 32, 48, 64, 80, 96, 112, 128])
@pytest.mark.parametrize("Hq,Hk", [(6, 2), (3, 3)])
def test_prompt_dims_and_heads(D, Hq, Hk):
    run_prompt([70, 129], [70, 129], Hq, Hk, D, seed=D)


@pytest.mark.parametrize("Hq,Hk", [(32, 8), (8, 1), (40, 5), (16, 16), (24, 12), (71, 71)])
def test_prompt_head_layouts(Hq, Hk):
    run_prompt([37, 90], [37, 90], Hq, Hk, 64, seed=Hq)


@pytest.mark.parametrize("causal", [True, False])
def test_prompt_packed_with_empty_short_and_ahead(causal):
    """No query, no key, fewer keys than queries (rows without keys), contexts in front."""
    nq = [0, 1, 64, 200, 33, 100, 5, 130, 0, 1]
    nk = [7, 1, 64, 0, 20, 300, 1000, 129, 0, 257]
    out, lse = run_prompt(nq, nk, 4, 2, 64, causal, seed=3)
    assert (out[65:265] == 0).all() and torch.isinf(lse[65:265]).all()
    run_prompt(nq, nk, 4, 1, 128, causal, seed=4)


def test_prompt_slices_of_one_product_and_odd_strides():
    run_prompt([100, 61], [100, 61], 8, 2, 128, seed=5, fused=True)
    run_prompt([100, 61], [100, 61], 8, 2, 96, seed=6, lead=8)


def test_prompt_peaked_rows_and_large_scores():
    """Maxima that keep rising, and scores in the hundreds: the running maximum is taken over many times."""
    run_prompt([300], [300], 2, 2, 128, seed=7, spread=6.0)
    run_prompt([300], [300], 2, 2, 64, seed=8, spread=1.0, scale=3.0)
    g = gen(9)
    n, D = 400, 64
    qq, v = rows(g, n, 1, D), rows(g, n, 1, D)
    k = (qq.float().mean(0, keepdim=True) * 0 + 1).expand(n, 1, D).to(torch.bfloat16).contiguous()
    k.mul_(torch.arange(n, device=DEV)[:, None, None] / 8.0)                       # each key above the one before, for queries of one sign
    qq.abs_()
    cu = torch.tensor([0, n], dtype=torch.int32, device=DEV)
    out, lse = torch.empty_like(qq), torch.empty((n, 1), dtype=torch.float32, device=DEV)
    q.attn_prompt(qq, k, v, cu, cu, out, scale=1.0, lse=lse)
    ref = reference(qq[:, 0].double(), k[:, 0].double(), v[:, 0].double(), torch.arange(n, device=DEV) + 1, 1.0)
    check(out[:, 0], lse[:, 0], ref, D, "rising")


def test_prompt_long():
    run_prompt([3000, 1100], [3000, 2100], 2, 1, 128, seed=10)
    run_prompt([2100], [2100], 2, 2, 64, seed=11)


def test_prompt_many_workgroups():
    """Enough queries that the variant for full launches runs."""
    run_prompt([700, 1, 515, 260, 1300], [700, 1, 600, 260, 1300], 40, 8, 128, seed=12)
    run_prompt([700, 1, 515, 260, 1300], [700, 1, 600, 260, 1300], 40, 40, 64, seed=13)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("D", [64, 128, 80])
def test_prompt_few_queries_many_keys(causal, D):
    """Keys of a query cut into parts: parts that a query does not reach, short sequences that are not cut, and rows without keys among them."""
    assert q.attention._lib().attn_prompt_workspace_bytes(5, 399, 12290, 2, 1, D) > 0
    run_prompt([130, 1, 7, 200, 61], [6000, 2050, 7, 4213, 20], 2, 1, D, causal, seed=18)
    run_prompt([1], [9001], 1, 1, D, causal, seed=19)
    run_prompt([700], [700], 1, 1, D, causal, seed=20)


@pytest.mark.parametrize("causal", [True, False])
def test_prompt_more_sequences_than_lanes(causal):
    """150 sequences, some of several tiles, empty ones and contexts among them: every tile is somebody's."""
    nq = [(37 * i) % 61 if i % 29 else 150 + i for i in range(150)]
    nk = [n + (0, 0, 200, -5)[i % 4] if n > 5 else n for i, n in enumerate(nq)]
    run_prompt(nq, nk, 2, 1, 64, causal, seed=17)


@pytest.mark.parametrize("Hq,Hk", [(4, 2), (4, 1), (12, 3), (3, 3)])
@pytest.mark.parametrize("causal", [True, False])
def test_prompt_parts_among_more_sequences_than_lanes(causal, Hq, Hk):
    """100 sequences of which a few are cut, one of them with tiles of queries that are cut into different numbers of parts."""
    nq = [(13 * i) % 19 for i in range(100)]
    nk = [n + (0, 30, -3)[i % 3] if n > 3 else n for i, n in enumerate(nq)]
    nq[3], nk[3], nq[70], nk[70], nq[71], nk[71], nq[99], nk[99] = 1, 40000, 700, 2100, 9, 30000, 130, 21000
    assert q.attention._lib().attn_prompt_workspace_bytes(100, sum(nq), sum(nk), Hq, Hk, 64) > 0
    run_prompt(nq, nk, Hq, Hk, 64, causal, seed=21)


def test_prompt_neighbours_do_not_leak():
    """Sequences of NaN and infinity beside others, and rows behind the last sequence."""
    g = gen(14)
    lens = [50, 70, 64]
    T = sum(lens) + 9
    qq, k, v = rows(g, T, 4, 64), rows(g, T, 2, 64), rows(g, T, 2, 64)
    for x in (qq, k, v):
        x[50:120] = NAN if x is not v else math.inf
        x[184:] = NAN
    cu = torch.tensor([0, 50, 120, 184], dtype=torch.int32, device=DEV)
    out = torch.full((T, 4, 64), 3.0, dtype=torch.bfloat16, device=DEV)
    q.attn_prompt(qq, k, v, cu, cu, out)
    assert (out[184:] == 3).all()                                               # no sequence's rows: untouched
    for a, b in ((0, 50), (120, 184)):
        for h in range(4):
            ref = reference(qq[a:b, h].double(), k[a:b, h // 2].double(), v[a:b, h // 2].double(), torch.arange(b - a, device=DEV) + 1, 0.125)
            check(out[a:b, h], None, ref, 64, (a, h))


def test_prompt_offsets_out_of_range_are_clamped():
    g = gen(15)
    n = 40
    qq, k, v = rows(g, n, 2, 64), rows(g, n, 2, 64), rows(g, n, 2, 64)
    out = torch.zeros((n, 2, 64), dtype=torch.bfloat16, device=DEV)
    good = torch.zeros_like(out)
    q.attn_prompt(qq, k, v, *(torch.tensor([0, 30, 40], dtype=torch.int32, device=DEV),) * 2, good)
    wild = torch.tensor([-5, 30, 1 << 30], dtype=torch.int32, device=DEV)
    q.attn_prompt(qq, k, v, wild, wild, out)
    assert torch.equal(out, good)
    down = torch.tensor([0, 30, 10], dtype=torch.int32, device=DEV)             # the second sequence has no row
    out.fill_(7)
    q.attn_prompt(qq, k, v, down, down, out)
    assert torch.equal(out[:30], good[:30]) and (out[30:] == 7).all()


def test_prompt_is_the_same_every_time_and_on_another_stream():
    g = gen(16)
    n, cu = 600, torch.tensor([0, 600], dtype=torch.int32, device=DEV)
    qq, k, v = rows(g, n, 8, 128), rows(g, n, 2, 128), rows(g, n, 2, 128)
    a, b = torch.empty_like(qq), torch.empty_like(qq)
    q.attn_prompt(qq, k, v, cu, cu, a)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        q.attn_prompt(qq, k, v, cu, cu, b)
    s.synchronize()
    assert torch.equal(a.view(torch.int16), b.view(torch.int16))


# ---- cache ----

def table(lens, page, seed, width=None):
    """Pages drawn at random; -1 behind each sequence's last."""
    need = [-(-n // page) for n in lens]
    n_pages = sum(need) + 2
    t = np.full((len(lens), width or max(1, max(need))), -1, dtype=np.int32)
    order, at = np.random.default_rng(seed).permutation(n_pages), 0
    for i, n in enumerate(need):
        t[i, :n] = order[at:at + n]
        at += n
    return torch.from_numpy(t).to(DEV), n_pages


def fresh(n_pages, Hk, page, D, fp8):
    """A cache whose every slot holds NaN (fp8: and the largest scale byte)."""
    c = q.AttnCache.empty(n_pages, Hk, page, D, fp8)
    for x in (c.k, c.v):
        x.fill_(0x7F if fp8 else NAN)
    if fp8:
        c.k_scale.fill_(255)
        c.v_scale.fill_(255)
    return c


def quantised(x):
    """What the fp8 cache holds for bf16 rows, from the definition in 64 bits."""
    x = x.double().cpu()
    part, n = torch.frexp(x.abs().amax(-1, keepdim=True))
    e = torch.where(part > 0, n - 9 + (part > 0.875).to(n.dtype), torch.full_like(n, -126)).clamp(min=-126).double()
    y = x * torch.exp2(-e)
    step = torch.exp2((torch.frexp(y)[1] - 4).clamp(min=-9).double())
    most = 1.875 * 2.0 ** 127                                          # 2^128 is no bf16
    return (torch.round(y / step) * step * torch.exp2(e)).clamp(-most, most).to(DEV)


def rotated(x, pos, f, layout, mscale):
    x = x.double()
    ang = pos.double()[:, None, None] * torch.tensor(f, dtype=torch.float64, device=DEV)
    c, s, n = torch.cos(ang) * mscale, torch.sin(ang) * mscale, len(f)
    i = torch.arange(n, device=DEV)
    a, b = (i, i + n) if layout == "half" else (2 * i, 2 * i + 1)
    r = x.clone()
    r[..., a], r[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
    size = x.abs().clone()
    size[..., a] = size[..., b] = x[..., a].abs() + x[..., b].abs()
    return r, size * mscale


CACHES = [(16, 128, 4), (64, 64, 2), (32, 80, 1), (256, 112, 3), (128, 16, 5), (16, 48, 2)]


@pytest.mark.parametrize("page,D,Hk", CACHES)
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_append_and_read(page, D, Hk, fp8, layout):
    g, Hq = gen(page + D), 2 * Hk
    before, lens = [0, 3, page - 1, 2 * page, 100000 // page * page + 5], [1, 40, 3, page + 1, 9]
    seq = torch.tensor(np.repeat(np.arange(5), lens).astype(np.int32), device=DEV)
    pos = torch.tensor(np.concatenate([b + np.arange(n) for b, n in zip(before, lens)]).astype(np.int32), device=DEV)
    T = len(seq)
    order = torch.randperm(T, generator=torch.Generator().manual_seed(1)).to(DEV)            # tokens in any order
    seq, pos = seq[order].contiguous(), pos[order].contiguous()
    pages, n_pages = table([b + n for b, n in zip(before, lens)], page, 2)
    c = fresh(n_pages, Hk, page, D, fp8)
    f, m = q.attn_rope_frequencies(D if D % 32 else D // 2, 10000.0, "ramp", 4.0)
    rope = q.AttnRope(torch.tensor(f, dtype=torch.float64, device=DEV), layout, m)
    qq, k, v = rows(g, T, Hq, D, pad=16), rows(g, T, Hk, D, pad=8), rows(g, T, Hk, D)
    qo, ko = torch.full((T, Hq, D), NAN, dtype=torch.bfloat16, device=DEV), torch.full((T, Hk, D), NAN, dtype=torch.bfloat16, device=DEV)
    bad = torch.zeros(1, dtype=torch.int32, device=DEV)
    assert q.attn_append(c, qq, k, v, seq, pos, pages, rope, qo, ko, bad) == q.MOE_OK
    for got, x in ((qo, qq), (ko, k)):
        want, size = rotated(x, pos, f, layout, m)
        slack = size * (2.0 ** -22 + 2 * 2.0 ** -24)
        assert ((got.double() - want).abs() <= slack + HALF * (want.abs() + slack)).all()
    k2, v2 = torch.empty_like(ko), torch.empty_like(ko)
    q.attn_read(c, seq, pos, pages, k2, v2, bad)
    assert torch.equal(k2.double(), quantised(ko) if fp8 else ko.double())
    assert torch.equal(v2.double(), quantised(v) if fp8 else v.double())
    assert int(bad) == 0
    # the slots of the tokens are what was written, no other slot
    at = pages[seq.long(), pos.long() // page].long()
    used = torch.zeros((n_pages, page), dtype=torch.bool, device=DEV)
    used[at, pos.long() % page] = True
    for x in (c.k, c.v):
        rest = x.transpose(1, 2)[~used]
        assert (rest == 0x7F).all() if fp8 else rest.isnan().all()
    if fp8:
        assert (c.k_scale.transpose(1, 2)[~used] == 255).all() and (c.v_scale.transpose(1, 2)[~used] == 255).all()


def test_append_in_place_without_rotation_and_without_queries():
    g = gen(20)
    T, Hk, D = 37, 2, 64
    pages, n_pages = table([T], 16, 3)
    pos = torch.arange(T, dtype=torch.int32, device=DEV)
    seq = torch.zeros_like(pos)
    f, m = q.attn_rope_frequencies(64)
    rope = q.AttnRope(torch.tensor(f, dtype=torch.float64, device=DEV))
    qq, k, v = rows(g, T, 4, D), rows(g, T, Hk, D), rows(g, T, Hk, D)
    qo, ko = torch.empty_like(qq), torch.empty_like(k)
    c = fresh(n_pages, Hk, 16, D, False)
    q.attn_append(c, qq, k, v, seq, pos, pages, rope, qo, ko)
    q2, k2, c2 = qq.clone(), k.clone(), fresh(n_pages, Hk, 16, D, False)
    q.attn_append(c2, q2, k2, v, seq, pos, pages, rope, q2, k2)
    assert torch.equal(q2, qo) and torch.equal(k2, ko)
    c3 = fresh(n_pages, Hk, 16, D, False)
    q.attn_append(c3, None, k, v, seq, pos, pages, None, None)                   # no rotation: keys as they are
    k3, v3 = torch.empty_like(k), torch.empty_like(v)
    q.attn_read(c3, seq, pos, pages, k3, v3)
    assert torch.equal(k3, k) and torch.equal(v3, v)


def test_append_far_positions_keep_their_angle():
    g = gen(21)
    pos = torch.tensor([0, 1, 131071, 1 << 20, (1 << 24) + 1, (1 << 30) + 12345], dtype=torch.int32, device=DEV)
    T, D = len(pos), 128
    f, m = q.attn_rope_frequencies(D)
    rope = q.AttnRope(torch.tensor(f, dtype=torch.float64, device=DEV), "half", m)
    qq, k = rows(g, T, 1, D), rows(g, T, 1, D)
    pages = torch.zeros((1, 1), dtype=torch.int32, device=DEV)
    c = fresh(1, 1, 256, D, False)
    qo, ko, bad = torch.empty_like(qq), torch.empty_like(k), torch.zeros(1, dtype=torch.int32, device=DEV)
    q.attn_append(c, qq, k, k, torch.zeros_like(pos), pos, pages, rope, qo, ko, bad)
    for got, x in ((qo, qq), (ko, k)):
        want, size = rotated(x, pos, f, "half", m)
        slack = size * (2.0 ** -22 + 2 * 2.0 ** -24)
        assert ((got.double() - want).abs() <= slack + HALF * (want.abs() + slack)).all()
    assert int(bad) == 4                                                        # four positions behind the sequence's one page: rotated, not kept


def test_rows_of_extremes_in_the_fp8_cache():
    """Zero rows, the smallest and largest bf16, maxima at the edge between two scales, values that round to zero or half way."""
    D = 32
    r = []
    for top in (0.0, 1.75, 1.7578125, 2.0, 448.0, 450.0, 2.0 ** -126, 2.0 ** -133, 1.1754943508222875e-38, 3.3e38, 1e-30):
        x = torch.zeros(D)
        x[3] = -top
        x[5] = top * 0.531                                             # half way between codes, among others
        x[7:23] = (top * (torch.arange(1, 17) / 17.0).double() * 2.0 ** -torch.arange(16.0).double()).float()
        r.append(x)
    v = torch.stack(r).to(torch.bfloat16).to(DEV).unsqueeze(1)
    T = v.shape[0]
    pos = torch.arange(T, dtype=torch.int32, device=DEV)
    pages = torch.zeros((1, 1), dtype=torch.int32, device=DEV)
    c = fresh(1, 1, 16, D, True)
    q.attn_append(c, None, v, v, torch.zeros_like(pos), pos, pages, None, None)
    k2, v2 = torch.empty_like(v), torch.empty_like(v)
    q.attn_read(c, torch.zeros_like(pos), pos, pages, k2, v2)
    want = quantised(v)
    normal = (want.abs() >= 2.0 ** -126) | (want == 0)
    assert torch.equal(v2.double()[normal], want[normal]) and torch.equal(k2, v2)
    assert (v2.double() - want).abs()[~normal].max() <= 2.0 ** -126 if (~normal).any() else True     # below the smallest normal: may go to zero


def test_places_out_of_range():
    g = gen(22)
    T, Hk, D, page = 9, 2, 64, 16
    #        good  good  seq<0 seq>   pos<0 behind page-1 page>  good
    seq = torch.tensor([0, 1, -1, 2, 0, 0, 1, 1, 0], dtype=torch.int32, device=DEV)
    pos = torch.tensor([0, 17, 3, 3, -1, 32, 0, 18, 31], dtype=torch.int32, device=DEV)
    pages = torch.tensor([[3, 0], [-1, 2]], dtype=torch.int32, device=DEV)
    pages[0, 1], pages[1, 1] = 1, 4                                              # the pool has 4 pages: 4 is none
    k, v = rows(g, T, Hk, D), rows(g, T, Hk, D)
    c = fresh(4, Hk, page, D, False)
    bad = torch.zeros(1, dtype=torch.int32, device=DEV)
    ko = torch.full_like(k, 5.0)
    q.attn_append(c, None, k, v, seq, pos, pages, None, None, ko, bad)
    good = torch.tensor([0, 8], device=DEV)
    # tokens 1, 2, 3, 5, 6, 7 have no slot; token 4 is padding: written nowhere, counted nowhere
    assert int(bad) == 6
    assert torch.equal(ko[pos >= 0], k[pos >= 0]) and (ko[4] == 5).all()
    assert int((~c.k.isnan()).sum()) == 2 * Hk * D
    k2, v2 = torch.full_like(k, 9.0), torch.full_like(v, 9.0)
    q.attn_read(c, seq, pos, pages, k2, v2, bad)
    assert int(bad) == 12
    assert torch.equal(k2[good], k[good]) and torch.equal(v2[good], v[good])
    rest = torch.ones(T, dtype=torch.bool, device=DEV)
    rest[good] = False
    assert (k2[rest] == 0).all() and (v2[rest] == 0).all()


# ---- decode ----

def run_decode(lens, Hq, Hk, D, page=16, fp8=False, seed=0, spread=1.0, width=None, pad=0):
    g = gen(seed)
    pages, n_pages = table(lens, page, seed, width)
    c = fresh(n_pages, Hk, page, D, fp8)
    B, T = len(lens), sum(lens)
    seq = torch.from_numpy(np.repeat(np.arange(B), lens).astype(np.int32)).to(DEV)
    pos = torch.from_numpy(np.concatenate([np.arange(n) for n in lens] + [np.zeros(0)]).astype(np.int32)).to(DEV)
    k, v = rows(g, T, Hk, D, spread), rows(g, T, Hk, D)
    if T:
        q.attn_append(c, None, k, v, seq, pos, pages, None, None)
        q.attn_read(c, seq, pos, pages, k, v)                                    # what the cache holds
    qq = rows(g, B, Hq, D, spread, pad=pad)
    ln = torch.tensor(lens, dtype=torch.int32, device=DEV)
    ws = q.attn_decode_workspace(c, B, Hq)
    out, lse = torch.full((B, Hq, D), NAN, dtype=torch.bfloat16, device=DEV), torch.full((B, Hq), NAN, dtype=torch.float32, device=DEV)
    bad = torch.zeros(1, dtype=torch.int32, device=DEV)
    assert q.attn_decode(c, qq, pages, ln, out, ws, lse=lse, bad=bad) == q.MOE_OK
    torch.cuda.synchronize()
    assert int(bad) == 0
    at = 0
    for b, n in enumerate(lens):
        for hk in range(Hk):
            hs = slice(hk * Hq // Hk, (hk + 1) * Hq // Hk)
            x = qq[b, hs].double()
            ref = reference(x, k[at:at + n, hk].double(), v[at:at + n, hk].double(), torch.full((x.shape[0],), n, device=DEV), D ** -0.5)
            check(out[b, hs], lse[b, hs], ref, D, (b, hk, n))
        at += n
    counters = q.attention._lib().attn_decode_counter_bytes(B, Hq, Hk)
    assert (ws[:counters] == 0).all()
    return c, qq, pages, ln, out, ws


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("page", [16, 64, 256])
def test_decode_lengths(page, fp8):
    run_decode([0, 1, 2, 15, 16, 17, 31, 32, 33, 127, 128, 129, 255, 256, 257, 600], 8, 2, 128, page, fp8, seed=page)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("D", [16, 32, 48, 64, 80, 96, 112, 128])
def test_decode_dims(D, fp8):
    run_decode([5, 130, 77], 6, 2, D, 32, fp8, seed=D, pad=8)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("Hq,Hk", [(1, 1), (5, 5), (32, 8), (15, 1), (16, 1), (17, 1), (71, 1), (64, 2)])
def test_decode_head_layouts(Hq, Hk, fp8):
    run_decode([100, 0, 333], Hq, Hk, 64, 16, fp8, seed=Hq)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("lens", [[20000], [9001, 1, 0, 4096], [5000, 70, 3000] * 5])
def test_decode_pieces(lens, fp8):
    """Sequences long enough to be cut, alone and among short ones."""
    run_decode(lens, 8, 2, 128, 64, fp8, seed=len(lens))


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("D", [64, 128])
def test_decode_ranges(D, fp8):
    """Keys enough, in sequences uneven enough, that workgroups have ranges of them: short and empty sequences within a range, at its ends, and long ones over many."""
    lens = [0, 9000, 1, 0, 4096, 12000, 130, 7000, 0, 300, 15000, 5, 0, 2500, 128, 129, 600, 0]
    c, qq, pages, ln, out, ws = run_decode(lens, 16, 8, D, 64, fp8, seed=22)
    again = torch.full_like(out, NAN)
    q.attn_decode(c, qq, pages, ln, again, ws)
    assert torch.equal(again.view(torch.int16), out.view(torch.int16))


@pytest.mark.parametrize("fp8", [False, True])
def test_decode_ranges_with_lens_and_pages_out_of_range(fp8):
    """A length below 0 and pages that are none among sequences that are cut: counted once each."""
    lens, P = [40, 9000, 4096, 12000, 3, 7000, 15000, 2500], 64
    c, qq, pages, ln, out, ws = run_decode(lens, 16, 8, 64, P, fp8, seed=25)
    hole, wild, bad = pages.clone(), ln.clone(), torch.zeros(1, dtype=torch.int32, device=DEV)
    hole[2, 3], hole[2, 40], wild[4] = -1, c.n_pages, -7
    got, lse = torch.full_like(out, NAN), torch.zeros(8, 16, dtype=torch.float32, device=DEV)
    q.attn_decode(c, qq, hole, wild, got, ws, lse=lse, bad=bad)
    assert int(bad) == 3 and (got[4] == 0).all() and torch.isinf(lse[4]).all()
    pos = torch.arange(4096, dtype=torch.int32, device=DEV)
    k, v = (torch.empty(4096, 8, 64, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    q.attn_read(c, torch.full_like(pos, 2), pos, pages, k, v)
    seen = [i for i in range(4096) if i // P not in (3, 40)]
    for hk in range(8):
        x = qq[2, 2 * hk:2 * hk + 2].double()
        ref = reference(x, k[seen, hk].double(), v[seen, hk].double(), torch.full((2,), len(seen), device=DEV), 64 ** -0.5)
        check(got[2, 2 * hk:2 * hk + 2], lse[2, 2 * hk:2 * hk + 2], ref, 64, hk)
    q.attn_decode(c, qq, pages, ln, got, ws, bad=bad)
    assert int(bad) == 3 and torch.equal(got.view(torch.int16), out.view(torch.int16))


def test_decode_ranges_of_many_sequences():
    run_decode([(613 * i) % 997 for i in range(150)], 8, 8, 64, 16, False, seed=23)
    run_decode([(613 * i) % 997 if i % 7 else 0 for i in range(150)], 34, 2, 64, 16, True, seed=24)


def test_decode_many_sequences():
    run_decode([(37 * i) % 97 for i in range(200)], 4, 2, 64, 16, False, seed=1, width=9)


def test_decode_peaked_scores():
    run_decode([700, 300], 8, 2, 128, 16, False, seed=2, spread=5.0)
    run_decode([700, 300], 8, 2, 128, 16, True, seed=3, spread=5.0)


def test_decode_again_is_the_same_bits():
    c, qq, pages, ln, out, ws = run_decode([9000, 4000, 17], 8, 2, 128, 64, seed=4)
    for _ in range(3):
        again = torch.full_like(out, NAN)
        q.attn_decode(c, qq, pages, ln, again, ws)
        assert torch.equal(again.view(torch.int16), out.view(torch.int16))


def test_decode_lens_and_pages_out_of_range():
    c, qq, pages, ln, out, ws = run_decode([100, 64, 40], 4, 2, 64, 16, seed=5)
    bad = torch.zeros(1, dtype=torch.int32, device=DEV)
    got = torch.full_like(out, NAN)
    full = pages.clone()
    full[1, 4:], full[2, 3:] = full[1, 0], full[2, 0]                           # all entries are pages
    wild = torch.tensor([100, -7, 1 << 20], dtype=torch.int32, device=DEV)
    q.attn_decode(c, qq, full, wild, got, ws, bad=bad)
    assert int(bad) == 2 and torch.equal(got[0], out[0]) and (got[1] == 0).all()
    # a page that is none: its 16 keys are left out, as if the sequence ended before them
    hole = pages.clone()
    hole[0, 6], hole[1, 3] = -1, c.n_pages
    bad.zero_()
    q.attn_decode(c, qq, hole, ln, got, ws, bad=bad)
    assert int(bad) == 2
    want = torch.full_like(out, NAN)
    q.attn_decode(c, qq, pages, torch.tensor([96, 48, 40], dtype=torch.int32, device=DEV), want, ws)
    assert torch.equal(got.view(torch.int16), want.view(torch.int16))


def test_a_query_of_nan_shows_and_stays_alone():
    """Its output and lse are NaN, not those of a query without keys; the others' bits are what they were."""
    c, qq, pages, ln, out, ws = run_decode([700, 3, 9000], 8, 2, 128, 16, seed=8)
    lse = torch.zeros(3, 8, dtype=torch.float32, device=DEV)
    got, sick = torch.zeros_like(out), qq.contiguous()
    sick[0, 3] = sick[2, 5] = NAN
    q.attn_decode(c, sick, pages, ln, got, ws, lse=lse)
    hit = torch.zeros(3, 8, dtype=torch.bool, device=DEV)
    hit[0, 3] = hit[2, 5] = True
    assert torch.equal(lse.isnan(), hit) and got[hit].isnan().all() and torch.equal(got[~hit], out[~hit])
    g = gen(9)                                                                  # many keys: cut into parts
    x, k, v = rows(g, 40, 8, 64), rows(g, 9000, 2, 64), rows(g, 9000, 2, 64)
    cq, ck = torch.tensor([0, 40], dtype=torch.int32, device=DEV), torch.tensor([0, 9000], dtype=torch.int32, device=DEV)
    hit = torch.zeros(40, 8, dtype=torch.bool, device=DEV)
    hit[7, 1] = hit[39, 6] = True
    for m in (9000, 300):
        ck[1] = m
        a, b, lse = torch.zeros_like(x), torch.zeros_like(x), torch.zeros(40, 8, dtype=torch.float32, device=DEV)
        q.attn_prompt(x, k, v, cq, ck, a)
        q.attn_prompt(torch.where(hit[:, :, None], torch.full_like(x, NAN), x), k, v, cq, ck, b, lse=lse)
        assert torch.equal(lse.isnan(), hit) and b[hit].isnan().all() and torch.equal(b[~hit], a[~hit])


def test_workspace_refused():
    c, qq, pages, ln, out, ws = run_decode([10], 2, 1, 64, 16, seed=6)
    with pytest.raises(q.MoeError) as e:
        q.attn_decode(c, qq, pages, ln, out, ws[:-256])
    assert e.value.code == q.MOE_E_WORKSPACE
    for args in ((c, qq.float(), pages, ln, out, ws), (c, qq, pages.long(), ln, out, ws), (c, qq, pages, ln.long(), out, ws), (c, qq, pages, ln, out[:, :1], ws)):
        with pytest.raises(q.MoeError):
            q.attn_decode(*args)


def test_calls_in_a_graph():
    """A decode step recorded once and replayed with other tokens, against the same calls made one by one."""
    B, Hq, Hk, D, page = 3, 8, 2, 128, 16
    g = gen(30)
    pages = torch.arange(B * 8, dtype=torch.int32, device=DEV).view(B, 8)
    f, m = q.attn_rope_frequencies(D)
    rope = q.AttnRope(torch.tensor(f, dtype=torch.float64, device=DEV))
    qq, k, v = rows(g, B, Hq, D), rows(g, B, Hk, D), rows(g, B, Hk, D)
    pos, lens = torch.zeros(B, dtype=torch.int32, device=DEV), torch.ones(B, dtype=torch.int32, device=DEV)

    def state():
        c = q.AttnCache.empty(B * 8, Hk, page, D, True)
        return c, torch.empty_like(qq), torch.empty_like(qq), q.attn_decode_workspace(c, B, Hq)

    def step(s):
        c, qo, out, ws = s
        q.attn_append(c, qq, k, v, None, pos, pages, rope, qo)
        q.attn_decode(c, qo, pages, lens, out, ws)

    one, two = state(), state()
    step(two)                                                                     # warm
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(one)
    for i in range(20):
        for x in (qq, k, v):
            x.copy_(torch.randn(x.shape, generator=g, device=DEV))
        pos.fill_(i)
        lens.fill_(i + 1)
        graph.replay()
        step(two)
        torch.cuda.synchronize()
        assert torch.equal(one[2].view(torch.int16), two[2].view(torch.int16)), i


def test_parts_and_ranges_in_a_graph():
    """What cuts keys up looks at the lengths of the replay, not at those of the recording."""
    g = gen(31)
    x, k, v = rows(g, 40, 8, 64), rows(g, 9000, 2, 64), rows(g, 9000, 2, 64)
    cq, ck = (torch.tensor(n, dtype=torch.int32, device=DEV) for n in ([0, 30, 40], [0, 8000, 9000]))
    assert q.attention._lib().attn_prompt_workspace_bytes(2, 40, 9000, 8, 2, 64) > 0
    c, qq, pages, ln, first, ws = run_decode([9000, 40, 12000, 4096, 3, 7000, 15000, 2500], 16, 8, 64, 64, seed=26)
    out, dec = torch.zeros_like(x), torch.zeros_like(first)

    def step(out, dec):
        q.attn_prompt(x, k, v, cq, ck, out)
        q.attn_decode(c, qq, pages, ln, dec, ws)

    step(out, dec)                                                                # warm
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(out, dec)
    for q1, k1, cut in [(30, 8000, 1), (1, 20, 1), (39, 9000, 30), (20, 4500, 2), (30, 8000, 1)]:
        cq[1], ck[1] = q1, k1
        ln.copy_(torch.tensor([9000, 40, 12000, 4096, 3, 7000, 15000, 2500], device=DEV) // cut)
        graph.replay()
        again, dagain = torch.zeros_like(out), torch.zeros_like(dec)
        step(again, dagain)
        torch.cuda.synchronize()
        assert torch.equal(out.view(torch.int16), again.view(torch.int16)), (q1, k1)
        assert torch.equal(dec.view(torch.int16), dagain.view(torch.int16)), cut
    assert torch.equal(dec.view(torch.int16), first.view(torch.int16))
