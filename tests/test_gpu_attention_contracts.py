"""What the attention calls promise beside their formulas (-m gpu): workspaces that calls share, calls of any size, offsets that
descend, calls of nothing, the smallest values of the 8-bit cache, bits that do not depend on other sequences;
and the tiles of heads of 128 against the formula."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2503_09304_amd as q
from paper_2503_09304_amd import attention
from test_gpu_attention import DEV, NAN, check, fresh, gen, quantised, rows, run_prompt, table

pytestmark = pytest.mark.gpu


def batch(lens, Hq, Hk, D, page, fp8, seed):
    """A cache that holds `lens` tokens of each sequence, and a query each."""
    g = gen(seed)
    pages, n_pages = table(lens, page, seed)
    c = fresh(n_pages, Hk, page, D, fp8)
    seq = torch.repeat_interleave(torch.arange(len(lens), dtype=torch.int32), torch.tensor(lens)).to(DEV)
    pos = torch.cat([torch.arange(n, dtype=torch.int32) for n in lens]).to(DEV)
    k, v = rows(g, len(seq), Hk, D), rows(g, len(seq), Hk, D)
    q.attn_append(c, None, k, v, seq, pos, pages, None, None)
    return c, rows(g, len(lens), Hq, D), pages, torch.tensor(lens, dtype=torch.int32, device=DEV)


def decode(c, qq, pages, lens, ws, n):
    out, lse = torch.full_like(qq[:n], NAN), torch.full(qq.shape[:2], NAN, dtype=torch.float32, device=DEV)[:n]
    q.attn_decode(c, qq[:n], pages[:n], lens[:n], out, ws, lse=lse)
    return out, lse


def same(a, b):
    return all(torch.equal(x.view(torch.int16), y.view(torch.int16)) for x, y in zip(a, b))


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("spare", [0, 300])
def test_decode_batches_of_any_size_share_a_workspace(fp8, spare):
    """Sequences that are cut, in batches that shrink and grow: the bits of a workspace of their own, and all counters zero after each call."""
    lens = [3000, 1500, 700, 33] * 16                                            # pieces of even batches, ranges of the uneven whole
    wide, narrow = batch(lens, 32, 8, 128, 64, fp8, 40), batch(lens[:20], 12, 3, 64, 16, fp8, 41)
    own = q.attn_decode_workspace(wide[0], 64, 32)
    ws = torch.zeros(own.numel() + spare, dtype=torch.uint8, device=DEV)
    counters = attention._lib().attn_decode_counter_bytes(64, 32, 8)
    for case, n in [(wide, 64), (wide, 32), (wide, 1), (wide, 64), (narrow, 20), (wide, 64), (wide, 9), (narrow, 3), (wide, 63), (wide, 64)]:
        got = decode(*case, ws, n)
        assert (ws[:counters] == 0).all(), n
        c, qq = case[:2]
        want = decode(*case, q.attn_decode_workspace(c, n, qq.shape[1]), n)
        assert not got[0].isnan().any() and not got[1].isnan().any() and same(got, want), n


def test_decode_of_more_workgroups_than_a_launch_takes():
    """16400 sequences of 1024 heads, 0 to 2 tokens long, on one page: 2^24 workgroups and more."""
    n, H, D = 16400, 1024, 16
    g = gen(42)
    k, v = rows(g, 2, H, D), rows(g, 2, H, D)
    c = fresh(1, H, 16, D, False)
    pages = torch.zeros((n, 1), dtype=torch.int32, device=DEV)
    q.attn_append(c, None, k, v, torch.zeros(2, dtype=torch.int32, device=DEV), torch.arange(2, dtype=torch.int32, device=DEV), pages, None, None)
    lens = (torch.arange(n, device=DEV) % 3).to(torch.int32)
    qq = torch.randn(n, H, D, generator=g, device=DEV, dtype=torch.bfloat16)
    out, lse = decode(c, qq, pages, lens, q.attn_decode_workspace(c, n, H), n)
    one, two = v[0].double(), v[1].double()
    for at in range(0, n, 1640):
        x, size = qq[at:at + 1640].double(), lens[at:at + 1640]
        s = torch.stack([(x * k[j].double()).sum(-1) for j in range(2)], -1) * D ** -0.5
        big = torch.stack([(x * k[j].double()).abs().sum(-1) for j in range(2)], -1).amax(-1) * D ** -0.5
        s = s.masked_fill(torch.arange(2, device=DEV) >= size[:, None, None], -torch.inf)
        rl = torch.logsumexp(s, -1)
        p = torch.exp(s - torch.where(torch.isinf(rl), torch.zeros_like(rl), rl)[..., None])
        ref = [p[..., :1] * one + p[..., 1:] * two, rl, p[..., :1] * one.abs() + p[..., 1:] * two.abs(), big]
        check(out[at:at + 1640].flatten(0, 1), lse[at:at + 1640].flatten(), [r.flatten(0, 1) for r in ref], D, at)


def prompt(qq, k, v, cq, ck, causal):
    cq, ck = (torch.from_numpy(np.asarray(x, dtype=np.int32)).to(DEV) for x in (cq, ck))
    out, lse = torch.full_like(qq, 7.0), torch.full(qq.shape[:2], 7.0, dtype=torch.float32, device=DEV)
    q.attn_prompt(qq, k, v, cq, ck, out, causal=causal, lse=lse)
    return out, lse


def held(cu, n):
    """Entries clamped to the range and to the entry before them."""
    return np.maximum.accumulate(np.clip(cu, 0, n))


@pytest.mark.parametrize("causal", [True, False])
def test_offsets_that_descend_in_the_middle(causal):
    """Each entry is at least the one before it: the bits of offsets that are so already, no row another sequence's, rows of none untouched."""
    g = gen(43)
    for Hq, Hk, D in [(2, 2, 64), (8, 2, 128)]:
        qq, k, v = rows(g, 300, Hq, D), rows(g, 300, Hk, D), rows(g, 300, Hk, D)
        for cq, ck in [([0, 30, 10, 40], [0, 30, 10, 40]), ([5, 250, 20, 260, 30, 270, 40], [0, 100, 200, 210, 230, 250, 300]),
                       ([0, 100, 150, 160, 200], [0, 90, 20, 300, 10]), ([0, 1 << 30, 5, 9], [-5, -9, 300, 7])]:
            got, want = prompt(qq, k, v, cq, ck, causal), prompt(qq, k, v, held(cq, 300), held(ck, 300), causal)
            assert same(got, want), (cq, ck)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("n", [3, 64, 65, 150, 200])
def test_offsets_of_any_kind(n, causal):
    """Among up to 200 sequences: descents at any place, some of them between the 64 that are looked at together, and entries out of range; uncut, and cut into parts."""
    r, g, Hq, Hk, D = np.random.default_rng(n), gen(44), 4, 1, 64
    for T, M in [(1500, 1500), (150, 700 * max(n, 13))]:
        qq, k, v = rows(g, T, Hq, D), rows(g, M, Hk, D), rows(g, M, Hk, D)
        assert (attention._lib().attn_prompt_workspace_bytes(n, T, M, Hq, Hk, D) > 0) == (T == 150)
        for share in (0.02, 0.3):
            cu = []
            for m in (T, M):
                x = np.sort(r.integers(0, m + 1, n + 1))
                wild = r.random(n + 1) < share
                x[wild] = r.integers(-m, 2 * m, wild.sum())
                x[n // 2] = x[n // 2 - 1] // 2
                cu.append(x)
            got, want = prompt(qq, k, v, *cu, causal), prompt(qq, k, v, held(cu[0], T), held(cu[1], M), causal)
            assert same(got, want), share


@pytest.mark.parametrize("n_pages", [0, 3])
def test_calls_of_nothing(n_pages):
    """No tokens, no queries, no sequences, no keys."""
    Hq, Hk, D = 8, 2, 64
    c = fresh(4, Hk, 16, D, False)
    bf, none = dict(dtype=torch.bfloat16, device=DEV), torch.empty(0, dtype=torch.int32, device=DEV)
    pages = torch.empty((0, n_pages), dtype=torch.int32, device=DEV)
    qq, k = torch.empty((0, Hq, D), **bf), torch.empty((0, Hk, D), **bf)
    assert q.attn_append(c, qq, k, k, none, none, pages, None, qq, k) == q.MOE_OK
    assert q.attn_append(c, None, k, k, None, none, pages, None, None) == q.MOE_OK
    assert q.attn_read(c, none, none, pages, k, k) == q.MOE_OK
    assert q.attn_decode(c, qq, pages, none, qq, q.attn_decode_workspace(c, 0, Hq), lse=torch.empty((0, Hq), device=DEV)) == q.MOE_OK
    for cu in ([0], [0, 0, 0]):
        cu = torch.tensor(cu, dtype=torch.int32, device=DEV)
        assert q.attn_prompt(qq, k, k, cu, cu, qq) == q.MOE_OK
    cq, ck = torch.tensor([0, 5], dtype=torch.int32, device=DEV), torch.tensor([0, 0], dtype=torch.int32, device=DEV)
    out, lse = torch.full((5, Hq, D), 7.0, **bf), torch.zeros((5, Hq), device=DEV)
    assert q.attn_prompt(torch.ones((5, Hq, D), **bf), k, k, cq, ck, out, lse=lse) == q.MOE_OK
    assert (out == 0).all() and (lse == -torch.inf).all() and c.k.isnan().all() and c.v.isnan().all()


def test_the_smallest_values_in_the_fp8_cache():
    """Rows whose largest element is 2^-133 to 2^-110: below 2^-126 too what is read back is what the definition gives, bit for bit."""
    D, g = 64, gen(45)
    top = torch.exp2(-torch.arange(110, 134, device=DEV).double())[:, None, None]
    x = torch.rand(24, 1, D, generator=g, device=DEV).double() * 2 - 1
    x[:, :, :8] = torch.exp2(-torch.arange(8, device=DEV).double())               # the largest and 7 halvings of it
    v = (x * top).to(torch.bfloat16)
    pos, seq = torch.arange(24, dtype=torch.int32, device=DEV), torch.zeros(24, dtype=torch.int32, device=DEV)
    pages, n_pages = table([24], 16, 0)
    c = fresh(n_pages, 1, 16, D, True)
    q.attn_append(c, None, v, -v, seq, pos, pages, None, None)
    k2, v2 = torch.empty_like(v), torch.empty_like(v)
    q.attn_read(c, seq, pos, pages, k2, v2)
    want = quantised(v)
    assert (want.abs() < 2.0 ** -126).any() and (want != 0).any(2).all()
    assert torch.equal(k2.double(), want) and torch.equal(v2.double(), -want)


def uncut(qq, k, v, cq, ck, D, causal):
    """attn_prompt of the C library without a workspace, which the binding always gives."""
    out, lse = torch.full_like(qq, 7.0), torch.full(qq.shape[:2], 7.0, dtype=torch.float32, device=DEV)
    held_rows = [(C.c_int64 * 3)(t.data_ptr(), t.stride(0), t.stride(1)) for t in (qq, k, v, out)]
    cq, ck = (torch.tensor(x, dtype=torch.int32, device=DEV) for x in (cq, ck))
    rc = attention._lib().attn_prompt(*held_rows, lse.data_ptr(), cq.data_ptr(), ck.data_ptr(), len(cq) - 1, len(qq), len(k), qq.shape[1], k.shape[1], D, D ** -0.5,
                                      causal, None, 0, torch.cuda.current_stream().cuda_stream)
    assert rc == q.MOE_OK
    torch.cuda.synchronize()
    return out, lse


@pytest.mark.parametrize("causal", [0, 1])
@pytest.mark.parametrize("Hq,Hk,D", [(8, 2, 128), (6, 2, 64), (3, 3, 80)])
def test_a_prompt_that_is_not_cut_has_the_same_bits_in_any_company(Hq, Hk, D, causal):
    g = gen(46)
    nq, nk = [1, 33, 200, 64, 5, 129], [1, 700, 200, 3000, 2, 129]
    cq, ck = (np.concatenate([[0], np.cumsum(n)]).tolist() for n in (nq, nk))
    qq, k, v = rows(g, cq[-1], Hq, D, 3.0), rows(g, ck[-1], Hk, D), rows(g, ck[-1], Hk, D)
    whole = uncut(qq, k, v, cq, ck, D, causal)
    for b in range(len(nq)):
        a, z, ka, kz = cq[b], cq[b + 1], ck[b], ck[b + 1]
        alone = uncut(qq[a:z], k[ka:kz], v[ka:kz], [0, z - a], [0, kz - ka], D, causal)
        assert same(alone, [x[a:z] for x in whole]), b


@pytest.mark.parametrize("Hq,Hk,D,queries", [(32, 8, 128, 32), (16, 4, 128, 32), (8, 1, 128, 128), (32, 8, 112, 32), (16, 4, 96, 32), (12, 2, 128, 64), (24, 12, 128, 64), (40, 8, 128, 128)])
@pytest.mark.parametrize("causal", [True, False])
def test_tiles_shared_by_heads(Hq, Hk, D, queries, causal):
    """Workgroups of 32 queries of four heads of up to 128, 64 of two, 128 of one: prompts that fill the chip, a context among them, against the formula in 64 bits."""
    nq, nk = [700, 1, 515, 33, 1300, 64], [700, 1, 900, 33, 1300, 20]
    L = attention._lib()
    assert L.attn_prompt_workspace_bytes(6, sum(nq), sum(nk), Hq, Hk, D) == 0
    assert 1 << L._ZN5qattn15prompt_log_tileEiiiii(6, sum(nq), Hq, Hk, 1) == queries
    run_prompt(nq, nk, Hq, Hk, D, causal, seed=Hq + D)


@pytest.mark.parametrize("Hq,Hk,queries", [(32, 8, 32), (4, 1, 32), (6, 3, 64), (5, 1, 128)])
@pytest.mark.parametrize("causal", [True, False])
def test_tiles_shared_by_heads_in_parts(Hq, Hk, queries, causal):
    """The same with keys that are cut into parts: chunks of a few queries on long contexts, heads of 128."""
    nq, nk = [16, 70, 1], [4000, 2500, 7001]
    L = attention._lib()
    size = L.attn_prompt_workspace_bytes(3, sum(nq), sum(nk), Hq, Hk, 128)
    parts = size // (sum(nq) * Hq * 130 * 4)
    assert parts > 1 and 1 << L._ZN5qattn15prompt_log_tileEiiiii(3, sum(nq), Hq, Hk, parts) == queries
    run_prompt(nq, nk, Hq, Hk, 128, causal, seed=Hq)


def test_a_long_prompt_of_the_benchmarks_heads():
    """Heads of 128, four to a key/value head, 5000 tokens: many tiles of keys, maxima that are taken over."""
    run_prompt([5000], [5000], 32, 8, 128, seed=47, spread=2.0)
