"""What the attention calls promise beside their formulas (-m gpu): workspaces that calls share."""
import pytest
import torch

import paper_2503_09304_amd as q
from test_gpu_attention import DEV, NAN, fresh, gen, rows, table

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
    counters = q.attention._lib().attn_decode_counter_bytes(64, 32, 8)
    for case, n in [(wide, 64), (wide, 32), (wide, 1), (wide, 64), (narrow, 20), (wide, 64), (wide, 9), (narrow, 3), (wide, 63), (wide, 64)]:
        got = decode(*case, ws, n)
        assert (ws[:counters] == 0).all(), n
        c, qq = case[:2]
        want = decode(*case, q.attn_decode_workspace(c, n, qq.shape[1]), n)
        assert not got[0].isnan().any() and not got[1].isnan().any() and same(got, want), n
