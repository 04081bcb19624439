"""A row of dense_norm is the same bits whatever stands beside it, on both sides of every number of rows at which another kernel takes over (-m gpu)."""
import pytest
import torch

import paper_2503_09304_amd as q
from test_gpu_dense import BF, DEV, F32, gen, rows

pytestmark = pytest.mark.gpu


def norm(x, w, add, fp8):
    shape = x.shape
    out = torch.zeros(shape, dtype=torch.uint8 if fp8 else BF, device=DEV)
    scale = torch.zeros((*shape[:-1], shape[-1] // 32), dtype=torch.uint8, device=DEV) if fp8 else None
    q.dense_norm(x, w, out, add=add, scale=scale)
    return [out] if scale is None else [out, scale]


@pytest.mark.parametrize("D", [64, 512, 1024, 2048, 2080, 2816, 4096, 4128, 16384])
@pytest.mark.parametrize("add", [None, BF, F32])
@pytest.mark.parametrize("fp8", [False, True])
def test_any_number_of_rows(D, add, fp8):
    g = gen(D)
    x, a = rows(g, (8300, D)), None if add is None else rows(g, (8300, D), add)
    w = 1 + 0.2 * torch.randn(D, generator=g, device=DEV)
    whole = norm(x, w, a, fp8)
    for n in (1, 1024, 1025, 3000):
        few = norm(x[:n], w, None if a is None else a[:n], fp8)
        assert all(torch.equal(f, t[:n]) for f, t in zip(few, whole)), n


def test_heads_are_rows():
    g = gen(1)
    x = rows(g, (1500, 2, 4096))
    whole, few = norm(x, None, None, False)[0], norm(x[:512], None, None, False)[0]
    assert torch.equal(whole[:512], few) and torch.equal(whole[7], norm(x[7], None, None, False)[0])
