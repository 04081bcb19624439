"""dense_linear's variants against 64 bits, each on shapes that its rule gives to it (-m gpu); bars as in test_gpu_dense.py."""
import pytest
import torch

from test_gpu_dense import BF, DEV, F8, F32, HALF, KINDS, NAN, by_c, decoded, eight_bit, gen, matrix, q, rows, weights

pytestmark = pytest.mark.gpu


def check(T, R, K, x_type, out_type, workspace=True, seed=0):
    """The C call with what it asks for, or without a workspace; out has odd rows' ends and NaN behind them."""
    g = gen(seed + 7 * T + R + K)
    m = matrix(g, R, K)
    x, scale = (rows(g, (T, K), pad=8), None) if x_type is BF else eight_bit(g, T, K, 16)
    whole = torch.full((T, R + 3), NAN, dtype=out_type, device=DEV)
    out, M = whole[:, :R], q.DenseMatrix4(*m)
    need = by_c(x, scale, M, out, None, None) if workspace else 0
    ws = torch.full((need + 16,), 0xFF, dtype=torch.uint8, device=DEV)
    by_c(x, scale, M, out, ws.data_ptr() if need else None, need)
    torch.cuda.synchronize()
    d, w = (x.double() if scale is None else decoded(x, scale)), weights(*m)
    ref, S = d @ w.t(), d.abs() @ w.abs().t()
    err = ((K + 16) * 2.0 ** -24 + (2.0 ** -11 if scale is not None and out_type is BF else 0)) * S
    bad = (out.double() - ref).abs() > err + (HALF if out_type is BF else 2.0 ** -24) * (ref.abs() + err)
    assert not bad.any(), (T, R, K, x_type, out_type, int(bad.sum()), bad.nonzero()[:4].tolist())
    assert whole[:, R:].isnan().all() and (ws[need:] == 0xFF).all()


# Rows of more than 64 blocks of 128 columns, whose scales come to LDS in turn where there is no workspace: the last one a few columns, and in every place of a round of four.
LONG = [(1, 5000, 8224), (9, 17199, 8448), (15, 22902, 9280), (16, 40, 8224), (16, 100, 14336), (30, 4099, 8544), (33, 70, 16416), (17, 16900, 8288), (34, 16609, 8864),
        (61, 4096, 14336), (67, 16, 8352), (102, 15831, 8992), (200, 130, 24576), (300, 2050, 8224), (771, 964, 8960), (653, 4016, 12960), (2090, 40, 8320),
        (2218, 298, 8992), (3345, 1057, 8320), (3455, 1047, 8224)]


@pytest.mark.parametrize("x_type,out_type", [(F8, BF), (F8, F32)])
@pytest.mark.parametrize("T,R,K", LONG)
def test_long_rows_in_8_bits_without_a_workspace(T, R, K, x_type, out_type):
    check(T, R, K, x_type, out_type, workspace=False)
