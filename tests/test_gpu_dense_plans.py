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


# Shapes of every plan that the rule gives: kernel, tiles, waves, one range or some, blocks ahead; rows, tokens and columns that fill no tile.  The last five are the kernel
# for many tokens: few and many groups of rows, tokens that end inside a tile.
SHAPES = {BF: [(1, 32753, 13472), (2, 21667, 13120), (1, 32007, 16192), (5, 8185, 13600), (7, 26237, 3264), (7, 6817, 12576), (2, 16059, 16224), (5, 4089, 14400), (19, 7209, 4384),
               (15, 3799, 8032), (3, 7987, 15264), (12, 1355, 15840), (2924, 247, 832), (3097, 23, 8416), (722, 577, 1440), (314, 279, 6848), (147, 769, 5312), (123, 79, 15520),
               (57, 15665, 672), (932, 87, 7392), (4620, 131, 992), (4719, 41, 3104), (3354, 263, 672), (2223, 67, 4512), (143, 33063, 800), (5725, 267, 672), (2763, 131, 10976),
               (4405, 131, 3232), (547, 10941, 672), (1449, 4315, 672), (207, 26063, 672), (7096, 773, 704), (1900, 7169, 608)],
          F8: [(1, 32753, 13472), (7, 17587, 4896), (7, 26237, 3264), (8, 8587, 8736), (6, 34285, 2912), (11, 3751, 14496), (3, 14375, 13920), (11, 4093, 15968), (19, 7209, 4384),
               (13, 3941, 11616), (7, 6817, 12576), (12, 1879, 16352), (1402, 393, 1088), (3097, 23, 8416), (722, 577, 1440), (314, 279, 6848), (147, 769, 5312), (91, 497, 13280),
               (57, 15665, 672), (932, 87, 7392), (4620, 131, 992), (4719, 41, 3104), (35, 24319, 704), (2223, 67, 4512), (69, 34721, 864), (5725, 267, 672), (2763, 131, 10976),
               (34, 3113, 11456), (549, 14641, 672), (1099, 7517, 672), (209, 32971, 832), (5011, 1591, 672), (1900, 7169, 608)]}


@pytest.mark.parametrize("x_type,out_type", KINDS)
@pytest.mark.parametrize("i", range(33))
def test_every_plan(i, x_type, out_type):
    check(*SHAPES[x_type][i], x_type, out_type)
