"""dense_linear over all scale bytes of the matrix and of 8-bit rows, with products brought back into range by the other side's powers of two (-m gpu).

Bars as in test_gpu_dense.py: (K + 16) 2^-24 S, 2^-11 S more for the scaled products (8-bit rows, bf16 out), and the output's rounding.  What is not exact by the header has
its own assertions: weights and widened elements of 2^128 and more, and widened elements below 2^-133."""
import math

import pytest
import torch

import paper_2503_09304_amd as q
from test_gpu_dense import BF, DEV, F32, F8, HALF, KINDS, decoded, eight_bit, gen, weights

pytestmark = pytest.mark.gpu
K, R = 96, 256                                                    # rows of every byte, 255 (NaN) as well


def compared(out, x, scale, codes, scales, x_type, out_type, among=None):
    d, w = (x.double() if scale is None else decoded(x, scale)), weights(codes, scales)
    ref, S = d @ w.t(), d.abs() @ w.abs().t()
    err = ((K + 16) * 2.0 ** -24 + (2.0 ** -11 if x_type is F8 and out_type is BF else 0)) * S
    bad = ~((out.double() - ref).abs() <= err + (HALF if out_type is BF else 2.0 ** -24) * (ref.abs() + err))
    bad = bad if among is None else bad & among
    assert not bad.any(), (int(bad.sum()), bad.nonzero()[:4].tolist())


def rows_of(g, T, power, x_type):
    """Rows whose elements are normal ones times 2^power."""
    if x_type is BF:
        return (torch.randn(T, K, generator=g, device=DEV) * 2.0 ** power).to(BF), None
    x, _ = eight_bit(g, T, K)                                     # elements of 60 at the root of their mean square
    return x, torch.full((T, K // 32), 121 + power, dtype=torch.uint8, device=DEV)


@pytest.mark.parametrize("T", [1, 7, 40, 300])
@pytest.mark.parametrize("x_type,out_type", KINDS)
def test_every_byte_of_the_matrix(T, x_type, out_type):
    """Bytes 0 to 69 with rows around 2^80, to 185 with rows around 1, to 254 with rows around 2^-80; elements whose weight is 2^128 or more come last, by themselves."""
    g = gen(T)
    codes = torch.randint(0, 256, (R, K // 2), generator=g, device=DEV, dtype=torch.uint8)
    scales = torch.arange(R, device=DEV).to(torch.uint8).view(R, 1).repeat(1, K // 32)
    inside = torch.ones((1, R), dtype=torch.bool, device=DEV)
    inside[:, 255] = False
    if not (x_type is F8 and out_type is BF):
        codes[253] &= 0xDD                                        # elements of 0, 0.5, 2 and 3 are left: below 2^128; of byte 254 those of 0 to 1.5
        codes[254] &= 0xBB
    M = q.DenseMatrix4(codes, scales)
    for lo, hi, power in ((0, 70, 80), (70, 186, 0), (186, 255, -80)):
        x, scale = rows_of(g, T, power, x_type)
        out = torch.zeros((T, R), dtype=out_type, device=DEV)
        q.dense_linear(x, M, out, scale=scale)
        among = inside.clone()
        among[:, :lo] = among[:, hi:] = False
        compared(out.nan_to_num(math.inf), x, scale, codes, scales.clamp(max=254), x_type, out_type, among)
        assert out[:, 255].isnan().all() and out[:, lo:hi].isfinite().all()


@pytest.mark.parametrize("T", [1, 40, 300])
@pytest.mark.parametrize("x_type,out_type", KINDS)
def test_weights_over_bf16_s_range(T, x_type, out_type):
    """Infinite as bf16 operands, exact as the scaled products' own."""
    codes = torch.zeros((16, K // 2), dtype=torch.uint8, device=DEV)
    codes[:, 5] = torch.arange(16, device=DEV).to(torch.uint8)   # column 10
    x, scale = rows_of(gen(5), T, -80, x_type)
    if x_type is BF:
        x.abs_()
    else:
        x &= 0x7F
    for byte, least in ((252, 8), (253, 4), (254, 2)):
        scales = torch.full((16, K // 32), byte, dtype=torch.uint8, device=DEV)
        out = torch.zeros((T, 16), dtype=out_type, device=DEV)
        q.dense_linear(x, q.DenseMatrix4(codes, scales), out, scale=scale)
        if x_type is F8 and out_type is BF:
            compared(out, x, scale, codes, scales, x_type, out_type)
            continue
        over = (weights(codes, scales)[:, 10].abs() >= 2.0 ** 128).expand(T, 16) & (x[:, 10:11] != 0)
        assert over[0].sum() == 2 * sum(v >= least for v in (0, 0.5, 1, 1.5, 2, 3, 4, 6))
        assert torch.equal(out.isfinite(), ~over)
        compared(out.nan_to_num(), x, scale, codes, scales, x_type, out_type, ~over)


@pytest.mark.parametrize("T", [1, 40, 300])
@pytest.mark.parametrize("out_type", [BF, F32])
@pytest.mark.parametrize("byte", [0, 1, 2, 3, 40, 127, 200, 246, 247, 248, 254])
def test_every_byte_of_8_bit_rows(T, out_type, byte):
    """With an fp32 output widened elements are rounded to multiples of 2^-133 (bf16's least) and infinite from 2^128 on; the scaled products take all of them."""
    g = gen(byte)
    codes = torch.randint(0, 256, (R, K // 2), generator=g, device=DEV, dtype=torch.uint8)
    scales = torch.full((R, K // 32), min(max(254 - byte, 50), 200), dtype=torch.uint8, device=DEV)
    x = torch.arange(K, device=DEV).to(torch.uint8).repeat(T, 1) + 40 * (torch.arange(T, device=DEV) % 4).to(torch.uint8).view(T, 1)
    x = torch.where(x & 0x7F == 0x7F, x - 1, x)                   # every element that is a number, of both signs, in four rows
    scale = torch.full((T, K // 32), byte, dtype=torch.uint8, device=DEV)
    out = torch.zeros((T, R), dtype=out_type, device=DEV)
    q.dense_linear(x, q.DenseMatrix4(codes, scales), out, scale=scale)
    d = decoded(x, scale)
    if out_type is BF:
        compared(out, x, scale, codes, scales, F8, BF)
        return
    over = (d.abs() >= 2.0 ** 128).any(1)
    assert not out[over].isfinite().all(1).any() and out[~over].isfinite().all()
    assert T == 1 or (byte > 246) == bool(over.any())                    # one row has the first 96 elements alone
    d = torch.round(d * 2.0 ** 133) * 2.0 ** -133 if byte < 3 else d
    w = weights(codes, scales)
    ref, S = d @ w.t(), d.abs() @ w.abs().t()
    bad = (out.double() - ref).abs() > ((K + 16) * 2.0 ** -24 + 2.0 ** -24) * S
    assert not bad[~over].any(), bad.nonzero()[:4].tolist()
