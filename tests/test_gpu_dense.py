"""dense_norm and dense_linear against plain implementations in 64 bits (-m gpu).

Bars.  HALF = 2^-8 is a rounding to bf16.  dense_norm: r is compared bit for bit.  The sum of its squares is an fp32 sum of positive terms: 64
in a row at most, 6 exchanges, 8 waves, and what the mean, eps, the root (2^-23) and three products add: below 2^-17 of the result.  weight + shift is rounded once:
2^-24 (|weight| + |shift|) of r * inv.  An 8-bit element is half a step off: 2^-4 of the value, or 2^-10 of its scale where that is more; the scale
is that of the largest of 32 within 2^-17.
dense_linear: fp32 sums of K exact products, in any order: at most (K + 16) 2^-24 S with S = sum |x w|, then the output's rounding.  The scaled products drop what
is below 2^-14 of the largest of the few products that they add first, each time a part of a product up to 4 times its power of two: less than 2^-11 S."""
import math

import numpy as np
import pytest
import torch

import paper_2503_09304_amd as q

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
HALF = torch.finfo(torch.bfloat16).eps / 2
NAN = float("nan")
BF, F32, F8 = torch.bfloat16, torch.float32, torch.float8_e4m3fn


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def rows(g, shape, dtype=BF, pad=0, lead=0, spread=1.0):
    """[T, D] or [T, heads, D] with `pad` elements of NaN behind each token's and `lead` in front of all."""
    T, width = shape[0], math.prod(shape[1:])
    x = torch.full((T * (width + pad) + lead,), NAN, dtype=dtype, device=DEV)
    x = x[lead:].view(T, width + pad)[:, :width].unflatten(1, shape[1:]) if T else torch.empty(shape, dtype=dtype, device=DEV)
    x.copy_(torch.randn(*shape, generator=g, device=DEV) * spread * torch.exp(torch.randn(T, *[1] * (len(shape) - 1), generator=g, device=DEV)))
    return x


def decoded(codes, scale):
    v = codes.view(F8).double().unflatten(-1, (-1, 32))
    return (v * torch.pow(2.0, scale.double() - 127.0).unsqueeze(-1)).flatten(-2)


def scale_byte(largest):
    part, n = torch.frexp(largest)                       # 448 = 0.875 * 2^9
    return (n - 9 + (part > 0.875).int() + 127).clamp(min=1).masked_fill(largest == 0, 1)


def check_norm(x, weight, add=None, shift=0.0, eps=1e-6, fp8=False, pad=0, inplace=False, no_total=False):
    shape = x.shape
    if add is None:
        r = x.float()
    else:
        r = (x.float() + add.float()).to(add.dtype)
    d = r.double()
    inv = 1.0 / torch.sqrt(d.square().mean(-1, keepdim=True) + eps)
    w = torch.ones(shape[-1], dtype=torch.float64, device=DEV) if weight is None else weight.double() + shift
    ref = d * inv * w
    err = 2.0 ** -17 * ref.abs() + (0 if weight is None else 2.0 ** -24 * (d * inv).abs() * (weight.double().abs() + abs(shift)))
    T, width = shape[0], math.prod(shape[1:])
    out = torch.full((T, width + pad), NAN if not fp8 else 0, dtype=torch.uint8 if fp8 else BF, device=DEV)
    if fp8:
        out.fill_(0x7F)
    mine = out[:, :width].unflatten(1, shape[1:])
    scale = torch.full((*shape[:-1], shape[-1] // 32), 7, dtype=torch.uint8, device=DEV) if fp8 else None
    total = None if add is None or no_total else add if inplace else torch.full(shape, NAN, dtype=add.dtype, device=DEV)
    assert q.dense_norm(x, weight, mine, eps=eps, add=add, total=total, scale=scale, shift=shift) == q.MOE_OK
    torch.cuda.synchronize()
    if total is not None:
        assert torch.equal(total, r)
    behind = out[:, width:]
    assert (behind == 0x7F).all() if fp8 else behind.isnan().all()
    if not fp8:
        assert ((mine.double() - ref).abs() <= err + HALF * (ref.abs() + err)).all()
        return mine
    big = ref.abs().unflatten(-1, (-1, 32)).amax(-1)
    assert ((scale == scale_byte(big * (1 - 2.0 ** -16))) | (scale == scale_byte(big * (1 + 2.0 ** -16)))).all()
    step = torch.pow(2.0, scale.double() - 127.0).repeat_interleave(32, -1)
    v = decoded(mine, scale)
    assert ((v - ref).abs() <= err + torch.maximum(2.0 ** -4 * (ref.abs() + err), 2.0 ** -10 * step)).all()
    return mine, scale


@pytest.mark.parametrize("D", [8, 16, 64, 72, 128, 136, 264, 512, 520, 1000, 1032, 2048, 2056, 4096, 4104, 8192, 8200, 16384, 16392, 32768])
@pytest.mark.parametrize("T", [1, 3, 1100])
def test_norm_sizes(D, T):
    g = gen(D + T)
    w = (1 + 0.2 * torch.randn(D, generator=g, device=DEV))
    check_norm(rows(g, (T, D)), w.to(BF))
    check_norm(rows(g, (T, D)), w, add=rows(g, (T, D), F32, spread=3.0))
    check_norm(rows(g, (T, D)), None, add=rows(g, (T, D), BF, spread=3.0))


@pytest.mark.parametrize("D", [32, 64, 96, 288, 512, 544, 1024, 1056, 4096, 4128, 8192, 16384, 32768])
@pytest.mark.parametrize("T,add", [(1, BF), (5, F32), (1030, None)])
def test_norm_in_8_bits(D, T, add):
    g = gen(D + T)
    a = None if add is None else rows(g, (T, D), add, pad=16)
    check_norm(rows(g, (T, D), pad=8), (0.2 * torch.randn(D, generator=g, device=DEV)), add=a, shift=1.0, fp8=True, pad=32)


@pytest.mark.parametrize("T,H,D", [(1, 1, 64), (7, 5, 128), (301, 32, 128), (33, 3, 80), (2, 1024, 8), (9, 2, 2048), (700, 2, 4096), (3, 2, 8192)])
@pytest.mark.parametrize("fp8", [False, True])
def test_norm_of_heads(T, H, D, fp8):
    if fp8 and D % 32:
        D += 32 - D % 32
    g = gen(T + H + D)
    x = rows(g, (T, H + 3, D), pad=24, lead=8)[:, 1:H + 1]        # slices of a wider row
    w = 1 + 0.2 * torch.randn(D, generator=g, device=DEV)
    check_norm(x, w.to(BF), fp8=fp8, pad=16)
    # heads first in memory; one residual row for all tokens
    y = rows(g, (H, T, D)).transpose(0, 1)
    check_norm(y, w, add=rows(g, (1, H, D), F32).expand(T, H, D), fp8=fp8)


def test_norm_in_place():
    g = gen(1)
    for T, D in ((3, 4096), (1500, 4096), (2, 20000), (4, 96)):
        for t in (BF, F32):
            check_norm(rows(g, (T, D)), None, add=rows(g, (T, D), t).contiguous(), inplace=True)
        x, add = rows(g, (T, D)), rows(g, (T, D))
        want = check_norm(x, None, add=add, no_total=True)
        for same in (x, add):
            kept = same.clone()
            q.dense_norm(x, None, same, add=add)
            assert torch.equal(same, want)
            same.copy_(kept)


def test_norm_rows_do_not_depend_on_others():
    g = gen(2)
    x = rows(g, (1300, 4096))
    whole = check_norm(x, None)
    x[5] = NAN
    x[7, 11] = math.inf
    out = torch.empty_like(x)
    q.dense_norm(x, None, out)
    keep = torch.ones(1300, dtype=torch.bool, device=DEV)
    keep[5] = keep[7] = False
    assert torch.equal(out[keep], whole[keep]) and out[5].isnan().all() and out[7, 11].isnan()
    few = torch.empty_like(x[9:12])
    q.dense_norm(x[9:12], None, few)
    assert torch.equal(few, whole[9:12]) or ((few.float() - whole[9:12].float()).abs() <= 2 * HALF * whole[9:12].float().abs()).all()
    codes, scale = torch.zeros((1300, 4096), dtype=torch.uint8, device=DEV), torch.zeros((1300, 128), dtype=torch.uint8, device=DEV)
    q.dense_norm(x, None, codes, scale=scale)
    assert (scale[5] == 255).all() and (codes[5] & 0x7F == 0x7F).all() and scale[7, 0] == 255 and (scale[8] != 255).all()


def test_norm_extremes():
    zero = torch.zeros((2, 64), dtype=BF, device=DEV)
    assert (check_norm(zero, None) == 0).all()
    codes, scale = check_norm(zero, None, fp8=True)
    assert (codes == 0).all() and (scale == 1).all()
    g = gen(3)
    check_norm(rows(g, (4, 256), spread=2.0 ** 50), None, fp8=True)
    check_norm(rows(g, (4, 256), spread=2.0 ** -60), None, eps=1e-30)
    # 249 * 2^120 is nearest to the code that stands for 2^128
    huge = torch.full((32,), 44 * 2.0 ** 120, device=DEV)
    x = torch.zeros((1, 32), dtype=BF, device=DEV)
    x[0, 0] = 1.0
    codes, scale = (torch.zeros(n, dtype=torch.uint8, device=DEV) for n in ((1, 32), (1, 1)))
    q.dense_norm(x, huge, codes, scale=scale)
    assert int(scale) == 247 and float(decoded(codes, scale)[0, 0]) == 240 * 2.0 ** 120
    q.dense_norm(x, huge * 1.1, codes, scale=scale)               # over fp32's range itself
    assert int(scale) == 255


def test_norm_far_rows():
    """Offsets over 2^31 elements."""
    big = torch.empty(18 << 27, dtype=BF, device=DEV)
    x = big.as_strided((17, 512), ((1 << 27) + 8, 1))
    x.copy_(torch.randn(17, 512, generator=gen(4), device=DEV))
    out = torch.empty_strided((17, 512), (512, 1), dtype=BF, device=DEV)
    q.dense_norm(x, None, out)
    near = torch.empty_like(out)
    q.dense_norm(x.contiguous(), None, near)
    assert torch.equal(out, near)
    q.dense_norm(near, None, x, add=near)
    q.dense_norm(near, None, out, add=near)
    assert torch.equal(x.contiguous(), out)


# ---- products ----

E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def matrix(g, R, K, spread=3):
    codes = torch.randint(0, 256, (R, K // 2), generator=g, device=DEV, dtype=torch.uint8)
    scales = torch.randint(124 - spread, 124 + spread + 1, (R, K // 32), generator=g, device=DEV, dtype=torch.uint8)
    return codes, scales


def weights(codes, scales):
    table = torch.tensor(E2M1 + [-v for v in E2M1], dtype=torch.float64, device=DEV)
    c = codes.long()
    w = table[torch.stack([c & 15, c >> 4], -1)].flatten(1).unflatten(1, (-1, 32))
    return (w * torch.pow(2.0, scales.double() - 127.0).unsqueeze(-1)).flatten(1)


def eight_bit(g, T, K, pad=0):
    """Rows in 8 bits, uint8 [T, K] with `pad` NaN codes behind each, and their scales."""
    codes = torch.full((T, K + pad), 0x7F, dtype=torch.uint8, device=DEV)
    codes[:, :K] = torch.randn(T, K, generator=g, device=DEV).mul_(60).to(F8).view(torch.uint8)
    return codes[:, :K], torch.randint(118, 125, (T, K // 32), generator=g, device=DEV, dtype=torch.uint8)


def check_linear(T, R, K, x_type=BF, out_type=BF, seed=0, pad=0, out_pad=0, x=None, m=None):
    g = gen(seed + 7 * T + R + K)
    codes, scales = matrix(g, R, K) if m is None else m
    scale = None
    if x is None:
        if x_type is BF:
            x = rows(g, (T, K), pad=pad, lead=pad)
        else:
            x, scale = eight_bit(g, T, K, pad)
    M = q.DenseMatrix4(codes, scales)
    whole = torch.full((T, R + out_pad), NAN, dtype=out_type, device=DEV)
    out = whole[:, :R]
    assert q.dense_linear(x, M, out, scale=scale) == q.MOE_OK
    torch.cuda.synchronize()
    d, w = (x.double() if scale is None else decoded(x, scale)), weights(codes, scales)
    ref, S = d @ w.t(), d.abs() @ w.abs().t()
    err = (K + 16) * 2.0 ** -24 * S
    if scale is not None and out_type is BF:
        err = err + 2.0 ** -11 * S
    half = HALF if out_type is BF else 2.0 ** -24
    bad = (out.double() - ref).abs() > err + half * (ref.abs() + err)
    assert not bad.any(), (T, R, K, x_type, out_type, int(bad.sum()), bad.nonzero()[:4].tolist())
    assert whole[:, R:].isnan().all()
    return out


KINDS = [(BF, BF), (BF, F32), (F8, BF), (F8, F32)]


@pytest.mark.parametrize("x_type,out_type", KINDS)
@pytest.mark.parametrize("T", [1, 2, 15, 16, 17, 31, 33, 64, 65, 100, 128, 129, 200, 257, 400, 513, 1025])
def test_linear_tokens(T, x_type, out_type):
    check_linear(T, 272, 640, x_type, out_type, pad=16, out_pad=3)


@pytest.mark.parametrize("x_type,out_type", KINDS)
@pytest.mark.parametrize("K", [32, 64, 96, 128, 160, 480, 512, 544, 1024, 1056, 2016, 4096, 8224])
def test_linear_columns(K, x_type, out_type):
    check_linear(3, 48, K, x_type, out_type)
    check_linear(70, 48, K, x_type, out_type, out_pad=1)
    check_linear(300, 300, K, x_type, out_type)


@pytest.mark.parametrize("x_type,out_type", KINDS)
@pytest.mark.parametrize("R", [1, 2, 3, 5, 15, 16, 17, 33, 63, 64, 65, 127, 255, 256, 257, 511, 1000, 4099])
def test_linear_rows(R, x_type, out_type):
    check_linear(1, R, 256, x_type, out_type)
    check_linear(37, R, 288, x_type, out_type, out_pad=5)
    check_linear(530, R, 288, x_type, out_type)


@pytest.mark.parametrize("T,R,K", [(1, 6144, 4096), (16, 32000, 2048), (61, 4096, 14336), (2, 16, 1 << 16), (1000, 4096, 1408), (9, 64, 14336), (130, 2816, 2048), (3000, 520, 4096),
                                   (48, 1024, 8192), (300, 128, 8192)])
def test_linear_sizes(T, R, K):
    for x_type, out_type in KINDS:
        check_linear(T, R, K, x_type, out_type)


@pytest.mark.parametrize("T", [1, 40, 300])
@pytest.mark.parametrize("x_type,out_type", KINDS)
def test_linear_every_scale_byte(T, x_type, out_type):
    """Powers of two from 2^-127 on; x is scaled against them so that products stay in range.  NaN (255) spoils its row of the matrix alone."""
    g = gen(9)
    K, R = 32, 256
    codes = torch.randint(0, 256, (R, K // 2), generator=g, device=DEV, dtype=torch.uint8)
    scales = torch.arange(256, device=DEV).to(torch.uint8).view(R, 1)
    if x_type is BF:
        x, scale = torch.randn(T, K, generator=g, device=DEV).to(BF), None
    else:
        x, scale = eight_bit(g, T, K)
    out = torch.zeros((T, R), dtype=out_type, device=DEV)
    q.dense_linear(x, q.DenseMatrix4(codes, scales), out, scale=scale)
    d = x.double() if scale is None else decoded(x, scale)
    w = weights(codes, scales)
    ref, S = d @ w.t(), d.abs() @ w.abs().t()
    assert out[:, 255].isnan().all()
    fine = slice(3, 240)                                          # subnormal sums below, overflow above
    err = 2.0 ** -11 * S
    assert ((out.double() - ref).abs() <= err + 2.0 ** -8 * (ref.abs() + err) + 2.0 ** -126)[:, fine].all()
    assert not out[:, fine].isnan().any()


def test_linear_tokens_do_not_spoil_each_other():
    g = gen(11)
    for T in (5, 40, 300):
        codes, scales = matrix(g, 80, 160)
        M = q.DenseMatrix4(codes, scales)
        x = rows(g, (T, 160))
        a, b = (torch.empty((T, 80), dtype=BF, device=DEV) for _ in range(2))
        q.dense_linear(x, M, a)
        x[3] = NAN
        q.dense_linear(x, M, b)
        keep = torch.arange(T, device=DEV) != 3
        assert torch.equal(a[keep], b[keep]) and b[3].isnan().all()
        e, s = eight_bit(g, T, 160)
        q.dense_linear(e, M, a, scale=s)
        s[3, 1] = 255
        q.dense_linear(e, M, b, scale=s)
        assert torch.equal(a[keep], b[keep]) and b[3].isnan().all()


def test_linear_strides_of_zero_far_rows_and_shared_inputs():
    g = gen(12)
    codes, scales = matrix(g, 33, 96)
    M = q.DenseMatrix4(codes, scales)
    one = rows(g, (1, 96))
    out = torch.empty((70, 33), dtype=F32, device=DEV)
    q.dense_linear(one.expand(70, 96), M, out)
    assert (out == out[0]).all()
    big = torch.empty(18 << 27, dtype=BF, device=DEV)
    for T in (17,):
        x = big.as_strided((T, 96), ((1 << 27) + 8, 1))
        x.copy_(torch.randn(T, 96, generator=g, device=DEV))
        a, b = (torch.empty((T, 33), dtype=BF, device=DEV) for _ in range(2))
        q.dense_linear(x, M, a)
        q.dense_linear(x.contiguous(), M, b)
        assert torch.equal(a, b)
        far = big.as_strided((T, 33), ((1 << 27) + 5, 1))
        near = x.contiguous()
        q.dense_linear(near, M, far)
        assert torch.equal(far.contiguous(), a)


# ---- as they are used ----

def test_empty_calls():
    g = gen(13)
    codes, scales = matrix(g, 32, 64)
    M = q.DenseMatrix4(codes, scales)
    none = torch.empty((0, 64), dtype=BF, device=DEV)
    assert q.dense_norm(none, None, torch.empty_like(none)) == q.MOE_OK
    assert q.dense_norm(torch.empty((0, 3, 64), dtype=BF, device=DEV), None, torch.empty((0, 3, 64), dtype=BF, device=DEV)) == q.MOE_OK
    assert q.dense_linear(none, M, torch.empty((0, 32), dtype=BF, device=DEV)) == q.MOE_OK


@pytest.mark.parametrize("T", [1, 23, 200])
def test_a_layer_s_calls_in_a_graph_and_on_another_stream(T):
    """norm (8 bits) -> product -> norm -> product, replayed with other inputs between the program's own eager calls."""
    g = gen(14 + T)
    H, F = 512, 1056
    up, down = q.DenseMatrix4(*matrix(g, F, H)), q.DenseMatrix4(*matrix(g, H, F))
    w1, w2 = (1 + 0.1 * torch.randn(n, generator=g, device=DEV) for n in (H, F))
    x, res = (torch.empty((T, H), dtype=t, device=DEV) for t in (BF, F32))

    def layer():
        h, hs, total = torch.empty((T, H), dtype=F8, device=DEV), torch.empty((T, H // 32), dtype=torch.uint8, device=DEV), torch.empty_like(res)
        q.dense_norm(x, w1, h, add=res, total=total, scale=hs)
        u, n, y = torch.empty((T, F), dtype=BF, device=DEV), torch.empty((T, F), dtype=BF, device=DEV), torch.empty((T, H), dtype=F32, device=DEV)
        q.dense_linear(h, up, u, scale=hs)
        q.dense_norm(u, w2, n)
        q.dense_linear(n, down, y)
        return total, y

    def fill(seed):
        s = gen(seed)
        x.copy_(torch.randn(T, H, generator=s, device=DEV))
        res.copy_(torch.randn(T, H, generator=s, device=DEV))

    fill(0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        layer()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kept = layer()
    for i in range(5):
        fill(i)
        graph.replay()
        got = [t.clone() for t in kept]
        eager = layer()
        torch.cuda.synchronize()
        for a, b in zip(got, eager):
            assert torch.equal(a, b)
        with torch.cuda.stream(side):
            side.wait_stream(torch.cuda.default_stream())
            other = layer()
        side.synchronize()
        for a, b in zip(other, eager):
            assert torch.equal(a, b)


def test_refusals_leave_outputs_alone():
    g = gen(15)
    M = q.DenseMatrix4(*matrix(g, 32, 64))
    x, out = rows(g, (4, 64)), torch.full((4, 64), 5.0, dtype=BF, device=DEV)
    y = torch.full((4, 32), 5.0, dtype=BF, device=DEV)
    for call in (lambda: q.dense_norm(x, None, out, eps=0.0), lambda: q.dense_norm(x, None, out, add=x.half()), lambda: q.dense_norm(x, None, out, total=x),
                 lambda: q.dense_norm(x[:, ::2], None, out[:, :32]), lambda: q.dense_norm(x, torch.ones(63, device=DEV), out), lambda: q.dense_norm(x, None, out[:1].expand(4, 64)),
                 lambda: q.dense_norm(x, None, out.view(torch.uint8)[:, :64]), lambda: q.dense_norm(x.cpu(), None, out), lambda: q.dense_norm(x, None, out, shift=NAN, eps=NAN),
                 lambda: q.dense_linear(x, M, y, scale=x), lambda: q.dense_linear(x[:, :32], M, y), lambda: q.dense_linear(x.view(torch.uint8)[:, :64], M, y),
                 lambda: q.dense_linear(x, M, y[:1].expand(4, 32)), lambda: q.dense_linear(x, M, y.half())):
        with pytest.raises(q.MoeError):
            call()
    torch.cuda.synchronize()
    assert (out == 5.0).all() and (y == 5.0).all()


def by_c(x, scale, M, out, ws, nb):
    """The C call itself, with a workspace of the caller's."""
    import ctypes as C
    from paper_2503_09304_amd import dense as d

    class Rows(C.Structure):
        _fields_ = [("data", C.c_void_p), ("scale", C.c_void_p), ("ts", C.c_int64), ("hs", C.c_int64), ("type", C.c_int32)]

    kind = d._TYPES[x.dtype]
    r = [Rows(t.data_ptr(), None if s is None else s.data_ptr(), t.stride(0), 0, d._TYPES[t.dtype]) for t, s in ((x, scale), (out, None))]
    need = d._lib().dense_linear_workspace_bytes(len(x), M.rows, M.cols, kind, r[1].type)
    if nb is not None:
        rc = d._lib().dense_linear(C.addressof(r[0]), M._at, C.addressof(r[1]), len(x), ws, nb, torch.cuda.current_stream().cuda_stream)
        assert rc == q.MOE_OK, q.moe_last_error()
    return need


@pytest.mark.parametrize("x_type,out_type", KINDS)
@pytest.mark.parametrize("T,R,K", [(1, 64, 4096), (1, 128, 32768), (16, 33, 8192), (40, 100, 4096), (61, 4096, 14336), (200, 65, 6144), (300, 128, 8192)])
def test_linear_workspaces(T, R, K, x_type, out_type):
    """Whatever stands in a workspace, nothing behind it is touched; with less than what is asked for, or none, the product is the same within its bar."""
    g = gen(16 + T)
    m = matrix(g, R, K)
    x, scale = (rows(g, (T, K)), None) if x_type is BF else eight_bit(g, T, K)
    M = q.DenseMatrix4(*m)
    outs = [torch.full((T, R), NAN, dtype=out_type, device=DEV) for _ in range(5)]
    need = by_c(x, scale, M, outs[0], None, None)
    assert (need > 0 or K <= 4096) and need % (T * (-(-R // 16) * 16) * 4) == 0
    ws = torch.full((need + 4096,), 0xFF, dtype=torch.uint8, device=DEV)
    for out, at, nb in zip(outs, (ws.data_ptr(), ws.data_ptr(), ws.data_ptr(), None, None), (need, need + 4096, need - 1, 0, need)):
        by_c(x, scale, M, out, at, nb)
        torch.cuda.synchronize()
        assert (ws[need:] == 0xFF).all()
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[2], outs[3]) and torch.equal(outs[3], outs[4])
    d, w = (x.double() if scale is None else decoded(x, scale)), weights(*m)
    ref, err = d @ w.t(), ((K + 16) * 2.0 ** -24 + (2.0 ** -11 if scale is not None and out_type is BF else 0)) * (d.abs() @ w.abs().t())
    for out in (outs[0], outs[2]):
        assert ((out.double() - ref).abs() <= err + (HALF if out_type is BF else 2.0 ** -24) * (ref.abs() + err)).all()


def test_two_graphs_of_one_memory_pool():
    """Calls with workspaces, captured into graphs that take turns on the same memory."""
    g = gen(17)
    A, B = q.DenseMatrix4(*matrix(g, 48, 8192)), q.DenseMatrix4(*matrix(g, 8192, 512))
    x = [torch.empty((T, 8192), dtype=BF, device=DEV) for T in (3, 40)]

    def run(v):
        y, h, z = (torch.empty((len(v), n), dtype=BF, device=DEV) for n in (48, 48, 48))
        q.dense_linear(v, A, y)
        q.dense_norm(y, None, h)
        wide = torch.empty((len(v), 8192), dtype=BF, device=DEV)
        q.dense_linear(h.repeat(1, 11)[:, :512].contiguous(), B, wide)
        q.dense_linear(wide, A, z)
        return z

    for v in x:
        v.copy_(torch.randn(v.shape, generator=g, device=DEV))
        run(v)
    torch.cuda.synchronize()
    graphs, kept, pool = [], [], None
    for v in x:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], pool=pool):
            kept.append(run(v))
        pool = graphs[0].pool()
    for i in range(4):
        for v, graph, out in zip(x, graphs, kept):
            v.copy_(torch.randn(v.shape, generator=g, device=DEV))
            graph.replay()
            got = out.clone()
            assert torch.equal(got, run(v))


def test_two_threads_on_two_streams():
    import threading
    g = gen(18)
    M = q.DenseMatrix4(*matrix(g, 48, 8192))
    x, add = [rows(g, (T, 8192)) for T in (5, 90)], [rows(g, (T, 8192), F32) for T in (5, 90)]
    bad = []

    def run(i):
        h, t, y = torch.empty_like(x[i]), torch.empty_like(add[i]), torch.empty((len(x[i]), 48), dtype=F32, device=DEV)
        q.dense_norm(x[i], None, h, add=add[i], total=t)
        q.dense_linear(h, M, y)
        return y

    want = [run(i) for i in range(2)]
    torch.cuda.synchronize()

    def work(i):
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(200):
                y = run(i)
                torch.cuda.current_stream().synchronize()
                if not torch.equal(y, want[i]):
                    bad.append(i)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not bad
