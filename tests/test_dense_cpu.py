"""Host side of the dense calls (include/qdense.h) and of the router by scores, without a GPU: symbols, argument checks that refuse before anything is
enqueued, sizes, the calls' arguments with recording stubs in place of the kernels' launchers, and the binding with stand-ins for tensors."""
import ctypes as C
import math
import os
import random
import re
import subprocess

import pytest
import torch

import paper_2503_09304_amd as q
from paper_2503_09304_amd import attention as at
from paper_2503_09304_amd import binding as b
from paper_2503_09304_amd import dense as d
from test_attention_cpu import FAKE, pointer, refused
from test_attention_host import Recorded, Stand, two_gpus  # noqa: F401

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
STUB = os.path.join(ROOT, "tests", "host_stub")
CSRC = os.path.join(ROOT, "paper_2503_09304_amd", "csrc")
BF, F32, F8 = d.DENSE_BF16, d.DENSE_F32, d.DENSE_FP8


def test_library_exports_every_declared_symbol():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "qdense.h")).read(), flags=re.S)
    names = set(re.findall(r"\b(dense_[a-z_0-9]+)\s*\(", text))
    assert {"dense_norm", "dense_pack4", "dense_linear", "dense_linear_workspace_bytes", "dense_matrix4_code_bytes", "dense_matrix4_scale_bytes"} <= names
    for n in names:
        assert hasattr(q.lib(), n), n


def test_host_side_with_recorded_launches(tmp_path):
    exe = str(tmp_path / "dense_test")
    cmd = ["g++", "-std=c++17", "-O1", "-Wall", "-fsanitize=address,undefined", "-I", STUB, "-I", os.path.join(ROOT, "include"), "-I", CSRC,
           "-x", "c++", os.path.join(CSRC, "qdense_api.hip"), os.path.join(STUB, "dense_test.cpp"), "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and "all dense host checks passed" in r.stdout, (r.stdout + r.stderr)[-3000:]


class Rows(C.Structure):
    _fields_ = [("data", C.c_void_p), ("scale", C.c_void_p), ("token_stride", C.c_int64), ("head_stride", C.c_int64), ("type", C.c_int32)]


def rows(kind=BF, ts=512, hs=128, data=FAKE, scale=None):
    return pointer(Rows(data, scale if scale is not None else FAKE if kind == F8 else 0, ts, hs, kind))


def matrix(codes=FAKE, scales=FAKE, R=48, K=256):
    return pointer(d._Matrix(codes, scales, R, K))


def norm(x=None, add=None, total=None, out=None, weight=FAKE, wt=F32, shift=0.0, eps=1e-6, n=4, heads=4, dim=128):
    return d._lib().dense_norm(x or rows(), add, total, out or rows(data=3 * FAKE), weight, wt, shift, eps, n, heads, dim, None)


NORMS = [(dict(n=-1), "n_tokens"), (dict(n=(1 << 30) + 1, heads=1), "n_tokens"), (dict(n=1 << 28, heads=8), "heads"), (dict(heads=0), "heads"), (dict(heads=1025), "heads"),
         (dict(dim=0), "dim"), (dict(dim=4), "dim"), (dict(dim=100), "dim"), (dict(dim=32776), "dim"), (dict(out=rows(F8), dim=120), "dim"), (dict(out=rows(F32)), "out"),
         (dict(x=rows(F32)), "x must"), (dict(x=rows(F8)), "x must"), (dict(add=rows(F8)), "add must"), (dict(add=rows(7)), "add must"), (dict(total=rows()), "total needs"),
         (dict(add=rows(), total=rows(F32)), "type"), (dict(eps=0.0), "eps"), (dict(eps=-1.0), "eps"), (dict(eps=math.nan), "eps"), (dict(eps=math.inf), "eps"),
         (dict(wt=F8), "weights"), (dict(weight=FAKE + 8), "weight"), (dict(shift=math.inf), "shift"), (dict(x=rows(data=0)), "null"), (dict(x=rows(data=FAKE + 8)), "aligned"),
         (dict(x=rows(ts=508)), "strides"), (dict(x=rows(hs=132)), "strides"), (dict(x=rows(ts=-512)), "strides"), (dict(add=rows(F32, ts=510)), "strides"),
         (dict(out=rows(F8, ts=520)), "strides"), (dict(out=rows(F8, scale=0)), "scale"), (dict(out=rows(scale=FAKE)), "scale"), (dict(out=rows(ts=120)), "overlap"),
         (dict(out=rows(hs=120)), "overlap"), (dict(add=rows(), total=rows(ts=0)), "overlap"), (dict(add=rows(data=5 * FAKE), total=rows()), "total may"),
         (dict(add=rows(F32), total=rows(F32, data=3 * FAKE)), "total may"), (dict(add=rows(data=5 * FAKE), total=rows(data=5 * FAKE, ts=1024)), "total may"),
         (dict(out=rows(ts=1024)), "out may"), (dict(out=rows(F8)), "out may")]


@pytest.mark.parametrize("kw,word", NORMS)
def test_norm_refused(kw, word):
    refused(norm(**kw), word)


def test_null_rows_and_empty_calls():
    L, ok = d._lib(), rows()
    refused(L.dense_norm(None, None, None, ok, None, BF, 0.0, 1e-6, 4, 1, 128, None), "null")
    refused(L.dense_norm(ok, None, None, None, None, BF, 0.0, 1e-6, 4, 1, 128, None), "null")
    refused(L.dense_linear(None, matrix(), ok, 4, None, 0, None), "null")
    refused(L.dense_linear(ok, matrix(), None, 4, None, 0, None), "null")
    refused(L.dense_linear(ok, None, ok, 4, None, 0, None), "null")
    assert norm(n=0, x=rows(data=0), out=rows(data=0)) == q.MOE_OK
    assert L.dense_linear(rows(data=0), matrix(), rows(data=0), 0, None, 0, None) == q.MOE_OK


def linear(x=None, w=None, out=None, n=4, ws=0, nb=0):
    return d._lib().dense_linear(x or rows(), w or matrix(), out or rows(data=3 * FAKE), n, ws, nb, None)


MATRICES = [(dict(codes=0), "null"), (dict(scales=0), "null"), (dict(codes=FAKE + 8), "aligned"), (dict(scales=FAKE + 4), "aligned"), (dict(R=0), "rows"), (dict(R=-1), "rows"),
            (dict(R=(1 << 24) + 1), "rows"), (dict(K=0), "cols"), (dict(K=16), "cols"), (dict(K=48), "cols"), (dict(K=(1 << 20) + 32), "cols")]


@pytest.mark.parametrize("kw,word", MATRICES)
def test_matrices_refused(kw, word):
    refused(linear(w=matrix(**kw)), word)
    refused(d._lib().dense_pack4(5 * FAKE, 7 * FAKE, matrix(**kw), None), word)


@pytest.mark.parametrize("kw,word,code", [
    (dict(n=-1), "n_tokens", None), (dict(n=(1 << 24) + 1), "n_tokens", None), (dict(x=rows(F32)), "x must", None), (dict(out=rows(F8)), "out must", None),
    (dict(x=rows(data=FAKE + 2)), "aligned", None), (dict(x=rows(ts=260)), "strides", None), (dict(x=rows(F8, ts=264)), "strides", None), (dict(x=rows(F8, scale=0)), "scale", None),
    (dict(x=rows(scale=FAKE)), "scale", None), (dict(out=rows(data=0)), "null", None), (dict(out=rows(data=3 * FAKE + 1)), "aligned", None),
    (dict(out=rows(F32, data=3 * FAKE + 2)), "aligned", None), (dict(out=rows(data=3 * FAKE, ts=47)), "overlap", None), (dict(out=rows()), "overlap", None),
    (dict(ws=5 * FAKE + 8, nb=1 << 20), "workspace", q.MOE_E_WORKSPACE), (dict(ws=FAKE, nb=1 << 20), "overlap", None)])
def test_linear_refused(kw, word, code):
    refused(linear(**kw), word, q.MOE_E_ARG if code is None else code)


def test_pack_refused():
    L = d._lib()
    refused(L.dense_pack4(None, 7 * FAKE, matrix(), None), "null")
    refused(L.dense_pack4(5 * FAKE, None, matrix(), None), "null")
    refused(L.dense_pack4(5 * FAKE + 8, 7 * FAKE, matrix(), None), "aligned")
    refused(L.dense_pack4(FAKE, 7 * FAKE, matrix(), None), "in place")
    refused(L.dense_pack4(5 * FAKE, FAKE, matrix(), None), "in place")


def test_sizes():
    L = d._lib()
    for R, K, codes, scales in [(1, 32, 1024, 256), (16, 128, 1024, 256), (17, 128, 2048, 512), (16, 160, 2048, 256), (16, 512, 4096, 256), (16, 544, 5120, 512),
                                (1 << 24, 1 << 20, 1 << 43, 1 << 39)]:
        assert L.dense_matrix4_code_bytes(R, K) == codes and L.dense_matrix4_scale_bytes(R, K) == scales
    for R, K in [(0, 32), ((1 << 24) + 1, 32), (16, 0), (16, 16), (16, (1 << 20) + 32), (-1, 64), (16, -64)]:
        assert L.dense_matrix4_code_bytes(R, K) == 0 and L.dense_matrix4_scale_bytes(R, K) == 0 and L.dense_linear_workspace_bytes(4, R, K, BF, BF) == 0
    for n, x, o in [(0, BF, BF), (-1, BF, BF), ((1 << 24) + 1, BF, BF), (4, F32, BF), (4, BF, F8)]:
        assert L.dense_linear_workspace_bytes(n, 64, 64, x, o) == 0


def test_workspaces_hold_whole_ranges_and_stay_small():
    """A workspace is [ranges][tokens][rows up to a multiple of 16] of 4 bytes, ranges of at least one block of 128 columns; never more than 256 MB."""
    L, rng = d._lib(), random.Random(1)
    some = 0
    for i in range(4000):
        n, R, K = (int(2 ** rng.uniform(0, top)) for top in ((24, 24, 15), (6, 18, 15), (12, 16, 15))[i % 3])
        for x in (BF, F8):
            nb = L.dense_linear_workspace_bytes(n, R, 32 * K, x, BF)
            one = n * (-(-R // 16) * 16) * 4
            assert nb % one == 0 and nb // one != 1 and nb // one <= -(-32 * K // 128) and nb <= 1 << 28
            assert nb == L.dense_linear_workspace_bytes(n, R, 32 * K, x, F32)
            some += nb > 0
    assert some > 1000


def test_route_scored_refused():
    L, h = q.lib(), C.c_void_p()
    cfg = q.MoeConfig(60, 8, 64, 64, q.MOE_BF16, 16, 64, 0)
    assert L.moe_create(C.byref(cfg), 256 * 4096, q.moe_workspace_bytes(cfg), C.byref(h)) == q.MOE_OK
    w = q.MoeWeights(1, 1, 1, 1, q.MOE_W_ROWMAJOR)

    def call(score=1, groups=6, take=3, best=2, renorm=1, factor=1.0, n=0, x=1, w=w, ctx=h):
        c = b._Scoring(score, None, None, groups, take, best, renorm, factor)
        return L.moe_route_scored(ctx, x, n, C.byref(w) if w is not None else None, C.byref(c), None)

    for kw, word in [(dict(score=2), "score"), (dict(score=-1), "score"), (dict(groups=0), "groups"), (dict(groups=7), "groups"), (dict(groups=120), "groups"), (dict(groups=-6), "groups"),
                     (dict(take=0), "top_groups"), (dict(take=7), "top_groups"), (dict(best=0), "group_best"), (dict(best=5), "group_best"),
                     (dict(groups=60, take=60, best=2), "group_best"), (dict(groups=30, take=3, best=1), "fewer than k"), (dict(factor=math.nan), "factor"),
                     (dict(factor=math.inf), "factor"), (dict(n=65), "n_tokens"), (dict(n=-1), "n_tokens"), (dict(n=4, x=None), "null x"), (dict(w=None), "weight"),
                     (dict(ctx=None), "context")]:
        refused(call(**kw), word)
    refused(L.moe_route_scored(h, 1, 0, C.byref(w), None, None), "scoring")
    L.moe_destroy(h)


def test_scorings_refused():
    for bad in (dict(score="tanh"), dict(logit_bias=torch.zeros(4)), dict(choice_bias=Stand((4,), torch.float64)), dict(choice_bias=Stand((2, 2), torch.float32))):
        with pytest.raises(q.MoeError) as e:
            q.MoeScoring(**bad)
        assert e.value.code == q.MOE_E_ARG


@pytest.fixture
def dense_gpus(two_gpus, monkeypatch):  # noqa: F811
    monkeypatch.setattr(d, "_lib", lambda: two_gpus)
    return two_gpus



def calls():
    """Of each call: itself, and its tensors by name."""
    bf, f32, u8, f8 = torch.bfloat16, torch.float32, torch.uint8, torch.float8_e4m3fn
    M = object.__new__(q.DenseMatrix4)
    M.rows, M.cols, M._at = 48, 64, 1 << 21

    def linear(c):
        M._device = c["codes"].on
        return q.dense_linear(c["x"], M, c["out"], scale=c["scale"])

    return {"dense_norm": (lambda c: q.dense_norm(c["x"], c["weight"], c["out"], add=c["add"], total=c["total"], scale=c["scale"]),
                           dict(x=Stand((4, 2, 64), bf), weight=Stand((64,), f32), out=Stand((4, 2, 64), f8), scale=Stand((4, 2, 2), u8), add=Stand((4, 2, 64), f32),
                                total=Stand((4, 2, 64), f32))),
            "dense_linear": (linear, dict(codes=Stand((48, 32), u8), x=Stand((4, 64), f8), scale=Stand((4, 2), u8), out=Stand((4, 48), f32)))}


@pytest.mark.parametrize("name", ["dense_norm", "dense_linear"])
def test_calls_go_to_the_device_of_their_tensors(name, dense_gpus):
    call, tensors = calls()[name]
    for device in (0, 1):
        for t in tensors.values():
            t.on = device
        assert call(tensors) == q.MOE_OK
        assert dense_gpus.last == (name, device, dense_gpus.last[2]) and dense_gpus.now == [0]


@pytest.mark.parametrize("name", ["dense_norm", "dense_linear"])
def test_tensors_of_two_devices_are_refused(name, dense_gpus):
    call, tensors = calls()[name]
    for odd in tensors:
        for device in (0, -1):
            for n, t in tensors.items():
                t.on = device if n == odd else 1
            with pytest.raises(q.MoeError) as e:
                call(tensors)
            assert e.value.code == q.MOE_E_ARG and dense_gpus.last is None, odd


@pytest.mark.parametrize("name,odd,change", [
    ("dense_norm", "x", dict(shape=(4, 2, 32))), ("dense_norm", "x", dict(shape=(4, 64))), ("dense_norm", "x", dict(shape=(4,))), ("dense_norm", "x", dict(dtype=torch.float32)),
    ("dense_norm", "weight", dict(shape=(32,))), ("dense_norm", "weight", dict(dtype=torch.float16)), ("dense_norm", "out", dict(dtype=torch.float16)),
    ("dense_norm", "out", dict(dtype=torch.bfloat16)), ("dense_norm", "scale", dict(shape=(4, 2, 1))), ("dense_norm", "scale", dict(dtype=torch.int8)),
    ("dense_norm", "add", dict(dtype=torch.bfloat16)), ("dense_norm", "total", dict(dtype=torch.bfloat16)), ("dense_norm", "total", dict(shape=(5, 2, 64))),
    ("dense_linear", "x", dict(shape=(4, 32))), ("dense_linear", "x", dict(shape=(5, 64))), ("dense_linear", "x", dict(shape=(4, 1, 64))), ("dense_linear", "x", dict(dtype=torch.float16)),
    ("dense_linear", "x", dict(dtype=torch.bfloat16)), ("dense_linear", "scale", dict(shape=(4, 1))), ("dense_linear", "out", dict(shape=(4, 32))),
    ("dense_linear", "out", dict(dtype=torch.float8_e4m3fn))])
def test_shapes_and_types_refused(name, odd, change, dense_gpus):
    call, tensors = calls()[name]
    for k, v in change.items():
        setattr(tensors[odd], k, v)
    with pytest.raises(q.MoeError) as e:
        call(tensors)
    assert e.value.code == q.MOE_E_ARG and dense_gpus.last is None


@pytest.mark.parametrize("name,long", [("dense_norm", ("x", "out", "scale", "add", "total")), ("dense_linear", ("x", "scale", "out"))])
def test_counts_of_33_bits_are_refused(name, long, dense_gpus):
    call, tensors = calls()[name]
    for t in long:
        tensors[t].shape = (tensors[t].shape[0] + (1 << 32), *tensors[t].shape[1:])
    with pytest.raises(q.MoeError) as e:
        call(tensors)
    assert e.value.code == q.MOE_E_ARG and dense_gpus.last is None


def test_matrices_of_odd_sources_are_refused():
    u8 = torch.uint8
    for codes, scales in ((Stand((48,), u8), Stand((48, 2), u8)), (Stand((48, 32), torch.int8), Stand((48, 2), u8)), (Stand((48, 32), u8), Stand((48, 1), u8)),
                          (Stand((48, 32), u8), Stand((48, 2), u8, 0)), (Stand((1 << 31, 32), u8), Stand((1 << 31, 2), u8)), (torch.zeros(48, 32, dtype=u8), torch.zeros(48, 2, dtype=u8))):
        with pytest.raises(q.MoeError) as e:
            q.DenseMatrix4(codes, scales)
        assert e.value.code == q.MOE_E_ARG


def test_two_workgroups_of_many_tokens_share_a_cu(tmp_path):
    """256 threads are a wave on each SIMD of 512 registers: two workgroups need at most 256 registers and 80 KB of LDS."""
    from test_kernel_resources import usage
    many = {n: u for n, u in usage("dense_linear_many.hip", tmp_path).items() if "linear_manyILi0E" in n or "linear_manyILi1E" in n}
    alone = tuple(f"ILi{x}ELi{v}E" for x in range(3) for v in ("4ELi4ELi1ELi4ELi2", "4ELi2ELi2ELi4ELi2", "2ELi2ELi2ELi4ELi2", "1ELi1ELi4ELi4ELi2"))        # one a CU
    some = {n: u for n, u in usage("dense_linear_some.hip", tmp_path).items() if not n.split("linear_some")[1].startswith(alone)}
    assert len(many) == 2 and len(some) == 18
    for name, (regs, lds) in {**many, **some}.items():
        assert regs <= 256 and lds <= 80 * 1024, (name, regs, lds)
