"""Host side of the attention calls (include/qattn.h), without a GPU: symbols, argument checks that refuse before anything
is enqueued, workspace sizes, and the rotary frequencies against formulas of their own."""
import ctypes as C
import math
import os
import re
import subprocess

import numpy as np
import pytest

import paper_2503_09304_amd as q
from paper_2503_09304_amd import attention as at
from paper_2503_09304_amd import build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 1 << 20                    # addresses that these calls never look at


def test_library_exports_every_declared_symbol():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "qattn.h")).read(), flags=re.S)
    names = set(re.findall(r"\b(attn_[a-z_]+)\s*\(", text))
    assert {"attn_append", "attn_read", "attn_prompt", "attn_decode", "attn_rope_frequencies"} <= names
    for n in names:
        assert hasattr(q.lib(), n), n


class Rows(C.Structure):
    _fields_ = [("data", C.c_void_p), ("token_stride", C.c_int64), ("head_stride", C.c_int64)]


class Place(C.Structure):
    _fields_ = [("seq", C.c_void_p), ("pos", C.c_void_p), ("pages", C.c_void_p), ("n_seqs", C.c_int32), ("seq_pages", C.c_int32)]


KEEP = []


def pointer(s):
    KEEP.append(s)
    return C.addressof(s)


def rows(ts=512, hs=128, data=FAKE):
    return pointer(Rows(data, ts, hs))


def rope(*args):
    return pointer(at._Rope(*args))


def cache(**kw):
    d = dict(k=FAKE, v=FAKE, k_scale=0, v_scale=0, n_pages=8, heads_kv=4, page_tokens=64, dim=128, format=q.ATTN_BF16)
    d.update(kw)
    return pointer(at._Cache(**d))


def place(**kw):
    d = dict(seq=FAKE, pos=FAKE, pages=FAKE, n_seqs=2, seq_pages=4)
    d.update(kw)
    return pointer(Place(**d))


def refused(rc, word, code=q.MOE_E_ARG):
    assert rc == code, (rc, q.moe_last_error())
    assert word in q.moe_last_error(), q.moe_last_error()


BAD_CACHES = [(dict(k=0), "null"), (dict(format=2), "format"), (dict(format=q.ATTN_FP8), "scale"), (dict(n_pages=0), "n_pages"),
              (dict(heads_kv=0), "heads_kv"), (dict(page_tokens=8), "page_tokens"), (dict(page_tokens=48), "page_tokens"),
              (dict(page_tokens=512), "page_tokens"), (dict(dim=136), "dim"), (dict(dim=0), "dim"), (dict(dim=72), "dim"), (dict(v=FAKE + 8), "aligned"),
              (dict(format=q.ATTN_FP8, k_scale=FAKE + 2, v_scale=FAKE), "aligned")]


@pytest.mark.parametrize("kw,word", BAD_CACHES)
def test_caches_refused(kw, word):
    L, c = at._lib(), cache(**kw)
    refused(L.attn_read(c, place(), 4, rows(), rows(), None, None), word)
    refused(L.attn_append(c, rows(), rows(), rows(), rows(), None, 4, 4, place(), None, None, None), word)
    refused(L.attn_decode(c, rows(), rows(), None, 2, 4, FAKE, 4, FAKE, 1.0, FAKE, 1 << 30, None, None), word)


BAD_ROWS = [(None, "null"), (rows(data=0), "null"), (rows(data=FAKE + 8), "aligned"), (rows(ts=500), "strides"), (rows(hs=100), "strides"),
            (rows(ts=-512), "strides")]


@pytest.mark.parametrize("r,word", BAD_ROWS)
def test_rows_refused(r, word):
    L, c = at._lib(), cache()
    ok = rows()
    refused(L.attn_read(c, place(), 4, r, ok, None, None), word)
    refused(L.attn_read(c, place(), 4, ok, r, None, None), word)
    refused(L.attn_append(c, ok, r, ok, ok, None, 4, 4, place(), None, None, None), word)
    refused(L.attn_append(c, ok, ok, r, ok, None, 4, 4, place(), None, None, None), word)
    refused(L.attn_prompt(r, ok, ok, ok, None, FAKE, FAKE, 1, 4, 4, 4, 4, 128, 1.0, 1, None, 0, None), word)
    refused(L.attn_prompt(ok, r, ok, ok, None, FAKE, FAKE, 1, 4, 4, 4, 4, 128, 1.0, 1, None, 0, None), word)
    refused(L.attn_prompt(ok, ok, r, ok, None, FAKE, FAKE, 1, 4, 4, 4, 4, 128, 1.0, 1, None, 0, None), word)
    refused(L.attn_prompt(ok, ok, ok, r, None, FAKE, FAKE, 1, 4, 4, 4, 4, 128, 1.0, 1, None, 0, None), word)
    refused(L.attn_decode(c, r, ok, None, 2, 4, FAKE, 4, FAKE, 1.0, FAKE, 1 << 30, None, None), word)
    refused(L.attn_decode(c, ok, r, None, 2, 4, FAKE, 4, FAKE, 1.0, FAKE, 1 << 30, None, None), word)


def test_append_and_read_refusals():
    L, c, ok = at._lib(), cache(), rows()

    def append(heads=4, n=4, p=place(), turn=None, qq=ok, qo=ok):
        return L.attn_append(c, qq, ok, ok, qo, None, heads, n, p, turn, None, None)

    refused(append(n=-1), "n_tokens")
    refused(append(heads=6), "heads_q")
    refused(append(heads=0), "together")
    refused(append(qo=None), "together")
    refused(append(p=place(pos=0)), "pos")
    refused(append(p=place(pages=0)), "pages")
    refused(append(p=place(n_seqs=0)), "n_seqs")
    refused(append(p=place(seq_pages=0)), "seq_pages")
    refused(append(turn=rope(0, 64, 0, 1.0)), "inv_freq")
    refused(append(turn=rope(FAKE, 24, 0, 1.0)), "dims")
    refused(append(turn=rope(FAKE, 144, 0, 1.0)), "dims")
    refused(append(turn=rope(FAKE, -16, 0, 1.0)), "dims")
    refused(append(turn=rope(FAKE, 64, 2, 1.0)), "layout")
    refused(append(turn=rope(FAKE, 64, 0, math.inf)), "mscale")
    refused(L.attn_read(c, None, 4, ok, ok, None, None), "place")
    assert append(n=0) == q.MOE_OK and L.attn_read(c, place(), 0, None, None, None, None) == q.MOE_OK       # nothing to do


def test_prompt_and_decode_refusals():
    L, c, ok = at._lib(), cache(), rows()

    def prompt(n_seqs=1, n_q=4, n_k=4, Hq=8, Hk=4, D=128, scale=1.0, cu=FAKE, ws=0):
        return L.attn_prompt(ok, ok, ok, ok, None, cu, cu, n_seqs, n_q, n_k, Hq, Hk, D, scale, 1, ws, 1 << 40, None)

    def decode(n=2, Hq=8, pages=FAKE, sp=4, lens=FAKE, scale=1.0, ws=FAKE, nb=1 << 40):
        return L.attn_decode(c, ok, ok, None, n, Hq, pages, sp, lens, scale, ws, nb, None, None)

    for kw, word in [(dict(Hq=6), "heads"), (dict(Hk=0), "heads"), (dict(Hq=2048, Hk=1024), "heads"), (dict(D=120), "dim"), (dict(n_seqs=-1), "negative"),
                     (dict(n_q=-1), "negative"), (dict(n_k=-1), "negative"), (dict(n_seqs=(1 << 20) + 1), "2^20"), (dict(scale=0.0), "scale"), (dict(scale=-1.0), "scale"),
                     (dict(scale=math.nan), "scale"), (dict(scale=math.inf), "scale"), (dict(cu=0), "cu_q")]:
        refused(prompt(**kw), word)
    refused(L.attn_prompt(ok, rows(ts=(1 << 24) + 8), ok, ok, None, FAKE, FAKE, 1, 4, 4, 4, 4, 128, 1.0, 1, None, 0, None), "2^24")
    refused(prompt(ws=FAKE + 8), "workspace", q.MOE_E_WORKSPACE)
    assert prompt(n_seqs=0) == q.MOE_OK and prompt(n_q=0) == q.MOE_OK
    for kw, word in [(dict(n=-1), "n_seqs"), (dict(n=65536), "n_seqs"), (dict(Hq=6), "heads"), (dict(pages=0), "pages"), (dict(lens=0), "lens"),
                     (dict(sp=0), "seq_pages"), (dict(sp=1 << 24), "seq_pages"), (dict(n=65535, sp=1 << 18), "2^38"), (dict(scale=math.nan), "scale")]:
        refused(decode(**kw), word)
    need = L.attn_decode_workspace_bytes(2, 8, 4, 128)
    for kw in (dict(ws=0), dict(ws=FAKE + 64), dict(nb=need - 1)):
        refused(decode(**kw), "workspace", q.MOE_E_WORKSPACE)
    assert decode(n=0) == q.MOE_OK


def test_decode_workspace_sizes():
    L = at._lib()
    for n, Hq, Hk, D in [(0, 1, 1, 16), (1, 32, 8, 128), (64, 32, 8, 128), (7, 71, 1, 64), (3, 5, 5, 112), (65535, 1024, 1024, 128)]:
        whole, counters = L.attn_decode_workspace_bytes(n, Hq, Hk, D), L.attn_decode_counter_bytes(n, Hq, Hk)
        tiles = Hk * -(-(Hq // Hk) // 16)
        assert counters % 256 == 0 and counters >= 4 * n * tiles
        # a piece of every sequence at least, each 16 rows of sums with their maximum and total
        assert whole - counters >= 4 * max(1, n) * tiles * 16 * (D + 2)
    for bad in [(-1, 8, 8, 64), (65536, 8, 8, 64), (4, 8, 3, 64), (4, 0, 0, 64), (4, 8, 8, 60)]:
        assert L.attn_decode_workspace_bytes(*bad) == 0
    assert L.attn_decode_workspace_bytes(4, 8, 8, 64) > 0


def test_prompt_workspace_sizes():
    """Only where queries leave CUs idle and keys are many: a part of the sums and two floats a row and head."""
    size = at._lib().attn_prompt_workspace_bytes
    assert size(1, 16384, 16384, 32, 8, 128) == 0 and size(1, 17, 17, 32, 8, 128) == 0 and size(64, 64, 64 * 4096, 32, 8, 128) == 0
    for n, n_q, n_k, Hq, Hk, D in [(1, 128, 16384, 8, 8, 128), (6, 2434, 16801, 16, 16, 64), (1, 1, 1 << 20, 1, 1, 16)]:
        one = n_q * Hq * (D + 2) * 4
        assert size(n, n_q, n_k, Hq, Hk, D) % one == 0 and 2 <= size(n, n_q, n_k, Hq, Hk, D) // one <= 16
    assert size(1, 128, 16384, 8, 3, 128) == 0 and size(0, 128, 16384, 8, 8, 128) == 0 and size(1, 128, 0, 8, 8, 128) == 0


def test_frequencies():
    f, m = q.attn_rope_frequencies(128, 10000.0)
    i = np.arange(64)
    plain = 10000.0 ** (-i / 64)
    assert m == 1.0 and np.allclose(f, plain, rtol=1e-14, atol=0)
    f, m = q.attn_rope_frequencies(128, 10000.0, "linear", 8.0)
    assert m == 1.0 and np.allclose(f, plain / 8, rtol=1e-14, atol=0)
    f, m = q.attn_rope_frequencies(64, 10000.0, "base", 8.0)
    # the fastest pair stays, the slowest is divided by the factor
    assert m == 1.0 and f[0] == 1.0 and np.isclose(f[31], 10000.0 ** (-62 / 64) / 8, rtol=1e-12)
    f, m = q.attn_rope_frequencies(128, 10000.0, "ramp", 32.0, trained=4096.0, fast=32.0, slow=1.0)
    turns = 4096 * plain / (2 * math.pi)
    assert np.isclose(m, 0.1 * math.log(32.0) + 1, rtol=1e-7)
    r = np.array(f) / plain
    lo, hi = np.flatnonzero(turns > 32).max(), np.flatnonzero(turns < 1).min()       # pairs that turn more often than `fast`, less than `slow`
    assert np.allclose(r[:lo + 1], 1.0, rtol=1e-14) and np.allclose(r[hi:], 1 / 32, rtol=1e-13) and (np.diff(r[lo:hi + 1]) < 0).all()
    steps = np.diff(r[lo:hi + 1])
    assert np.allclose(steps, -(1 - 1 / 32) / (hi - lo), rtol=1e-10)
    f, m = q.attn_rope_frequencies(128, 500000.0, "waves", 8.0, trained=8192.0, fast=4.0, slow=1.0)
    plain = 500000.0 ** (-i / 64)
    wave = 2 * math.pi / plain
    r = np.array(f) / plain
    assert m == 1.0 and np.allclose(r[wave < 8192 / 4], 1.0, rtol=1e-14) and np.allclose(r[wave > 8192], 1 / 8, rtol=1e-13)
    mid = (wave >= 8192 / 4) & (wave <= 8192)
    t = (8192 / wave[mid] - 1.0) / 3.0
    assert mid.any() and np.allclose(r[mid], (1 - t) / 8 + t, rtol=1e-12)
    # factor 1 changes nothing
    for s in ("linear", "base", "ramp", "waves"):
        assert np.allclose(q.attn_rope_frequencies(96, 10000.0, s, 1.0)[0], q.attn_rope_frequencies(96, 10000.0)[0], rtol=1e-14)


@pytest.mark.parametrize("kw", [dict(dims=0), dict(dims=7), dict(dims=130), dict(base=1.0), dict(base=math.inf), dict(base=math.nan), dict(scaling="linear", factor=0.5),
                                dict(scaling="ramp", factor=math.nan), dict(dims=2, scaling="base", factor=2.0), dict(scaling="ramp", factor=2.0, trained=0.0),
                                dict(scaling="waves", factor=2.0, fast=1.0, slow=1.0), dict(scaling="waves", factor=2.0, slow=0.0), dict(scaling="other")])
def test_frequencies_refused(kw):
    with pytest.raises(q.MoeError) as e:
        q.attn_rope_frequencies(**dict(dict(dims=64), **kw))
    assert e.value.code == q.MOE_E_ARG


def test_registers_and_lds_of_the_attention_kernels(tmp_path):
    """Workgroups of 256 threads are a wave on each SIMD of 512 registers: what shares a CU by them and by 160 KB of LDS, and nothing in scratch."""
    seen = {}
    for src in ("attn_prompt", "attn_decode"):
        cmd = [build.HIPCC, *build.FLAGS, "--cuda-device-only", "-Rpass-analysis=kernel-resource-usage", "-c", os.path.join(build.CSRC, src + ".hip"),
               "-o", str(tmp_path / "kernels.o")]
        r = subprocess.run(cmd, capture_output=True, text=True, timeout=300)
        assert r.returncode == 0, r.stderr[-4000:]
        for part in r.stderr.split("Function Name: ")[1:]:
            get = lambda what: int(re.search(what + r": (\d+)", part).group(1))  # noqa: E731
            regs, lds = get(r"\bVGPRs") + get(r"\bAGPRs"), get(r"LDS Size \[bytes/block\]")
            assert get(r"ScratchSize \[bytes/lane\]") == 0, part.split()[0]
            seen[part.split()[0]] = min(512 // (-(-regs // 8) * 8), 160 * 1024 // max(lds, 1))
    for name, least in (("prompt_tileILi128E", 2), ("prompt_tileILi64E", 3), ("decode_pieceILi128E", 3), ("decode_pieceILi64E", 4)):
        found = [n for k, n in seen.items() if name in k]
        assert found and min(found) >= least, (name, seen)


def test_tensors_refused_by_the_binding():
    import torch
    bf = torch.zeros((4, 2, 64), dtype=torch.bfloat16)
    for call in (lambda: at._heads(bf, "q", 4, 2, 64),                                                       # not on the GPU
                 lambda: at.AttnCache(torch.zeros((2, 2, 16, 64)), torch.zeros((2, 2, 16, 64))),    # no bf16 or float8
                 lambda: at.AttnCache(torch.zeros((2, 2, 16, 64), dtype=torch.uint8), torch.zeros((2, 2, 16, 64), dtype=torch.uint8)),
                 lambda: at.AttnCache(bf, bf), lambda: at.AttnRope(torch.zeros(32, dtype=torch.float64), "other")):
        with pytest.raises(q.MoeError):
            call()
    assert C.sizeof(Rows) == 8 * at._ROWS == 24 and C.sizeof(at._Cache) == 56 and C.sizeof(Place) == 8 * at._PLACE == 32 and C.sizeof(at._Rope) == 24
