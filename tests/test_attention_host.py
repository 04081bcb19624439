"""Host side of the attention calls on the CPU: qattn_api.hip compiled as plain C++ with recording stubs in place of the kernels'
launchers (tests/host_stub/attn_test.cpp), and the binding with stand-ins for tensors."""
import math
import os
import subprocess

import pytest
import torch

import paper_2503_09304_amd as q
from paper_2503_09304_amd import attention as at
from test_attention_cpu import FAKE, cache, refused, rows

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
STUB = os.path.join(ROOT, "tests", "host_stub")
CSRC = os.path.join(ROOT, "paper_2503_09304_amd", "csrc")


def test_host_side_with_recorded_launches(tmp_path):
    """Decode calls of different sizes on one workspace: the sums of one never stand on the counters of another."""
    exe = str(tmp_path / "attn_test")
    cmd = ["g++", "-std=c++17", "-O1", "-Wall", "-I", STUB, "-I", os.path.join(ROOT, "include"), "-I", CSRC,
           "-x", "c++", os.path.join(CSRC, "qattn_api.hip"), os.path.join(STUB, "attn_test.cpp"), "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and "all attention host checks passed" in r.stdout, r.stdout[-3000:]


def test_prompts_of_more_rows_than_a_tile_counts():
    """Up to the end of its last tile of 128 a row's number has to stay below 2^31."""
    L, ok = at._lib(), rows()
    for n_q, n_k in [((1 << 31) - 1, 4), (4, (1 << 31) - 1), ((1 << 30) + 1, 4), (4, (1 << 30) + 1)]:
        refused(L.attn_prompt(ok, ok, ok, ok, None, FAKE, FAKE, 1, n_q, n_k, 8, 4, 128, 1.0, 1, None, 0, None), "2^30")
        assert L.attn_prompt_workspace_bytes(1, n_q, n_k, 8, 4, 128) == 0
    assert L.attn_prompt_workspace_bytes(1, 16, 1 << 20, 8, 4, 128) > 0


def test_scales_whose_power_of_two_overflows():
    L, ok, c = at._lib(), rows(), cache()
    for scale in (2.0 ** 127.9, 2.4e38):
        refused(L.attn_prompt(ok, ok, ok, ok, None, FAKE, FAKE, 1, 4, 4, 8, 4, 128, scale, 1, None, 0, None), "scale")
        refused(L.attn_decode(c, ok, ok, None, 2, 8, FAKE, 4, FAKE, scale, FAKE, 1 << 30, None, None), "scale")
    assert L.attn_prompt(ok, ok, ok, ok, None, FAKE, FAKE, 1, 0, 4, 8, 4, 128, 2.0 ** 127, 1, None, 0, None) == q.MOE_OK


class Stand:
    """Stands for a tensor on GPU `device`: what the binding looks at."""
    def __init__(self, shape, dtype, device=1):
        self.shape, self.dtype, self.on, self.device, self.is_cuda = tuple(shape), dtype, device, f"cuda:{device}", True

    def get_device(self):
        return self.on

    def dim(self):
        return len(self.shape)

    def stride(self):
        return tuple(math.prod(self.shape[i + 1:]) for i in range(len(self.shape)))

    def numel(self):
        return math.prod(self.shape)

    def data_ptr(self):
        return 1 << 20

    def is_contiguous(self):
        return True


class Recorded:
    """Stands for the library: which call came last, and which device was current."""
    def __init__(self, now):
        self.now, self.last = now, None

    def __getattr__(self, name):
        def call(*args):
            if name.endswith("_bytes"):
                return 0
            self.last = (name, self.now[-1], args[-1])
            return 0
        return call


def calls():
    """Of each call: itself, and its tensors by name."""
    bf, i32, f32 = torch.bfloat16, torch.int32, torch.float32
    heads, T = lambda h: Stand((4, h, 64), bf), 4  # noqa: E731
    place = dict(seq=Stand((T,), i32), pos=Stand((T,), i32), pages=Stand((2, 3), i32), bad=Stand((1,), i32))
    cache = dict(k=Stand((9, 2, 16, 64), torch.uint8), v=Stand((9, 2, 16, 64), torch.uint8), k_scale=Stand((9, 2, 16), torch.uint8), v_scale=Stand((9, 2, 16), torch.uint8))
    freq = Stand((32,), torch.float64)
    of = lambda c: at.AttnCache(c["cache_k"], c["cache_v"], c["cache_k_scale"], c["cache_v_scale"])  # noqa: E731
    cached = {"cache_" + n: t for n, t in cache.items()}
    return {
        "attn_append": (lambda c: at.attn_append(of(c), c["q"], c["k"], c["v"], c["seq"], c["pos"], c["pages"], at.AttnRope(c["freq"]), c["q_out"], c["k_out"], c["bad"]),
                        dict(cached, **place, q=heads(4), k=heads(2), v=heads(2), q_out=heads(4), k_out=heads(2), freq=freq)),
        "attn_read": (lambda c: at.attn_read(of(c), c["seq"], c["pos"], c["pages"], c["k_out"], c["v_out"], c["bad"]),
                      dict(cached, **place, k_out=heads(2), v_out=heads(2))),
        "attn_prompt": (lambda c: at.attn_prompt(c["q"], c["k"], c["v"], c["cu_q"], c["cu_k"], c["out"], lse=c["lse"]),
                        dict(q=heads(4), k=heads(2), v=heads(2), out=heads(4), cu_q=Stand((3,), i32), cu_k=Stand((3,), i32), lse=Stand((4, 4), f32))),
        "attn_decode": (lambda c: at.attn_decode(of(c), c["q"], c["pages"], c["lens"], c["out"], c["workspace"], lse=c["lse"], bad=c["bad"]),
                        dict(cached, q=heads(4), out=heads(4), pages=Stand((4, 3), i32), lens=Stand((4,), i32), lse=Stand((4, 4), f32), bad=place["bad"],
                             workspace=Stand((1 << 20,), torch.uint8))),
    }


@pytest.fixture
def two_gpus(monkeypatch):
    """Device 0 is current; the streams of device d are number 100 + d."""
    now = [0]

    class Guard:
        def __init__(self, device):
            self.device = device

        def __enter__(self):
            now.append(self.device)

        def __exit__(self, *args):
            now.pop()

    library = Recorded(now)
    monkeypatch.setattr(at, "_lib", lambda: library)
    monkeypatch.setattr(at, "_raw_stream", lambda d: 100 + d)
    monkeypatch.setattr(at, "_current_device", lambda: now[-1], raising=False)
    monkeypatch.setattr(torch.cuda, "device", Guard)
    return library


@pytest.mark.parametrize("name", ["attn_append", "attn_read", "attn_prompt", "attn_decode"])
def test_calls_go_to_the_device_of_their_tensors(name, two_gpus):
    call, tensors = calls()[name]
    for device in (0, 1):
        for t in tensors.values():
            t.on = device
        assert call(tensors) == q.MOE_OK
        assert two_gpus.last == (name, device, 100 + device) and two_gpus.now == [0]


@pytest.mark.parametrize("name", ["attn_append", "attn_read", "attn_prompt", "attn_decode"])
def test_tensors_of_two_devices_are_refused(name, two_gpus):
    call, tensors = calls()[name]
    for odd in tensors:
        for device in (0, -1):
            for n, t in tensors.items():
                t.on = device if n == odd else 1
            with pytest.raises(q.MoeError) as e:
                call(tensors)
            assert e.value.code == q.MOE_E_ARG and two_gpus.last is None, odd


@pytest.mark.parametrize("name,long", [("attn_append", ("k", "v", "q", "q_out", "k_out", "seq", "pos")), ("attn_append", ("q",)), ("attn_append", ("pages",)), ("attn_read", ("k_out", "v_out", "seq", "pos")),
                                       ("attn_prompt", ("q", "out", "lse")), ("attn_prompt", ("k", "v")), ("attn_prompt", ("cu_q", "cu_k")),
                                       ("attn_decode", ("q", "out", "lse", "pages", "lens"))])
def test_counts_of_33_bits_are_refused(name, long, two_gpus):
    """2^32 rows more than there are: the library's 32 bits would be the rows that there are."""
    call, tensors = calls()[name]
    for t in long:
        tensors[t].shape = (tensors[t].shape[0] + (1 << 32), *tensors[t].shape[1:])
    with pytest.raises(q.MoeError) as e:
        call(tensors)
    assert e.value.code == q.MOE_E_ARG and two_gpus.last is None
