"""Host side of the attention calls on the CPU: qattn_api.hip compiled as plain C++ with recording stubs in place of the kernels'
launchers (tests/host_stub/attn_test.cpp), and the binding with stand-ins for tensors."""
import os
import subprocess

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
