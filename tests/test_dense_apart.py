"""Outputs of the dense calls whose rows overlap are refused, whichever of the two strides brings them together (on the CPU)."""
import os
import subprocess

from test_dense_cpu import CSRC, ROOT, STUB


def test_every_layout_of_few_rows(tmp_path):
    exe = str(tmp_path / "apart_test")
    cmd = ["g++", "-std=c++17", "-O1", "-Wall", "-fsanitize=address,undefined", "-I", STUB, "-I", os.path.join(ROOT, "include"), "-I", CSRC,
           "-x", "c++", os.path.join(CSRC, "qdense_api.hip"), os.path.join(STUB, "dense_apart_test.cpp"), "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and "all rows that overlap are refused" in r.stdout, (r.stdout + r.stderr)[-3000:]
