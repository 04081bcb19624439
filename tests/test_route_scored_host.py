"""What the router by scores promises its compiler, on the CPU."""
import os
import re
import subprocess

from paper_2503_09304_amd import build


def test_one_array_of_sums_and_logits(tmp_path):
    """A router whose hidden size is one range has its sums in the logits' array, which the choice reads and writes: neither pointer may be
    promised to be the only one to its memory."""
    out = str(tmp_path / "route_scored.ll")
    r = subprocess.run([build.HIPCC, *build.FLAGS, "--cuda-device-only", "-S", "-emit-llvm", os.path.join(build.CSRC, "route_scored.hip"), "-o", out], capture_output=True,
                       text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-4000:]
    found = re.findall(r"^define [^\n]*amdgpu_kernel void @(\S*score_topk\S*?)\((.*)\)[^)]*\{", open(out).read(), flags=re.M)
    assert len(found) == 5 * (4 + 3)
    for name, args in found:
        pointers = re.findall(r"ptr addrspace\(1\)[^%]*%", args)
        assert len(pointers) == 4, (name, args)                     # sums, logits, experts, weights
        assert "noalias" not in pointers[0] and "noalias" not in pointers[1], (name, args)
