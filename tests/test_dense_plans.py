"""The rule that picks dense_linear's kernel, tiles and ranges of columns, run on the CPU."""
import ctypes as C
import os
import random
import subprocess
from collections import namedtuple

import pytest

from test_dense_cpu import BF, CSRC, F8, STUB, d

Plan = namedtuple("Plan", "tiles rows ks share ranges range_blocks us bytes")
MANY = 8                                                           # tiles of the kernel for many tokens
ALL = 1 << 40


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("plan") / "plan.so")
    r = subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-shared", "-fPIC", "-I", CSRC, os.path.join(STUB, "plan_lib.cpp"), "-o", so], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    L = C.CDLL(so)
    L.plan.argtypes = [C.c_int] * 4 + [C.c_long, C.c_void_p, C.POINTER(C.c_float), C.POINTER(C.c_long)]

    def call(T, R, K, bf16=True, nb=ALL):
        out, us, need = (C.c_int * 6)(), C.c_float(), C.c_long()
        L.plan(T, R, K, int(bf16), nb, out, C.byref(us), C.byref(need))
        return Plan(*out, us.value, need.value)

    return call


def shapes(n, seed=1):
    rng = random.Random(seed)
    for i in range(n):
        T, R, K = (int(2 ** rng.uniform(0, top)) for top in ((13, 15, 9), (6, 15, 9), (11, 13, 9))[i % 3])
        yield T, R, 32 * K


def test_the_workspace_asked_for_is_the_plan_s(plan):
    for T, R, K in shapes(2000):
        for bf16 in (True, False):
            p = plan(T, R, K, bf16)
            assert p.bytes == d._lib().dense_linear_workspace_bytes(T, R, K, BF if bf16 else F8, BF)
            assert plan(T, R, K, bf16, p.bytes) == p                  # more than that changes nothing


def test_with_less_the_best_plan_without_ranges(plan):
    """Not the kernel for many tokens, whatever their number: only where it is the best."""
    cut = 0
    for T, R, K in shapes(3000):
        for bf16 in (True, False):
            full = plan(T, R, K, bf16)
            if full.bytes == 0:
                continue
            cut += 1
            none = plan(T, R, K, bf16, 0)
            assert none.ranges == 1 and none.bytes == 0 and plan(T, R, K, bf16, full.bytes - 1) == none
            assert none.tiles != MANY or T > 64
            assert full.us <= none.us or not bf16 and K > 8192
    assert cut > 500


def test_a_down_projection_of_61_tokens(plan):
    for bf16 in (True, False):
        full, none = plan(61, 4096, 14336, bf16), plan(61, 4096, 14336, bf16, 0)
        assert full.ranges >= 2 and full.us < 17 and none.ranges == 1 and none.us < 20 and none.tiles != MANY


def test_ranges_whose_scales_are_in_lds_at_once(plan):
    """8-bit rows: 64 blocks of 128 columns, where there is a workspace; in the kernel whose waves do not wait for each other always."""
    for T, R, K in shapes(3000, 2):
        for nb in (ALL, 0):
            p = plan(T, R, K, False, nb)
            if p.tiles != MANY and p.share > 0 and (nb or p.share == 1):
                assert p.range_blocks <= 64


def test_long_rows_in_8_bits_reach_every_kernel_that_takes_them(plan):
    """The shapes of test_gpu_dense_plans.py: each variant whose range is longer than its scales' place, whole rounds of blocks and odd ones behind it."""
    from test_gpu_dense_plans import LONG
    met = {p[:4] for p in (plan(*s, False, 0) for s in LONG) if p.range_blocks > 64 and p.tiles != MANY and p.share}
    wanted = {p[:4] for p in (plan(T, R, K + 8192, False, 0) for T, R, K in shapes(6000, 3)) if p.tiles != MANY and p.share}
    assert met == wanted, (met ^ wanted)


def variant(p, T, R):
    """What tells one plan's code from another's: kernel, tiles, waves, sums by ranges or whole, and with the largest tiles how many blocks are asked for ahead."""
    if p.tiles == MANY:
        return MANY
    groups = -(-(-(-R // 16)) // (4 * p.rows)) * -(-T // (16 * p.tiles)) * p.ranges
    return p[:4] + (p.ranges > 1,) + ((groups <= 256,) if (p.tiles, p.rows) == (4, 4) else ())


@pytest.mark.parametrize("bf16", [True, False])
def test_every_plan_is_compared_on_the_gpu(plan, bf16):
    """Whatever the rule gives on shapes of the whole range stands among those of test_gpu_dense_plans.py: a change of its constants that leaves a variant without one fails here."""
    from test_gpu_dense_plans import BF, F8, SHAPES
    mine = SHAPES[BF if bf16 else F8]
    met = {variant(plan(*s, bf16), s[0], s[1]) for s in mine}
    rng, wanted = random.Random(4), set()
    for _ in range(40000):
        T, R, K = int(2 ** rng.uniform(0, 13)), int(2 ** rng.uniform(0, 15.1)), 32 * int(2 ** rng.uniform(0, 9))
        wanted.add(variant(plan(T, R, K, bf16), T, R))
    assert len(wanted) > 20 and wanted <= met, wanted - met
    many = [s for s in mine if plan(*s, bf16).tiles == MANY]
    assert any(s[1] > 8 * 256 * 3 for s in many) and any(s[0] > 1024 for s in many) and all(s[0] % 16 and s[1] % 16 and s[2] % 128 for s in many)
    # groups of eight tiles of rows, the last one whole or not
    assert len({-(-s[1] // 256) % 8 for s in many}) > 2
