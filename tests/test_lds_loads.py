"""CPU check of the built kernels that bring operands from memory to LDS past the registers.  Those loads stand in inline assembly, where the compiler
neither inserts wait states nor counts what is under way, so the built code has to keep by itself, along every path: a wait state between a write of
m0 and the load whose place in LDS it gives, five between a vector instruction that writes a scalar register and the load that takes its address from
it, and, where a wait leaves the newest N loads under way, at least N others behind the newest of these."""
import re

import pytest

from test_mfma_hazards import kernels, listing, regs, within

NAMES = {"dense_linear": 12, "dense_linear_some": 30, "dense_linear_many": 3, "route_scored": 6}         # kernels with such loads
VMEM = ("global_", "buffer_", "scratch_", "flat_")
SCALAR = re.compile(r"\bs(?:\[(\d+):(\d+)\]|(\d+)\b)")


def to_lds(ins):
    return ins.startswith("global_load_lds_") or ins.startswith("buffer_load_") and ins.endswith(" lds")


def scalars(text):
    return {i for lo, hi, one in SCALAR.findall(text) for i in (range(int(lo), int(hi) + 1) if lo else (int(one),))}


def hazards(code):
    out = []
    for at, (x, _) in enumerate(code):
        if re.match(r"s_\w+ m0\b", x):
            out += [(x, code[j][0]) for j in within(code, at, 1, 1) if to_lds(code[j][0])]
        elif x.startswith("v_"):
            written = scalars(x.split(", ")[0])          # of v_readfirstlane, v_readlane, comparisons
            for j in within(code, at, 5, 1) if written else ():
                if to_lds(code[j][0]) and written & scalars(code[j][0]):
                    out.append((x, code[j][0]))
    return out


def preceding(code):
    before = {}
    for i, (x, target) in enumerate(code):
        for j in ([] if x.startswith(("s_branch", "s_endpgm")) else [i + 1]) + ([target] if target is not None else []):
            before.setdefault(j, []).append(i)
    return before


def behind(code, before, at):
    """The fewest memory instructions between the newest load to LDS and instruction `at`, over all paths; None where no path has such a load."""
    least, todo, found = {at: 0}, [at], None
    while todo:
        i = min(todo, key=least.get)
        todo.remove(i)
        for j in before.get(i, []):
            if to_lds(code[j][0]):
                found = least[i] if found is None else min(found, least[i])
                continue
            n = least[i] + code[j][0].startswith(VMEM)
            if n < least.get(j, 1 << 30):
                least[j] = n
                todo.append(j)
    return found


def unwaited(code):
    """Barriers that some path reaches with a load to LDS under way."""
    before, out = preceding(code), []
    for barrier, (x, _) in enumerate(code):
        if not x.startswith("s_barrier"):
            continue
        todo, seen = [barrier], {barrier}
        while todo:
            for j in before.get(todo.pop(), []):
                y = code[j][0]
                if j in seen:
                    continue
                seen.add(j)
                if to_lds(y):
                    out.append((barrier, j))
                    continue
                m = re.search(r"vmcnt\((\d+)\)", y)
                if m:
                    n = behind(code, before, j)
                    if n is None or n >= int(m.group(1)):
                        continue
                todo.append(j)
    return out


@pytest.mark.parametrize("name", NAMES)
def test_wait_states(name, tmp_path):
    found = [(k, c) for k, c in kernels(name, tmp_path) if any(to_lds(x) for x, _ in c)]
    assert len(found) == NAMES[name]
    for kernel, code in found:
        assert not hazards(code), (kernel, len(hazards(code)), hazards(code)[:3])


@pytest.mark.parametrize("name", ["dense_linear", "dense_linear_many", "route_scored"])
def test_nothing_on_its_way_to_lds_at_a_barrier(name, tmp_path):
    """The counted wait of the router's products leaves loads of weights under way, which the compiler placed; the other two wait for all.
    (dense_linear_some counts loads to LDS alone, all in inline assembly.)"""
    for kernel, code in kernels(name, tmp_path):
        if any(to_lds(x) for x, _ in code):
            assert any(x.startswith("s_barrier") for x, _ in code) and not unwaited(code), (kernel, unwaited(code)[:3])


LOAD = "global_load_lds_dwordx4 v[2:3], off"
BASE = "global_load_lds_dwordx4 v2, s[4:5]"


def one(lines):
    return listing("0000000000001000 <k>:\n" + "".join(
        "\t%-58s // %012X:%s\n" % (x.split(" @")[0], 0x1000 + 4 * i, " <k+0x%x>" % (4 * int(x.split(" @")[1])) if " @" in x else "") for i, x in enumerate(lines)))["k"]


@pytest.mark.parametrize("good,lines", [
    (False, ["s_mov_b32 m0, s3", LOAD]),
    (True, ["s_mov_b32 m0, s3", "s_nop 0", LOAD]),
    (True, ["s_mov_b32 m0, s3", "s_mov_b32 exec_hi, 0", LOAD]),
    (False, ["s_add_i32 m0, s3, 16", LOAD]),
    (False, ["v_readfirstlane_b32 s5, v9", "s_mov_b32 m0, s3", "s_nop 2", BASE]),
    (True, ["v_readfirstlane_b32 s5, v9", "s_mov_b32 m0, s3", "s_nop 3", BASE]),
    (True, ["v_readfirstlane_b32 s6, v9", "s_nop 0", BASE]),
])
def test_scan_finds_planted_hazards(good, lines):
    assert (not hazards(one(lines))) == good


@pytest.mark.parametrize("good,lines", [
    (True, [LOAD, "global_load_dword v1, v2, s[2:3]", "s_waitcnt vmcnt(1)", "s_barrier"]),
    (False, [LOAD, "s_waitcnt vmcnt(1)", "s_barrier"]),
    (False, ["global_load_dword v1, v2, s[2:3]", LOAD, "s_waitcnt vmcnt(1)", "s_barrier"]),
    (False, [LOAD, "s_cbranch_scc1 1 @3", "global_load_dword v1, v2, s[2:3]", "s_waitcnt vmcnt(1)", "s_barrier"]),      # along the jump
    (True, [LOAD, "global_load_dword v1, v2, s[2:3]", "s_waitcnt vmcnt(1)", "s_barrier", "global_load_dword v1, v2, s[2:3]", "s_cbranch_scc1 -4 @2"]),
    (False, [LOAD, "global_load_dword v1, v2, s[2:3]", "s_waitcnt vmcnt(1)", "s_barrier", LOAD, "s_cbranch_scc1 -4 @2"]),
])
def test_scan_finds_waits_that_are_too_short(good, lines):
    assert (not unwaited(one(lines))) == good
