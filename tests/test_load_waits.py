"""Loads into LDS whose scalar operands a vector instruction has just written: found in assembly, and absent from the built kernels."""
import pytest

from paper_2603_05500_amd.load_waits import MEMORY, parse, too_close
from tests.test_built_code import listing  # noqa: F401
from tests.test_abi import clib  # noqa: F401

LOAD = ";;#ASMSTART\ns_nop 0\nbuffer_load_dwordx4 v3, s[40:43], 0 offen lds\n;;#ASMEND\n"
BACK = "v_readlane_b32 s43, v226, 36\n"
MASKED = ";;#ASMSTART\nv_cndmask_b32 v5, v3, v4, s[8:9]\nbuffer_load_dwordx4 v5, s[40:43], 0 offen lds\n;;#ASMEND\n"


@pytest.mark.parametrize("code,found", [
    (BACK + LOAD, 1), (BACK + "s_mov_b32 m0, s7\n" + LOAD, 1), (BACK + "v_add_u32 v1, v2, v3\n" * 3 + LOAD, 1),
    (BACK + "v_add_u32 v1, v2, v3\n" * 4 + LOAD, 0), (BACK + "s_nop 3\n" + LOAD, 0), (BACK + "s_nop 2\n" + LOAD, 1),
    (BACK.replace("s43", "s44") + LOAD, 0), (BACK.replace("s43", "s39") + LOAD, 0), (BACK.replace("s43", "s40") + LOAD, 1),
    ("s_mov_b32 s43, s1\n" + LOAD, 0), ("v_readfirstlane_b32 s41, v1\n" + LOAD, 1), ("v_cmp_gt_u32_e64 s[42:43], v1, v2\n" + LOAD, 1),
    ("v_readlane_b32 s9, v226, 36\n" + MASKED, 1), ("v_readlane_b32 s9, v226, 36\ns_nop 0\n" + MASKED, 1), ("v_readlane_b32 s9, v226, 36\ns_nop 1\n" + MASKED, 0),
    ("v_add_co_u32_e64 v1, s[40:41], v2, v3\n" + LOAD, 1),
    # over a branch, taken and not, and along a loop
    (BACK + "s_cbranch_scc1 .LBB0_2\ns_nop 7\n.LBB0_2:\n" + LOAD, 1), (BACK + "s_branch .LBB0_3\n" + LOAD + ".LBB0_3:\ns_nop 7\n", 0),
    (".LBB0_1:\n" + LOAD + "s_nop 7\n" + BACK + "s_cbranch_scc1 .LBB0_1\n", 1), (".LBB0_1:\n" + LOAD + "s_nop 7\n" + BACK + "s_nop 4\ns_cbranch_scc1 .LBB0_1\n", 0),
    # what the compiler writes itself it sees to
    (BACK + "buffer_load_dword v3, v4, s[40:43], 0 offen\n", 0),
])
def test_found(code, found):
    assert len(too_close(code)) == found


def test_no_such_load_is_built(listing):  # noqa: F811
    bad, kernel, recent = set(), "", []
    for line in listing:
        if line.endswith(">:"):
            kernel = line
            continue
        count, out, read, need, _ = parse(line) or (1, set(), set(), 0, None)
        if need == MEMORY and "lds" in line:
            passed = 0
            for c, written in reversed(recent):
                if passed < need and written & read:
                    bad.add(kernel)
                passed += c
        recent = recent[-5:] + [(count, out)]
    assert not bad, sorted(bad)
