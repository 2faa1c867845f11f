"""What the instruction set asks of the built kernels and the compiler does not see to inside inline assembly."""
import os
import re
import shutil
import subprocess

import pytest

import paper_2603_05500_amd as px
from tests.test_abi import clib  # noqa: F401

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"


@pytest.fixture(scope="module")
def listing(clib, tmp_path_factory):  # noqa: F811
    """The instructions of every kernel in order, a label as its name ending in ':'."""
    if not os.path.exists(OBJDUMP):
        pytest.skip("no llvm-objdump here")
    at = tmp_path_factory.mktemp("code")
    shutil.copy(px.LIB_PATH, at / "lib.so")
    subprocess.run([OBJDUMP, "--offloading", "lib.so"], cwd=at, check=True, capture_output=True)
    lines = []
    for f in sorted(at.glob("lib.so.*gfx950")):
        out = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", "--no-leading-addr", str(f)], check=True, capture_output=True, text=True).stdout
        lines += [t for t in (l.split("//")[0].strip() for l in out.splitlines()) if t]
    assert sum(l.startswith("s_endpgm") for l in lines) > 100
    return lines


def test_lds_loads_wait_for_m0(listing):
    """A load straight into LDS takes its address from M0, and needs an instruction between M0's write and itself."""
    loads, bad, kernel, before = 0, set(), "", ""
    for line in listing:
        if line.endswith(">:"):
            kernel = line
            continue      # code falls through labels: what comes before one counts
        if re.match(r"\w+_load_lds_|\w+_load_\w+ .*\blds$", line):
            loads += 1
            if re.match(r"[sv]_\w+ m0\b", before):
                bad.add(kernel)
        before = line
    assert loads > 1000
    assert not bad, sorted(bad)
