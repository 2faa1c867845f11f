"""The check of hand-written loads in the build: with the compiler's own output, with waits, and along the branches of what was built."""
import os
import re
import shutil
import subprocess

import pytest

import paper_2603_05500_amd as px
from paper_2603_05500_amd import build
from paper_2603_05500_amd.load_waits import too_close
from tests.test_abi import clib  # noqa: F401
from tests.test_built_code import OBJDUMP

needs_compiler = pytest.mark.skipif(not os.path.exists(build.HIPCC), reason="no hipcc here")

# Descriptors, bases and masks that vector instructions bring into scalar registers right before the loads that take them.
SOURCE = r"""
#include "grouped_stream.h"
using namespace poetx;
extern "C" __global__ void loads(const uint32_t* p, uint32_t* out) {
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  const uint32_t at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds;
  grouped::u32x4 r;
  for (int i = 0; i < 4; ++i) r[i] = __builtin_amdgcn_readfirstlane(p[threadIdx.x + i]);
  KIND
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  out[threadIdx.x] = ((uint32_t*)lds)[threadIdx.x];
}
"""
KINDS = {
    "16 bytes": "grouped::dma16b(r, 16 * threadIdx.x, at);",
    "4 bytes": "grouped::dma4b(r, 4 * threadIdx.x, at);",
    "masked": "grouped::dma16b_but((uint64_t)r[1] << 32 | r[0], r, 16 * threadIdx.x, at);",
    "base": "dense::dma16g<0>((const void*)((uint64_t)r[1] << 32 | r[0]), 16 * threadIdx.x, at);",
}


@needs_compiler
@pytest.mark.parametrize("kind", KINDS)
def test_found_and_mended(tmp_path, kind):
    source, obj = tmp_path / "loads.hip", tmp_path / "loads.o"
    source.write_text(SOURCE.replace("KIND", KINDS[kind]))
    assert build.compile_one(str(source), str(obj)), "the plain build has a load that reads too soon"
    text = (tmp_path / "loads-hip-amdgcn-amd-amdhsa-gfx950.s").read_text()
    assert too_close(text) == []
    block = re.search(r";;#ASMSTART\s*\n([^;]*_load_[^;]*);;#ASMEND", text)[1].split("\n")
    assert block[0].strip() == "s_nop 4"
    # and without the waits
    bare = text.replace("s_nop 4\n", "s_nop 0\n")
    assert too_close(bare)


def test_unmarked_load_is_an_error():
    load = "buffer_load_dwordx4 v3, s[40:43], 0 offen lds\n"
    assert too_close(";;#ASMSTART\n" + load + ";;#ASMEND\n") == []
    for line in (load, "global_load_lds_dwordx4 v2, s[4:5]\n"):
        with pytest.raises(ValueError):
            too_close(";#OTHER_START\n" + line + ";#OTHER_END\n")
    assert too_close("buffer_load_dwordx4 v[0:3], v3, s[40:43], 0 offen\n") == []


def test_no_such_load_along_branches(clib, tmp_path):  # noqa: F811
    """The library as it was linked, each branch followed."""
    if not os.path.exists(OBJDUMP):
        pytest.skip("no llvm-objdump here")
    shutil.copy(px.LIB_PATH, tmp_path / "lib.so")
    subprocess.run([OBJDUMP, "--offloading", "lib.so"], cwd=tmp_path, check=True, capture_output=True)
    loads = branches = 0
    for f in sorted(tmp_path.glob("lib.so.*gfx950")):
        out = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", "--no-leading-addr", "--symbolize-operands", str(f)], check=True, capture_output=True, text=True).stdout
        lines, kernel = [], 0
        for line in (l.split("//")[0].strip() for l in out.splitlines()):
            local = re.fullmatch(r"<(L\d+)>:", line)
            branch = re.fullmatch(r"(s_c?branch\w*) (L\d+)", line)
            if local:
                lines.append(f"{kernel}.{local[1]}:")                  # labels are counted anew in every kernel
            elif line.endswith(">:"):
                kernel += 1
                lines.append("s_endpgm")                               # nothing falls into a kernel
            elif branch:
                branches += 1
                lines.append(f"{branch[1]} {kernel}.{branch[2]}")
            elif re.search(r"_load_lds_|\blds$", line):
                loads += 1
                masked = lines and lines[-1].startswith("v_cndmask_b32") and re.split(r"[ ,]+", lines[-1])[1] == re.split(r"[ ,]+", line)[1]
                lines[-1:] = [";;#ASMSTART", lines[-1], line, ";;#ASMEND"] if masked else [*lines[-1:], ";;#ASMSTART", line, ";;#ASMEND"]
            elif line:
                lines.append(line)
        assert too_close("\n".join(lines)) == []
    assert loads > 1000 and branches > 1000
