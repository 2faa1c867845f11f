"""Build libpoetx.so (gfx950) in-tree with hipcc."""
from __future__ import annotations

import glob
import os
import subprocess
import sys
import tempfile
from concurrent.futures import ThreadPoolExecutor

try:
    from .load_waits import too_close
except ImportError:      # run as a file
    from load_waits import too_close

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
LIB = os.path.join(PKG, "libpoetx.so")
LIMITS = os.path.join(PKG, "poetx_limits")          # measurement tool (csrc/diag/limits.hip)

FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared", "-fno-gpu-rdc",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-Wall", "-Wno-unused-function", "-Wno-unused-value"]


def sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.hip")))


def build(verbose: bool = False) -> str:
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    noise = "is not a recognized feature for this target"

    def run(cmd):
        if verbose:
            print(" ".join(cmd), flush=True)
        r = subprocess.run(cmd, capture_output=True, text=True)
        err = "\n".join(l for l in r.stderr.splitlines() if noise not in l)
        if r.returncode != 0:
            raise RuntimeError("hipcc failed:\n" + err)
        if verbose and err.strip():
            print(err, file=sys.stderr)

    # one object per source, a few at a time: their kernels share nothing
    with tempfile.TemporaryDirectory() as tmp:
        objects = [os.path.join(tmp, os.path.basename(s)[:-4] + ".o") for s in sources()]
        compile_flags = [f for f in FLAGS if f != "-shared"]

        def compile_one(source, obj):
            for waits in ([], ["-DPOETX_LOAD_WAITS"]):
                run([hipcc, *compile_flags, *waits, "--save-temps=obj", "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-c", source, "-o", obj])
                with open(obj[:-2] + "-hip-amdgcn-amd-amdhsa-gfx950.s") as f:
                    found = too_close(f.read())
                if not found:
                    return
                if verbose:
                    print(source + ": loads that need waits:", *found, sep="\n  ", flush=True)
            raise RuntimeError(f"{source}: scalar operands read too soon: {found}")

        with ThreadPoolExecutor(max_workers=min(8, os.cpu_count() or 1)) as pool:
            list(pool.map(compile_one, sources(), objects))
        run([hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", "-fno-gpu-rdc", *objects, "-o", LIB])
    # the measurement tool: machine ceilings next to the dense kernel and its feed-less variants
    tool = [hipcc, "--offload-arch=gfx950", "-O3", "-std=c++17", "-Xclang", "-target-feature", "-Xclang",
            "-packed-fp32-ops", "-Wno-unused-value", "-Wno-unused-result", "-I", os.path.join(ROOT, "include"), "-I", CSRC,
            os.path.join(CSRC, "diag", "limits.hip"), "-o", LIMITS]
    run(tool)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
