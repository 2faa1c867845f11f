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
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
LIB = os.path.join(PKG, "libpoetx.so")
LIMITS = os.path.join(PKG, "poetx_limits")          # measurement tool (csrc/diag/limits.hip)

FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared", "-fno-gpu-rdc",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-Wall", "-Wno-unused-function", "-Wno-unused-value", "-Wno-unused-private-field"]


def sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.hip")))


def run(cmd, verbose: bool = False):
    if verbose:
        print(" ".join(cmd), flush=True)
    r = subprocess.run(cmd, capture_output=True, text=True)
    err = "\n".join(l for l in r.stderr.splitlines() if "is not a recognized feature for this target" not in l)
    if r.returncode != 0:
        raise RuntimeError("hipcc failed:\n" + err)
    if verbose and err.strip():
        print(err, file=sys.stderr)


def compile_one(source: str, obj: str, verbose: bool = False):
    """One object; with waits in front of its hand-written loads where the assembly has one that needs them.  Returns what needed them."""
    first = None
    for waits in ([], ["-DPOETX_LOAD_WAITS"]):
        run([HIPCC, *(f for f in FLAGS if f != "-shared"), *waits, "--save-temps=obj", "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-c", source, "-o", obj], verbose)
        with open(obj[:-2] + "-hip-amdgcn-amd-amdhsa-gfx950.s") as f:
            found = too_close(f.read())
        first = found if first is None else first
        if not found:
            return first
        if verbose:
            print(source + ": loads that need waits:", *found, sep="\n  ", flush=True)
    raise RuntimeError(f"{source}: scalar operands read too soon: {found}")


def build(verbose: bool = False) -> str:
    # one object per source, a few at a time: their kernels share nothing.  The last one is of the measurement tool: machine ceilings next to the dense kernel and its feed-less variants
    with tempfile.TemporaryDirectory() as tmp:
        todo = [*sources(), os.path.join(CSRC, "diag", "limits.hip")]
        objects = [os.path.join(tmp, os.path.basename(s)[:-4] + ".o") for s in todo]
        with ThreadPoolExecutor(max_workers=min(8, os.cpu_count() or 1)) as pool:
            list(pool.map(lambda s, o: compile_one(s, o, verbose), todo, objects))
        run([HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-fno-gpu-rdc", *objects[:-1], "-o", LIB], verbose)
        run([HIPCC, "--offload-arch=gfx950", objects[-1], "-o", LIMITS], verbose)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
