"""Which rows of a 4-bit weight the decoding kernel of the gated block loads: for every hidden size up to some tiles, that each load its descriptors let through lies in the group's own
weights, and that every row whose products are used is let through.  The arithmetic is the kernel's own, compiled for the host."""
import os
import shutil
import subprocess

import pytest

import paper_2603_05500_amd as px

PROGRAM = r"""
#include "values_tile.h"
#include <cstdio>
#include <initializer_list>
using namespace poetx::values;
int main() {
  for (int n = 1; n <= 400; ++n)
    for (int width : {64, 128})
      for (int units = 1; units <= 3; ++units)
        for (int n0 = 0; n0 < (n + 127) / 128 * 128; n0 += width) {
          const int ldb = units * 64, reach = gated_reach(n, n0, width), cols = n - n0 < width ? n - n0 : width;
          for (int u = 0; u < units; ++u) {
            // bytes that the descriptors let through: as they start, and none below zero on the way
            auto left = [&](int bytes) { return (unsigned)(u > 0 && bytes < 0 ? 0 : bytes); };
            const unsigned codes = left(reach * ldb - 64 * u), scales = left((reach * units - u) * 4);
            for (int r = 0; r < 2 * width; ++r) {
              const int row = gated_row(r, n, width), column = r % width;
              bool through = false;
              for (int chunk = 0; chunk < 4; ++chunk) {
                const unsigned at = (unsigned)(row * ldb + 16 * chunk);
                through = (unsigned long long)at + 16 <= codes && codes <= 0x7fffffffu;
                if ((unsigned long long)at + 16 <= codes && (long long)n0 * ldb + 64 * u + at + 16 > 2ll * n * ldb) return printf("codes: n %d, width %d, n0 %d, row %d, unit %d of %d\n", n, width, n0, r, u, units), 1;
              }
              const unsigned at = (unsigned)(row * units * 4);
              if ((unsigned long long)at + 4 <= scales && (long long)(n0 * units + u) * 4 + at + 4 > 8ll * n * units) return printf("scales: n %d, width %d, n0 %d, row %d\n", n, width, n0, r), 1;
              const int wanted = r < width ? n0 + r : n + n0 + r - width;
              if (column < cols && (n0 + row != wanted || !through)) return printf("not loaded: n %d, width %d, n0 %d, row %d\n", n, width, n0, r), 1;
            }
          }
        }
  return 0;
}
"""


def test_loads_stay_in_the_group(tmp_path):
    compiler = shutil.which("g++") or shutil.which("clang++")
    if not compiler:
        pytest.skip("no host compiler")
    (tmp_path / "loads.cpp").write_text(PROGRAM)
    csrc = os.path.join(os.path.dirname(os.path.abspath(px.__file__)), "csrc")
    subprocess.run([compiler, "-std=c++17", "-O1", "-I", csrc, "loads.cpp", "-o", "loads"], cwd=tmp_path, check=True)
    run = subprocess.run([str(tmp_path / "loads")], capture_output=True, text=True)
    assert run.returncode == 0, run.stdout
