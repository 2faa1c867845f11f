"""The gated block with offsets that are not in order or point outside the rows, on every kernel: every row has the group that the header says, and nothing else is touched.
The oracle takes offsets as test_gpu_grouped_offsets.py does; bounds as in test_gpu_gated.py."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from tests.test_gpu_gated import Block, run_backward, run_recompute
from tests.test_gpu_grouped_offsets import disorder

pytestmark = pytest.mark.gpu

# A shape for every kernel of the block, with more than one group: groups, rows, d_in, d_hidden, dtype, weight.
KERNELS = {
    "few": (4, 100, 128, 64, "bf16", "dense"), "few f32": (4, 100, 128, 64, "f32", "dense"), "few mx4": (4, 100, 128, 64, "bf16", "mx4"),
    "edge 32": (6, 128, 72, 480, "bf16", "dense"), "edge 32 odd": (3, 2082, 160, 33, "bf16", "dense"), "edge 32 deep": (3, 1450, 2112, 32, "bf16", "dense"),
    "edge 32 deep odd": (5, 1124, 2095, 33, "bf16", "dense"), "edge 64": (8, 139, 40, 448, "bf16", "dense"), "edge 64 odd": (8, 162, 41, 371, "bf16", "dense"),
    "128": (4, 2315, 1800, 216, "bf16", "dense"), "128 narrow": (4, 3523, 1928, 132, "bf16", "dense"), "256 x 128": (6, 5561, 736, 328, "bf16", "dense"),
    "256 x 128 narrow": (5, 2132, 528, 933, "bf16", "dense"), "256": (4, 929, 680, 3560, "bf16", "dense"), "256 narrow": (5, 1126, 536, 3180, "bf16", "dense"),
    "in ranges": (6, 3183, 4352, 40, "bf16", "dense"), "in ranges narrow": (3, 4034, 4792, 34, "bf16", "dense"),
    "laid anew 256 x 128": (3, 4123, 1206, 752, "bf16", "dense"), "laid anew 256 narrow": (4, 7346, 861, 602, "bf16", "dense"),
    "edge 32 f32": (8, 35, 40, 1064, "f32", "dense"), "edge 64 f32": (6, 36, 32, 1600, "f32", "dense"), "64 f32": (8, 39, 72, 3936, "f32", "dense"),
    "64 f32 narrow": (4, 4921, 784, 65, "f32", "dense"), "128 f32": (2, 7940, 1952, 896, "f32", "dense"), "128 f32 narrow": (2, 8059, 1956, 754, "f32", "dense"),
    "in ranges f32": (4, 4148, 1488, 32, "f32", "dense"), "in ranges f32 narrow": (4, 2133, 1920, 58, "f32", "dense"),
    "laid anew f32": (3, 2302, 1253, 232, "f32", "dense"), "laid anew in ranges f32": (3, 1661, 2505, 264, "f32", "dense"),
    "decoded 64 x 128": (4, 70, 40, 2746, "bf16", "mx4"), "decoded 128 x 128": (6, 5031, 488, 336, "bf16", "mx4"), "decoded 128 x 256": (4, 830, 616, 3720, "bf16", "mx4"),
    "decoded in ranges": (3, 1853, 3752, 54, "bf16", "mx4"), "few mx4 laid anew": (3, 1541, 62, 57, "bf16", "mx4"), "decoded laid anew": (6, 4092, 172, 58, "bf16", "mx4"),
    "decoded laid anew in ranges": (3, 1587, 3815, 64, "bf16", "mx4"), "written out": (3, 16184, 32, 840, "bf16", "mx4"), "written out narrow": (2, 11205, 32, 1219, "bf16", "mx4"),
}


@pytest.mark.parametrize("kernel,kind", [(k, kind) for k, s in KERNELS.items() for kind in ("back and forth", "first in the middle", "some anywhere", "outside")[: 4 if s[1] * s[2] * s[3] < 1 << 27 else 2]])
def test_block(lib, kernel, kind):
    groups, rows, m, n, dtype, weight = KERNELS[kernel]
    offsets = disorder(kind, groups, rows)
    ends = np.maximum.accumulate(np.clip(offsets, 0, rows))
    b = Block(np.diff(ends).tolist(), m, n, dtype, "silu" if n % 2 else "gelu", weight, before=int(ends[0]), extra=rows - int(ends[-1]))
    assert b.off.tolist() == ends.tolist() and b.rows == rows
    b.off = torch.from_numpy(offsets.astype(np.int32)).cuda()
    run_backward(b, "same")
    run_backward(b, "mx8")
    run_recompute(b)
