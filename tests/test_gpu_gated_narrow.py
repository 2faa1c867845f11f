"""The gated block of hidden sizes below a block of 32 and enough rows to leave the kernels for a handful: tiles that lie wholly behind the last column, for the codes of zero there.
Bounds as in test_gpu_gated.py; groups are many, so that the last one's weights end the buffer after some tiles' beginning."""
from __future__ import annotations

import pytest

from tests.test_gpu_gated import run_all

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("counts,m,n", [
    ([16376], 512, 24), ([9000, 0, 7400, 3600], 1032, 16), ([33000], 136, 8), ([20000], 264, 31), ([4500] * 4 + [40], 200, 30),      # 4-bit weights decoded on the way
    ([16500, 16500], 72, 1), ([16384], 260, 33), ([9000, 9000], 130, 47),
])
@pytest.mark.parametrize("weight", ["mx4", "dense"])
def test_fewer_columns_than_a_block(lib, counts, m, n, weight):
    run_all(counts, m, n, "bf16", "gelu" if n % 2 else "silu", weight, before=3, extra=5)


@pytest.mark.parametrize("counts,m,n", [([16376], 128, 24), ([20000], 72, 5), ([9000, 0, 7400], 68, 31)])
def test_fewer_columns_than_a_block_fp32(lib, counts, m, n):
    run_all(counts, m, n, "f32", "silu", before=3, extra=5)
